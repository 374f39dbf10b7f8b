"""Rotary positions, and a paged cache held in 8 bits, as a serving loop calls them, and their plain forms.

A case is a dict of plain values. Its "op" is the call:

  rope      dkv_rope: the rows of a projection turned by their positions, before a dense cache is pruned
  append    dkv_rope_append: a step's q and new K turned by their positions, K and V written to their pages (16-bit, or 8-bit
            with a scale a row)
  compact   dkv_quant_compact: the kept rows of pruned sequences into 8-bit pages
  attn      dkv_quant_attn: attention of a step's tokens over 8-bit pages

Positions: pair i of a row's first `rot` elements turns by the angle p f_i, f_i = theta^(-2 i / rot), or a long context's scaled
f_i; a pair is (i, i + rot / 2), or (2 i, 2 i + 1) where they are interleaved. Angles of far positions are products in 64 bits.

8 bits: a row of 128 elements x is held as e4m3 values x / 2^e, rounded to nearest, and one scale 2^e, with the least e that
keeps them within 448.

A slab is one (layer, sequence slot, KV head), h = (l B + b) Hkv + g; row r of slab h is row table[h][r // P] P + r % P of the
pools (P rows a page). Lengths differ from slab to slab, as pruning leaves them. Sizes come from the case alone ("mix" seeds
them), values from the seed.
"""
import math

import numpy as np
import torch

own = False

HEAD = 128     # elements of a row
SINK, RECENT = 128, 1024
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _rotary(rot=128, inter=False, theta=10000.0, scaling="none", factor=1.0, context=0, low=0.0, high=0.0):
    """rot: elements turned, 0: none. scaling: none; linear: f / factor; ntk: a larger theta; bands: wavelengths over
    context / low are divided, those under context / high kept, between them a mix; yarn: the same by turns within the context
    (low .. high), with a factor on the values."""
    return {"rot": rot, "inter": inter, "theta": theta, "scaling": scaling, "factor": factor, "context": context, "low": low,
            "high": high}


PLAIN = _rotary()
BANDS = _rotary(128, False, 500000.0, "bands", 8.0, 8192, 1.0, 4.0)
YARN = _rotary(64, True, 10000.0, "yarn", 16.0, 4096, 1.0, 32.0)
NTK = _rotary(96, False, 10000.0, "ntk", 4.0)
LINEAR = _rotary(32, True, 10000.0, "linear", 4.0)
NONE = _rotary(0)


def _rope(name, heads, T, start, rotary, dtype="bf16", fused=True, mix=1):
    return {"name": name, "op": "rope", "heads": heads, "T": T, "start": start, "dtype": dtype, "fused": fused, "mix": mix, **rotary}


def _append(name, H, Hkv, B, ctx, tokens, page, rotary, bits=8, dtype="bf16", decode=0.0, far=0, fused=True, pad=0, mix=1):
    """ctx and tokens: (least, most) of a sequence; decode: share of the sequences that bring one token; far: what positions
    lie behind the rows of the cache, as tokens were pruned; fused: q, k and v are slices of one projection; pad: rows of the
    batch behind the last sequence."""
    return {"name": name, "op": "append", "L": 2, "H": H, "Hkv": Hkv, "B": B, "ctx_min": ctx[0], "ctx_max": ctx[1],
            "tok_min": tokens[0], "tok_max": tokens[1], "page": page, "bits": bits, "dtype": dtype, "decode": decode, "far": far,
            "fused": fused, "pad": pad, "mix": mix, **rotary}


def _compact(name, L, H, Hkv, B, admitted, ctx, D, W, rate, page, dtype="bf16", mix=1):
    """admitted: pruned sequences, which go to slots of a pool of B."""
    return {"name": name, "op": "compact", "L": L, "H": H, "Hkv": Hkv, "B": B, "admitted": admitted, "ctx_min": ctx[0],
            "ctx_max": ctx[1], "D": D, "W": W, "rate": rate, "page": page, "dtype": dtype, "mix": mix}


def _attn(name, H, Hkv, B, ctx, tokens, page, dtype="bf16", decode=0.0, causal=True, fused=True, pad=0, mix=1):
    return {"name": name, "op": "attn", "L": 2, "H": H, "Hkv": Hkv, "B": B, "ctx_min": ctx[0], "ctx_max": ctx[1],
            "tok_min": tokens[0], "tok_max": tokens[1], "page": page, "dtype": dtype, "decode": decode, "causal": causal,
            "fused": fused, "pad": pad, "mix": mix}


def listed():
    return [
        # K of a 16K prompt of a layer, in the projection that made it, before it is pruned.
        _rope("rope-k-16k", 8, 16384, 0, BANDS, mix=21),
        # Four layers' K and more of a long prompt's second part, each pair of neighbours turned, half of the head.
        _rope("rope-far-fp16", 28, 30001, 131072, YARN, dtype="fp16", fused=False, mix=22),
        # The next token of 16 sequences over pruned contexts: latency.
        _append("append-tokens-b16", 32, 8, 16, (1500, 24000), (1, 1), 64, BANDS, far=100000, mix=23),
        # A new turn of 4K tokens.
        _append("append-turn-4k", 32, 8, 1, (9000, 9000), (4096, 4096), 64, BANDS, far=120000, mix=24),
        # Ragged turns to 16-bit pages, a part of the head turned.
        _append("append-ragged-16bit", 28, 4, 5, (0, 6000), (0, 1500), 16, NTK, bits=16, dtype="fp16", fused=False, pad=7, mix=25),
        # A 16K prompt of the 32-layer model admitted after pruning.
        _compact("compact-16k", 32, 32, 8, 4, 1, (16384, 16384), 32, 476, 0.35, 64, mix=26),
        # Three ragged prompts of the 28-layer model, small pages.
        _compact("compact-ragged", 28, 28, 4, 8, 3, (700, 9001), 64, 123, 0.25, 16, dtype="fp16", mix=27),
        # One sequence's next token over 4K context, pruned: launch latency and the ends of the pass.
        _attn("token-4k", 32, 8, 1, (1800, 1800), (1, 1), 16, mix=28),
        # A decode step of 16 ragged sequences.
        _attn("tokens-b16", 32, 8, 16, (3000, 24000), (1, 1), 64, mix=29),
        # Five drafted tokens or so a sequence, seven heads a group.
        _attn("draft-b4-g7", 28, 4, 4, (2500, 30000), (3, 7), 32, dtype="fp16", fused=False, mix=30),
        # A serving step: some sequences bring a new turn, the others their next token.
        _attn("mixed-b12", 32, 8, 12, (0, 20000), (50, 2000), 64, decode=0.7, pad=9, mix=31),
        # A long new turn over a pruned 128K context.
        _attn("turn-4k-over-45k", 32, 8, 1, (45300, 45300), (4096, 4096), 64, mix=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["rope", "append", "append", "compact", "attn", "attn", "attn"])
    H, Hkv = rng.choice([(32, 8), (28, 4), (32, 4), (16, 8), (4, 4), (40, 8)])
    page, mix = rng.choice([16, 32, 64, 128]), rng.randrange(1 << 30)
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    rotary = rng.choice([PLAIN, BANDS, YARN, NTK, LINEAR])
    if op == "rope":
        return _rope(None, rng.choice([1, 4, 8, 28, 32]), _log(rng, 1, 20000), rng.randint(0, 1 << 20), rotary, dtype,
                     rng.random() < 0.5, mix)
    if op == "compact":
        B = _log(rng, 1, 16)
        top = _log(rng, 500, 12000)
        D = rng.randint(8, 96)
        return _compact(None, rng.randint(1, 16), H, Hkv, B, rng.randint(1, min(B, 4)), (rng.randint(1, top), top), D,
                        max(1, -(-max(1, top - SINK - RECENT) // D)), rng.uniform(0.1, 0.7), page, dtype, mix)
    kind = rng.choice(["token", "few", "turn", "mixed"])
    if kind == "token":
        B, tok, dec = _log(rng, 1, 32), (1, 1), 0.0
    elif kind == "few":
        B, tok, dec = _log(rng, 1, 16), (rng.randint(0, 2), rng.randint(2, 17)), 0.0
    elif kind == "turn":
        B, n = _log(rng, 1, 4), _log(rng, 18, 2500)
        tok, dec = (rng.randint(1, n), n), 0.0
    else:
        B, n = _log(rng, 2, 16), _log(rng, 18, 1500)
        tok, dec = (rng.randint(1, n), n), rng.uniform(0.3, 0.9)
    top = _log(rng, 300, max(301, min(30000, 4096 * 42000 // (B * tok[1]))))
    ctx = (rng.randint(0, top), top)
    if op == "append":
        return _append(None, H, Hkv, B, ctx, tok, page, rng.choice([rotary, rotary, rotary, NONE]), rng.choice([8, 8, 16]), dtype,
                       dec, rng.randint(0, 1 << 20), rng.random() < 0.6, rng.randint(0, 9), mix)
    return _attn(None, H, Hkv, B, ctx, tok, page, dtype, dec, rng.random() < 0.8, rng.random() < 0.6, rng.randint(0, 9), mix)


# ------------------------------------------------------------ sizes

def _lengths(case):
    """Rows of every slab before the step, int64 [L, B, Hkv]: of a context, pruning leaves each slab its own part."""
    r = np.random.default_rng([case["mix"], 1])
    L, B, Hkv = case["L"], case["B"], case["Hkv"]
    ctx = r.integers(case["ctx_min"], case["ctx_max"] + 1, B)
    return np.floor(ctx[None, :, None] * r.uniform(0.55, 1.0, (L, B, Hkv))).astype(np.int64)


def _tokens(case):
    """New tokens of every sequence, int64 [B]."""
    r = np.random.default_rng([case["mix"], 2])
    n = r.integers(case["tok_min"], case["tok_max"] + 1, case["B"])
    n = np.where(r.random(case["B"]) < case["decode"], 1, n).astype(np.int64)
    n[0] = max(n[0], 1)  # never an empty step
    return n


def _pages_of(rows, page):
    return -(-rows // page)


def _keep(case):
    """Plan of a compact case: (pattern uint8 [L, H, D], contexts [admitted], slots [admitted], kept positions of each
    plan slab as a list of arrays). A position is kept by the sink, the recent window, or its bin's bit of any head."""
    r = np.random.default_rng([case["mix"], 3])
    L, H, Hkv, D, W = (case[k] for k in ("L", "H", "Hkv", "D", "W"))
    G, n = H // Hkv, case["admitted"]
    ctx = r.integers(case["ctx_min"], case["ctx_max"] + 1, n)
    seq = np.sort(r.permutation(case["B"])[:n])
    M = (r.random((L, H, D)) < 1 - (1 - case["rate"]) ** (1 / G)).astype(np.uint8)
    U = M.reshape(L, Hkv, G, D).any(2)
    kept = []
    for l in range(L):
        for T in ctx:
            p = np.arange(T)
            window = (p < SINK) | (p >= T - RECENT)
            d = np.clip((T - RECENT - 1 - p) // W, 0, D - 1)
            kept += [np.nonzero(window | U[l, g][d])[0] for g in range(Hkv)]
    return M, ctx, seq, kept


def work(case):
    row = 2 * HEAD
    if case["op"] == "rope":
        n = case["T"] * case["heads"]
        return {"bytes": 2 * n * row + 4 * case["T"], "flops": 3 * n * case["rot"]}
    P, H, Hkv = case["page"], case["H"], case["Hkv"]
    if case["op"] == "compact":
        _, _, _, kept = _keep(case)
        rows = sum(len(k) for k in kept)
        return {"bytes": rows * (2 * row + 2 * (HEAD + 1) + 4) + sum(_pages_of(len(k), P) for k in kept) * 4, "flops": 0}
    ln, n = _lengths(case)[1], _tokens(case)
    T, live = int(n.sum()), n > 0
    after = ln + n[:, None]
    if case["op"] == "append":
        held = HEAD + 1 if case["bits"] == 8 else row
        pages = int((_pages_of(after, P) - ln // P)[live].sum())
        return {"bytes": T * (2 * H * row + 2 * Hkv * (row + held) + 4) + 4 * pages, "flops": 3 * T * (H + Hkv) * case["rot"]}
    rows = int(after[live].sum())
    if case["causal"]:
        pairs = int((ln * n[:, None] + (n * (n + 1) // 2)[:, None]).sum())
    else:
        pairs = int((after * n[:, None]).sum())
    pages = int(_pages_of(after[live], P).sum())
    return {"bytes": 2 * T * H * row + 2 * rows * (HEAD + 1) + 4 * pages, "flops": 4 * HEAD * pairs * (H // Hkv)}


# ------------------------------------------------------------ inputs

def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(DEV)


def _place(rows, page, spare, seed):
    """A pool whose pages lie in any order: (table int32 [slabs, widest], pages of the pool). `rows`: rows of every slab."""
    pages = _pages_of(rows.reshape(-1), page)
    total = int(pages.sum())
    order = np.random.default_rng([seed, 5]).permutation(total + spare).astype(np.int32)
    table = np.full((pages.size, max(int(pages.max(initial=0)), 1)), -1, np.int32)
    table[np.arange(table.shape[1])[None, :] < pages[:, None]] = order[:total]
    return table, total + spare


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dtype)


def _rows(n, dtype, gen):
    """n rows of a cache, some keys' outliers among them; made in parts to keep the 32-bit copy small."""
    out = torch.empty((n, HEAD), dtype=dtype, device=DEV)
    for i in range(0, n, 1 << 20):
        part = out[i:i + (1 << 20)]
        part.copy_(_randn(part.shape, dtype, gen))
    out[torch.rand(n, generator=gen, device=DEV) < 0.01] *= 4
    out[:, :2] *= 8  # dimensions that are larger than the others, as keys have them
    return out


def _frequencies(case):
    """(radians a position of every pair, float64; the factor on the values)."""
    rot, f, c = case["rot"], case["factor"], case["context"]
    theta = case["theta"] * f ** (rot / (rot - 2)) if case["scaling"] == "ntk" else case["theta"]
    w = theta ** (-2.0 * np.arange(rot // 2) / rot)
    if case["scaling"] == "linear":
        return w / f, 1.0
    if case["scaling"] == "bands":
        turns = c * w / (2 * np.pi)  # within the context
        keep = np.clip((turns - case["low"]) / (case["high"] - case["low"]), 0, 1)
        return w * (keep + (1 - keep) / f), 1.0
    if case["scaling"] == "yarn":
        at = [rot * math.log(c / (t * 2 * math.pi)) / (2 * math.log(theta)) for t in (case["high"], case["low"])]
        first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        keep = 1 - np.clip((np.arange(rot // 2) - first) / max(last - first, 1e-3), 0, 1)
        return w * (keep + (1 - keep) / f), 0.1 * math.log(f) + 1
    return w, 1.0


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op, dt = case["op"], DTYPES[case["dtype"]]
    s = {"case": case}
    if case.get("rot"):
        freq, s["magnitude"] = _frequencies(case)
        s["freq"] = torch.from_numpy(freq).to(DEV)
    if op == "rope":
        T, heads = case["T"], case["heads"]
        s["x"] = _randn((T, heads * (3 if case["fused"] else 1), HEAD), dt, gen)[:, :heads]
        s.update(positions=_dev(case["start"] + np.arange(T)), out=torch.zeros((T, heads, HEAD), dtype=dt, device=DEV))
    elif op == "compact":
        P, L, B, Hkv = (case[k] for k in ("page", "L", "B", "Hkv"))
        M, ctx, seq, kept = _keep(case)
        ln = np.zeros((L, B, Hkv), np.int64)
        ln[:, seq] = np.array([len(k) for k in kept]).reshape(L, len(seq), Hkv)
        table, pages = _place(ln, P, 9, seed)
        T = int(ctx.max())
        K, V = (_rows(L * len(seq) * Hkv * T, dt, gen).view(L, len(seq), Hkv, T, HEAD) for _ in range(2))
        s.update(table=_dev(table), len=_dev(ln.reshape(-1)), K=K, V=V, seq=_dev(seq), pages=pages, pattern=M, ctx=ctx,
                 kept=_dev(np.concatenate(kept), torch.int64), counts=_dev([len(k) for k in kept], torch.int64))
        _pools(case, s)
    else:
        P, B, H, Hkv = (case[k] for k in ("page", "B", "H", "Hkv"))
        ln, n = _lengths(case), _tokens(case)
        after = ln + n[None, :, None]
        table, pages = _place(after, P, 5, seed)
        T = int(n.sum()) + case["pad"]
        cu = np.concatenate([[0], np.cumsum(n)])
        heads = (H, Hkv, Hkv) if op == "append" else (H, Hkv)  # (the attention's q lies in its projection too)
        if case["fused"]:
            base = _randn((T, sum(heads), HEAD), dt, gen)
            x = base.split(heads, 1)
        else:
            x = [_randn((T, m, HEAD), dt, gen) for m in heads]
        s.update(table=_dev(table), len=_dev(after.reshape(-1)), cu=_dev(cu), q=x[0], pages=pages, cu_host=cu, len_host=after[1],
                 out=torch.zeros((T, H, HEAD), dtype=dt, device=DEV), most=int(n.max()))
        if op == "append":
            pos = np.concatenate([case["far"] + int(ln[:, b].max()) + np.arange(m) for b, m in enumerate(n)] + [np.zeros(case["pad"], np.int64)])
            s.update(k=x[1], v=x[2], positions=_dev(pos))
            _pools(case, s)
        else:
            s["Kp"], s["Ks"] = _quantised(_rows(pages * P, dt, gen))
            s["Vp"], s["Vs"] = _quantised(_randn((pages * P, HEAD), dt, gen))
    if own:
        _prepare_own(case, s)
    return s


def _pools(case, s):
    rows, wide = s["pages"] * case["page"], case.get("bits") == 16
    for name in ("Kp", "Vp"):
        s[name] = torch.zeros((rows, HEAD), dtype=DTYPES[case["dtype"]] if wide else torch.uint8, device=DEV)
        if not wide:
            s[name] = s[name].view(E4M3)
            s[name[0] + "s"] = torch.ones(rows, dtype=torch.uint8, device=DEV).view(E8M0)


def _prepare_own(case, s):
    from paper_2609_32663_gb300 import dkv
    if case.get("rot"):
        s["rotary"] = dkv.dkv_rotary_make(case["rot"], case["theta"], interleaved=case["inter"], scaling=case["scaling"],
                                          factor=case["factor"], context=case["context"], low=case["low"], high=case["high"])
    s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    if case["op"] == "rope":
        return
    s["geometry"] = dkv.Pages(L=case["L"], B=case["B"], H=case["H"], H_kv=case["Hkv"], page_rows=case["page"],
                              num_pages=s["pages"], max_pages=s["table"].shape[1])
    if case["op"] == "compact":
        shape = dkv.Shape(L=case["L"], H=case["H"], H_kv=case["Hkv"], D=case["D"], sink=SINK, recent=RECENT, bin_width=case["W"])
        s["plan"] = dkv.dkv_map_pattern(s["pattern"], s["ctx"], shape)
    if case["op"] == "attn":
        s["work"] = torch.empty(dkv.dkv_quant_workspace_bytes(s["geometry"]), dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------ one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return _own(op, s)
    return {"rope": _plain_rope, "append": _plain_append, "compact": _plain_compact, "attn": _plain_attn}[op](s)


def _own(op, s):
    from paper_2609_32663_gb300 import dkv
    if op == "rope":
        dkv.dkv_rope(s["x"], s["positions"], s["rotary"], s["out"])
        return s["out"]
    if op == "append":
        dkv.dkv_rope_append(s["geometry"], 1, s["q"], s["k"], s["v"], s["positions"], s["cu"], s["table"], s["len"], s["Kp"],
                            s["Vp"], s["out"], Ks=s.get("Ks"), Vs=s.get("Vs"), rotary=s.get("rotary"), status=s["status"])
        return _appended(s)
    if op == "compact":
        dkv.dkv_quant_compact(s["geometry"], s["plan"], s["K"], s["V"], s["table"], s["len"], s["Kp"], s["Vp"], s["Ks"], s["Vs"],
                              seq=s["seq"], status=s["status"])
        return s["Kp"], s["Vp"], s["Ks"], s["Vs"]
    dkv.dkv_quant_attn(s["geometry"], 1, s["q"], s["cu"], s["table"], s["len"], s["Kp"], s["Vp"], s["Ks"], s["Vs"], s["out"],
                       s["work"], causal=s["case"]["causal"], max_tokens=s["most"], status=s["status"])
    return s["out"]


def _appended(s):
    return (s["out"], s["Kp"], s["Vp"]) + ((s["Ks"], s["Vs"]) if "Ks" in s else ())


def _power(u):
    """2^(u - 127) in 32 bits."""
    return (u.int() << 23).view(torch.float32)


def _quantised(x):
    """(e4m3 values, scales as powers of two) of rows."""
    x = x.float()
    m, p = torch.frexp(x.abs().amax(-1))
    u = torch.clamp(p + 118 + (m > 0.875).int(), 1, 253)  # 448 = 0.875 2^9; 2^e is held as e + 127
    return (x * _power(254 - u)[..., None]).to(E4M3), u.to(torch.uint8).view(E8M0)


def _values(codes, scales):
    return codes.view(E4M3).float() * _power(scales)[..., None]


def _turned(s, x, positions):
    """Rows x [T, heads, 128] turned by their positions, in 32 bits."""
    c, x = s["case"], x.float()
    if not c["rot"]:
        return x
    angle = positions.double()[:, None] * s["freq"]
    cos, sin = ((f(angle) * s["magnitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    rot, half = c["rot"], c["rot"] // 2
    y = x.clone()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if c["inter"] else (slice(0, half), slice(half, rot))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _plain_rope(s):
    s["out"].copy_(_turned(s, s["x"], s["positions"]))
    return s["out"]


def _new_rows(s):
    """Pool rows [tokens, Hkv] of the step's tokens in layer 1."""
    c = s["case"]
    P, B, Hkv = (c[k] for k in ("page", "B", "Hkv"))
    cu = s["cu"].long()
    b = torch.repeat_interleave(torch.arange(B, device=DEV), cu.diff())
    h = (B + b)[:, None] * Hkv + torch.arange(Hkv, device=DEV)
    r = s["len"].long()[h] - (cu[b + 1] - torch.arange(b.numel(), device=DEV))[:, None]
    return s["table"][h, r // P].long() * P + r % P


def _plain_append(s):
    to, n = _new_rows(s), int(s["cu_host"][-1])
    s["out"][:n] = _turned(s, s["q"][:n], s["positions"][:n]).to(s["out"].dtype)
    k, v = _turned(s, s["k"][:n], s["positions"][:n]), s["v"][:n]
    if "Ks" not in s:
        s["Kp"][to], s["Vp"][to] = k.to(s["Kp"].dtype), v
        return _appended(s)
    for x, name in ((k, "K"), (v, "V")):
        codes, scales = _quantised(x)
        s[name + "p"].view(torch.uint8)[to] = codes.view(torch.uint8)
        s[name + "s"].view(torch.uint8)[to] = scales.view(torch.uint8)
    return _appended(s)


def _kept_rows(s):
    """(rows of the dense caches, pool rows) of the kept positions."""
    c = s["case"]
    P, B, Hkv = c["page"], c["B"], c["Hkv"]
    T, n, counts = s["K"].shape[3], s["seq"].numel(), s["counts"]
    i = torch.repeat_interleave(torch.arange(counts.numel(), device=DEV), counts)
    r = torch.arange(i.numel(), device=DEV) - (torch.cumsum(counts, 0) - counts)[i]
    l, j, g = i // (n * Hkv), i // Hkv % n, i % Hkv
    slab = (l * B + s["seq"].long()[j]) * Hkv + g
    r = r + s["len"].long()[slab] - counts[i]
    return i * T + s["kept"], s["table"][slab, r // P].long() * P + r % P


def _plain_compact(s):
    at, to = _kept_rows(s)
    for x, name in ((s["K"], "K"), (s["V"], "V")):
        codes, scales = _quantised(x.reshape(-1, HEAD)[at])
        s[name + "p"].view(torch.uint8)[to] = codes.view(torch.uint8)
        s[name + "s"].view(torch.uint8)[to] = scales.view(torch.uint8)
    return s["Kp"], s["Vp"], s["Ks"], s["Vs"]


def _plain_attn(s):
    c = s["case"]
    P, B, H, Hkv = (c[k] for k in ("page", "B", "H", "Hkv"))
    G, cu = H // Hkv, s["cu_host"]
    tf32 = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    Kp, Vp, Ks, Vs = (s[k].view(torch.uint8) for k in ("Kp", "Vp", "Ks", "Vs"))
    for b in range(B):
        t0, n = int(cu[b]), int(cu[b + 1] - cu[b])
        if n == 0:
            continue
        h = (B + b) * Hkv + torch.arange(Hkv, device=DEV)[:, None]
        m = s["len"].long()[h]
        r = torch.arange(int(s["len_host"][b].max()), device=DEV)
        at = s["table"][h, r.expand(Hkv, -1) // P].long().clamp(min=0) * P + r % P
        K, V = _values(Kp[at], Ks[at]), _values(Vp[at], Vs[at])
        step = max(1, (1 << 29) // (H * r.numel()))
        for i in range(0, n, step):
            q = s["q"][t0 + i:t0 + min(i + step, n)].unflatten(1, (Hkv, G)).transpose(0, 1).float()
            x = torch.matmul(q.flatten(1, 2), K.transpose(1, 2)).unflatten(1, q.shape[1:3]) * HEAD ** -0.5
            sees = m - n + i + 1 + torch.arange(q.shape[1], device=DEV) if c["causal"] else m.expand(-1, q.shape[1])
            x = torch.where(r < sees[:, :, None, None], x, -math.inf)
            w = torch.exp(x - x.amax(-1, keepdim=True))
            w = w / w.sum(-1, keepdim=True)
            o = torch.matmul(w.flatten(1, 2), V).unflatten(1, q.shape[1:3])
            s["out"][t0 + i:t0 + i + q.shape[1]] = o.transpose(0, 1).flatten(1, 2).to(s["out"].dtype)
    torch.backends.cuda.matmul.allow_tf32 = tf32
    return s["out"]


# ------------------------------------------------------------ from the definition, in 64 bits

def _turned_exactly(s, x, positions):
    """As complex numbers, in 64 bits."""
    c, x = s["case"], x.double()
    if not c["rot"]:
        return x
    head = x[..., :c["rot"]]
    pair = head.unflatten(-1, (-1, 2)) if c["inter"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
    z = torch.view_as_complex(pair.contiguous())
    p = positions.double()[:, None] * torch.from_numpy(_frequencies(c)[0]).to(DEV)
    z = torch.view_as_real(z * torch.polar(torch.full_like(p, s["magnitude"]), p)[:, None])
    return torch.cat([z.flatten(-2) if c["inter"] else z.transpose(-1, -2).flatten(-2), x[..., c["rot"]:]], -1)


def _held_exactly(x):
    """(e4m3 values, scales) of rows, as numbers in 64 bits."""
    x = x.double()
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True).clamp(min=448 * 2.0 ** -126) / 448)
    scale = _power64(e - (m == 0.5).int())  # the least power of two that is not below
    y = x / scale
    quantum = _power64(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)  # 4 significant bits
    return torch.round(y / quantum) * quantum, scale[..., 0]


def _power64(e):
    return (e.long() + 1023 << 52).view(torch.float64)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rope":
        return _turned_exactly(s, s["x"], s["positions"])
    if op == "attn":
        return _attended_exactly(case, s)
    pools = {name: s[name].double() for name in ("Kp", "Vp", "Ks", "Vs") if name in s}
    if op == "compact":
        at, to = _kept_rows(s)
        rows = [s[name].reshape(-1, HEAD)[at] for name in "KV"]
    else:
        to, n = _new_rows(s), int(s["cu_host"][-1])
        rows = [_turned_exactly(s, s["k"][:n], s["positions"][:n]), s["v"][:n].double()]
    for x, name in zip(rows, "KV"):
        if "Ks" in s:
            pools[name + "p"][to], pools[name + "s"][to] = _held_exactly(x)
        else:
            pools[name + "p"][to] = x
    if op == "compact":
        return tuple(pools.values())
    q = s["out"].double()
    q[:n] = _turned_exactly(s, s["q"][:n], s["positions"][:n])
    return (q, *pools.values())


def _attended_exactly(case, s):
    P, B, H, Hkv = (case[k] for k in ("page", "B", "H", "Hkv"))
    table = s["table"].cpu().numpy().astype(np.int64)
    K, V = (s[x + "p"].double() * s[x + "s"].double()[:, None] for x in "KV")
    out = s["out"].double()
    G, tokens = H // Hkv, np.diff(s["cu_host"])
    for b in range(B):
        n, t0 = int(tokens[b]), int(s["cu_host"][b])
        for g in range(Hkv):
            if n == 0:
                continue
            h, m = (B + b) * Hkv + g, int(s["len_host"][b, g])
            r = np.arange(m)
            at = torch.from_numpy(table[h][r // P] * P + r % P).to(DEV)
            for j in range(G):
                q = s["q"][t0:t0 + n, g * G + j].double()
                for i in range(0, n, 1024):
                    part = q[i:i + 1024]
                    z = (part @ K[at].t()).div_(math.sqrt(HEAD))
                    if case["causal"]:
                        z.masked_fill_(torch.ones(z.shape, dtype=torch.bool, device=DEV).triu(m - n + i + 1), -math.inf)
                    out[t0 + i:t0 + i + part.shape[0], g * G + j] = torch.softmax(z, -1) @ V[at]
    return out
