"""The paged cache's operators as a serving loop calls them, and their plain forms.

A case is a dict of plain values. Its "op" is the call:

  tables    dkv_page_tables: pages for a step's new tokens, the block tables, the slot map and the token offsets
  release   dkv_page_release: the pages of ended sequences go back to the free list
  compact   dkv_page_compact: the kept rows of pruned sequences into their pages
  chunk     dkv_chunk_attn: one layer's new tokens appended to the pages, and their attention

A slab is one (layer, sequence slot, KV head), h = (l B + b) Hkv + g; row r of slab h is row
table[h][r // P] P + r % P of the page pools (P rows a page). Lengths differ from slab to slab, as pruning leaves them.
Sizes come from the case alone ("mix" seeds them), values from the seed.
"""
import math

import numpy as np
import torch

own = False

HEAD = 128     # elements of a row
SINK, RECENT = 128, 1024
DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _chunk(name, H, Hkv, B, ctx, tokens, page, dtype="bf16", decode=0.0, causal=True, fused=True, pad=0, L=2, mix=1):
    """ctx and tokens: (least, most) of a sequence; decode: share of the sequences that bring one token; fused: q, k and
    v are slices of one projection; pad: rows of the batch behind the last sequence."""
    return {"name": name, "op": "chunk", "L": L, "H": H, "Hkv": Hkv, "B": B, "ctx_min": ctx[0], "ctx_max": ctx[1],
            "tok_min": tokens[0], "tok_max": tokens[1], "page": page, "dtype": dtype, "decode": decode, "causal": causal,
            "fused": fused, "pad": pad, "mix": mix}


def _tables(name, L, Hkv, B, ctx, tokens, page, pad=0, mix=1):
    return {"name": name, "op": "tables", "L": L, "Hkv": Hkv, "H": 4 * Hkv, "B": B, "ctx_min": ctx[0], "ctx_max": ctx[1],
            "tok_min": tokens[0], "tok_max": tokens[1], "decode": 0.0, "page": page, "pad": pad, "mix": mix}


def _release(name, L, Hkv, B, ctx, page, ended, mix=1):
    return {"name": name, "op": "release", "L": L, "Hkv": Hkv, "H": 4 * Hkv, "B": B, "ctx_min": ctx[0], "ctx_max": ctx[1],
            "page": page, "ended": ended, "mix": mix}


def _compact(name, L, H, Hkv, B, admitted, ctx, D, W, rate, page, dtype="bf16", mix=1):
    """admitted: pruned sequences, which go to slots of a pool of B."""
    return {"name": name, "op": "compact", "L": L, "H": H, "Hkv": Hkv, "B": B, "admitted": admitted, "ctx_min": ctx[0],
            "ctx_max": ctx[1], "D": D, "W": W, "rate": rate, "page": page, "dtype": dtype, "mix": mix}


def listed():
    return [
        # A decode step of 16 sequences on a 32-layer model: one page now and then. Latency.
        _tables("tables-step-b16", 32, 8, 16, (1500, 24000), (1, 1), 64, mix=3),
        # New turns of eight sequences at once; the slot map is the bulk of it.
        _tables("tables-turns-b8", 32, 8, 8, (0, 48000), (100, 4000), 16, pad=5, mix=4),
        # A few sequences of a 28-layer model end.
        _release("release-b16", 28, 4, 16, (100, 6000), 64, 0.2, mix=5),
        # Half of a large batch with long tables ends.
        _release("release-b64", 32, 8, 64, (2000, 60000), 16, 0.5, mix=6),
        # A 16K prompt of the 32-layer model admitted after pruning.
        _compact("compact-16k", 32, 32, 8, 4, 1, (16384, 16384), 32, 476, 0.35, 64, mix=7),
        # Three ragged prompts of the 28-layer model, small pages.
        _compact("compact-ragged", 28, 28, 4, 8, 3, (700, 9001), 64, 123, 0.25, 16, dtype="fp16", mix=8),
        # One sequence's next token over 4K context, pruned: launch latency and the ends of the pass.
        _chunk("token-4k", 32, 8, 1, (1800, 1800), (1, 1), 16, mix=9),
        # A decode step of 16 ragged sequences.
        _chunk("tokens-b16", 32, 8, 16, (3000, 24000), (1, 1), 64, mix=10),
        # Five drafted tokens or so a sequence, seven heads a group.
        _chunk("draft-b4-g7", 28, 4, 4, (2500, 30000), (3, 7), 32, dtype="fp16", fused=False, mix=11),
        # Questions over a cache that is not changed for them to see one another: every query sees every row.
        _chunk("queries-b2", 32, 8, 2, (5000, 13000), (200, 777), 128, causal=False, pad=3, mix=12),
        # A serving step: some sequences bring a new turn, the others their next token.
        _chunk("mixed-b12", 32, 8, 12, (0, 20000), (50, 2000), 64, decode=0.7, pad=9, mix=13),
        # A long new turn over a pruned 128K context.
        _chunk("turn-4k-over-45k", 32, 8, 1, (45300, 45300), (4096, 4096), 64, mix=14),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["tables", "release", "compact", "chunk", "chunk", "chunk"])
    H, Hkv = rng.choice([(32, 8), (28, 4), (32, 4), (16, 8), (8, 8), (24, 8)])
    page, mix = rng.choice([16, 32, 64, 128]), rng.randrange(1 << 30)
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if op == "tables":
        L, B = rng.randint(1, 40), _log(rng, 1, 64)
        most = max(1, min(4000, (1 << 22) // (L * Hkv * B)))
        tok = _log(rng, 1, most)
        return _tables(None, L, Hkv, B, (_log(rng, 1, 2000) - 1, _log(rng, 2000, 30000)),
                       (rng.randint(0, tok), tok), page, rng.randint(0, 9), mix)
    if op == "release":
        return _release(None, rng.randint(1, 40), Hkv, _log(rng, 1, 64), (_log(rng, 1, 2000) - 1, _log(rng, 2000, 30000)), page,
                        rng.uniform(0.1, 1.0), mix)
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
    return _chunk(None, H, Hkv, B, (rng.randint(0, top), top), tok, page, dtype, dec, rng.random() < 0.8, rng.random() < 0.6,
                  rng.randint(0, 9), rng.randint(1, 2), mix)


# ------------------------------------------------------------ sizes

def _lengths(case):
    """Rows of every slab before the call, int64 [L, B, Hkv]: of a context, pruning leaves each slab its own part."""
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
    P, L, B, Hkv = case["page"], case["L"], case["B"], case["Hkv"]
    if case["op"] == "tables":
        ln, n = _lengths(case), _tokens(case)
        after = ln + n[None, :, None]
        pages = int((_pages_of(after, P) - _pages_of(ln, P)).sum())
        partial = int(((ln % P != 0) & (after > ln)).sum())
        return {"bytes": 8 * ln.size + 8 * pages + 4 * partial + 4 * L * Hkv * int(n.sum()) + 8 * B, "flops": 0}
    if case["op"] == "release":
        ln = _lengths(case)
        ended = _ended(case)
        return {"bytes": 8 * ln.size + 8 * int(_pages_of(ln[:, ended], P).sum()) + 4 * B, "flops": 0}
    if case["op"] == "compact":
        _, _, _, kept = _keep(case)
        rows = sum(len(k) for k in kept)
        return {"bytes": rows * (2 * 2 * 2 * HEAD + 4) + sum(_pages_of(len(k), P) for k in kept) * 4, "flops": 0}
    ln, n = _lengths(case)[case["L"] - 1], _tokens(case)
    H, T = case["H"], int(n.sum())
    live = n > 0
    rows = int((ln + n[:, None])[live].sum())
    if case["causal"]:
        pairs = int((ln * n[:, None] + (n * (n + 1) // 2)[:, None]).sum())
    else:
        pairs = int(((ln + n[:, None]) * n[:, None]).sum())
    row = 2 * HEAD
    pages = int(_pages_of((ln + n[:, None])[live], P).sum())
    return {"bytes": 2 * T * H * row + 2 * rows * row + 2 * T * Hkv * row + 4 * pages, "flops": 4 * HEAD * pairs * (H // Hkv)}


def _ended(case):
    r = np.random.default_rng([case["mix"], 4])
    e = r.random(case["B"]) < case["ended"]
    e[r.integers(case["B"])] = True
    return e


# ------------------------------------------------------------ inputs

def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(DEV)


def _place(rows, page, spare, seed, slack=0):
    """A pool whose pages lie in any order: (table int32 [slabs, widest + slack], free list, free pages). `rows`: rows of
    every slab. The free list holds `spare` pages."""
    pages = _pages_of(rows.reshape(-1), page)
    total = int(pages.sum())
    order = np.random.default_rng([seed, 5]).permutation(total + spare).astype(np.int32)
    table = np.full((pages.size, max(int(pages.max(initial=0)) + slack, 1)), -1, np.int32)
    table[np.arange(table.shape[1])[None, :] < pages[:, None]] = order[:total]
    free = np.full(total + spare, -1, np.int32)
    free[:spare] = order[total:]
    return table, free, spare


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dtype)


def _rows(n, dtype, gen):
    """n rows of a cache, some keys' outliers among them; made in parts to keep the 32-bit copy small."""
    out = torch.empty((n, HEAD), dtype=dtype, device=DEV)
    for i in range(0, n, 1 << 20):
        part = out[i:i + (1 << 20)]
        part.copy_(_randn(part.shape, dtype, gen))
    out[torch.rand(n, generator=gen, device=DEV) < 0.01] *= 4
    return out


def prepare(case, seed):
    P, L, B, H, Hkv = (case[k] for k in ("page", "L", "B", "H", "Hkv"))
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case}
    op = case["op"]
    if op == "tables":
        ln, n = _lengths(case), _tokens(case)
        after = ln + n[None, :, None]
        need = int((_pages_of(after, P) - _pages_of(ln, P)).sum())
        table, free, count = _place(ln, P, need + 17, seed, int((_pages_of(after, P) - _pages_of(ln, P)).max()))
        cap = int(n.sum()) + case["pad"]
        s.update(table=_dev(table), free=_dev(free), free_count=_dev([count]), len=_dev(ln.reshape(-1)), tokens=_dev(n),
                 new_len=torch.zeros(ln.size, dtype=torch.int32, device=DEV),
                 new_count=torch.zeros(1, dtype=torch.int32, device=DEV),
                 cu=torch.zeros(B + 1, dtype=torch.int32, device=DEV),
                 slots=torch.full((L, max(cap, 1), Hkv), -1, dtype=torch.int32, device=DEV))
    elif op == "release":
        ln = _lengths(case)
        table, free, count = _place(ln, P, 33, seed)
        s.update(table=_dev(table), free=_dev(free), free_count=_dev([count]), len=_dev(ln.reshape(-1)), ended=_dev(_ended(case)),
                 new_len=torch.zeros(ln.size, dtype=torch.int32, device=DEV),
                 new_count=torch.zeros(1, dtype=torch.int32, device=DEV))
    elif op == "compact":
        dt = DTYPES[case["dtype"]]
        M, ctx, seq, kept = _keep(case)
        ln = np.zeros((L, B, Hkv), np.int64)
        ln[:, seq] = np.array([len(k) for k in kept]).reshape(L, len(seq), Hkv)
        table, free, _ = _place(ln, P, 9, seed)
        T = int(ctx.max())
        K, V = (_rows(L * len(seq) * Hkv * T, dt, gen).view(L, len(seq), Hkv, T, HEAD) for _ in range(2))
        Kp = torch.zeros((free.size * P, HEAD), dtype=dt, device=DEV)
        s.update(table=_dev(table), len=_dev(ln.reshape(-1)), K=K, V=V, Kp=Kp, Vp=torch.zeros_like(Kp), seq=_dev(seq),
                 slabs=[(l * B + int(b)) * Hkv + g for l in range(L) for b in seq for g in range(Hkv)])
        if own:
            s["plan"] = _plan(case, M, ctx)
        else:
            s["kept"] = _dev(np.concatenate(kept), torch.int64)
            s["counts"] = _dev([len(k) for k in kept], torch.int64)
    else:
        dt = DTYPES[case["dtype"]]
        ln, n = _lengths(case), _tokens(case)
        after = ln + n[None, :, None]
        table, free, _ = _place(after, P, 5, seed)
        T = int(n.sum()) + case["pad"]
        Kp = _rows(free.size * P, dt, gen)
        Vp = _randn(Kp.shape, dt, gen)
        if case["fused"]:
            qkv = _randn((T, H + 2 * Hkv, HEAD), dt, gen)
            q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        else:
            q, k, v = (_randn((T, m, HEAD), dt, gen) for m in (H, Hkv, Hkv))
        cu = np.concatenate([[0], np.cumsum(n)])
        s.update(table=_dev(table), len=_dev(after.reshape(-1)), cu=_dev(cu), q=q, k=k, v=v, Kp=Kp, Vp=Vp,
                 out=torch.zeros((T, H, HEAD), dtype=dt, device=DEV), cu_host=cu, len_host=after[L - 1])
    if own:
        _prepare_own(case, s)
    return s


def _geometry(case, s):
    from paper_2609_32663_gb300 import dkv
    pages = s["Kp"].shape[0] // case["page"] if "Kp" in s else s["free"].numel()
    return dkv.Pages(L=case["L"], B=case["B"], H=case["H"], H_kv=case["Hkv"], page_rows=case["page"], num_pages=pages,
                     max_pages=s["table"].shape[1])


def _prepare_own(case, s):
    from paper_2609_32663_gb300 import dkv
    s["pages"] = _geometry(case, s)
    s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    if case["op"] in ("tables", "release"):
        s["work"] = torch.empty(dkv.dkv_page_workspace_bytes(s["pages"]), dtype=torch.uint8, device=DEV)
    if case["op"] == "chunk":
        s["work"] = torch.empty(dkv.dkv_chunk_workspace_bytes(s["pages"]), dtype=torch.uint8, device=DEV)


def _plan(case, M, ctx):
    from paper_2609_32663_gb300 import dkv
    shape = dkv.Shape(L=case["L"], H=case["H"], H_kv=case["Hkv"], D=case["D"], sink=SINK, recent=RECENT, bin_width=case["W"])
    return dkv.dkv_map_pattern(M, ctx, shape)


# ------------------------------------------------------------ one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return _own(op, s)
    return {"tables": _plain_tables, "release": _plain_release, "compact": _plain_compact, "chunk": _plain_chunk}[op](s)


def _own(op, s):
    from paper_2609_32663_gb300 import dkv
    if op == "tables":
        dkv.dkv_page_tables(s["pages"], s["len"], s["new_len"], s["table"], s["free"], s["free_count"], s["new_count"], s["work"],
                            tokens=s["tokens"], cu_tokens=s["cu"], slots=s["slots"], status=s["status"])
        return s["table"], s["new_len"], s["new_count"], s["cu"], s["slots"]
    if op == "release":
        dkv.dkv_page_release(s["pages"], s["ended"], s["len"], s["new_len"], s["table"], s["free"], s["free_count"],
                             s["new_count"], s["work"], status=s["status"])
        return s["free"], s["new_len"], s["new_count"]
    if op == "compact":
        dkv.dkv_page_compact(s["pages"], s["plan"], s["K"], s["V"], s["table"], s["len"], s["Kp"], s["Vp"], seq=s["seq"],
                             status=s["status"])
        return s["Kp"], s["Vp"]
    dkv.dkv_chunk_attn(s["pages"], s["case"]["L"] - 1, s["q"], s["k"], s["v"], s["cu"], s["table"], s["len"], s["Kp"], s["Vp"],
                       s["out"], s["work"], causal=s["case"]["causal"], status=s["status"])
    return s["out"], s["Kp"], s["Vp"]


def _plain_tables(s):
    c = s["case"]
    P, L, B, Hkv = c["page"], c["L"], c["B"], c["Hkv"]
    ln = s["len"].long()
    n = s["tokens"].long().view(1, B, 1).expand(L, B, Hkv).reshape(-1)
    had, has = (ln + P - 1) // P, (ln + n + P - 1) // P
    need = has - had
    end = torch.cumsum(need, 0)
    slab = torch.repeat_interleave(torch.arange(ln.numel(), device=DEV), need)
    k = torch.arange(slab.numel(), device=DEV)
    count = s["free_count"].long()
    s["table"][slab, had[slab] + k - (end - need)[slab]] = s["free"][count - 1 - k]
    s["new_len"].copy_(ln + n)
    s["new_count"].copy_(count - end[-1:])
    s["cu"][0] = 0
    s["cu"][1:] = torch.cumsum(s["tokens"], 0)
    b = torch.repeat_interleave(torch.arange(B, device=DEV), s["tokens"].long())
    t = torch.arange(b.numel(), device=DEV)
    slab = (torch.arange(L, device=DEV).view(L, 1, 1) * B + b.view(1, -1, 1)) * Hkv + torch.arange(Hkv, device=DEV)
    r = ln[slab] + (t - s["cu"].long()[b]).view(1, -1, 1)
    s["slots"][:, :b.numel()] = (s["table"][slab, r // P].long() * P + r % P).int()
    return s["table"], s["new_len"], s["new_count"], s["cu"], s["slots"]


def _plain_release(s):
    c = s["case"]
    P, L, B, Hkv = c["page"], c["L"], c["B"], c["Hkv"]
    ln = s["len"].long()
    gone = (s["ended"] != 0).view(1, B, 1).expand(L, B, Hkv).reshape(-1)
    pages = torch.where(gone, (ln + P - 1) // P, 0)
    mine = torch.arange(s["table"].shape[1], device=DEV)[None, :] < pages[:, None]
    back = s["table"][mine]
    count = s["free_count"].long()
    s["free"][count + torch.arange(back.numel(), device=DEV)] = back
    s["new_len"].copy_(torch.where(gone, 0, ln))
    s["new_count"].copy_(count + back.numel())
    return s["free"], s["new_len"], s["new_count"]


def _plain_compact(s):
    c = s["case"]
    P, L, B, Hkv = c["page"], c["L"], c["B"], c["Hkv"]
    T, n = s["K"].shape[3], s["seq"].numel()
    counts = s["counts"]
    i = torch.repeat_interleave(torch.arange(counts.numel(), device=DEV), counts)
    r = torch.arange(i.numel(), device=DEV) - (torch.cumsum(counts, 0) - counts)[i]
    l, j, g = i // (n * Hkv), i // Hkv % n, i % Hkv
    slab = (l * B + s["seq"].long()[j]) * Hkv + g
    r = r + s["len"].long()[slab] - counts[i]
    to = s["table"][slab, r // P].long() * P + r % P
    at = i * T + s["kept"]
    s["Kp"][to] = s["K"].reshape(-1, HEAD)[at]
    s["Vp"][to] = s["V"].reshape(-1, HEAD)[at]
    return s["Kp"], s["Vp"]


def _plain_chunk(s):
    c = s["case"]
    P, L, B, H, Hkv = (c[k] for k in ("page", "L", "B", "H", "Hkv"))
    G, cu = H // Hkv, s["cu_host"]
    tf32 = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    for b in range(B):
        t0, n = int(cu[b]), int(cu[b + 1] - cu[b])
        if n == 0:
            continue
        h = ((L - 1) * B + b) * Hkv + torch.arange(Hkv, device=DEV)[:, None]
        m = s["len"].long()[h]

        def place(r):
            return s["table"][h, r // P].long().clamp(min=0) * P + r % P

        new = place(m - n + torch.arange(n, device=DEV))
        s["Kp"][new] = s["k"][t0:t0 + n].transpose(0, 1)
        s["Vp"][new] = s["v"][t0:t0 + n].transpose(0, 1)
        r = torch.arange(int(s["len_host"][b].max()), device=DEV)
        at = place(r.expand(Hkv, -1))
        K, V = s["Kp"][at].float(), s["Vp"][at].float()
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
    return s["out"], s["Kp"], s["Vp"]


# ------------------------------------------------------------ from the definition, in 64 bits

def exact(case, seed):
    if case["op"] in ("tables", "release"):
        return None  # whole numbers
    s = prepare(case, seed)
    P, L, B, H, Hkv = (case[k] for k in ("page", "L", "B", "H", "Hkv"))
    table = s["table"].cpu().numpy().astype(np.int64)

    def places(h, first, last):
        r = np.arange(first, last)
        return torch.from_numpy(table[h][r // P] * P + r % P).to(DEV)

    Kp, Vp = s["Kp"].double(), s["Vp"].double()
    if case["op"] == "compact":
        _, _, _, kept = _keep(case)
        n = s["seq"].numel()
        for i, h in enumerate(s["slabs"]):
            to, at = places(h, 0, len(kept[i])), torch.from_numpy(kept[i]).to(DEV)
            l, j, g = i // (n * Hkv), i // Hkv % n, i % Hkv
            Kp[to], Vp[to] = s["K"][l, j, g, at].double(), s["V"][l, j, g, at].double()
        return Kp, Vp
    out = s["out"].double()
    G, tokens = H // Hkv, np.diff(s["cu_host"])
    for b in range(B):
        n, t0 = int(tokens[b]), int(s["cu_host"][b])
        for g in range(Hkv):
            if n == 0:
                continue
            h, m = ((L - 1) * B + b) * Hkv + g, int(s["len_host"][b, g])
            at = places(h, 0, m)
            K = torch.cat([Kp[at[:m - n]], s["k"][t0:t0 + n, g].double()])
            V = torch.cat([Vp[at[:m - n]], s["v"][t0:t0 + n, g].double()])
            Kp[at[m - n:]], Vp[at[m - n:]] = K[m - n:], V[m - n:]
            for j in range(G):
                q = s["q"][t0:t0 + n, g * G + j].double()
                for i in range(0, n, 1024):
                    part = q[i:i + 1024]
                    z = (part @ K.t()).div_(math.sqrt(HEAD))
                    if case["causal"]:
                        z.masked_fill_(torch.ones(z.shape, dtype=torch.bool, device=DEV).triu(m - n + i + 1), -math.inf)
                    out[t0 + i:t0 + i + part.shape[0], g * G + j] = torch.softmax(z, -1) @ V
    return out, Kp, Vp
