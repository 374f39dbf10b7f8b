"""dkv_rope and dkv_rope_append against their definition in 64 bits: layouts, parts of the head, far and negative positions,
head counts, strides, in place, both types, 16-bit and 8-bit pages, and what lies in unused places."""
import numpy as np
import pytest
import torch

import paged
import quant
from paper_2609_32663_gb300 import dkv

pytestmark = pytest.mark.gpu
NAN = float("nan")
TYPES = [torch.bfloat16, torch.float16]


def dev(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x)).to(dtype).cuda()


def frequencies(rot, theta=10000.0):
    return theta ** (-2 * np.arange(rot // 2) / rot)


def randn(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [16, 48, 64, 112, 128])
def test_layouts(cuda, dtype, interleaved, rot):
    T, heads = 37, 3
    f = frequencies(rot)
    x = randn((T, heads, 128), dtype, rot)
    pos = np.random.default_rng(rot).integers(0, 200000, T)
    r = dkv.dkv_rotary_custom(f, interleaved=interleaved, magnitude=1.25)
    out = torch.full(x.shape, NAN, dtype=dtype, device="cuda")
    dkv.dkv_rope(x.cuda(), dev(pos), r, out)
    want, size = quant.turned(x, pos, f, interleaved, 1.25)
    quant.assert_turned(out, want, size, dtype)
    assert torch.equal(out[..., rot:].cpu(), x[..., rot:])  # what is not turned keeps its bits


@pytest.mark.parametrize("T,heads", [(1, 1), (1, 41), (5, 32), (3, 33), (2431, 1), (2432, 9), (5001, 2)])
def test_sizes(cuda, T, heads):
    x = randn((T, heads, 128), torch.float16, T)
    f = frequencies(128, 5e5)
    pos = np.arange(T) + 77777
    out = torch.full(x.shape, NAN, dtype=x.dtype, device="cuda")
    dkv.dkv_rope(x.cuda(), dev(pos), dkv.dkv_rotary_make(128, 5e5), out)
    want, size = quant.turned(x, pos, f, False)
    quant.assert_turned(out, want, size, x.dtype)


def test_far_and_negative_positions(cuda):
    """The angle is exact at every 32-bit position, also where the frequency is above one."""
    pos = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1 << 24, (1 << 24) + 1, 999_999_937, -123456789])
    f = np.array([1.0, 1e-3, 3.14159265, 6.2831853, 0.7071, 1e-9, 1e5, 0.0])
    x = randn((len(pos), 2, 128), torch.float16, 1)
    out = torch.full(x.shape, NAN, dtype=x.dtype, device="cuda")
    dkv.dkv_rope(x.cuda(), dev(pos), dkv.dkv_rotary_custom(f, interleaved=True), out)
    want, size = quant.turned(x, pos, f, True)
    quant.assert_turned(out, want, size, x.dtype)


def test_strided_and_in_place(cuda):
    """A slice of a projection turned in place: the other slices, and the same rows elsewhere, keep their bits."""
    T, f = 300, frequencies(64)
    x = randn((T, 12, 128), torch.bfloat16, 3)
    pos = np.arange(T)
    d, r = x.cuda(), dkv.dkv_rotary_make(64)
    dkv.dkv_rope(d[:, 4:9], dev(pos), r, d[:, 4:9])
    want, size = quant.turned(x[:, 4:9], pos, f, False)
    quant.assert_turned(d[:, 4:9], want, size, x.dtype)
    assert torch.equal(d[:, :4].cpu(), x[:, :4]) and torch.equal(d[:, 9:].cpu(), x[:, 9:])
    wide = torch.full((T, 9, 128), NAN, dtype=x.dtype, device="cuda")
    dkv.dkv_rope(x.cuda()[:, 4:9], dev(pos), r, wide[:, 2:7])
    assert torch.equal(wide[:, 2:7], d[:, 4:9]) and torch.isnan(wide[:, [0, 1, 7, 8]].float()).all()


def test_values_that_are_not_finite_stay_in_their_pair(cuda):
    x = randn((4, 2, 128), torch.bfloat16, 4)
    clean = x.clone()
    x[1, 0, 5], x[2, 1, 100], x[3, 0, 127] = NAN, float("inf"), -float("inf")
    pos, r = dev(np.arange(4)), dkv.dkv_rotary_make(96)
    out, ref = (torch.empty(x.shape, dtype=x.dtype, device="cuda") for _ in range(2))
    dkv.dkv_rope(x.cuda(), pos, r, out)
    dkv.dkv_rope(clean.cuda(), pos, r, ref)
    bad = torch.zeros(x.shape, dtype=torch.bool)
    bad[1, 0, 5] = bad[1, 0, 53] = bad[2, 1, 100] = bad[3, 0, 127] = True
    assert torch.isnan(out[1, 0, [5, 53]].float()).all()
    assert out[2, 1, 100] == float("inf") and out[3, 0, 127] == -float("inf")
    assert torch.equal(out.cpu()[~bad], ref.cpu()[~bad])


def test_calls_on_other_streams_and_devices_buffers(cuda):
    x, pos, r = randn((64, 4, 128), torch.bfloat16, 5), np.arange(64), dkv.dkv_rotary_make()
    d, p = x.cuda(), dev(pos)
    out = torch.empty_like(d)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    dkv.dkv_rope(d, p, r, out, stream=s)
    with torch.cuda.stream(s):
        again = torch.empty_like(d)
        dkv.dkv_rope(d, p, r, again)
    s.synchronize()
    assert torch.equal(out, again)
    with pytest.raises(dkv.DkvError):
        dkv.dkv_rope(d, torch.arange(64, dtype=torch.int32), r, out)
    with pytest.raises(dkv.DkvError, match="positions"):
        dkv.dkv_rope(d, dev(np.arange(63)), r, out)


def test_captured_with_new_positions(cuda):
    """A graph keeps the rotary that it was captured with, and reads positions when it runs."""
    x, f = randn((40, 2, 128), torch.float16, 6), frequencies(128)
    d, p, out, r = x.cuda(), dev(np.arange(40)), torch.empty(x.shape, dtype=x.dtype, device="cuda"), dkv.dkv_rotary_make()
    dkv.dkv_rope(d, p, r, out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dkv.dkv_rope(d, p, r, out)
    for i in range(64):
        r.c.turns[i] = 0
    for start in (0, 5000):
        p.copy_(dev(np.arange(40) + start))
        g.replay()
        torch.cuda.synchronize()
        want, size = quant.turned(x, np.arange(40) + start, f, False)
        quant.assert_turned(out, want, size, x.dtype)


# ------------------------------------------------------------ append

class Append:
    """A call's buffers. Pools hold what no row is written with: NaN codes (or NaN), scale bytes 255."""

    def __init__(self, lens, page, tokens, dtype=torch.bfloat16, H=None, bits=8, rot=64, interleaved=False, seed=0, pad=0, fused=True):
        self.c = c = paged.Cache(lens, page, dtype=dtype, seed=seed, H=H)
        self.tokens, self.bits, self.interleaved, self.dtype = tokens, bits, interleaved, dtype
        self.f = frequencies(rot) if rot else None
        self.rotary = dkv.dkv_rotary_custom(self.f, interleaved=interleaved, magnitude=1.1) if rot else None
        T = sum(tokens) + pad
        self.pos = np.random.default_rng(seed).integers(0, 1 << 20, T)
        x = randn((T, c.H + 2 * c.Hkv, 128), dtype, seed)
        x[::3] *= 37
        x[1::5, -1] = 0  # rows of V that are all zero
        self.host = [x[:, :c.H], x[:, c.H:c.H + c.Hkv], x[:, c.H + c.Hkv:]]
        d = x.cuda()
        self.q, self.k, self.v = ([d[:, :c.H], d[:, c.H:c.H + c.Hkv], d[:, c.H + c.Hkv:]] if fused else
                                  [y.contiguous().cuda() for y in self.host])
        self.cu_host = np.concatenate([[0], np.cumsum(tokens)])
        self.cu, self.table, self.len, self.positions = dev(self.cu_host), dev(c.table), dev(c.lens), dev(self.pos)
        rows = c.pages.num_pages * page
        if bits == 8:
            self.pools = [torch.full((rows, 128), 0x7f, dtype=torch.uint8, device="cuda") for _ in "KV"]
            self.scales = [torch.full((rows,), 255, dtype=torch.uint8, device="cuda") for _ in "KV"]
        else:
            self.pools, self.scales = [torch.full((rows, 128), NAN, dtype=dtype, device="cuda") for _ in "KV"], [None, None]
        self.out = torch.full((T, c.H, 128), NAN, dtype=dtype, device="cuda")
        self.status = dev([0])

    def run(self, layer, **kw):
        dkv.dkv_rope_append(self.c.pages, layer, self.q, self.k, self.v, self.positions, self.cu, self.table, self.len, *self.pools,
                            self.out, *self.scales, rotary=self.rotary, status=self.status, **kw)
        torch.cuda.synchronize()
        return self

    def turned(self, i):
        x = self.host[i]
        if self.f is None or i == 2:
            return x.double(), torch.zeros_like(x, dtype=torch.float64)
        return quant.turned(x, self.pos, self.f, self.interleaved, 1.1)

    def places(self, layer, skip=()):
        """(token, head, pool row) of every new row."""
        c, at = self.c, []
        for b in range(c.B):
            n, t0 = int(self.tokens[b]), int(self.cu_host[b])
            for g in range(c.Hkv):
                h = (layer * c.B + b) * c.Hkv + g
                m = int(c.lens[h])
                at += [(t0 + i, g, int(c.rows(h, m - n + i, m - n + i + 1)[0])) for i in range(n) if m - n + i >= 0 and b not in skip]
        return at

    def check(self, layer, skip=()):
        n, dtype = int(self.cu_host[-1]), self.dtype
        want, size = self.turned(0)
        if self.q is not None:
            quant.assert_turned(self.out[:n], want[:n], size[:n], dtype, "q")
            assert torch.isnan(self.out[n:].float()).all()
        at = self.places(layer, skip)
        t, g, rows = (np.array([x[i] for x in at], np.int64) for i in range(3))
        for i in (1, 2):
            x, size = (y[t, g] for y in self.turned(i))
            pool = self.pools[i - 1].cpu()
            others = np.setdiff1d(np.arange(pool.shape[0]), rows)
            if self.bits == 16:
                quant.assert_turned(pool[rows], x, size, dtype, "pool")
                assert torch.isnan(pool[others].float()).all()
                continue
            scales = self.scales[i - 1].cpu()
            assert (pool[others] == 0x7f).all() and (scales[others] == 255).all()
            if i == 2 or self.f is None:  # bits: the row as it was given
                codes, u = quant.held(x)
                assert np.array_equal(scales[rows].numpy(), u) and np.array_equal(pool[rows].numpy(), codes)
                continue
            # A turned row: its largest element is known to 2^-21 of its pair, and so is its scale, unless that lies on a border.
            off = 2.0 ** -21 * size
            least = quant.scale_bytes((x.abs() - off).clamp(min=0).numpy())
            most = quant.scale_bytes((x.abs() + off).numpy())
            u = scales[rows].numpy()
            assert ((u == least) | (u == most)).all()
            scale = torch.exp2(torch.from_numpy(u).double() - 127)[:, None]
            err = (quant.values(pool[rows].numpy(), u) - x).abs()
            assert (err <= torch.maximum(2.0 ** -4 * (x.abs() + off), 2.0 ** -10 * scale) + off).all()


def lens_of(L, B, Hkv, ctx, tokens, seed):
    less = np.random.default_rng(seed).integers(0, 6, (L, B, Hkv))
    return np.maximum(np.asarray(ctx)[None, :, None] - less, 0) + np.asarray(tokens)[None, :, None]


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("ctx,tokens,pad", [([0], [1], 0), ([15], [1], 0), ([16, 300, 0], [1, 0, 2], 3), ([100, 3, 0, 127], [40, 1, 129, 0], 1)])
def test_append(cuda, bits, page, ctx, tokens, pad):
    a = Append(lens_of(2, len(ctx), 2, ctx, tokens, page), page, tokens, H=8, bits=bits, pad=pad, seed=page)
    a.run(1).check(1)
    assert int(a.status) == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rot,interleaved", [(0, False), (128, False), (128, True), (32, True), (96, False)])
@pytest.mark.parametrize("G,Hkv,fused", [(1, 5, True), (7, 3, False)])
def test_append_layouts(cuda, dtype, rot, interleaved, G, Hkv, fused):
    for bits in (8, 16):
        tokens = [3, 0, 17]
        a = Append(lens_of(1, 3, Hkv, [33, 5, 100], tokens, rot), 16, tokens, dtype, G * Hkv, bits, rot, interleaved, rot, 2, fused)
        a.run(0).check(0)
        assert int(a.status) == 0


def test_many_tokens(cuda):
    tokens = [2500, 1, 900]
    a = Append(lens_of(1, 3, 1, [10, 700, 0], tokens, 1), 64, tokens, H=2, rot=128)
    a.run(0).check(0)


def test_q_in_place_q_alone_and_rows_alone(cuda):
    tokens = [4, 9]
    a = Append(lens_of(1, 2, 2, [20, 0], tokens, 2), 16, tokens, H=4, pad=1)
    untouched = a.q[13:].clone()
    a.out = a.q
    dkv.dkv_rope_append(a.c.pages, 0, a.q, None, None, a.positions, a.cu, a.table, a.len, None, None, a.q, rotary=a.rotary,
                        status=a.status)
    want, size = a.turned(0)
    quant.assert_turned(a.q[:13], want[:13], size[:13], a.dtype)
    assert torch.equal(a.q[13:], untouched)
    assert all((p == 0x7f).all() for p in a.pools)
    assert torch.equal(a.k.cpu(), a.host[1]) and torch.equal(a.v.cpu(), a.host[2])
    a.q = a.out = None
    a.run(0).check(0)
    assert int(a.status) == 0


def test_values_that_are_not_finite_are_held_as_nan(cuda):
    """An infinity, a NaN and the type's largest and smallest values in 8 bits; the scale goes by what is finite."""
    for dtype in TYPES:
        tokens = [6]
        a = Append(np.array([[[6]]]), 16, tokens, dtype, H=1, rot=0)
        v = a.host[2]
        v[0, 0, 3], v[1, 0, 4], v[2, 0, 5] = NAN, float("inf"), -float("inf")
        v[3, 0, 6], v[3, 0, 7] = torch.finfo(dtype).max, torch.finfo(dtype).min
        v[4] = torch.finfo(dtype).smallest_normal
        v[5] = torch.finfo(dtype).smallest_normal / 2
        a.v.copy_(v)
        a.run(0).check(0)


@pytest.mark.parametrize("bits", [8, 16])
def test_bad_pages_and_lengths_are_reported(cuda, bits):
    """They are not followed; other sequences' rows are written."""
    for kind in ("page", "negative", "long", "short"):
        tokens = [2, 3, 2]
        a = Append(lens_of(1, 3, 1, [40, 50, 60], tokens, 1), 16, tokens, H=4, bits=bits)
        if kind == "page":
            a.table[1] = 1 << 30
        elif kind == "negative":
            a.table[1] = -5
        else:
            a.len[1] = 1 << 30 if kind == "long" else 0
        a.run(0).check(0, skip=(1,))
        assert int(a.status) == dkv.DKV_DEV_PAGE_RANGE, kind


def test_bad_offsets_write_nothing(cuda):
    tokens = [2, 3, 2]
    for cu in ([1, 2, 5, 7], [0, 3, 2, 7], [0, 2, 5, 8], [0, -1, 5, 7], [0, 2, 5, 1 << 30]):
        a = Append(lens_of(1, 3, 1, [40, 50, 60], tokens, 1), 16, tokens, H=4)
        a.cu.copy_(dev(cu))
        a.run(0)
        assert int(a.status) == dkv.DKV_DEV_PAGE_RANGE
        assert torch.isnan(a.out.float()).all() and all((p == 0x7f).all() for p in a.pools) and all((s == 255).all() for s in a.scales)


@pytest.mark.parametrize("H,Hkv,tokens", [(100, 100, [3, 1]), (64, 8, [700, 0, 5]), (8, 1, [1]), (3, 3, [2500, 1])])
def test_many_and_few_heads(cuda, H, Hkv, tokens):
    """Tokens cut into several items, and whole."""
    for bits in (8, 16):
        a = Append(lens_of(1, len(tokens), Hkv, [20] * len(tokens), tokens, H), 32, tokens, H=H, bits=bits, rot=128, pad=1, seed=H)
        a.run(0).check(0)
        assert int(a.status) == 0


def test_no_token_at_all(cuda):
    a = Append(lens_of(1, 2, 1, [20, 0], [0, 0], 1), 16, [0, 0], H=2, pad=40)
    a.run(0)
    assert int(a.status) == 0 and torch.isnan(a.out.float()).all() and all((p == 0x7f).all() for p in a.pools)


def test_two_streams_at_once(cuda):
    calls = [(Append(lens_of(1, 2, 2, [200, 10], [5 + 600 * i, 1], i), 16, [5 + 600 * i, 1], H=8, seed=i), torch.cuda.Stream()) for i in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for a, s in calls:
            dkv.dkv_rope_append(a.c.pages, 0, a.q, a.k, a.v, a.positions, a.cu, a.table, a.len, *a.pools, a.out, *a.scales, rotary=a.rotary,
                                status=a.status, stream=s)
    torch.cuda.synchronize()
    for a, _ in calls:
        a.check(0)
        assert int(a.status) == 0


def test_captured_append(cuda):
    """A graph reads offsets, lengths, tables and positions when it runs; rows behind fewer tokens stay."""
    a = Append(lens_of(1, 2, 1, [20, 9], [4, 30], 1), 16, [4, 30], H=2)
    a.run(0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dkv.dkv_rope_append(a.c.pages, 0, a.q, a.k, a.v, a.positions, a.cu, a.table, a.len, *a.pools, a.out, *a.scales, rotary=a.rotary,
                            status=a.status)
    for x, v in ((a.out, NAN), (a.pools[0], 0x7f), (a.pools[1], 0x7f), (a.scales[0], 255), (a.scales[1], 255)):
        x.fill_(v)
    a.pos = a.pos[::-1].copy() + 5
    a.positions.copy_(dev(a.pos))
    g.replay()
    torch.cuda.synchronize()
    a.check(0)
    a.out.fill_(NAN)
    a.cu.copy_(dev([0, 4, 4]))
    a.len.copy_(dev(np.array([a.c.lens[0], a.c.lens[1] - 30])))
    g.replay()
    torch.cuda.synchronize()
    assert int(a.status) == 0 and torch.isfinite(a.out[:4].float()).all() and torch.isnan(a.out[4:].float()).all()


def test_pool_places_past_32_bits(cuda):
    """8-bit pools of more than 4 GB: pages at their end."""
    page, num, tokens = 128, 340_000, [3, 70]
    a = Append(lens_of(1, 2, 1, [300, 100], tokens, 1), page, tokens, H=2)
    small = a.c.pages.num_pages
    wide = [torch.full((num * page, *x.shape[1:]), int(x.flatten()[0]), dtype=torch.uint8, device="cuda") for x in a.pools + a.scales]
    table = torch.where(a.table < small, a.table + (num - small), a.table)
    g = dkv.Pages(L=1, B=2, H=2, H_kv=1, page_rows=page, num_pages=num, max_pages=a.table.shape[1])
    dkv.dkv_rope_append(g, 0, a.q, a.k, a.v, a.positions, a.cu, table, a.len, *wide[:2], a.out, *wide[2:], rotary=a.rotary, status=a.status)
    torch.cuda.synchronize()
    a.pools, a.scales = [x[-small * page:] for x in wide[:2]], [x[-small * page:] for x in wide[2:]]
    a.check(0)
    assert int(a.status) == 0 and all((x[:1 << 20] == x[0]).all() for x in wide[:2])


def test_more_sequences_than_threads(cuda):
    tokens = [b % 3 for b in range(512)]
    a = Append(lens_of(1, 512, 1, [b % 40 for b in range(512)], tokens, 1), 16, tokens, H=2)
    a.run(0).check(0)
    assert int(a.status) == 0


def test_an_injected_launch_failure_is_told(cuda, monkeypatch):
    a = Append(np.array([[[3]]]), 16, [3], H=1)
    monkeypatch.setenv("DKV_FAULT", "launch")
    with pytest.raises(dkv.DkvError, match="injected") as e:
        a.run(0)
    assert e.value.status == dkv.DKV_ERR_CUDA
