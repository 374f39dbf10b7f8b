"""dkv_chunk_attn against its definition in 64 bits: token counts around the tiles, ragged and empty sequences, every
group size and page size, both types, strided inputs, and what lies in masked and unused places."""
import numpy as np
import pytest
import torch

import paged
from paper_2609_32663_gb300 import dkv

pytestmark = pytest.mark.gpu
NAN = float("nan")


def inputs(cache, tokens, seed, pad=0, fused=True):
    T = int(sum(tokens)) + pad
    gen = torch.Generator().manual_seed(seed)
    qkv = torch.randn((T, cache.H + 2 * cache.Hkv, paged.HEAD), generator=gen).to(cache.dtype)
    cu = np.concatenate([[0], np.cumsum(tokens)]).astype(np.int32)
    parts = [qkv[:, :cache.H], qkv[:, cache.H:cache.H + cache.Hkv], qkv[:, cache.H + cache.Hkv:]]
    return cu, (parts if fused else [x.contiguous() for x in parts])


class Call:
    """The call's buffers on the GPU; inputs that are slices of one projection stay slices."""

    def __init__(self, cache, layer, qkv, cu, causal=True, append=True, scale=0.0, dev="cuda"):
        self.cache, self.layer, self.causal, self.scale = cache, layer, causal, scale
        base = qkv[0]._base
        if base is not None and all(x._base is base for x in qkv):
            d, H, Hk = base.to(dev), cache.H, cache.Hkv
            self.q, k, v = d[:, :H], d[:, H:H + Hk], d[:, H + Hk:]
        else:
            self.q, k, v = (x.to(dev) for x in qkv)
        self.k, self.v = (k, v) if append else (None, None)
        self.Kp, self.Vp = cache.Kp.to(dev), cache.Vp.to(dev)
        self.table = torch.from_numpy(cache.table).to(dev)
        self.len = torch.from_numpy(cache.lens.astype(np.int32)).to(dev)
        self.cu = torch.from_numpy(np.asarray(cu, np.int32)).to(dev)
        self.out = torch.full((self.q.shape[0], cache.H, paged.HEAD), NAN, dtype=cache.dtype, device=dev)
        self.work = torch.full((dkv.dkv_chunk_workspace_bytes(cache.pages),), 0xa5, dtype=torch.uint8, device=dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)

    def run(self, **kw):
        dkv.dkv_chunk_attn(self.cache.pages, self.layer, self.q, self.k, self.v, self.cu, self.table, self.len, self.Kp,
                           self.Vp, self.out, self.work, causal=self.causal, scale=self.scale, status=self.status, **kw)
        return self


def check(cache, layer, tokens, causal=True, append=True, pad=0, fused=True, seed=1, scale=0.0):
    cu, qkv = inputs(cache, tokens, seed, pad, fused)
    c = Call(cache, layer, qkv, cu, causal, append, scale).run()
    torch.cuda.synchronize()
    want, size, Kp, Vp = paged.attention(cache, layer, qkv[0], qkv[1] if append else None, qkv[2] if append else None, cu,
                                         causal, scale or None)
    assert int(c.status) == 0
    paged.assert_attention(c.out, want, size, cache.dtype, f"tokens {tokens}")
    for got, exp in ((c.Kp, Kp), (c.Vp, Vp)):
        assert torch.equal(torch.nan_to_num(got.double().cpu(), 99.0), torch.nan_to_num(exp, 99.0)), "pools differ"


def lens_of(L, B, Hkv, ctx, tokens, seed):
    """Lengths after the tokens' append: a context of ctx[b] rows, less some for every slab but the first."""
    r = np.random.default_rng(seed)
    less = r.integers(0, 6, (L, B, Hkv))
    less[0, :, 0] = 0
    return np.maximum(np.asarray(ctx)[None, :, None] - less, 0) + np.asarray(tokens)[None, :, None]


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("ctx,tokens", [
    ([0], [1]), ([1], [1]), ([126], [1]), ([127], [1]), ([128], [1]), ([1000], [1]),
    ([300, 0, 5, 700], [1, 1, 1, 1]),
    ([250, 130, 0, 513], [3, 0, 17, 2]),
    ([0], [33]), ([90], [65]), ([0, 400], [129, 40]),
    ([40, 1200, 3], [31, 1, 150]),
])
def test_lengths_and_pages(cuda, page, ctx, tokens):
    lens = lens_of(2, len(ctx), 2, ctx, tokens, page)
    check(paged.Cache(lens, page, H=8, seed=page), 1, tokens)


@pytest.mark.parametrize("G,Hkv", [(1, 3), (2, 2), (3, 1), (4, 1), (5, 2), (6, 1), (7, 2), (8, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_group_sizes(cuda, G, Hkv, dtype):
    tokens = [1, 128 // G + 1, 3, 2 * (128 // G) + 1]
    lens = lens_of(1, 4, Hkv, [333, 60, 0, 129], tokens, G)
    check(paged.Cache(lens, 32, H=G * Hkv, seed=G, dtype=dtype), 0, tokens, fused=bool(G & 1))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("pad", [0, 5])
def test_masks_and_padding(cuda, causal, append, pad):
    tokens = [5, 1, 70, 0]
    lens = lens_of(2, 4, 2, [200, 129, 64, 10], tokens, 3)
    check(paged.Cache(lens, 64, H=8), 0, tokens, causal=causal, append=append, pad=pad)


def test_scale(cuda):
    check(paged.Cache(lens_of(1, 2, 1, [100, 300], [2, 40], 1), 16, H=4), 0, [2, 40], scale=0.03)


def test_slab_shorter_than_its_tokens(cuda):
    """Rows are in the pools already and a slab holds fewer than there are queries: the first queries see no row."""
    cache = paged.Cache(np.array([[[3, 0], [40, 1]]]), 16, H=8)
    check(cache, 0, [5, 41], append=False)
    check(cache, 0, [5, 41], append=False, causal=False)


@pytest.mark.parametrize("n,ctx", [(40, 100), (1, 300), (200, 0)])
def test_long_and_many(cuda, n, ctx):
    """More sequences than CTAs."""
    B = 90 if n == 1 else 5
    tokens = [n] * B
    check(paged.Cache(lens_of(1, B, 2, [ctx] * B, tokens, 4), 16, H=4), 0, tokens)


def test_later_tokens_hold_anything(cuda):
    """Infinities, NaN and the type's lowest value in K and V of a later token change no earlier token's output."""
    for dtype in (torch.bfloat16, torch.float16):
        tokens = [70, 4]
        cache = paged.Cache(lens_of(1, 2, 2, [90, 128], tokens, 5), 16, H=8, dtype=dtype)
        cu, qkv = inputs(cache, tokens, 2)
        q, k, v = (x.clone() for x in qkv)
        k[50, 0], v[50, 0, 3] = NAN, NAN
        v[60, 1] = float("inf")
        k[61, 1] = torch.finfo(dtype).min
        v[73, :, 7], k[73, 1, 0] = -float("inf"), float("inf")
        c = Call(cache, 0, (q, k, v), cu).run()
        want, size, _, _ = paged.attention(cache, 0, q, k, v, cu, True)
        got = c.out.double().cpu()
        first = [(slice(0, 50), slice(0, 8)), (slice(50, 60), slice(4, 8)), (slice(70, 73), slice(0, 8))]
        for t, h in first:
            paged.assert_attention(got[t, h], want[t, h], size[t, h], dtype, str((t, h)))
        # From the NaN key on, its heads are NaN; a NaN or infinity of V stays in its dimension.
        assert torch.isnan(got[50:70, :4]).all()
        assert torch.isinf(got[60:61, 4:]).all()
        assert (got[73, :4, 7] == -float("inf")).all() and torch.isfinite(got[73, :4, :7]).all()


def test_bad_page_numbers_and_lengths_are_reported(cuda):
    """Out-of-range page numbers and lengths on the device are not followed; other sequences keep their results."""
    tokens = [2, 3, 2]
    cache = paged.Cache(lens_of(1, 3, 1, [40, 50, 60], tokens, 1), 16, H=4)
    cu, qkv = inputs(cache, tokens, 3)
    want, size, _, _ = paged.attention(cache, 0, *qkv, cu, True)
    for kind in ("page", "negative", "long"):
        c = Call(cache, 0, qkv, cu)
        if kind == "page":
            c.table[1, :4] = 1 << 30
        elif kind == "negative":
            c.table[1, :4] = -5
        else:
            c.len[1] = 1 << 30
        c.run()
        assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE
        for t in (slice(0, 2), slice(5, 7)):
            paged.assert_attention(c.out[t], want[t], size[t], cache.dtype, kind)


def test_repeats_are_bit_exact(cuda):
    tokens = [1, 200, 1, 7]
    cache = paged.Cache(lens_of(1, 4, 2, [4000, 900, 30, 2500], tokens, 1), 64, H=8)
    cu, qkv = inputs(cache, tokens, 3)
    c = Call(cache, 0, qkv, cu).run()
    first = c.out.clone()
    for _ in range(5):
        c.out.fill_(NAN)
        c.work.fill_(0xff)
        c.run()
        assert torch.equal(c.out, first)


def test_captured_and_replayed(cuda):
    """A captured call reads token counts, lengths and tables at replay; two graphs of one workspace replay in turn."""
    cases, graphs = [], []
    stream = torch.cuda.Stream()
    for i, tokens in enumerate(([1, 1], [1, 60])):
        cache = paged.Cache(lens_of(1, 2, 2, [700, 90 + i], tokens, i), 32, H=8, seed=i)
        cu, qkv = inputs(cache, tokens, i)
        c = Call(cache, 0, qkv, cu)
        c.work = cases[0][0].work if cases else c.work
        cases.append((c, paged.attention(cache, 0, *qkv, cu, True)))
        c.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            c.run()
        graphs.append(g)
    for _ in range(3):
        for g, (c, (want, size, _, _)) in zip(graphs, cases):
            c.out.fill_(NAN)
            g.replay()
            torch.cuda.synchronize()
            paged.assert_attention(c.out, want, size, c.cache.dtype)
    # The same graph after the step's tokens became fewer: the rows behind stay.
    c = cases[1][0]
    c.cu.copy_(torch.tensor([0, 1, 1], dtype=torch.int32))
    c.out.fill_(NAN)
    graphs[1].replay()
    torch.cuda.synchronize()
    assert torch.isfinite(c.out[0]).all() and torch.isnan(c.out[1:]).all()


def test_two_streams_at_once(cuda):
    """Calls with workspaces of their own may overlap."""
    calls = []
    for i in range(2):
        tokens = [1, 90, 1]
        cache = paged.Cache(lens_of(1, 3, 2, [3000, 500, 1000 * i], tokens, i), 64, H=8, seed=i)
        cu, qkv = inputs(cache, tokens, i)
        calls.append((Call(cache, 0, qkv, cu), paged.attention(cache, 0, *qkv, cu, True), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for c, _, s in calls:
            c.run(stream=s)
    torch.cuda.synchronize()
    for c, (want, size, _, _), _ in calls:
        paged.assert_attention(c.out, want, size, c.cache.dtype)


def test_long_cache_offsets_pass_32_bits(cuda):
    """A pool of more than 2^31 elements and more than 4 GB: pages at its end."""
    page, num = 128, 170_000
    tokens = [3, 1]
    cache = paged.Cache(lens_of(1, 2, 1, [300, 200], tokens, 1), page, H=4)
    cu, qkv = inputs(cache, tokens, 4)
    want, size, _, _ = paged.attention(cache, 0, *qkv, cu, True)
    c = Call(cache, 0, qkv, cu)
    small = cache.pages.num_pages
    Kp = torch.zeros((num * page, paged.HEAD), dtype=cache.dtype, device="cuda")
    Vp = torch.zeros_like(Kp)
    Kp[-small * page:] = c.Kp
    Vp[-small * page:] = c.Vp
    c.Kp, c.Vp = Kp, Vp
    c.table = torch.where(c.table < small, c.table + (num - small), c.table)
    c.cache.pages = dkv.Pages(L=1, B=2, H=4, H_kv=1, page_rows=page, num_pages=num, max_pages=cache.table.shape[1])
    c.run()
    assert int(c.status) == 0
    paged.assert_attention(c.out, want, size, cache.dtype)


def test_copies_that_never_land_are_reported(cuda, monkeypatch):
    """Page copies that deliver half their bytes: every wait runs out, the call ends with the status bit, outputs stay
    unwritten, and the next call is right."""
    tokens = [1, 70]
    cache = paged.Cache(lens_of(1, 2, 1, [500, 90], tokens, 1), 16, H=4)
    cu, qkv = inputs(cache, tokens, 3)
    c = Call(cache, 0, qkv, cu)
    monkeypatch.setenv("DKV_FAULT", "copy")
    c.run()
    torch.cuda.synchronize()
    monkeypatch.delenv("DKV_FAULT")
    assert int(c.status) & dkv.DKV_DEV_TMA_TIMEOUT
    assert torch.isnan(c.out).all()
    c.status.zero_()
    c.run()
    want, size, _, _ = paged.attention(cache, 0, *qkv, cu, True)
    assert int(c.status) == 0
    paged.assert_attention(c.out, want, size, cache.dtype)


def test_many_short_units_in_one_share(cuda):
    """Sequences of few rows, so that a CTA has many units of one or two tiles, with turns between them."""
    tokens = [1, 3, 1, 80, 1, 0, 2, 1] * 12
    cache = paged.Cache(lens_of(1, len(tokens), 4, [20, 200, 140, 5, 300, 9, 0, 127] * 12, tokens, 6), 16, H=16)
    cu, qkv = inputs(cache, tokens, 3)
    c = Call(cache, 0, qkv, cu).run()
    want, size, _, _ = paged.attention(cache, 0, *qkv, cu, True)
    paged.assert_attention(c.out, want, size, cache.dtype)


@pytest.mark.parametrize("causal,dtype", [(True, torch.bfloat16), (False, torch.float16)])
def test_units_of_two_and_three_pieces(cuda, causal, dtype):
    """Units a little longer than a CTA's share: whichever CTA is last joins them, from what is stored and what it
    still holds, and the result is the same bits beside other work."""
    tokens, H, Hkv = [640], 32, 4
    cache = paged.Cache(lens_of(1, 1, Hkv, [1450], tokens, 3), 32, dtype=dtype, H=H)
    cu, qkv = inputs(cache, tokens, 5)
    c = Call(cache, 0, qkv, cu, causal).run()
    torch.cuda.synchronize()
    want, size, _, _ = paged.attention(cache, 0, *qkv, cu, causal)
    paged.assert_attention(c.out, want, size, dtype, "pieces")
    first, side, x = c.out.clone(), torch.cuda.Stream(), torch.randn((2048, 2048), device="cuda")
    for i in range(60):
        c.out.fill_(NAN)
        if i % 2:
            with torch.cuda.stream(side):
                for _ in range(1 + i % 5):
                    x = torch.sin(x)
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.out.view(torch.int16), first.view(torch.int16)), f"call {i} differs"
    assert int(c.status) == 0


def test_more_slabs_than_costs_fit(cuda):
    """Past 20,480 slabs a layer the costs are kept for groups of slabs."""
    B, Hkv = 512, 42
    tokens = [1 + b % 3 if b % 9 == 0 else 0 for b in range(B)]
    tokens[301] = 150
    ctx = np.array([b % 4 * 37 if tokens[b] else 0 for b in range(B)])
    lens = np.broadcast_to((ctx + tokens)[None, :, None], (1, B, Hkv)).copy()
    lens[0, 301, 5:] += 90
    check(paged.Cache(lens, 16), 0, tokens)


@pytest.mark.parametrize("tokens,ctx", [([1], 300), ([40], 200), ([1, 5], 0)])
def test_scores_of_minus_infinity_alone_give_zeros(cuda, tokens, ctx):
    cache = paged.Cache(lens_of(1, len(tokens), 2, [ctx] * len(tokens), tokens, 2), 16, H=8)
    cu, qkv = inputs(cache, tokens, 1, fused=False)
    qkv[0] = qkv[0].abs() + 1
    c = Call(cache, 0, qkv, cu, append=False)
    c.Kp.fill_(-float("inf"))
    c.run()
    assert int(c.status) == 0 and (c.out == 0).all()
