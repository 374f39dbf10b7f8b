"""dkv_quant_attn and dkv_quant_compact against their definition in 64 bits: token counts around the blocks and tiles, ragged and
empty sequences, every group size and page size, both types, scales far apart, and what lies in masked and unused places."""
import numpy as np
import pytest
import torch

import paged
import quant
from paper_2609_32663_gb300 import dkv
from test_gpu_chunk import lens_of
from test_gpu_rope import dev

pytestmark = pytest.mark.gpu
NAN = float("nan")


class Call:
    def __init__(self, c8, layer, q, cu, causal=True, scale=0.0, most=0):
        self.c8, self.layer, self.causal, self.scale, self.most = c8, layer, causal, scale, most
        self.q = q.cuda()
        self.pools = [x.cuda() for x in (c8.K8, c8.V8, c8.Ks, c8.Vs)]
        self.cu, self.table, self.len = dev(cu), dev(c8.cache.table), dev(c8.cache.lens)
        self.out = torch.full(q.shape, NAN, dtype=q.dtype, device="cuda")
        self.work = torch.full((dkv.dkv_quant_workspace_bytes(c8.pages),), 0xa5, dtype=torch.uint8, device="cuda")
        self.status = dev([0])

    def run(self, **kw):
        dkv.dkv_quant_attn(self.c8.pages, self.layer, self.q, self.cu, self.table, self.len, *self.pools, self.out, self.work,
                           causal=self.causal, scale=self.scale, max_tokens=self.most, status=self.status, **kw)
        return self


def inputs(c8, tokens, seed, pad=0):
    q = torch.randn((int(sum(tokens)) + pad, c8.cache.H, 128), generator=torch.Generator().manual_seed(seed)).to(c8.dtype)
    return np.concatenate([[0], np.cumsum(tokens)]).astype(np.int32), q


def check(c8, layer, tokens, causal=True, pad=0, seed=1, scale=0.0, most=0, q=None):
    cu, q0 = inputs(c8, tokens, seed, pad)
    q = q0 if q is None else q
    c = Call(c8, layer, q, cu, causal, scale, most).run()
    want, size = quant.attention(c8, layer, q, cu, causal, scale or None)
    assert int(c.status) == 0
    weights = quant.weight_rounding(tokens, c8.cache.H // c8.cache.Hkv, q.dtype, q.shape[0], most)
    quant.assert_attention(c.out, want, size, q.dtype, f"tokens {tokens}", weights)
    return c


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("ctx,tokens", [
    ([0], [1]), ([1], [1]), ([14], [1]), ([15], [1]), ([31], [1]), ([32], [1]), ([255], [1]), ([1000], [1]),
    ([300, 0, 5, 700], [1, 1, 1, 1]),
    ([250, 130, 0, 513], [3, 0, 17, 2]),
    ([0], [33]), ([90], [65]), ([0, 400], [129, 40]),
    ([40, 1200, 3], [31, 1, 150]),
])
def test_lengths_and_pages(cuda, page, ctx, tokens):
    check(quant.Cache8(lens_of(2, len(ctx), 2, ctx, tokens, page), page, H=8, seed=page), 1, tokens)


@pytest.mark.parametrize("G,Hkv", [(1, 3), (2, 2), (3, 1), (4, 1), (5, 2), (6, 1), (7, 2), (8, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_group_sizes(cuda, G, Hkv, dtype):
    tokens = [1, 16 // G + 1, 3, 128 // G + 1, 2 * (128 // G) + 1]
    lens = lens_of(1, 5, Hkv, [333, 60, 0, 129, 40], tokens, G)
    check(quant.Cache8(lens, 32, H=G * Hkv, seed=G, dtype=dtype), 0, tokens)


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8])
@pytest.mark.parametrize("cols", [8, 16])
@pytest.mark.parametrize("causal", [True, False])
def test_few_tokens_a_sequence(cuda, G, cols, causal):
    """As many columns as the kernels of 8 and of 16 take, sequences of fewer beside them, rows that only the last ones see."""
    n = max(cols // G, 1)
    tokens = [n, 1, 0, n, max(n - 1, 1), n]
    for page, ctx in ((16, [0, 40, 3, 33, 500, 14]), (128, [1300, 0, 9, 255, 31, 4000])):
        check(quant.Cache8(lens_of(1, 6, 2, ctx, tokens, G), page, H=2 * G, seed=G), 0, tokens, causal=causal, most=n)


def test_no_token_at_all(cuda):
    """Sequences that bring nothing: nothing is written."""
    c8 = quant.Cache8(np.array([[[40], [0]]]), 16, H=4)
    _, q = inputs(c8, [0, 0], 1, pad=70)
    for most in (0, 1, 70):
        c = Call(c8, 0, q, [0, 0, 0], most=most).run()
        assert int(c.status) == 0 and torch.isnan(c.out.float()).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("pad", [0, 5])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_masks_and_padding(cuda, causal, pad, dtype):
    tokens = [5, 1, 70, 0, 2]
    c = check(quant.Cache8(lens_of(2, 5, 2, [200, 129, 64, 10, 0], tokens, 3), 64, H=8, dtype=dtype), 0, tokens, causal=causal, pad=pad)
    assert torch.isnan(c.out[78:].float()).all()


def test_scale(cuda):
    check(quant.Cache8(lens_of(1, 2, 1, [100, 300], [2, 40], 1), 16, H=4), 0, [2, 40], scale=0.03)


def test_slab_shorter_than_its_tokens(cuda):
    """Fewer rows than queries: the first queries see no row."""
    c8 = quant.Cache8(np.array([[[3, 0], [40, 1]]]), 16, H=8)
    for tokens in ([5, 41], [1, 2], [0, 300]):
        check(c8, 0, tokens)
        check(c8, 0, tokens, causal=False)


def test_more_sequences_than_ctas(cuda):
    tokens = [1, 2, 5] * 60
    check(quant.Cache8(lens_of(1, 180, 2, [30, 300, 0] * 60, tokens, 4), 16, H=4), 0, tokens)


def test_more_slabs_than_sums_fit(cuda):
    """Past 24,576 slabs a layer the tiles are summed for groups of slabs."""
    B, Hkv = 512, 50
    tokens = [1 + b % 3 if b % 9 == 0 else 0 for b in range(B)]
    tokens[301] = 150
    ctx = np.array([b % 4 * 37 if tokens[b] else 0 for b in range(B)])
    lens = np.broadcast_to((ctx + tokens)[None, :, None], (1, B, Hkv)).copy()
    lens[0, 301, 5:] += 90
    check(quant.Cache8(lens, 16), 0, tokens)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_one_long_sequence(cuda, dtype):
    """Units over all CTAs, with many pieces to join."""
    check(quant.Cache8(np.array([[[30011, 20000]]]), 64, H=8, dtype=dtype), 0, [1])
    check(quant.Cache8(np.array([[[9000, 5]]]), 16, H=16, dtype=dtype), 0, [3])


@pytest.mark.parametrize("G,tokens", [(7, [5]), (8, [16, 1]), (3, [50]), (4, [64, 2, 9]), (1, [200])])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("causal", [True, False])
def test_drafts_in_many_pieces(cuda, G, tokens, dtype, causal):
    """Units of up to 256 rows that many CTAs have a part of, joined in the same order each time."""
    ctx = [12003, 5, 2500][:len(tokens)]
    c8 = quant.Cache8(lens_of(1, len(tokens), 1, ctx, tokens, G), 32, H=G, dtype=dtype)
    c = check(c8, 0, tokens, causal, pad=3)
    assert torch.isnan(c.out[sum(tokens):].float()).all()
    before = c.out.clone()
    c.out.fill_(NAN)
    assert torch.equal(c.run().out[:sum(tokens)], before[:sum(tokens)])


def test_scales_far_apart(cuda):
    """Rows of V up to 2^40 apart, of K up to 2^6, and many rows of V that are all zero (their scale byte is 1) with weight."""
    r = np.random.default_rng(1)
    for tokens in ([1], [9], [150]):
        c8 = quant.Cache8(np.array([[[900, 431]]]) + tokens[0], 16, H=8)
        n = c8.Vs.numel()
        held = c8.Vs != 255
        c8.Vs[held] = torch.from_numpy((100 + r.integers(0, 40, n)).astype(np.uint8))[held]
        c8.Ks[held] = torch.from_numpy((113 + r.integers(0, 6, n)).astype(np.uint8))[held]
        zero = held & torch.from_numpy(r.random(n) < 0.5)
        c8.V8[zero], c8.Vs[zero] = 0, 1
        c8.sync()
        check(c8, 0, tokens)


def test_zero_rows_keep_their_weight(cuda):
    """A row of V that is all zero has the scale byte 1; thousands of them, with scores a little below one other row's, make most
    of the sum."""
    for tokens in ([1], [40]):
        rows = 4000 + tokens[0]
        c8 = quant.Cache8(np.array([[[rows]]]), 64, H=4)
        c8.K8[c8.cache.rows(0)] = 0
        at = c8.cache.rows(0)
        c8.V8[at[5:]], c8.Vs[at[5:]] = 0, 1
        c8.K8[at[5:]], c8.Ks[at[5:]] = 0xb8, 127  # -1 in every dim
        c8.sync()
        q = torch.full((tokens[0], 4, 128), 1.4, dtype=c8.dtype)
        check(c8, 0, tokens, q=q)


@pytest.mark.parametrize("size", [1e-30, 1e-3, 300.0, 6e4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_queries_of_any_size(cuda, size, dtype):
    """The scale undoes the queries' size, so that the scores are those of standard normal ones."""
    if dtype == torch.float16 and size < 1e-6:
        size = 1e-3
    tokens = [2, 40]
    c8 = quant.Cache8(lens_of(1, 2, 1, [100, 300], tokens, 1), 16, H=4, dtype=dtype)
    cu, q = inputs(c8, tokens, 3)
    q = (q.float().clamp(-1, 1) * size).to(dtype)
    check(c8, 0, tokens, q=q, scale=128 ** -0.5 / size)


@pytest.mark.parametrize("tokens", [[70, 4], [3, 4], [4, 4]])
def test_later_tokens_hold_anything(cuda, tokens):
    """NaN in K and V of a later token changes no earlier token's output, and is NaN for those that see it."""
    for dtype in (torch.bfloat16, torch.float16):
        c8 = quant.Cache8(lens_of(1, 2, 2, [90, 128], tokens, 5), 16, H=8, dtype=dtype)
        c = c8.cache
        n = tokens[0]
        last = [c.rows(h)[-tokens[h // 2]:] for h in range(4)]  # the new rows of each slab
        k1, v1 = (50, 60) if n == 70 else (2, 1)
        c8.K8[last[0][k1], 7] = 0x7f
        c8.V8[last[1][v1], :] = 0xff
        c8.V8[last[2][3], 9] = 0x7f
        c8.sync()
        cu, q = inputs(c8, tokens, 2)
        x = Call(c8, 0, q, cu, most=max(tokens)).run()
        want, size = quant.attention(c8, 0, q, cu)
        # (the definition's sums over what a token sees alone)
        quant.assert_attention(x.out, want, size, dtype)
        assert torch.isnan(want[k1, :4]).all() and torch.isnan(want[n + 3, :4, 9]).all() and torch.isfinite(want[0]).all()
        assert torch.isfinite(x.out[n:n + 3].float()).all()


@pytest.mark.parametrize("tokens", [[70, 4], [3, 4], [4, 4], [2, 2]])
@pytest.mark.parametrize("most", [0, 1])
@pytest.mark.parametrize("dtype,byte", [(torch.bfloat16, 240), (torch.bfloat16, 150), (torch.float16, 135)])
def test_later_tokens_may_be_far_larger(cuda, tokens, most, dtype, byte):
    """A later token's K and V of 448 2^113 (or of the largest that fp16 rows have) change no earlier token's output, and are most
    of the outputs that see them."""
    c8 = quant.Cache8(lens_of(1, 2, 2, [90, 128], tokens, 5), 16, H=8, dtype=dtype)
    c, n = c8.cache, tokens[0]
    last = [c.rows(h)[-tokens[h // 2]:] for h in range(4)]  # the new rows of each slab
    cu, q = inputs(c8, tokens, 2)
    first = Call(c8, 0, q, cu, most=max(tokens) if most else 0).run()  # (all rows as they were)
    for h in range(4):
        r = last[h][tokens[h // 2] - 1]
        c8.V8[r], c8.Vs[r] = 0x7e, byte
    c8.Ks[last[0][n - 1]] = min(byte, 140)
    c8.sync()
    x = Call(c8, 0, q, cu, most=max(tokens) if most else 0).run()
    want, size = quant.attention(c8, 0, q, cu)
    ends = [n - 1, sum(tokens) - 1]
    others = [i for i in range(sum(tokens)) if i not in ends]
    assert torch.equal(x.out[others], first.out[others])
    finite = want.abs() <= torch.finfo(dtype).max
    for t in ends:
        got, w, sz = x.out[t:t + 1, 4:].double().cpu(), want[t:t + 1, 4:], size[t:t + 1, 4:]
        ok = finite[t:t + 1, 4:]
        quant.assert_attention(torch.where(ok, got, w), w, sz, dtype)


@pytest.mark.parametrize("tokens", [[70, 4], [33, 40]])
@pytest.mark.parametrize("byte", [136, 140, 200, 247])
def test_later_rows_past_fp16_spoil_no_earlier_output(cuda, tokens, byte):
    """fp16 products over a row of V that fp16 does not hold: tokens that do not see it are as without it. (Their outputs may be
    computed another way then, so they are held to the definition.)"""
    c8 = quant.Cache8(lens_of(1, 2, 2, [90, 128], tokens, 5), 16, H=8, dtype=torch.float16)
    c, n = c8.cache, tokens[0]
    cu, q = inputs(c8, tokens, 2)
    want, size = quant.attention(c8, 0, q, cu)
    for h in range(4):
        r = c.rows(h)[-1]
        c8.V8[r, ::3], c8.Vs[r] = 0x7e, byte
        c8.Ks[r] = 140
    c8.sync()
    x = Call(c8, 0, q, cu).run()
    others = [i for i in range(sum(tokens)) if i not in (n - 1, sum(tokens) - 1)]
    quant.assert_attention(x.out[others], want[others], size[others], torch.float16)


@pytest.mark.parametrize("tokens,ctx", [([1], 300), ([40], 200), ([1, 5], 0)])
def test_scores_of_minus_infinity_alone_give_zeros(cuda, tokens, ctx):
    c8 = quant.Cache8(lens_of(1, len(tokens), 2, [ctx] * len(tokens), tokens, 2), 16, H=8)
    c8.K8[c8.Ks != 255] = 0xb8  # -1
    cu, q = inputs(c8, tokens, 1)
    q[:] = float("inf")
    c = Call(c8, 0, q, cu).run()
    assert int(c.status) == 0 and (c.out == 0).all()


@pytest.mark.parametrize("turn", [3, 60])
def test_bad_page_numbers_and_lengths_are_reported(cuda, turn):
    """They are not followed; other sequences keep their results."""
    tokens = [2, turn, 2]
    c8 = quant.Cache8(lens_of(1, 3, 1, [40, 50, 60], tokens, 1), 16, H=4)
    cu, q = inputs(c8, tokens, 3)
    want, size = quant.attention(c8, 0, q, cu)
    for kind in ("page", "negative", "long"):
        c = Call(c8, 0, q, cu)
        if kind == "page":
            c.table[1, :4] = 1 << 30
        elif kind == "negative":
            c.table[1, :4] = -5
        else:
            c.len[1] = 1 << 30
        c.run()
        assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE
        for t in (slice(0, 2), slice(2 + turn, 4 + turn)):
            quant.assert_attention(c.out[t], want[t], size[t], c8.dtype, kind)
        assert torch.isfinite(c.out.float()).all()


def test_bad_offsets_write_nothing(cuda):
    tokens = [2, 30, 2]
    c8 = quant.Cache8(lens_of(1, 3, 1, [40, 50, 60], tokens, 1), 16, H=4)
    _, q = inputs(c8, tokens, 3)
    for cu in ([1, 2, 32, 34], [0, 33, 32, 34], [0, 2, 32, 35], [0, -1, 5, 34], [0, 2, 5, 1 << 30]):
        c = Call(c8, 0, q, cu).run()
        assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE and torch.isnan(c.out.float()).all()


def test_more_tokens_than_were_said(cuda):
    """A sequence of more tokens than max_tokens is skipped and reported; with the right number it is not."""
    tokens = [2, 30, 4]
    c8 = quant.Cache8(lens_of(1, 3, 2, [40, 50, 60], tokens, 1), 16, H=8)
    cu, q = inputs(c8, tokens, 3)
    want, size = quant.attention(c8, 0, q, cu)
    for most in (4, 29):
        c = Call(c8, 0, q, cu, most=most).run()
        assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE
        assert torch.isnan(c.out[2:32].float()).all()
        for t in (slice(0, 2), slice(32, 36)):
            quant.assert_attention(c.out[t], want[t], size[t], c8.dtype)
    for most in (30, 31, 1000, -1):
        c = Call(c8, 0, q, cu, most=most).run()
        assert int(c.status) == 0
        quant.assert_attention(c.out, want, size, c8.dtype)


def test_repeats_are_bit_exact(cuda):
    for tokens in ([1, 200, 1, 7], [1, 1, 1, 3]):
        c8 = quant.Cache8(lens_of(1, 4, 2, [4000, 900, 30, 2500], tokens, 1), 64, H=8)
        cu, q = inputs(c8, tokens, 3)
        c = Call(c8, 0, q, cu).run()
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
        c8 = quant.Cache8(lens_of(1, 2, 2, [700, 90 + i], tokens, i), 32, H=8, seed=i)
        cu, q = inputs(c8, tokens, i)
        c = Call(c8, 0, q, cu)
        c.work = cases[0][0].work if cases else c.work
        cases.append((c, quant.attention(c8, 0, q, cu)))
        c.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            c.run()
        graphs.append(g)
    for _ in range(3):
        for g, (c, (want, size)) in zip(graphs, cases):
            c.out.fill_(NAN)
            g.replay()
            torch.cuda.synchronize()
            quant.assert_attention(c.out, want, size, c.c8.dtype)
    c = cases[1][0]
    c.cu.copy_(dev([0, 1, 1]))  # the step's tokens became fewer: the rows behind stay
    c.out.fill_(NAN)
    graphs[1].replay()
    torch.cuda.synchronize()
    assert torch.isfinite(c.out[0].float()).all() and torch.isnan(c.out[1:].float()).all()


def test_two_streams_at_once(cuda):
    """Calls with workspaces of their own may overlap."""
    calls = []
    for i in range(2):
        tokens = [1, 90, 1]
        c8 = quant.Cache8(lens_of(1, 3, 2, [3000, 500, 1000 * i], tokens, i), 64, H=8, seed=i)
        cu, q = inputs(c8, tokens, i)
        calls.append((Call(c8, 0, q, cu), quant.attention(c8, 0, q, cu), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for c, _, s in calls:
            c.run(stream=s)
    torch.cuda.synchronize()
    for c, (want, size), _ in calls:
        quant.assert_attention(c.out, want, size, c.c8.dtype)


def test_long_cache_offsets_pass_32_bits(cuda):
    """Pools of more than 4 GB: pages at their end."""
    page, num, tokens = 128, 340_000, [3, 70, 1]
    c8 = quant.Cache8(lens_of(1, 3, 1, [300, 100, 200], tokens, 1), page, H=4)
    cu, q = inputs(c8, tokens, 4)
    want, size = quant.attention(c8, 0, q, cu)
    c = Call(c8, 0, q, cu)
    small = c8.pages.num_pages
    for i, x in enumerate(c.pools):
        wide = torch.zeros((num * page, *x.shape[1:]), dtype=torch.uint8, device="cuda")
        wide[-small * page:] = x
        c.pools[i] = wide
    c.table = torch.where(c.table < small, c.table + (num - small), c.table)
    c8.pages = dkv.Pages(L=1, B=3, H=4, H_kv=1, page_rows=page, num_pages=num, max_pages=c8.cache.table.shape[1])
    c.run()
    assert int(c.status) == 0
    quant.assert_attention(c.out, want, size, c8.dtype)


@pytest.mark.parametrize("tokens", [[1, 3], [1, 70]])
def test_copies_that_never_land_are_reported(cuda, monkeypatch, tokens):
    """Page copies that deliver half their bytes: every wait runs out, the call ends with the status bit, outputs stay
    unwritten, and the next call is right."""
    c8 = quant.Cache8(lens_of(1, 2, 1, [500, 90], tokens, 1), 16, H=4)
    cu, q = inputs(c8, tokens, 3)
    c = Call(c8, 0, q, cu)
    monkeypatch.setenv("DKV_FAULT", "copy")
    c.run()
    torch.cuda.synchronize()
    monkeypatch.delenv("DKV_FAULT")
    assert int(c.status) & dkv.DKV_DEV_TMA_TIMEOUT
    assert torch.isnan(c.out.float()).all()
    c.status.zero_()
    c.run()
    want, size = quant.attention(c8, 0, q, cu)
    assert int(c.status) == 0
    quant.assert_attention(c.out, want, size, c8.dtype)


def test_buffers_of_other_types(cuda):
    """Pools and scales may be named by their own types; others are refused."""
    c8 = quant.Cache8(np.array([[[40]]]), 16, H=2)
    cu, q = inputs(c8, [1], 1)
    c = Call(c8, 0, q, cu)
    c.pools = [x.view(torch.float8_e4m3fn) for x in c.pools[:2]] + [x.view(torch.float8_e8m0fnu) for x in c.pools[2:]]
    c.run()
    want, size = quant.attention(c8, 0, q, cu)
    quant.assert_attention(c.out, want, size, c8.dtype)
    for i, bad in enumerate((torch.bfloat16, torch.float8_e5m2, torch.int8, torch.float8_e4m3fn)):
        keep, c.pools[i] = c.pools[i], torch.empty(c.pools[i].shape, dtype=bad, device="cuda")
        with pytest.raises(dkv.DkvError):
            c.run()
        c.pools[i] = keep


# ------------------------------------------------------------ prune-and-pack

def packed(L, H, Hkv, B, ctx, seq, page, dtype, seed):
    """A plan over some sequences, tables with room for them, and the calls' buffers."""
    r = np.random.default_rng(seed)
    D, W = 6, 37
    M = (r.random((L, H, D)) < 0.3).astype(np.uint8)
    shape = dkv.Shape(L=L, H=H, H_kv=Hkv, D=D, sink=9, recent=20, bin_width=W)
    plan = dkv.dkv_map_pattern(M, ctx, shape)
    ln, off, ioff, idx = dkv.dkv_plan_read(plan)
    before = r.integers(0, 40, (L, B, Hkv))
    lens = before.copy()
    lens[:, seq] += ln.reshape(L, len(seq), Hkv)
    cache = paged.Cache(lens, page, dtype=dtype, seed=seed, H=H)
    T = int(max(ctx)) + 3
    K, V = (torch.randn((L, len(seq), Hkv, T, 128), generator=torch.Generator().manual_seed(seed + i)).to(dtype) for i in range(2))
    return plan, cache, before, K, V, [idx[ioff[i]:ioff[i + 1]] for i in range(len(ln))]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("ctx,seq", [([1], [0]), ([29], [0]), ([251, 3, 100], [0, 2, 3]), ([0, 200], [1, 3])])
def test_compact(cuda, dtype, page, ctx, seq):
    L, H, Hkv, B = 2, 8, 2, 4
    plan, cache, before, K, V, kept = packed(L, H, Hkv, B, ctx, seq, page, dtype, page)
    K[..., 0, 0], V[..., max(ctx) // 2, 3] = 1e4, NAN
    rows = cache.pages.num_pages * page
    pools = [torch.full((rows, 128), 0x55, dtype=torch.uint8, device="cuda") for _ in "KV"] + [
        torch.full((rows,), 3, dtype=torch.uint8, device="cuda") for _ in "KV"]
    status = dev([0])
    dkv.dkv_quant_compact(cache.pages, plan, K.cuda(), V.cuda(), dev(cache.table), dev(cache.lens), *pools, seq=dev(seq), status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    want = [np.full((rows, 128), 0x55, np.uint8) for _ in "KV"] + [np.full(rows, 3, np.uint8) for _ in "KV"]
    for i, at in enumerate(kept):
        l, j, g = i // (len(seq) * Hkv), i // Hkv % len(seq), i % Hkv
        h = (l * B + seq[j]) * Hkv + g
        to = cache.rows(h, cache.lens[h] - len(at))
        for x in range(2):
            want[x][to], want[2 + x][to] = quant.held((K, V)[x][l, j, g, at.astype(np.int64)])
    for got, exp in zip(pools, want):
        got = got.cpu().numpy()
        nan = (exp & 0x7f) == 0x7f if exp.ndim == 2 else np.zeros(exp.shape, bool)
        assert np.array_equal(got[~nan], exp[~nan]) and ((got[nan] & 0x7f) == 0x7f).all()
    plan.close()


def test_compact_skips_what_is_out_of_range(cuda):
    plan, cache, before, K, V, kept = packed(1, 4, 1, 3, [200, 90], [0, 2], 16, torch.bfloat16, 1)
    rows = cache.pages.num_pages * 16

    def run(table, ln, seq):
        pools = [torch.full((rows, 128), 0x55, dtype=torch.uint8, device="cuda") for _ in "KV"] + [
            torch.full((rows,), 3, dtype=torch.uint8, device="cuda") for _ in "KV"]
        status = dev([0])
        dkv.dkv_quant_compact(cache.pages, plan, K.cuda(), V.cuda(), dev(table), dev(ln), *pools, seq=dev(seq), status=status)
        return int(status), pools

    good = run(cache.table, cache.lens, [0, 2])
    assert good[0] == 0
    table = cache.table.copy()
    table[2] = -1
    st, pools = run(table, cache.lens, [0, 2])
    at = cache.rows(2, before.reshape(-1)[2])
    assert st == dkv.DKV_DEV_PAGE_RANGE
    for x, y in zip(pools, good[1]):
        y = y.clone()
        y[at] = 0x55 if y.dim() == 2 else 3
        assert torch.equal(x, y)
    for ln, seq in ((cache.lens, [0, 5]), (cache.lens, [-1, 2]), (np.array([cache.lens[0], 0, 1 << 30]), [0, 2]), (np.zeros(3), [0, 2])):
        st, _ = run(cache.table, ln, seq)
        assert st == dkv.DKV_DEV_PAGE_RANGE
    plan.close()


# ------------------------------------------------------------ together

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_serving_loop(cuda, dtype):
    """Sequences admitted after pruning, steps of turns and next tokens with rotary positions, one sequence ends, all in 8 bits, with
    nothing between the calls: lengths, tables and counts are updated in place."""
    L, B, H, Hkv, page = 2, 3, 8, 2, 16
    NH = L * B * Hkv
    r = np.random.default_rng(1)
    M = (r.random((L, H, 5)) < 0.4).astype(np.uint8)
    ctx, seq = [150, 61], [0, 2]
    plan = dkv.dkv_map_pattern(M, ctx, dkv.Shape(L=L, H=H, H_kv=Hkv, D=5, sink=7, recent=11, bin_width=40))
    kept, off, ioff, idx = dkv.dkv_plan_read(plan)
    g = dkv.Pages(L=L, B=B, H=H, H_kv=Hkv, page_rows=page, num_pages=400, max_pages=30)
    ln, table, free, count, status = dev(np.zeros(NH)), dev(np.zeros((NH, 30))), dev(r.permutation(400)), dev([400]), dev([0])
    pools = [torch.full((400 * page, 128), 0x7f, dtype=torch.uint8, device="cuda") for _ in "KV"] + [
        torch.full((400 * page,), 255, dtype=torch.uint8, device="cuda") for _ in "KV"]
    pw = torch.empty(dkv.dkv_page_workspace_bytes(g), dtype=torch.uint8, device="cuda")
    aw = torch.empty(dkv.dkv_quant_workspace_bytes(g), dtype=torch.uint8, device="cuda")
    gen = torch.Generator().manual_seed(5)
    K, V = (torch.randn((L, 2, Hkv, 150, 128), generator=gen).to(dtype) for _ in range(2))
    rotary, f = dkv.dkv_rotary_make(64, interleaved=True), 10000.0 ** (-2 * np.arange(32) / 64)
    steps = [[3, 40, 1], [1, 1, 1], [1, 0, 20], [2, 1, 1]]
    qkv = [[torch.randn((sum(n) + 1, H + 2 * Hkv, 128), generator=gen).to(dtype) for _ in range(L)] for n in steps]
    pos = [np.concatenate([[1000 * b + 50 * i + np.arange(n)] for b, n in enumerate(s) for _ in [0] if n], axis=None) if sum(s) else np.zeros(0)
           for i, s in enumerate(steps)]
    dq, dp = [[x.cuda() for x in s] for s in qkv], [dev(np.append(p, 0)) for p in pos]
    dn, cu, ended = [dev(n) for n in steps], dev(np.zeros(B + 1)), dev([0, 1, 0])
    outs = [[torch.full((x.shape[0], H, 128), NAN, dtype=dtype, device="cuda") for x in s] for s in qkv]
    Kd, Vd, sd = K.cuda(), V.cuda(), dev(seq)
    torch.cuda.synchronize()
    dkv.dkv_page_tables(g, ln, ln, table, free, count, count, pw, plan=plan, seq=sd, status=status)
    dkv.dkv_quant_compact(g, plan, Kd, Vd, table, ln, *pools, seq=sd, status=status)
    snaps = []
    for i in range(len(steps)):
        if i == 2:
            dkv.dkv_page_release(g, ended, ln, ln, table, free, count, count, pw, status=status)
        dkv.dkv_page_tables(g, ln, ln, table, free, count, count, pw, tokens=dn[i], cu_tokens=cu, status=status)
        for layer in range(L):
            d = dq[i][layer]
            q, k, v = d[:, :H], d[:, H:H + Hkv], d[:, H + Hkv:]
            dkv.dkv_rope_append(g, layer, q, k, v, dp[i], cu, table, ln, *pools[:2], q, *pools[2:], rotary=rotary, status=status)
            dkv.dkv_quant_attn(g, layer, q, cu, table, ln, *pools, outs[i][layer], aw, max_tokens=max(steps[i]), status=status)
        snaps.append([x.clone() for x in (ln, table, *pools)])
    torch.cuda.synchronize()
    assert int(status) == 0
    # The slabs as lists of rows: (codes, scales) of what was written.
    slabs = [[np.zeros((0, 128)), np.zeros(0), np.zeros((0, 128)), np.zeros(0)] for _ in range(NH)]

    def grow(h, k, v):
        parts = [*quant.held(k), *quant.held(v)]
        slabs[h] = [np.concatenate([x, y]) for x, y in zip(slabs[h], parts)]

    for i, n in enumerate(kept):
        l, j, x = i // (2 * Hkv), i // Hkv % 2, i % Hkv
        at = idx[ioff[i]:ioff[i + 1]].astype(np.int64)
        grow((l * B + seq[j]) * Hkv + x, K[l, j, x, at], V[l, j, x, at])
    for i, n in enumerate(steps):
        if i == 2:
            for l in range(L):
                for x in range(Hkv):
                    slabs[(l * B + 1) * Hkv + x] = [np.zeros((0, 128)), np.zeros(0), np.zeros((0, 128)), np.zeros(0)]
        sln, stable, sK8, sV8, sKs, sVs = (x.cpu() for x in snaps[i])
        offsets = np.concatenate([[0], np.cumsum(n)])
        for layer in range(L):
            x = qkv[i][layer]
            got_q = dq[i][layer][:, :H].cpu()
            want_q, size_q = quant.turned(x[:sum(n), :H], pos[i], f, True)
            quant.assert_turned(got_q[:sum(n)], want_q, size_q, dtype)
            assert torch.equal(got_q[sum(n):], x[sum(n):, :H])
            k, _ = quant.turned(x[:sum(n), H:H + Hkv], pos[i], f, True)
            for b in range(B):
                for y in range(Hkv):
                    h = (layer * B + b) * Hkv + y
                    grow(h, k[offsets[b]:offsets[b + 1], y], x[offsets[b]:offsets[b + 1], H + Hkv + y])
                    m = len(slabs[h][0])
                    assert int(sln[h]) == m
                    r = np.arange(m)
                    at = stable[h].numpy()[r // page].astype(np.int64) * page + r % page
                    old = np.arange(m) < m - n[b]
                    assert np.array_equal(sV8[at].numpy(), slabs[h][2]) and np.array_equal(sVs[at].numpy(), slabs[h][3])
                    assert np.array_equal(sK8[at[old]].numpy(), slabs[h][0][old])
                    # turned keys: the GPU's own, which test_append holds to the definition, are what it attends to
                    near = (quant.values(sK8[at].numpy(), sKs[at].numpy()) - quant.values(slabs[h][0].astype(np.uint8), slabs[h][1])).abs()
                    assert (near <= 2.0 ** -3 * quant.values(slabs[h][0].astype(np.uint8), slabs[h][1]).abs() + 2e-2).all()
                    slabs[h][0], slabs[h][1] = sK8[at].numpy(), sKs[at].numpy()
                    Kv, Vv = quant.values(sK8[at].numpy(), sKs[at].numpy()), quant.values(sV8[at].numpy(), sVs[at].numpy())
                    for t in range(offsets[b], offsets[b + 1]):
                        s = m - (offsets[b + 1] - 1 - t)
                        heads = slice(y * (H // Hkv), (y + 1) * (H // Hkv))
                        w = torch.softmax(got_q[t, heads].double() @ Kv[:s].T / 128 ** 0.5, -1)
                        quant.assert_attention(outs[i][layer][t, heads], w @ Vv[:s], w @ Vv[:s].abs(), dtype, f"step {i}")
            assert torch.isnan(outs[i][layer][sum(n):].float()).all()
    plan.close()


def test_16_bit_pages_with_rotary_positions(cuda):
    """dkv_rope_append to 16-bit pages, then dkv_chunk_attn without rows of its own."""
    tokens, H, Hkv = [2, 50, 1], 8, 2
    cache = paged.Cache(lens_of(1, 3, Hkv, [100, 0, 300], tokens, 2), 32, H=H, dtype=torch.bfloat16)
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((53, H + 2 * Hkv, 128), generator=gen).to(torch.bfloat16)
    cu, pos, f = np.array([0, 2, 52, 53]), np.arange(53) * 7 + 9000, 10000.0 ** (-2 * np.arange(64) / 128)
    d, Kp, Vp = x.cuda(), cache.Kp.cuda(), cache.Vp.cuda()
    out, status = torch.full((53, H, 128), NAN, dtype=torch.bfloat16, device="cuda"), dev([0])
    work = torch.empty(dkv.dkv_chunk_workspace_bytes(cache.pages), dtype=torch.uint8, device="cuda")
    dcu, table, ln, dpos = dev(cu), dev(cache.table), dev(cache.lens), dev(pos)
    dkv.dkv_rope_append(cache.pages, 0, d[:, :H], d[:, H:H + Hkv], d[:, H + Hkv:], dpos, dcu, table, ln, Kp, Vp, d[:, :H],
                        rotary=dkv.dkv_rotary_make(), status=status)
    dkv.dkv_chunk_attn(cache.pages, 0, d[:, :H], None, None, dcu, table, ln, Kp, Vp, out, work, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    q, size = quant.turned(x[:, :H], pos, f, False)
    quant.assert_turned(d[:, :H], q, size, torch.bfloat16)
    cache.Kp, cache.Vp = Kp.cpu(), Vp.cpu()
    k, size = quant.turned(x[:, H:H + Hkv], pos, f, False)
    for b in range(3):
        for g in range(Hkv):
            at = cache.rows(b * Hkv + g)[-tokens[b]:]
            quant.assert_turned(cache.Kp[at], k[cu[b]:cu[b + 1], g], size[cu[b]:cu[b + 1], g], torch.bfloat16)
            assert torch.equal(cache.Vp[at], x[cu[b]:cu[b + 1], H + Hkv + g])
    want, size, _, _ = paged.attention(cache, 0, d[:, :H].cpu(), None, None, cu, True)
    paged.assert_attention(out, want, size, torch.bfloat16)
