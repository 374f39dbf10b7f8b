"""fp16 over 8-bit rows with elements that fp16 does not hold (scale bytes above 135), as fp16 keys turned with a magnitude above 1.4 may
have them, or rows of bf16 values: the outputs are the definition's, by whichever kernel a sequence's tokens take."""
import numpy as np
import pytest
import torch

import quant
from test_gpu_chunk import lens_of
from test_gpu_quant import Call, check, inputs

pytestmark = pytest.mark.gpu

HALF = torch.float16
# (heads a group, rows before, tokens): split units, pair units, pieces joined by the unit's CTAs and by the next kernel, beside few
CALLS = [(4, [200], [9]), (4, [200, 90], [2, 70]), (4, [300, 0, 129], [17, 1, 140]), (7, [260, 900], [5, 3]), (1, [150], [200]), (8, [12003], [3]), (2, [5000, 700], [1, 130]),
         (8, [2500, 30], [16, 260])]


def cache(G, ctx, tokens, page=32, Hkv=1):
    return quant.Cache8(lens_of(1, len(tokens), Hkv, ctx, tokens, G), page, H=G * Hkv, dtype=HALF, seed=G)


def some(c8, share, seed):
    """A part of the rows that slabs hold, the first of each slab among them."""
    held = c8.Ks != 255
    part = torch.from_numpy(np.random.default_rng(seed).random(held.numel()) < share)
    for h in range(c8.cache.lens.size):
        part[c8.cache.rows(h)[:1]] = True
    return held & part


@pytest.mark.parametrize("G,ctx,tokens", CALLS)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("share", [0.002, 0.4, 1.0])
def test_large_keys(cuda, G, ctx, tokens, causal, share):
    """Keys 2^18 times as large, and a scale that undoes that."""
    c8 = cache(G, ctx, tokens)
    c8.Ks[some(c8, share, G)] += 18
    c8.sync()
    assert int(c8.Ks[c8.Ks != 255].max()) > 135
    check(c8, 0, tokens, causal, scale=128 ** -0.5 * 2.0 ** -18)


@pytest.mark.parametrize("G,ctx,tokens", [c for c in CALLS if min(c[1]) >= 150])
@pytest.mark.parametrize("causal", [True, False])
def test_large_values(cuda, G, ctx, tokens, causal):
    """The first row of V of each slab past 2^16, with the weight of one of some hundred rows. (In one call 27 outputs, of a row with nearly
    all weight, are 65,520 to 228,538 by the definition: infinite, rounded to fp16, whose largest number is 65,504.)"""
    c8 = cache(G, ctx, tokens)
    for h in range(len(tokens)):
        c8.Vs[c8.cache.rows(h)[0]] = 136
    c8.sync()
    cu, q = inputs(c8, tokens, 1)
    c = Call(c8, 0, q, cu, causal).run()
    want, size = quant.attention(c8, 0, q, cu, causal)
    past, got = want.abs() >= 65520, c.out.double().cpu()
    assert int(c.status) == 0 and torch.equal(got[past], want[past].sign() * float("inf"))
    weights = quant.weight_rounding(tokens, G, HALF, q.shape[0])
    quant.assert_attention(torch.where(past, want, got), want, size, HALF, weights=weights)


@pytest.mark.parametrize("page", [16, 128])
def test_pages_heads_and_padding(cuda, page):
    tokens = [33, 0, 12, 150]
    c8 = cache(4, [100, 20, 333, 64], tokens, page, Hkv=3)
    c8.Ks[some(c8, 0.1, 1)] += 20
    c8.sync()
    c = check(c8, 0, tokens, pad=7, scale=128 ** -0.5 * 2.0 ** -20)
    assert torch.isnan(c.out[sum(tokens):].float()).all()


@pytest.mark.parametrize("tokens", [[6, 1], [40, 5], [150, 3]])
def test_the_same_sequence_by_either_kernel(cuda, tokens):
    """Beside a sequence of many tokens the last one's are few columns or many; its outputs are the definition's both times, and so are those
    of a call of its own."""
    c8 = cache(2, [400, 500], tokens)
    c8.Ks[some(c8, 0.3, 5)] += 18
    c8.sync()
    scale = 128 ** -0.5 * 2.0 ** -18
    c = check(c8, 0, tokens, scale=scale)
    alone = Call(c8, 0, c.q.cpu(), [0, 0, 0], scale=scale, most=tokens[1])
    alone.q, alone.out = c.q[tokens[0]:].contiguous(), alone.out[tokens[0]:].contiguous()
    alone.cu[2] = tokens[1]
    alone.run()
    both = [x[-tokens[1]:].double().cpu() for x in (alone.out, c.out)]
    assert int(alone.status) == 0
    assert float((both[0] - both[1]).norm() / both[1].norm()) <= 2.0 ** -9  # (each: half a step of fp16 a weight and an output)


def test_later_rows_do_not_show(cuda):
    """Rows that only the last token sees, of K and of V, at the largest scale; NaN among others that no token but the last sees."""
    for byte, code in ((136, 0x7e), (200, 0x70), (247, 0x7e), (140, 0x7f)):
        tokens = [70, 3]
        c8 = cache(4, [90, 128], tokens, 16, Hkv=2)
        cu, q = inputs(c8, tokens, 2)
        want, size = quant.attention(c8, 0, q, cu)
        for h in range(4):
            r = c8.cache.rows(h)[-1]
            c8.V8[r, ::3], c8.Vs[r], c8.Ks[r] = code, byte, min(byte, 220)
        c8.sync()
        x = Call(c8, 0, q, cu).run()
        others = [i for i in range(73) if i not in (69, 72)]
        quant.assert_attention(x.out[others], want[others], size[others], HALF)
        assert int(x.status) == 0


def test_bad_pages_among_them(cuda):
    """Their rows are zeros, with scores of 0, in units that are computed again too."""
    tokens = [40, 2]
    c8 = cache(4, [100, 100], tokens, 16)
    c8.Ks[some(c8, 0.5, 2)] += 18
    at = c8.cache.rows(0)[16:32]
    c8.K8[at], c8.V8[at] = 0, 0
    c8.sync()
    cu, q = inputs(c8, tokens, 1)
    scale = 128 ** -0.5 * 2.0 ** -18
    want, size = quant.attention(c8, 0, q, cu, scale=scale)
    for page in (-1, 1 << 30):
        c = Call(c8, 0, q, cu, scale=scale)
        c.table[0, 1] = page
        c.run()
        assert int(c.status) != 0
        quant.assert_attention(c.out, want, size, HALF)


def test_repeats_are_bit_exact(cuda):
    tokens = [3, 70]
    c8 = cache(8, [12003, 300], tokens)
    c8.Ks[some(c8, 0.01, 3)] += 18
    c8.sync()
    cu, q = inputs(c8, tokens, 3)
    c = Call(c8, 0, q, cu, scale=2.0 ** -22).run()
    first = c.out.clone()
    for _ in range(3):
        c.out.fill_(float("nan"))
        c.work.fill_(0xff)
        assert torch.equal(c.run().out, first)
