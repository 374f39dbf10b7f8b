"""dkv_quant_attn at the ends of its ranges: V of the least scales, and products of q and the softmax scale that pass fp32's range
by themselves."""
import pytest
import torch

import quant
from test_gpu_chunk import lens_of
from test_gpu_quant import Call, check, inputs

pytestmark = pytest.mark.gpu

TOKENS = [[1], [1, 3], [4, 1], [2, 40]]  # 4 heads a group: kernels of 8 and 16 columns, and of many beside one of 8


def cache(tokens, ctx, **kw):
    return quant.Cache8(lens_of(1, len(tokens), 2, [ctx] * len(tokens), tokens, 3), 16, H=8, **kw)


@pytest.mark.parametrize("byte", [1, 2, 5, 8, 10])
@pytest.mark.parametrize("tokens", TOKENS)
@pytest.mark.parametrize("ctx", [3, 150, 5000])
def test_values_of_the_least_scales(cuda, byte, tokens, ctx):
    """All rows of V at 2^(byte - 127). An output is off by half a step, 2^-8 of it (eps / 2: 8 bits of significand), or by 2^-134
    below 2^-126, as bf16's least step is 2^-133; so is each element of V in products of bf16, and their mean at most as much."""
    c8 = cache(tokens, ctx)
    held = c8.Vs != 255
    c8.Vs[held] = byte
    c8.sync()
    cu, q = inputs(c8, tokens, 1)
    c = Call(c8, 0, q, cu, most=max(tokens)).run()
    want, size = quant.attention(c8, 0, q, cu)
    weights = quant.weight_rounding(tokens, 4, q.dtype, q.shape[0], max(tokens))
    got = c.out.double().cpu()
    bound = torch.finfo(q.dtype).eps / 2 * want.abs() * (1 + 1e-3) + (weights + 4e-4) * size + 2 * 2.0 ** -134
    assert int(c.status) == 0
    err = ((got - want).abs() / bound).max()
    assert float(err) <= 1, f"{float(err):.3g} times the bound"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens", TOKENS)
@pytest.mark.parametrize("size,scale", [(0.0, 2.0 ** -30), (0.0, 1e-38), (0.0, 1e-45), (2.0 ** -14, 1e-45), (1.0, 1e-45), (2.0 ** -120, 2.0 ** -40)])
def test_scores_that_vanish(cuda, dtype, tokens, size, scale):
    """Scores of nearly 0: the output is the mean of the rows of V that are seen."""
    c8 = cache(tokens, 70, dtype=dtype)
    _, q = inputs(c8, tokens, 2)
    check(c8, 0, tokens, most=max(tokens), scale=scale, q=(q.double() * size).to(dtype))


@pytest.mark.parametrize("tokens", TOKENS)
def test_some_queries_of_zeros(cuda, tokens):
    """Beside others in the same call, with a small scale."""
    c8 = cache(tokens, 70)
    _, q = inputs(c8, tokens, 2)
    q[0, ::2] = 0
    q[-1, 1::3] = 0
    check(c8, 0, tokens, most=max(tokens), scale=2.0 ** -26, q=q)


@pytest.mark.parametrize("tokens", TOKENS)
def test_large_queries_and_scale(cuda, tokens):
    """Their product passes fp32's range; K is 0 in all rows, and so are the scores."""
    c8 = cache(tokens, 70)
    held = c8.Ks != 255
    c8.K8[held], c8.Ks[held] = 0, 1
    c8.sync()
    _, q = inputs(c8, tokens, 2)
    check(c8, 0, tokens, most=max(tokens), scale=2.0 ** 20, q=(q.double().sign() * 2.0 ** 127).to(q.dtype))
