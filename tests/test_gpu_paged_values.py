"""What the paged cache's calls do with values on the device that are out of range: offsets, lengths and page numbers
that no check on the host sees. Nothing is followed, the status word says so, and what is in range keeps its results."""
import numpy as np
import pytest
import torch

import paged
from paper_2609_32663_gb300 import dkv
from test_gpu_chunk import Call, inputs, lens_of

pytestmark = pytest.mark.gpu


def bits(t):
    return t.view(torch.int16).clone()


@pytest.mark.parametrize("append", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cu", [
    [4, 6, 9, 79], [1, 1, 1, 1], [-2, 2, 5, 75], [0, 5, 2, 75], [0, 2, 5, 83], [0, 2, 5, 1 << 30], [0, -1, 5, 75],
    [0, 2, 75, 5], [0, 2, 5, -(1 << 31)],
])
def test_bad_token_offsets_change_nothing(cuda, cu, dtype, append):
    """Offsets that do not start at 0 (a slice of a larger batch's), descend or pass the rows of the call."""
    tokens = [2, 3, 70]
    cache = paged.Cache(lens_of(1, 3, 2, [98, 300, 131], tokens, 1), 16, H=8, dtype=dtype)
    good, qkv = inputs(cache, tokens, 3, pad=7)
    c = Call(cache, 0, qkv, cu, append=append)
    before = bits(c.Kp), bits(c.Vp), bits(c.out)
    c.run()
    assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE
    for got, old in zip((c.Kp, c.Vp, c.out), before):
        assert torch.equal(bits(got), old)
    # The same buffers with offsets that hold.
    c.cu.copy_(torch.from_numpy(good))
    c.status.zero_()
    c.run()
    k, v = (qkv[1], qkv[2]) if append else (None, None)
    want, size, _, _ = paged.attention(cache, 0, qkv[0], k, v, good, True)
    assert int(c.status) == 0
    paged.assert_attention(c.out, want, size, dtype)


def test_bad_token_offsets_of_many_slots(cuda):
    """The pair that breaks the order lies behind the CTA's first 384 slots."""
    tokens = [1] * 512
    cache = paged.Cache(lens_of(1, 512, 1, [5] * 512, tokens, 1), 16, H=2)
    good, qkv = inputs(cache, tokens, 3)
    for at in (383, 384, 385, 511, 512):
        cu = good.copy()
        cu[at] += 600 if at == 512 else -2
        c = Call(cache, 0, qkv, cu)
        before = bits(c.Kp), bits(c.Vp), bits(c.out)
        c.run()
        assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE
        for got, old in zip((c.Kp, c.Vp, c.out), before):
            assert torch.equal(bits(got), old)


@pytest.mark.parametrize("over", [1, 2, 3, 100, -1])
def test_a_length_out_of_range_counts_as_empty(cuda, over):
    """A slab whose length passes its table (or is negative): none of its rows is written or read, though some of the
    new tokens' places would lie in the table."""
    tokens = [2, 3, 2]
    cache = paged.Cache(lens_of(1, 3, 1, [40, 61, 60], tokens, 1), 16, H=4, wider=0)
    cap = cache.pages.max_pages * 16
    assert cache.lens[1] == cap
    cu, qkv = inputs(cache, tokens, 3)
    want, size, Kp, Vp = paged.attention(cache, 0, *qkv, cu, True)
    c = Call(cache, 0, qkv, cu)
    c.len[1] = cap + over if over > 0 else over
    before = bits(c.Kp), bits(c.Vp)
    c.run()
    assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE
    mine = torch.from_numpy(cache.rows(1))
    for got, old in zip((c.Kp, c.Vp), before):
        assert torch.equal(bits(got)[mine], old[mine])
    assert not c.out[2:5].any()
    for t in (slice(0, 2), slice(5, 7)):
        paged.assert_attention(c.out[t], want[t], size[t], cache.dtype)
    for h in (0, 2):
        assert torch.equal(c.Kp.cpu()[cache.rows(h)].double(), Kp[cache.rows(h)])


def test_a_slab_shorter_than_its_new_tokens(cuda):
    """Tokens that the slab has no row for are skipped and reported, the others are placed."""
    tokens = [5, 1]
    cache = paged.Cache(np.array([[[3], [40]]]), 16, H=4)
    cu, qkv = inputs(cache, tokens, 3)
    c = Call(cache, 0, qkv, cu).run()
    assert int(c.status) == dkv.DKV_DEV_PAGE_RANGE
    Kp = cache.Kp.clone()
    Kp[cache.rows(0)] = qkv[1][2:5, 0]
    Kp[cache.rows(1)[-1]] = qkv[1][5, 0]
    assert torch.equal(bits(c.Kp.cpu()), bits(Kp))
