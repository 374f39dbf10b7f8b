"""Where dkv_rope and dkv_rope_append may read and write: other heads of the tokens that are read, as their rows do not overlap, and
heads whose elements pass 32 bits."""
import numpy as np
import pytest
import torch

import quant
from paper_2609_32663_gb300 import dkv
from test_gpu_rope import Append, dev, frequencies, lens_of, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("src,dst", [((0, 3), (3, 6)), ((4, 7), (0, 3)), ((1, 4), (6, 9)), ((6, 9), (5, 6))])
@pytest.mark.parametrize("T", [1, 2, 700])
def test_other_heads_of_a_projection(cuda, src, dst, T):
    n = min(src[1] - src[0], dst[1] - dst[0])
    src = (src[0], src[0] + n)
    x, f = randn((T, 9, 128), torch.bfloat16, T), frequencies(128)
    d = x.cuda()
    pos = np.arange(T) + 5
    dkv.dkv_rope(d[:, src[0]:src[1]], dev(pos), dkv.dkv_rotary_make(), d[:, dst[0]:dst[1]])
    want, size = quant.turned(x[:, src[0]:src[1]], pos, f, False)
    quant.assert_turned(d[:, dst[0]:dst[1]], want, size, x.dtype)
    others = [h for h in range(9) if not dst[0] <= h < dst[1]]
    assert torch.equal(d[:, others].cpu(), x[:, others])


def test_other_tokens_between(cuda):
    """Every other token's row is read, those between are written."""
    x, f = randn((40, 2, 128), torch.float16, 1), frequencies(128)
    d = x.cuda()
    dkv.dkv_rope(d[::2], dev(np.arange(20)), dkv.dkv_rotary_make(), d[1::2])
    want, size = quant.turned(x[::2], np.arange(20), f, False)
    quant.assert_turned(d[1::2], want, size, x.dtype)
    assert torch.equal(d[::2].cpu(), x[::2])


def test_append_to_other_heads(cuda):
    tokens = [4, 9]
    a = Append(lens_of(1, 2, 2, [20, 0], tokens, 2), 16, tokens, H=4, pad=1)
    wide = torch.full((14, 8, 128), float("nan"), dtype=a.dtype, device="cuda")
    wide[:, 2:6] = a.q
    a.q, a.out = wide[:, 2:6], wide[:, 6:]
    with pytest.raises(dkv.DkvError, match="q_out"):  # (another number of heads)
        a.run(0)
    wide = torch.full((14, 8, 128), float("nan"), dtype=a.dtype, device="cuda")
    wide[:, 4:] = a.q
    a.q, a.out = wide[:, 4:], wide[:, :4]
    a.run(0).check(0)
    assert int(a.status) == 0
    assert torch.equal(a.q.cpu(), a.host[0])


def test_rows_that_overlap_are_refused(cuda):
    d = torch.zeros((40, 8, 128), dtype=torch.bfloat16, device="cuda")
    r = dkv.dkv_rotary_make()
    for x, out in ((d[:, :3], d[:, 2:5]), (d[:, 2:5], d[:, :3]), (d[:-1, :4], d[1:, :4]), (d[1:, 5:], d[:-1, 4:7]), (d[:-1, 6:], d.view(-1, 128)[7:7 + 39 * 8].view(39, 8, 128)[:, :2]),
                   (d[:20, :2], d[::2, :2]), (d[::2, :4], d[:20, 4:])):
        with pytest.raises(dkv.DkvError, match="overlap"):
            dkv.dkv_rope(x, dev(np.arange(x.shape[0])), r, out)


def test_heads_whose_elements_pass_32_bits(cuda):
    """One token of 2^24 + 57 heads, in place: as 2^24 + 57 tokens of one head at the same position."""
    heads = 2 ** 24 + 57
    x = torch.randn((64, 128), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    d = x.repeat(heads // 64 + 1, 1)[:heads].unsqueeze(0)
    d[0, -50:] *= 3
    want = torch.empty((64 + 50, 1, 128), dtype=d.dtype, device="cuda")
    r = dkv.dkv_rotary_make()
    dkv.dkv_rope(torch.cat([x, d[0, -50:]]).unsqueeze(1), dev(np.full(114, 1234567)), r, want)
    dkv.dkv_rope(d, dev([1234567]), r, d)
    torch.cuda.synchronize()
    n = (heads - 50) // 64
    assert (d[0, :64 * n].view(n, 64, 128) == want[:64, 0]).all()
    assert torch.equal(d[0, 64 * n:-50], want[:heads - 50 - 64 * n, 0]) and torch.equal(d[0, -50:], want[64:, 0])
