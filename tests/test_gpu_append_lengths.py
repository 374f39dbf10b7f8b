"""dkv_rope_append with lengths out of range on the device, negative ones among them: their rows are skipped and reported, the other
sequences' are written."""
import pytest

from paper_2609_32663_gb300 import build, dkv
from test_gpu_bounds_build import _child
from test_gpu_rope import Append, lens_of

pytestmark = pytest.mark.gpu

INT_MIN, INT_MAX = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("tokens", [[2, 1, 2], [2, 3, 2], [1, 700, 5]])
@pytest.mark.parametrize("length", [INT_MIN, INT_MIN + 1, INT_MIN + 2, INT_MIN + 3, INT_MIN + 700, -700, -1, INT_MAX, INT_MAX - 1])
def test_lengths_out_of_range(cuda, bits, tokens, length):
    """A 32-bit n - behind of n near -2^31 is large and positive."""
    a = Append(lens_of(1, 3, 2, [40, 50, 60], tokens, 1), 16, tokens, H=4, bits=bits)
    a.len[2:4] = length  # (both slabs of sequence 1)
    a.run(0).check(0, skip=(1,))
    assert int(a.status) == dkv.DKV_DEV_PAGE_RANGE


def test_the_bounds_checked_build_finds_nothing(cuda):
    """Its kernels set DKV_DEV_BOUNDS for a place that is out of range."""
    rc, out = _child(build.build_library(debug=True), ["tests/test_gpu_append_lengths.py::test_lengths_out_of_range"])
    assert rc == 0, out[-3000:]
