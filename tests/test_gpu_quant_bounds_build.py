"""The bounds-checked build (libdkv_debug.so) over the suites of rotary positions and the 8-bit cache: their kernels check the
places that they compute themselves, skip one that is outside and set DKV_DEV_BOUNDS in the call's status word. The suites
compare that word with what each call should report, so a bit that is set fails them."""
import pytest

from test_gpu_bounds_build import _child

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("suite", ["rope", "quant"])
def test_bounds_checked_build_passes_the_suites(cuda, suite):
    from paper_2609_32663_gb300 import build
    rc, out = _child(build.build_library(debug=True), [f"tests/test_gpu_{suite}.py"])
    assert rc == 0, out[-3000:]
