"""What the binding of the paged cache refuses before a call is made: it answers without a GPU."""
from types import SimpleNamespace

import pytest
import torch

BF, HALF, I16 = torch.bfloat16, torch.float16, torch.int16


@pytest.fixture(scope="module")
def dkv():
    from paper_2609_32663_gb300 import build
    build.build_library()
    import paper_2609_32663_gb300.dkv as dkv
    return dkv


def refused(dkv, word, call, *args, **kw):
    with pytest.raises(dkv.DkvError, match=word) as e:
        call(*args, **kw)
    assert e.value.status == dkv.DKV_ERR_INVALID_ARG


def compact_args(dkv, K=BF, V=BF, Kp=BF, Vp=BF):
    g = dkv.Pages(L=1, B=1, H=2, H_kv=1, page_rows=16, num_pages=4, max_pages=4)
    plan = SimpleNamespace(shape=dkv.Shape(L=1, H=2, H_kv=1, D=1), B=1, address=1 << 20)
    i = torch.zeros(4, dtype=torch.int32)
    return [g, plan, torch.zeros((1, 1, 1, 40, 128), dtype=K), torch.zeros((1, 1, 1, 40, 128), dtype=V), i, i[:1],
            torch.zeros((64, 128), dtype=Kp), torch.zeros((64, 128), dtype=Vp)]


@pytest.mark.parametrize("types", [(HALF, HALF, BF, BF), (BF, HALF, BF, BF), (BF, BF, BF, HALF), (I16, I16, BF, HALF),
                                   (HALF, BF, HALF, BF), (torch.float32, BF, BF, BF)])
def test_rows_of_another_type_are_not_packed(dkv, types):
    refused(dkv, "different types", dkv.dkv_page_compact, *compact_args(dkv, *types), stream=0)


@pytest.mark.parametrize("types", [(BF,) * 4, (HALF,) * 4, (I16, I16, BF, BF), (HALF, HALF, I16, I16), (I16,) * 4])
def test_rows_of_one_type_pass_that_check(dkv, types):
    """The next check refuses them, as they lie on the host."""
    refused(dkv, "CUDA tensor", dkv.dkv_page_compact, *compact_args(dkv, *types), stream=0)


def test_what_is_no_tensor_is_refused(dkv):
    """An address where a size, shape or type is needed, nothing, or an array of the host."""
    import numpy as np
    g, plan, K, V, table, ln, Kp, Vp = compact_args(dkv)
    q = torch.zeros((1, 2, 128), dtype=BF)
    for what in (1 << 20, None, np.zeros(1 << 16, np.uint8)):
        name = type(what).__name__
        refused(dkv, f"workspace .*{name}", dkv.dkv_page_release, g, A, A, A, A, A, A, A, what, stream=0)
        refused(dkv, f"workspace .*{name}", dkv.dkv_page_tables, g, A, A, A, A, A, A, what, tokens=A, stream=0)
        refused(dkv, f"K .*{name}", dkv.dkv_page_compact, g, plan, what, V, table, ln, Kp, Vp, stream=0)
        refused(dkv, f"q .*{name}", dkv.dkv_chunk_attn, g, 0, what, None, None, A, A, A, A, A, A, None, stream=0)
    refused(dkv, "K .*ndarray", dkv.dkv_page_compact, g, plan, np.zeros(1), V, table, ln, Kp, Vp, T_stride=40, stream=0)
    refused(dkv, "q ", dkv.dkv_chunk_attn, g, 0, q, None, None, A, A, A, A, A, A, A, stream=0)


A = 1 << 20  # an address that no check follows


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are none: a launch must not follow them")
@pytest.mark.parametrize("name", ["page table", "page release", "chunk attention"])
def test_an_injected_launch_failure_is_told_from_others(dkv, monkeypatch, name):
    """Without a GPU every launch fails: only with the fault does the message say that it is the injected one."""
    import ctypes
    g, L = dkv.Pages(L=1, B=1, H=2, H_kv=1, page_rows=16, num_pages=4, max_pages=4), dkv.lib()
    call = {
        "page table": lambda: L.dkv_page_tables(g.ref, A, None, None, A, A, A, A, A, A, None, None, 0, A, 1 << 20, None, None),
        "page release": lambda: L.dkv_page_release(g.ref, A, A, A, A, A, A, A, A, 1 << 20, None, None),
        "chunk attention": lambda: L.dkv_chunk_attn(g.ref, 0, 0, 1, A, 256, None, None, 0, A, A, A, A, 2 * A, 1,
                                                    ctypes.c_float(0), 3 * A, A, 1 << 40, None, None),
    }[name]
    for fault in (False, True):
        monkeypatch.setenv("DKV_FAULT", "launch") if fault else monkeypatch.delenv("DKV_FAULT", raising=False)
        assert call() == dkv.DKV_ERR_CUDA
        said = L.dkv_last_error().decode()
        assert name.split()[0] in said and ("injected launch failure" in said) == fault


@pytest.mark.parametrize("kw", [dict(L=2**31 - 1, B=512, H=2**31 - 1, H_kv=2**31 - 1), dict(L=2**20, B=512, H=2**20, H_kv=2**20),
                                dict(L=1, B=512, H=2**17 + 1, H_kv=2**17 + 1), dict(L=2**20 + 1, B=1, H=1, H_kv=1)])
def test_a_geometry_of_too_many_slabs_is_named(dkv, kw):
    """Factors whose product passes 64 bits among them."""
    g = dkv.Pages(**kw, page_rows=16, num_pages=4, max_pages=4)
    refused(dkv, f"L={kw['L']} B={kw['B']} H_kv={kw['H_kv']}", dkv.dkv_page_workspace_bytes, g)
