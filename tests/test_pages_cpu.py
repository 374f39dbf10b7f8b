"""Argument checks of the paged cache's entry points: they answer without a GPU."""
import ctypes

import numpy as np
import pytest


@pytest.fixture(scope="module")
def dkv():
    from paper_2609_32663_gb300 import build
    build.build_library()
    import paper_2609_32663_gb300.dkv as dkv
    return dkv


def geometry(dkv, **kw):
    return dkv.Pages(**{**dict(L=2, B=3, H=8, H_kv=2, page_rows=16, num_pages=50, max_pages=9), **kw})


def test_workspace_sizes(dkv):
    g = geometry(dkv)
    assert dkv.dkv_page_workspace_bytes(g) >= 8 * g.slabs
    assert dkv.dkv_chunk_workspace_bytes(g) > 0


@pytest.mark.parametrize("kw", [
    dict(L=0), dict(B=0), dict(B=513), dict(H=7), dict(H=18), dict(H_kv=0), dict(head_dim=64), dict(page_rows=8),
    dict(page_rows=48), dict(page_rows=256), dict(num_pages=0), dict(num_pages=1 << 27), dict(max_pages=0),
    dict(max_pages=1 << 27, page_rows=16), dict(max_pages=(1 << 27) - 1, page_rows=16), dict(L=1 << 20, B=512),
])
def test_bad_geometry(dkv, kw):
    for f in (dkv.dkv_page_workspace_bytes, dkv.dkv_chunk_workspace_bytes):
        with pytest.raises(dkv.DkvError) as e:
            f(geometry(dkv, **kw))
        assert e.value.status == dkv.DKV_ERR_INVALID_ARG


# Addresses that the checks look at and no check follows.
A = 1 << 20


def tables_args(**kw):
    d = dict(tokens=A, plan=None, seq=None, len=A, new_len=A, table=A, free=A, count=A, new_count=A, cu=A, slots=A, most=10,
             work=A, bytes=1 << 20, status=None)
    d.update(kw)
    return list(d.values())


def refused(dkv, status, word):
    assert status == dkv.DKV_ERR_INVALID_ARG
    assert word in dkv.lib().dkv_last_error().decode()


@pytest.mark.parametrize("kw,word", [
    (dict(len=None), "NULL"), (dict(new_len=None), "NULL"), (dict(table=None), "NULL"), (dict(free=None), "NULL"),
    (dict(count=None), "NULL"), (dict(new_count=None), "NULL"), (dict(table=A + 2), "aligned"), (dict(status=A + 1), "aligned"),
    (dict(work=None), "workspace"), (dict(work=A + 8), "workspace"), (dict(bytes=100), "workspace"),
    (dict(tokens=None), "exactly one"), (dict(cu=None), "needs cu_tokens"), (dict(most=-1), "max_tokens"),
    (dict(most=1 << 31), "max_tokens"), (dict(cu=A + 2), "aligned"),
])
def test_tables_refusals(dkv, kw, word):
    g = geometry(dkv).c
    refused(dkv, dkv.lib().dkv_page_tables(ctypes.byref(g), *tables_args(**kw), None), word)


def test_release_refusals(dkv):
    g = geometry(dkv).c
    L = dkv.lib()
    refused(dkv, L.dkv_page_release(ctypes.byref(g), None, A, A, A, A, A, A, A, 1 << 20, None, None), "ended")
    refused(dkv, L.dkv_page_release(ctypes.byref(g), A, A, A, None, A, A, A, A, 1 << 20, None, None), "NULL")
    refused(dkv, L.dkv_page_release(None, A, A, A, A, A, A, A, A, 1 << 20, None, None), "pages is NULL")


def test_compact_refusals(dkv):
    g = geometry(dkv).c
    refused(dkv, dkv.lib().dkv_page_compact(ctypes.byref(g), None, None, A, A, 10, A, A, A, A, None, None), "plan is NULL")


def chunk_args(**kw):
    d = dict(layer=0, dtype=0, tokens=4, q=A, qs=8 * 128, k=A, v=A, ks=2 * 128, cu=A, table=A, len=A, Kp=A, Vp=2 * A, causal=1,
             scale=0.0, out=3 * A, work=A, bytes=1 << 40, status=None)
    d.update(kw)
    d["scale"] = ctypes.c_float(d["scale"])
    return list(d.values())


@pytest.mark.parametrize("kw,word", [
    (dict(layer=2), "layer"), (dict(layer=-1), "layer"), (dict(dtype=2), "dtype"), (dict(tokens=-1), "num_tokens"),
    (dict(tokens=1 << 30), "num_tokens"), (dict(q=None), "NULL"), (dict(cu=None), "NULL"), (dict(table=None), "NULL"),
    (dict(len=None), "NULL"), (dict(Kp=None), "NULL"), (dict(out=None), "NULL"), (dict(k=None), "both"), (dict(v=None), "both"),
    (dict(q=A + 8), "aligned"), (dict(k=A + 4), "aligned"), (dict(Vp=A + 2), "aligned"), (dict(out=A + 8), "aligned"),
    (dict(Vp=A), "different"), (dict(qs=8 * 128 - 8), "q_stride"), (dict(qs=8 * 128 + 4), "q_stride"), (dict(ks=128), "kv_stride"),
    (dict(ks=2 * 128 + 1), "kv_stride"), (dict(scale=float("nan")), "scale"), (dict(work=None), "workspace"),
    (dict(bytes=8), "workspace"), (dict(work=A + 4), "workspace"), (dict(status=A + 2), "aligned"),
])
def test_chunk_refusals(dkv, kw, word):
    g = geometry(dkv).c
    refused(dkv, dkv.lib().dkv_chunk_attn(ctypes.byref(g), *chunk_args(**kw), None), word)


def test_chunk_without_tokens_does_nothing(dkv):
    g = geometry(dkv).c
    assert dkv.lib().dkv_chunk_attn(ctypes.byref(g), *chunk_args(tokens=0, q=None, out=None), None) == dkv.DKV_OK


def test_binding_refuses_host_tensors(dkv):
    import torch
    g = geometry(dkv)
    i = torch.zeros(g.slabs, dtype=torch.int32)
    t = torch.zeros((g.slabs, g.max_pages), dtype=torch.int32)
    f, one, w = torch.zeros(g.num_pages, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1 << 16, dtype=torch.uint8)
    for call in (
        lambda: dkv.dkv_page_tables(g, i, i, t, f, one, one, w, tokens=torch.zeros(3, dtype=torch.int32), stream=0),
        lambda: dkv.dkv_page_release(g, torch.zeros(3, dtype=torch.int32), i, i, t, f, one, one, w, stream=0),
        lambda: dkv.dkv_chunk_attn(g, 0, torch.zeros((4, 8, 128), dtype=torch.bfloat16), None, None,
                                   torch.zeros(4, dtype=torch.int32), t, i, None, None, None, w, stream=0),
        lambda: dkv.dkv_chunk_attn(g, 0, torch.zeros((4, 8, 128)), None, None, None, t, i, None, None, None, w, stream=0),
    ):
        with pytest.raises(dkv.DkvError) as e:
            call()
        assert e.value.status == dkv.DKV_ERR_INVALID_ARG


def test_injected_launch_failure(dkv, monkeypatch):
    """Reported as an error (here the launch also fails for want of a GPU)."""
    monkeypatch.setenv("DKV_FAULT", "launch")
    if not __import__("torch").cuda.is_available():
        g = geometry(dkv).c
        assert dkv.lib().dkv_page_tables(ctypes.byref(g), *tables_args(), None) == dkv.DKV_ERR_CUDA
        assert b"page table" in dkv.lib().dkv_last_error()


@pytest.mark.parametrize("scale", [3e38, float("inf"), float("-inf")])
def test_scale_past_the_base_2_softmax_is_refused(dkv, scale):
    """Its product with log2(e) is infinite: every score of 0 would give NaN."""
    g = geometry(dkv).c
    refused(dkv, dkv.lib().dkv_chunk_attn(ctypes.byref(g), *chunk_args(scale=scale), None), "scale")


def test_seq_without_a_plan_is_refused(dkv):
    g = geometry(dkv).c
    refused(dkv, dkv.lib().dkv_page_tables(ctypes.byref(g), *tables_args(seq=A), None), "seq")
