"""Frequencies of rotary positions, and what the calls over rotary positions and 8-bit pages refuse: they answer without a GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

import quant

A = 1 << 20  # an address that no check follows


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


def radians(rotary):
    n = rotary.c.rot_dim // 2
    assert all(t == 0 for t in rotary.c.turns[n:])
    return np.array([t * 2.0 ** -64 * 2 * math.pi for t in rotary.c.turns[:n]])


@pytest.mark.parametrize("rot", [16, 32, 64, 96, 128])
@pytest.mark.parametrize("theta", [1.0, 10000.0, 5e5])
def test_frequencies(dkv, rot, theta):
    i = np.arange(rot // 2)
    f = theta ** (-2 * i / rot)
    # 2^-64 of a turn, and double precision
    close = dict(rtol=1e-14, atol=2.0 ** -64 * 7)
    np.testing.assert_allclose(radians(dkv.dkv_rotary_make(rot, theta)), f, **close)
    np.testing.assert_allclose(radians(dkv.dkv_rotary_make(rot, theta, scaling="linear", factor=2.5)), f / 2.5, **close)
    r = dkv.dkv_rotary_make(rot, theta, interleaved=True, scaling="ntk", factor=4)
    np.testing.assert_allclose(radians(r), (theta * 4 ** (rot / (rot - 2))) ** (-2 * i / rot), **close)
    assert r.c.interleaved == 1 and r.c.magnitude == 1
    wave = 2 * math.pi / f
    low, high, C, s = 1.0, 4.0, 8192, 8.0
    k = (C / wave - low) / (high - low)
    want = np.where(wave < C / high, f, np.where(wave > C / low, f / s, (1 - k) * f / s + k * f))
    np.testing.assert_allclose(radians(dkv.dkv_rotary_make(rot, theta, scaling="bands", factor=s, context=C, low=low, high=high)),
                               want, rtol=1e-13, atol=2.0 ** -64 * 7)


def test_yarn(dkv):
    rot, theta, s, C, low, high = 128, 10000.0, 16.0, 4096, 1.0, 32.0
    r = dkv.dkv_rotary_make(rot, theta, scaling="yarn", factor=s, context=C, low=low, high=high)
    # the pair that turns n times within C tokens
    pair = lambda n: rot * math.log(C / (n * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    i0, i1 = math.floor(pair(high)), math.ceil(pair(low))
    assert (i0, i1) == (20, 46)
    i = np.arange(rot // 2)
    f = theta ** (-2 * i / rot)
    ramp = np.clip((i - i0) / (i1 - i0), 0, 1)
    np.testing.assert_allclose(radians(r), f / s * ramp + f * (1 - ramp), rtol=1e-13)
    assert abs(r.c.magnitude - (0.1 * math.log(s) + 1)) < 1e-7


def test_custom_frequencies(dkv):
    f = np.array([0.0, 1.0, -1.0, 2 * math.pi, -1e-300, 1e5, 3.0, 1048575.0])
    r = dkv.dkv_rotary_custom(f, interleaved=True, magnitude=-0.5)
    got = radians(r)
    assert (r.c.rot_dim, r.c.interleaved, r.c.magnitude) == (16, 1, -0.5)
    # (the quotient by 2 pi is a double: 2^-53 of it)
    away = np.abs((got - f + math.pi) % (2 * math.pi) - math.pi)
    assert (away <= 1e-15 * (1 + np.abs(f))).all()


@pytest.mark.parametrize("kw,word", [
    (dict(rot_dim=8), "rot_dim"), (dict(rot_dim=144), "rot_dim"), (dict(rot_dim=24), "rot_dim"), (dict(rot_dim=0), "rot_dim"),
    (dict(theta=0.0), "theta"), (dict(theta=float("nan")), "theta"), (dict(theta=float("inf")), "theta"),
    (dict(scaling="other"), "scaling"), (dict(scaling="linear", factor=0.5), "factor"),
    (dict(scaling="ntk", factor=float("nan")), "factor"),
    (dict(scaling="bands", factor=2, context=0, low=1, high=4), "context"),
    (dict(scaling="bands", factor=2, context=10, low=4, high=4), "high"),
    (dict(scaling="yarn", factor=2, context=10, low=0, high=4), "low"),
    (dict(scaling="yarn", factor=2, context=10, low=1, high=4, theta=1.0), "theta"),
])
def test_bad_rotaries(dkv, kw, word):
    refused(dkv, word, dkv.dkv_rotary_make, **kw)


def test_bad_frequencies(dkv):
    for f in ([1.0] * 7, [1.0] * 72, [], [float("nan")] * 8, [float("inf")] * 8, [2.0 ** 20] * 8):
        refused(dkv, "rot_dim|freq", dkv.dkv_rotary_custom, f)
    refused(dkv, "magnitude", dkv.dkv_rotary_custom, [1.0] * 8, magnitude=float("inf"))
    refused(dkv, "magnitude", dkv.dkv_rotary_custom, [1.0] * 8, magnitude=1e39)
    lib = dkv.lib()
    assert lib.dkv_rotary_custom(None, 16, 0, A, 1.0) == dkv.DKV_ERR_INVALID_ARG
    assert lib.dkv_rotary_make(None, 16, 0, 1e4, 0, 1.0, 0, 0.0, 0.0) == dkv.DKV_ERR_INVALID_ARG
    assert lib.dkv_rotary_make(ctypes.byref(dkv.dkv_rotary()), 16, 0, 1e4, 7, 1.0, 0, 0.0, 0.0) == dkv.DKV_ERR_INVALID_ARG


def rope(dkv, rotary=None, **kw):
    r = rotary or dkv.dkv_rotary_make()
    a = dict(dtype=0, T=4, heads=2, x=A, xs=256, pos=A, out=2 * A, os=256, status=None) | kw
    return dkv.lib().dkv_rope(r.ref if r else None, a["dtype"], a["T"], a["heads"], a["x"], a["xs"], a["pos"], a["out"], a["os"],
                              a["status"], None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(T=-1), dict(heads=0), dict(status=A + 2), dict(T=1 << 30, heads=2), dict(x=None), dict(x=A + 8), dict(out=None),
                                dict(pos=None), dict(pos=A + 2), dict(xs=128), dict(xs=260), dict(os=128), dict(xs=1 << 40),
                                dict(out=A, os=512), dict(out=A + 256), dict(out=A - 256)])
def test_rope_refuses(dkv, kw):
    assert rope(dkv, **kw) == dkv.DKV_ERR_INVALID_ARG
    assert dkv.lib().dkv_last_error()


def test_rope_of_nothing_and_of_a_bad_rotary(dkv):
    assert rope(dkv, T=0) == dkv.DKV_OK
    for field, value in (("rot_dim", 130), ("rot_dim", 20), ("magnitude", float("nan"))):
        r = dkv.dkv_rotary_make()
        setattr(r.c, field, value)
        assert rope(dkv, r) == dkv.DKV_ERR_INVALID_ARG


def append(dkv, g=None, **kw):
    g = g or dkv.Pages(L=2, B=2, H=8, H_kv=2, page_rows=16, num_pages=4, max_pages=4)
    a = dict(layer=1, rotary=dkv.dkv_rotary_make(), dtype=1, T=3, pos=A, q=A, qs=1024, qo=2 * A, os=1024, k=3 * A, v=4 * A, ks=256,
             cu=A, table=A, len=A, Kp=5 * A, Vp=6 * A, Ks=7 * A, Vs=8 * A, status=A) | kw
    return dkv.lib().dkv_rope_append(g.ref, a["layer"], a["rotary"].ref if a["rotary"] else None, a["dtype"], a["T"], a["pos"], a["q"],
                                     a["qs"], a["qo"], a["os"], a["k"], a["v"], a["ks"], a["cu"], a["table"], a["len"], a["Kp"], a["Vp"],
                                     a["Ks"], a["Vs"], a["status"], None)


@pytest.mark.parametrize("kw", [dict(layer=2), dict(layer=-1), dict(dtype=3), dict(T=-1), dict(T=1 << 28), dict(pos=None), dict(pos=A + 1),
                                dict(rotary=None), dict(q=None), dict(qo=None), dict(k=None), dict(v=None), dict(Ks=None), dict(Vs=None),
                                dict(cu=None), dict(table=None), dict(len=None), dict(Kp=None), dict(Vp=None), dict(cu=A + 2),
                                dict(table=A + 1), dict(len=A + 3), dict(status=A + 1), dict(q=A + 8), dict(qo=A + 4), dict(k=A + 2),
                                dict(v=A + 8), dict(Kp=A + 8), dict(Vp=A + 8), dict(Ks=A + 8), dict(Vs=A + 8), dict(qs=1016), dict(qs=1028),
                                dict(os=1000), dict(ks=128), dict(ks=260), dict(Vp=5 * A), dict(Vs=7 * A), dict(qo=A + 2048),
                                dict(qo=A, os=2048)])
def test_append_refuses(dkv, kw):
    assert append(dkv, **kw) == dkv.DKV_ERR_INVALID_ARG
    assert dkv.lib().dkv_last_error()


def test_append_of_nothing(dkv):
    assert append(dkv, T=0) == dkv.DKV_OK
    assert append(dkv, q=None, qo=None, k=None, v=None) == dkv.DKV_OK


def test_bad_geometry(dkv):
    g = dkv.Pages(L=1, B=1, H=9, H_kv=1, page_rows=16, num_pages=4, max_pages=4)
    assert append(dkv, g, layer=0) == dkv.DKV_ERR_INVALID_ARG
    refused(dkv, "group size", dkv.dkv_quant_workspace_bytes, g)
    assert dkv.dkv_quant_workspace_bytes(dkv.Pages(L=1, B=1, H=8, H_kv=1, page_rows=16, num_pages=4, max_pages=4)) > 0


def attn(dkv, **kw):
    g = dkv.Pages(L=2, B=2, H=8, H_kv=2, page_rows=16, num_pages=4, max_pages=4)
    a = dict(layer=1, dtype=0, T=3, most=0, q=A, qs=1024, cu=A, table=A, len=A, Kp=A, Vp=A, Ks=A, Vs=A, scale=0.0, out=A, work=A,
             bytes=dkv.dkv_quant_workspace_bytes(g), status=A) | kw
    return dkv.lib().dkv_quant_attn(g.ref, a["layer"], a["dtype"], a["T"], a["most"], a["q"], a["qs"], a["cu"], a["table"], a["len"],
                                    a["Kp"], a["Vp"], a["Ks"], a["Vs"], 1, a["scale"], a["out"], a["work"], a["bytes"], a["status"], None)


@pytest.mark.parametrize("kw", [dict(layer=2), dict(dtype=2), dict(T=-1), dict(T=1 << 28), dict(q=None), dict(q=A + 8), dict(qs=1016), dict(qs=1025),
                                dict(cu=None), dict(cu=A + 1), dict(table=None), dict(len=None), dict(Kp=None), dict(Vp=A + 8), dict(Ks=None),
                                dict(Vs=A + 1), dict(out=None), dict(out=A + 4), dict(work=None), dict(work=A + 8), dict(bytes=100),
                                dict(status=A + 2), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38),
                                dict(dtype=1, scale=2e38)])
def test_attention_refuses(dkv, kw):
    assert attn(dkv, **kw) == dkv.DKV_ERR_INVALID_ARG
    assert dkv.lib().dkv_last_error()


def test_attention_of_nothing(dkv):
    assert attn(dkv, T=0) == dkv.DKV_OK


def test_the_binding_refuses_other_types_shapes_and_hosts(dkv):
    g = dkv.Pages(L=1, B=1, H=2, H_kv=1, page_rows=16, num_pages=4, max_pages=4)
    x = torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    r = dkv.dkv_rotary_make()
    refused(dkv, "float32", dkv.dkv_rope, x.float(), A, r, x, stream=0)
    refused(dkv, "dimensions", dkv.dkv_rope, x[0], A, r, x, stream=0)
    refused(dkv, "x must be a CUDA", dkv.dkv_rope, x, A, r, x, stream=0)
    refused(dkv, "x must be a CUDA", dkv.dkv_rope, 5, A, r, x, stream=0)
    refused(dkv, "q must be a CUDA", dkv.dkv_rope_append, g, 0, x, None, None, A, A, A, A, A, A, x, rotary=r, stream=0)
    refused(dkv, "q_out", dkv.dkv_rope_append, g, 0, x, None, None, A, A, A, A, A, A, None, rotary=r, stream=0)
    refused(dkv, "without q", dkv.dkv_rope_append, g, 0, None, None, None, A, A, A, A, A, A, None, rotary=r, stream=0)
    refused(dkv, "q must be a CUDA", dkv.dkv_quant_attn, g, 0, x, A, A, A, A, A, A, A, A, A, stream=0)
    refused(dkv, "int16", dkv.dkv_quant_attn, g, 0, x.view(torch.int16), A, A, A, A, A, A, A, A, A, stream=0)


def compact(dkv, K, V, **kw):
    from types import SimpleNamespace
    g = dkv.Pages(L=1, B=1, H=2, H_kv=1, page_rows=16, num_pages=4, max_pages=4)
    plan = SimpleNamespace(shape=dkv.Shape(L=1, H=2, H_kv=1, D=1), B=1, address=A)
    return dkv.dkv_quant_compact(g, plan, K, V, A, A, A, A, A, A, stream=0, **kw)


def test_compact_refuses_other_types(dkv):
    rows = {t: torch.zeros((1, 1, 1, 40, 128), dtype=t) for t in (torch.bfloat16, torch.float16, torch.float32, torch.int16)}
    BF, H = rows[torch.bfloat16], rows[torch.float16]
    for K, V, word in ((rows[torch.float32], BF, "float32"), (BF, rows[torch.int16], "int16"), (BF, H, "different types"),
                       (BF, BF[..., :10, :], "elements"), (BF, BF, "CUDA tensor"), (None, BF, "K must"), (BF, 7, "V must")):
        if word == "elements":
            refused(dkv, word, compact, dkv, K, V, T_stride=40)
        else:
            refused(dkv, word, compact, dkv, K, V)


def test_compact_refuses_in_c(dkv):
    """(A plan needs a GPU: what is checked before it.)"""
    g = dkv.Pages(L=1, B=1, H=2, H_kv=1, page_rows=16, num_pages=4, max_pages=4)
    call = dkv.lib().dkv_quant_compact
    assert call(g.ref, None, None, 0, A, A, 1, A, A, A, A, A, A, None, None) == dkv.DKV_ERR_INVALID_ARG
    assert call(g.ref, None, None, 5, A, A, 1, A, A, A, A, A, A, None, None) == dkv.DKV_ERR_INVALID_ARG
    assert call(None, None, None, 0, A, A, 1, A, A, A, A, A, A, None, None) == dkv.DKV_ERR_INVALID_ARG


def test_the_definition_of_8_bits_here():
    """The host's own e4m3 rounding against torch's, at every tie and in between, and scales at their borders."""
    grid = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    mid = (grid[1:] + grid[:-1]) / 2
    x = np.concatenate([grid, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9), np.random.default_rng(1).uniform(-448, 448, 5000)])
    x = np.concatenate([x, -x]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(quant.codes_of(x), want)
    for e in (-130, -126, -20, 0, 7, 119):
        u = quant.scale_bytes([[448 * 2.0 ** e, -1e-45], [np.nextafter(448 * 2.0 ** e, 1e300), np.inf], [np.nan, -448.0 * 2.0 ** e]])
        assert u.tolist() == [max(e, -126) + 127, max(e + 1, -126) + 127, max(e, -126) + 127]
