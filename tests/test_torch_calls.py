"""The compiled calls of dkv.py (csrc/dkv_torch.cpp): they do what the functions do by themselves, and leave to those whatever is
not as it should be."""
import ctypes
import gc

import numpy as np
import pytest
import torch

import quant
from paper_2609_32663_gb300 import build, dkv


@pytest.fixture(scope="module")
def calls():
    build.build_library()
    if build.build_torch_calls() is None:
        pytest.skip("no headers of Python or torch")
    module = dkv._torch_calls(torch.__version__)
    assert module is not None
    return module


@pytest.fixture(autouse=True)
def no_frames_left():
    """What was raised holds its frames' tensors until a collection, which other tests' looks at memory would see."""
    yield
    gc.collect()


def test_what_is_not_as_it_should_be_is_left_alone(calls):
    """Nothing is called (the entry point's address is none) and nothing raised, by objects of any kind at every place."""
    g = dkv.Pages(L=1, B=1, H=2, H_kv=1, page_rows=16, num_pages=4, max_pages=4)
    r = dkv.dkv_rotary_make()
    x = torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    lists = {"rope": [0, 0, None, r.at, x, i, x, None],
             "rope_append": [0, 0, None, g.at, 0, r.at, x, x, x, i, i, i, i, x, x, x, None, None, None],
             "quant_compact": [0, 0, None, g.at, 0, None, 1, 1, 1, x, x, 1, i, i, x, x, x, x, None],
             "quant_attn": [0, 0, None, g.at, 0, x, i, i, i, i, i, i, i, x, i, True, 0.0, 0, None]}
    for name, good in lists.items():
        f = getattr(calls, name)
        assert f(*good) is None and f(*good[:-1]) is None and f() is None  # (host tensors)
        hosts = {"rope": (2, 3), "rope_append": (2, 3, 5), "quant_compact": (2, 3, 4), "quant_attn": (2, 3)}[name]  # addresses: dkv.py's own
        for at in range(1, len(good)):
            for odd in (None, 1 << 80, "x", 0.5, object(), torch.zeros(2, 2).to_sparse(), torch.nn.Parameter(torch.zeros(3))):
                if at not in hosts:
                    assert f(*good[:at], odd, *good[at + 1:]) is None


def both(monkeypatch, run):
    """run() with the compiled calls and without."""
    T = dkv._torch()
    assert T.calls is not None
    first = run()
    with monkeypatch.context() as m:
        m.setattr(T, "calls", None)
        second = run()
    return first, second


def told(run):
    try:
        run()
    except (dkv.DkvError, TypeError, ctypes.ArgumentError) as e:
        return f"{type(e).__name__}: {e}"
    return "nothing"


class Spy:
    """The compiled calls, and how many of them answered."""

    def __init__(self, calls):
        self.calls, self.answered = calls, 0

    def __getattr__(self, name):
        def call(*a):
            s = getattr(self.calls, name)(*a)
            self.answered += s is not None
            return s
        return call


def make(dtype, bits, seed=0):
    """Arguments of a step's two calls on the GPU: two sequences, 3 and 1 tokens, a padded one, q and K, V slices of a projection."""
    c8 = quant.Cache8(np.array([[[40, 23], [9, 64]]]), 16, H=6, dtype=dtype)
    p, gen = c8.pages, torch.Generator().manual_seed(seed)
    qkv = torch.randn((5, 6 + 2 * 2, 128), generator=gen).to(dtype).cuda()
    dev = lambda x: torch.as_tensor(np.asarray(x)).to(torch.int32).cuda()
    n = p.num_pages * p.page_rows
    pools = [x.cuda() for x in (c8.K8, c8.V8)] if bits == 8 else [torch.zeros((n, 128), dtype=dtype, device="cuda") for _ in "KV"]
    scales = [x.cuda() for x in (c8.Ks, c8.Vs)]
    a = dict(pages=p, layer=0, q=qkv[:, :6], k_new=qkv[:, 6:8], v_new=qkv[:, 8:], positions=dev([5, 6, 7, 80, 0]), cu_tokens=dev([0, 3, 4]),
             table=dev(c8.cache.table), len=dev(c8.cache.lens), Kp=pools[0], Vp=pools[1], q_out=torch.zeros((5, 6, 128), dtype=dtype, device="cuda"),
             rotary=dkv.dkv_rotary_make(), status=dev([0]))
    if bits == 8:
        a.update(Ks=scales[0], Vs=scales[1])
    b = {k: a[k] for k in ("pages", "layer", "cu_tokens", "table", "len", "status", "Kp", "Vp")} | dict(
        q=a["q_out"], Ks=scales[0], Vs=scales[1], out=torch.zeros((5, 6, 128), dtype=dtype, device="cuda"),
        workspace=torch.zeros(dkv.dkv_quant_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    return a, b


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [8, 16])
def test_the_same_results(cuda, calls, monkeypatch, dtype, bits):
    spy = Spy(calls)
    monkeypatch.setattr(dkv._torch(), "calls", spy)

    def run():
        a, b = make(dtype, bits)
        got = [torch.zeros((5, 6, 128), dtype=dtype, device="cuda")]
        dkv.dkv_rope(a["q"], a["positions"], a["rotary"], got[0])
        dkv.dkv_rope_append(**a)
        dkv.dkv_rope_append(**a | dict(q=None, q_out=None, rotary=None, positions=None))
        dkv.dkv_rope_append(**a | dict(k_new=None, v_new=None))
        if bits == 8:
            dkv.dkv_quant_attn(**b)
            dkv.dkv_quant_attn(**b | dict(max_tokens=3, causal=False, scale=0.05, q=a["q"]))
        torch.cuda.synchronize()
        return got + [a[k] for k in ("q_out", "Kp", "Vp", "status")] + [b["Ks"], b["Vs"], b["out"]]

    first, second = both(monkeypatch, run)
    assert spy.answered == (6 if bits == 8 else 4)
    for x, y in zip(first, second):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.gpu
def test_the_same_refusals(cuda, calls, monkeypatch):
    a, b = make(torch.bfloat16, 8)
    wide = torch.zeros((5, 12, 128), dtype=torch.bfloat16, device="cuda")
    odd = {"host": lambda t: t.cpu(), "type": lambda t: t.to(torch.float64), "short": lambda t: t[:-1], "long": lambda t: torch.cat([t, t]),
           "apart": lambda t: torch.cat([t, t], -1)[..., ::2], "list": lambda t: [1], "flat": lambda t: t.reshape(-1, 1)}
    for args, call in ((a, dkv.dkv_rope_append), (b, dkv.dkv_quant_attn)):
        for name in args:
            if not isinstance(args[name], torch.Tensor) or name == "status":
                continue
            for kind, f in odd.items():
                bad = dict(args)
                bad[name] = f(args[name])
                first, second = both(monkeypatch, lambda: told(lambda: call(**bad)))
                assert first == second, (call.__name__, name, kind)
                # (a shape of as many elements is none, and a smaller q has other tokens)
                assert first != "nothing" or kind in ("flat", "apart", "type", "short", "long"), (call.__name__, name, kind)
        for more in (dict(layer=1), dict(layer=-1), dict(layer=1 << 40), dict(status=torch.zeros(1, device="cuda")), dict(pages=dkv.Pages(1, 2, 6, 2, 24, 9, 9))):
            first, second = both(monkeypatch, lambda: told(lambda: call(**args | more)))
            assert first == second, (call.__name__, more)
    for more in (dict(rotary=5), dict(k_new=None), dict(q_out=None), dict(Ks=None), dict(k_new=wide[:, :2]), dict(positions=None), dict(q=wide[:, ::2])):
        first, second = both(monkeypatch, lambda: told(lambda: dkv.dkv_rope_append(**a | more)))
        assert first == second != "nothing", more
    for more in (dict(workspace=b["workspace"][:100]), dict(scale=float("nan")), dict(scale=None), dict(max_tokens=None), dict(workspace=None)):
        first, second = both(monkeypatch, lambda: told(lambda: dkv.dkv_quant_attn(**b | more)))
        assert first == second != "nothing", more
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_compact_both_ways(cuda, calls, monkeypatch):
    from test_gpu_quant import packed
    plan, cache, _, K, V, _ = packed(2, 8, 2, 4, [251, 3, 100], [0, 2, 3], 16, torch.float16, 1)
    K, V, rows = K.cuda(), V.cuda(), cache.pages.num_pages * 16
    dev = lambda x: torch.as_tensor(np.asarray(x)).to(torch.int32).cuda()
    table, lens, seq, status = dev(cache.table), dev(cache.lens), dev([0, 2, 3]), dev([0])
    spy = Spy(calls)
    monkeypatch.setattr(dkv._torch(), "calls", spy)

    def run(**kw):
        pools = [torch.zeros((rows, 128), dtype=torch.uint8, device="cuda") for _ in "KV"] + [torch.zeros(rows, dtype=torch.uint8, device="cuda") for _ in "KV"]
        a = dict(K=K, V=V, table=table, len=lens, seq=seq, status=status, Ks=pools[2], Vs=pools[3]) | kw
        dkv.dkv_quant_compact(cache.pages, plan, Kp=pools[0], Vp=pools[1], **a)
        torch.cuda.synchronize()
        return pools

    first, second = both(monkeypatch, run)
    assert spy.answered == 1 and all(torch.equal(x, y) for x, y in zip(first, second)) and int(status) == 0 and first[2].any()
    first, second = both(monkeypatch, lambda: run(T_stride=K.shape[-2]))
    assert spy.answered == 2 and all(torch.equal(x, y) for x, y in zip(first, second))
    for bad in (dict(K=K[:1]), dict(K=K.bfloat16()), dict(V=V.transpose(0, 1)), dict(T_stride=1 << 20), dict(T_stride=0), dict(seq=seq[:2]), dict(table=table.float()),
                dict(K=K.cpu()), dict(Ks=None)):
        first, second = both(monkeypatch, lambda: told(lambda: run(**bad)))
        assert first == second != "nothing", bad.keys()
    plan.close()
    assert "freed" in told_value(lambda: run())


def told_value(run):
    with pytest.raises(ValueError) as e:
        run()
    return str(e.value)
