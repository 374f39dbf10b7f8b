"""Thin Python binding of the C ABI in include/dkv.h (libdkv.so).

Argument marshalling only: each function takes torch tensors (device buffers)
or numpy arrays (host inputs), passes raw pointers, sizes and the current CUDA
stream to the function of the same name in libdkv.so, and raises DkvError on a
non-zero status. Every step of the path runs in the library's CUDA kernels;
there is no Python or CPU fallback, and importing the functions fails loudly
when libdkv.so has not been built.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from functools import cached_property

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
# DKV_LIBRARY names another build of the same ABI to load instead, e.g. the
# bounds-checked libdkv_debug.so (build.build_library(debug=True)).
LIB_PATH = os.environ.get("DKV_LIBRARY") or os.path.join(_PKG, "libdkv.so")

DKV_OK, DKV_ERR_INVALID_ARG, DKV_ERR_CUDA, DKV_ERR_OOM, DKV_ERR_RANGE, DKV_ERR_TIMEOUT = range(6)
DKV_DEV_APPEND_OVERFLOW = 0x1
DKV_DEV_TMA_TIMEOUT = 0x2
DKV_DEV_MERGE_TIMEOUT = 0x4
DKV_DEV_BOUNDS = 0x8
DKV_DEV_PAGES_EXHAUSTED = 0x10
DKV_DEV_PAGE_RANGE = 0x20
DKV_BF16, DKV_FP16 = 0, 1

# Every entry point include/dkv.h declares.
EXPORTS = ("dkv_last_error", "dkv_map_pattern", "dkv_plan_dense", "dkv_plan_query", "dkv_plan_read",
           "dkv_compact", "dkv_decode_attn", "dkv_decode_partial", "dkv_decode_combine", "dkv_advance",
           "dkv_plan_status", "dkv_free", "dkv_decode_attn_noalloc", "dkv_budget", "dkv_topk_workspace_bytes",
           "dkv_topk_mask", "dkv_decode_multi", "dkv_map_pattern_inplace", "dkv_compact_inplace",
           "dkv_vmm_alloc", "dkv_vmm_trim", "dkv_vmm_pages_to_keep", "dkv_vmm_mapped_bytes", "dkv_vmm_page_bytes",
           "dkv_vmm_free", "dkv_page_workspace_bytes", "dkv_page_tables", "dkv_page_release", "dkv_page_compact",
           "dkv_chunk_workspace_bytes", "dkv_chunk_attn", "dkv_rotary_make", "dkv_rotary_custom", "dkv_rope", "dkv_rope_append",
           "dkv_quant_compact", "dkv_quant_workspace_bytes", "dkv_quant_attn")
DKV_ROPE_NONE, DKV_ROPE_LINEAR, DKV_ROPE_NTK, DKV_ROPE_BANDS, DKV_ROPE_YARN = range(5)


class DkvError(RuntimeError):
    def __init__(self, status, func, msg):
        super().__init__(f"{func} failed with status {status}: {msg}")
        self.status = status


class dkv_shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("L", "H", "H_kv", "D", "head_dim", "sink", "recent", "bin_width")]


@dataclass(frozen=True)
class Shape:
    """Model and pattern geometry (dkv_shape)."""
    L: int
    H: int
    H_kv: int
    D: int
    head_dim: int = 128
    sink: int = 128
    recent: int = 1024
    bin_width: int = 128

    def c(self):
        return dkv_shape(self.L, self.H, self.H_kv, self.D, self.head_dim, self.sink, self.recent,
                         self.bin_width)

    @property
    def G(self):
        return self.H // self.H_kv


class dkv_pages(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("L", "B", "H", "H_kv", "head_dim", "page_rows", "num_pages", "max_pages")]


@dataclass(frozen=True)
class Pages:
    """Geometry of a paged cache (dkv_pages): B sequence slots, pools of num_pages pages of page_rows rows, tables of
    max_pages entries a slab."""
    L: int
    B: int
    H: int
    H_kv: int
    page_rows: int
    num_pages: int
    max_pages: int
    head_dim: int = 128

    @cached_property
    def c(self):
        return dkv_pages(self.L, self.B, self.H, self.H_kv, self.head_dim, self.page_rows, self.num_pages, self.max_pages)

    @cached_property
    def ref(self):
        return ctypes.byref(self.c)

    @cached_property
    def at(self):
        return ctypes.addressof(self.c)

    @cached_property
    def slabs(self):
        return self.L * self.B * self.H_kv


class dkv_rotary(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("magnitude", ctypes.c_float),
                ("reserved", ctypes.c_int32), ("turns", ctypes.c_uint64 * 64)]


class Rotary:
    """Layout and frequencies of rotary positions (dkv_rotary), from dkv_rotary_make or dkv_rotary_custom."""

    def __init__(self):
        self.c = dkv_rotary()
        self.ref = ctypes.byref(self.c)
        self.at = ctypes.addressof(self.c)


_lib = None
_entry = {}  # addresses of the loaded library's entry points that csrc/dkv_torch.cpp calls


def lib(path: str | None = None):
    """Load libdkv.so (once) and declare its signatures."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is missing: build it with paper_2609_32663_gb300.build.build_library() "
                           "(or __graft_entry__.build()); there is no fallback path")
    L = ctypes.CDLL(p)
    V, I32, I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    PP = ctypes.POINTER(ctypes.c_void_p)
    L.dkv_last_error.restype = ctypes.c_char_p
    L.dkv_last_error.argtypes = []
    L.dkv_map_pattern.restype = ctypes.c_int
    L.dkv_map_pattern.argtypes = [V, V, I32, ctypes.POINTER(dkv_shape), I32, V, PP]
    L.dkv_map_pattern_inplace.restype = ctypes.c_int
    L.dkv_map_pattern_inplace.argtypes = [V, V, I32, ctypes.POINTER(dkv_shape), I32, I64, V, PP]
    L.dkv_compact_inplace.restype = ctypes.c_int
    L.dkv_compact_inplace.argtypes = [V, V, V, V]
    L.dkv_vmm_alloc.restype = ctypes.c_int
    L.dkv_vmm_alloc.argtypes = [I64, PP, PP]
    L.dkv_vmm_trim.restype = ctypes.c_int
    L.dkv_vmm_trim.argtypes = [V, V, I32, ctypes.POINTER(I64)]
    L.dkv_vmm_pages_to_keep.restype = None
    L.dkv_vmm_pages_to_keep.argtypes = [V, I64, I64, I32, I32, I64, I64, I64, V]
    L.dkv_vmm_mapped_bytes.restype = I64
    L.dkv_vmm_mapped_bytes.argtypes = [V]
    L.dkv_vmm_page_bytes.restype = I64
    L.dkv_vmm_page_bytes.argtypes = [V]
    L.dkv_vmm_free.restype = None
    L.dkv_vmm_free.argtypes = [V]
    L.dkv_plan_dense.restype = ctypes.c_int
    L.dkv_plan_dense.argtypes = [V, I32, ctypes.POINTER(dkv_shape), I64, V, PP]
    L.dkv_plan_query.restype = ctypes.c_int
    L.dkv_plan_query.argtypes = [V, ctypes.POINTER(I64), ctypes.POINTER(I64), PP, PP, PP, PP]
    L.dkv_plan_read.restype = ctypes.c_int
    L.dkv_plan_read.argtypes = [V, V, V, V, V, V]
    L.dkv_compact.restype = ctypes.c_int
    L.dkv_compact.argtypes = [V, V, V, I64, V, V, V]
    L.dkv_decode_attn.restype = ctypes.c_int
    L.dkv_decode_attn.argtypes = [V, I32, V, V, V, V, V, V, ctypes.c_float, V, V]
    L.dkv_decode_multi.restype = ctypes.c_int
    L.dkv_decode_multi.argtypes = [V, I32, V, I32, V, V, V, ctypes.c_float, V, V]
    L.dkv_decode_partial.restype = ctypes.c_int
    L.dkv_decode_partial.argtypes = [V, I32, V, V, V, V, V, V, ctypes.c_float, V]
    L.dkv_decode_combine.restype = ctypes.c_int
    L.dkv_decode_combine.argtypes = [V, I32, V, I32, V, V]
    L.dkv_advance.restype = ctypes.c_int
    L.dkv_advance.argtypes = [V, V, V]
    L.dkv_plan_status.restype = ctypes.c_int
    L.dkv_plan_status.argtypes = [V, ctypes.POINTER(I32), I32, V]
    L.dkv_decode_attn_noalloc.restype = ctypes.c_int
    L.dkv_decode_attn_noalloc.argtypes = [ctypes.POINTER(dkv_shape), I32, I32, I32, V, V, V, V, V, V, V, V, V,
                                          ctypes.c_float, V, V, V]
    L.dkv_free.restype = None
    L.dkv_free.argtypes = [V]
    L.dkv_budget.restype = I64
    L.dkv_budget.argtypes = [ctypes.c_double, I32, I32, I32]
    L.dkv_topk_workspace_bytes.restype = I64
    L.dkv_topk_workspace_bytes.argtypes = []
    L.dkv_topk_mask.restype = ctypes.c_int
    L.dkv_topk_mask.argtypes = [V, I64, I64, V, V, I64, V]
    PG = ctypes.POINTER(dkv_pages)
    L.dkv_page_workspace_bytes.restype = I64
    L.dkv_page_workspace_bytes.argtypes = [PG]
    L.dkv_page_tables.restype = ctypes.c_int
    L.dkv_page_tables.argtypes = [PG, V, V, V, V, V, V, V, V, V, V, V, I64, V, I64, V, V]
    L.dkv_page_release.restype = ctypes.c_int
    L.dkv_page_release.argtypes = [PG, V, V, V, V, V, V, V, V, I64, V, V]
    L.dkv_page_compact.restype = ctypes.c_int
    L.dkv_page_compact.argtypes = [PG, V, V, V, V, I64, V, V, V, V, V, V]
    L.dkv_chunk_workspace_bytes.restype = I64
    L.dkv_chunk_workspace_bytes.argtypes = [PG]
    L.dkv_chunk_attn.restype = ctypes.c_int
    L.dkv_chunk_attn.argtypes = [PG, I32, I32, I32, V, I64, V, V, I64, V, V, V, V, V, I32, ctypes.c_float, V, V, I64, V, V]
    RT, F64 = ctypes.POINTER(dkv_rotary), ctypes.c_double
    L.dkv_rotary_make.restype = ctypes.c_int
    L.dkv_rotary_make.argtypes = [RT, I32, I32, F64, I32, F64, I32, F64, F64]
    L.dkv_rotary_custom.restype = ctypes.c_int
    L.dkv_rotary_custom.argtypes = [RT, I32, I32, V, F64]
    L.dkv_rope.restype = ctypes.c_int
    L.dkv_rope.argtypes = [RT, I32, I32, I32, V, I64, V, V, I64, V, V]
    L.dkv_rope_append.restype = ctypes.c_int
    L.dkv_rope_append.argtypes = [PG, I32, RT, I32, I32, V, V, I64, V, I64, V, V, I64, V, V, V, V, V, V, V, V, V]
    L.dkv_quant_compact.restype = ctypes.c_int
    L.dkv_quant_compact.argtypes = [PG, V, V, I32, V, V, I64, V, V, V, V, V, V, V, V]
    L.dkv_quant_workspace_bytes.restype = I64
    L.dkv_quant_workspace_bytes.argtypes = [PG]
    L.dkv_quant_attn.restype = ctypes.c_int
    L.dkv_quant_attn.argtypes = [PG, I32, I32, I32, I32, V, I64, V, V, V, V, V, V, V, I32, ctypes.c_float, V, V, I64, V, V]
    if path is None:
        _lib = L
        _entry.update({n: ctypes.cast(getattr(L, n), V).value for n in ("dkv_rope", "dkv_rope_append", "dkv_quant_compact", "dkv_quant_attn")})
    return L


def _address(name):
    """Address of an entry point."""
    lib()
    return _entry[name]


def _check(status, func):
    if status != DKV_OK:
        raise DkvError(status, func, lib().dkv_last_error().decode(errors="replace"))


def _ptr(t):
    """Device (torch) or host (numpy) buffer -> address; None -> NULL."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _dev(t, name, dtypes=None, numel=None, min_numel=None):
    """Address of a device buffer argument, checked: a contiguous CUDA tensor of
    the expected element type and size (an int is taken as a raw device address,
    None as NULL). A host tensor passed here would make the kernel read host
    addresses, so it is refused before the call."""
    if t is None or isinstance(t, int):
        return t
    if (getattr(t, "is_cuda", False) and t.is_contiguous() and (dtypes is None or t.dtype in dtypes)
            and (numel is None or t.numel() == numel) and (min_numel is None or t.numel() >= min_numel)):
        return t.data_ptr()
    if not getattr(t, "is_cuda", False):
        why = "must be a CUDA tensor"
    elif not t.is_contiguous():
        why = "must be contiguous"
    elif dtypes is not None and t.dtype not in dtypes:
        why = f"has dtype {t.dtype}, expected one of {dtypes}"
    elif numel is not None and t.numel() != numel:
        why = f"has {t.numel()} elements, expected {numel}"
    else:
        why = f"has {t.numel()} elements, needs at least {min_numel}"
    raise DkvError(DKV_ERR_INVALID_ARG, "argument check", f"{name} {why}")


# Element types of the buffer arguments, and torch's own lookup of the current
# stream: resolved once, on the first call that takes tensors (the binding can be
# imported without torch). Per call these were a third of the binding's time.
_T = None


class _Torch:
    def __init__(self):
        import torch
        self.torch = torch
        self.bf16 = (torch.bfloat16, torch.int16)
        self.i32 = (torch.int32,)
        self.f32 = (torch.float32,)
        self.u8 = (torch.uint8,)
        self.e4m3 = (torch.uint8, torch.float8_e4m3fn)
        self.e8m0 = (torch.uint8,) + ((torch.float8_e8m0fnu,) if hasattr(torch, "float8_e8m0fnu") else ())
        C = torch._C
        self.raw_stream = getattr(C, "_cuda_getCurrentRawStream", None)
        self.device = getattr(C, "_cuda_getDevice", None)
        self.calls = _torch_calls(torch.__version__)


def _torch_calls(version):
    """The module of csrc/dkv_torch.cpp, which looks at a call's tensors and makes it. None where it was not built of these
    sources, or does not load: the functions below do the same themselves."""
    from .build import torch_calls
    try:
        path = torch_calls(version)
    except OSError:  # (no sources here)
        return None
    if not os.path.exists(path):
        return None
    from importlib.machinery import ExtensionFileLoader
    from importlib.util import module_from_spec, spec_from_file_location
    spec = spec_from_file_location("dkv_torch", path, loader=ExtensionFileLoader("dkv_torch", path))
    try:
        module = module_from_spec(spec)
        spec.loader.exec_module(module)
    except (ImportError, OSError) as e:
        import warnings
        warnings.warn(f"{path} does not load, so that calls take longer on the host: {e}")
        return None
    return module


def _torch():
    global _T
    if _T is None:
        _T = _Torch()
    return _T


def _bf16():
    return _torch().bf16


def _i32():
    return _torch().i32


def _f32():
    return _torch().f32


def _stream(stream):
    if stream is None:
        t = _torch()
        if t.raw_stream is not None and t.torch.cuda.is_initialized():
            return t.raw_stream(t.device())
        if not t.torch.cuda.is_available():
            return None
        return t.torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


class Plan:
    """Owner of a dkv_plan*; dkv_free runs on close() or garbage collection."""

    def __init__(self, handle, shape: Shape, B: int, dense: bool):
        self.handle = handle
        self.shape = shape
        self.B = B
        self.dense = dense
        self._info = None  # dkv_plan_query's answer: a plan's sizes and addresses never change

    def close(self):
        if self.handle:
            lib().dkv_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def address(self) -> int:
        if not self.handle:
            raise ValueError("plan already freed")
        return self.handle

    @property
    def _as_parameter_(self):
        return ctypes.c_void_p(self.address)


def dkv_map_pattern(M, ctx_len, shape: Shape, reserve_rows: int = 0, stream=None) -> Plan:
    M = np.ascontiguousarray(M, dtype=np.uint8)
    ctx = np.ascontiguousarray(ctx_len, dtype=np.int32)
    out = ctypes.c_void_p()
    sh = shape.c()
    _check(lib().dkv_map_pattern(_ptr(M), _ptr(ctx), len(ctx), ctypes.byref(sh), int(reserve_rows),
                                 _stream(stream), ctypes.byref(out)), "dkv_map_pattern")
    return Plan(out.value, shape, len(ctx), False)


def dkv_map_pattern_inplace(M, ctx_len, shape: Shape, T_stride: int, reserve_rows: int = 0, stream=None) -> Plan:
    """dkv_map_pattern with every slab at the start of its own dense region (off[h] = h T_stride)."""
    M = np.ascontiguousarray(M, dtype=np.uint8)
    ctx = np.ascontiguousarray(ctx_len, dtype=np.int32)
    out = ctypes.c_void_p()
    sh = shape.c()
    _check(lib().dkv_map_pattern_inplace(_ptr(M), _ptr(ctx), len(ctx), ctypes.byref(sh), int(reserve_rows),
                                         int(T_stride), _stream(stream), ctypes.byref(out)), "dkv_map_pattern_inplace")
    return Plan(out.value, shape, len(ctx), False)


def dkv_compact_inplace(plan: Plan, K, V, stream=None):
    """Move each slab's kept rows to the start of its region of K and V (in place)."""
    need = dkv_plan_query(plan).total_rows * 128
    _check(lib().dkv_compact_inplace(plan, _dev(K, "K", _bf16(), min_numel=need), _dev(V, "V", _bf16(), min_numel=need),
                                     _stream(stream)), "dkv_compact_inplace")


class VmmBuffer:
    """A page-backed device buffer (dkv_vmm_alloc); .tensor(shape, dtype) views it as a torch tensor."""

    def __init__(self, nbytes: int):
        h, p = ctypes.c_void_p(), ctypes.c_void_p()
        _check(lib().dkv_vmm_alloc(int(nbytes), ctypes.byref(h), ctypes.byref(p)), "dkv_vmm_alloc")
        self.handle, self.ptr, self.nbytes = h.value, p.value, int(nbytes)

    @property
    def _as_parameter_(self):
        return ctypes.c_void_p(self.handle)

    def tensor(self, shape, dtype):
        import torch
        typestr = {torch.bfloat16: "<i2", torch.int16: "<i2", torch.float32: "<f4", torch.uint8: "|u1"}[dtype]
        n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        assert n <= self.nbytes

        class _View:
            __cuda_array_interface__ = {"shape": tuple(int(x) for x in shape), "typestr": typestr,
                                        "data": (self.ptr, False), "version": 3}
        t = torch.as_tensor(_View(), device="cuda")
        return t.view(torch.bfloat16) if dtype == torch.bfloat16 else t

    def trim(self, plan, guard_rows: int = 16) -> int:
        freed = ctypes.c_int64()
        _check(lib().dkv_vmm_trim(self, plan, int(guard_rows), ctypes.byref(freed)), "dkv_vmm_trim")
        return freed.value

    def mapped_bytes(self) -> int:
        return int(lib().dkv_vmm_mapped_bytes(self))

    def page_bytes(self) -> int:
        return int(lib().dkv_vmm_page_bytes(self))

    def close(self):
        if self.handle:
            lib().dkv_vmm_free(self)
            self.handle = None


def dkv_vmm_pages_to_keep(len_host, T_stride: int, reserve: int, guard_rows: int, page_bytes: int, npages: int,
                          row_bytes: int = 256) -> np.ndarray:
    ln = np.ascontiguousarray(len_host, np.int32)
    keep = np.zeros(max(npages, 1), np.uint8)
    lib().dkv_vmm_pages_to_keep(_ptr(ln), ln.size, int(T_stride), int(reserve), int(guard_rows), int(row_bytes),
                                int(page_bytes), int(npages), _ptr(keep))
    return keep[:npages]


def dkv_plan_dense(ctx_len, shape: Shape, T_stride: int, stream=None) -> Plan:
    ctx = np.ascontiguousarray(ctx_len, dtype=np.int32)
    out = ctypes.c_void_p()
    sh = shape.c()
    _check(lib().dkv_plan_dense(_ptr(ctx), len(ctx), ctypes.byref(sh), int(T_stride), _stream(stream),
                                ctypes.byref(out)), "dkv_plan_dense")
    return Plan(out.value, shape, len(ctx), True)


@dataclass
class PlanInfo:
    total_rows: int
    kept_rows: int
    d_len: int
    d_off: int
    d_ioff: int | None
    d_idx: int | None


def dkv_plan_query(plan: Plan) -> PlanInfo:
    tr, kr = ctypes.c_int64(), ctypes.c_int64()
    pl, po, pi, px = (ctypes.c_void_p() for _ in range(4))
    _check(lib().dkv_plan_query(plan, ctypes.byref(tr), ctypes.byref(kr), ctypes.byref(pl),
                                ctypes.byref(po), ctypes.byref(pi), ctypes.byref(px)), "dkv_plan_query")
    plan._info = PlanInfo(tr.value, kr.value, pl.value, po.value, pi.value, px.value)
    return plan._info


def dkv_compact(plan: Plan, K, V, Kc, Vc, T_stride: int | None = None, stream=None):
    if T_stride is None:
        T_stride = K.shape[-2]
    sh = plan.shape
    dense = sh.L * plan.B * sh.H_kv * int(T_stride) * 128
    packed = dkv_plan_query(plan).total_rows * 128
    _check(lib().dkv_compact(plan, _dev(K, "K", _bf16(), min_numel=dense), _dev(V, "V", _bf16(), min_numel=dense),
                             int(T_stride), _dev(Kc, "Kc", _bf16(), min_numel=packed),
                             _dev(Vc, "Vc", _bf16(), min_numel=packed), _stream(stream)), "dkv_compact")


def _decode_ptrs(plan: Plan, q, k_new, v_new, n_appended, Kc, Vc, Q: int = 1):
    sh, B, T = plan.shape, plan.B, _torch()
    plan.address  # a freed plan is refused before its sizes are used
    rows = (plan._info or dkv_plan_query(plan)).total_rows * 128
    return (_dev(q, "q", T.bf16, B * Q * sh.H * 128),
            _dev(k_new, "k_new", T.bf16, B * sh.H_kv * 128),
            _dev(v_new, "v_new", T.bf16, B * sh.H_kv * 128),
            _dev(n_appended, "n_appended", T.i32, B),
            _dev(Kc, "Kc", T.bf16, None, rows), _dev(Vc, "Vc", T.bf16, None, rows))


def dkv_decode_attn(plan: Plan, layer: int, q, k_new, v_new, n_appended, Kc, Vc, out, scale: float = 0.0,
                    stream=None):
    qp, kp, vp, np_, kc, vc = _decode_ptrs(plan, q, k_new, v_new, n_appended, Kc, Vc)
    op = _dev(out, "out", _f32(), numel=plan.B * plan.shape.H * 128)
    _check(lib().dkv_decode_attn(plan.address, int(layer), qp, kp, vp, np_, kc, vc, scale, op, _stream(stream)),
           "dkv_decode_attn")


def dkv_decode_multi(plan: Plan, layer: int, q, num_queries: int, n_appended, Kc, Vc, out, scale: float = 0.0,
                     stream=None):
    """num_queries queries per sequence over the same compressed rows: q bf16
    [B][Q][H][128] -> out fp32 [B][Q][H][128]."""
    Q = max(int(num_queries), 1)
    qp, _, _, np_, kc, vc = _decode_ptrs(plan, q, None, None, n_appended, Kc, Vc, Q=Q)
    op = _dev(out, "out", _f32(), numel=plan.B * Q * plan.shape.H * 128)
    _check(lib().dkv_decode_multi(plan.address, int(layer), qp, int(num_queries), np_, kc, vc, scale, op,
                                  _stream(stream)), "dkv_decode_multi")


def dkv_decode_partial(plan: Plan, layer: int, q, k_new, v_new, n_appended, Kc, Vc, scale: float = 0.0,
                       stream=None):
    qp, kp, vp, np_, kc, vc = _decode_ptrs(plan, q, k_new, v_new, n_appended, Kc, Vc)
    _check(lib().dkv_decode_partial(plan, int(layer), qp, kp, vp, np_, kc, vc, ctypes.c_float(scale),
                                    _stream(stream)), "dkv_decode_partial")


def dkv_decode_combine(plan: Plan, layer: int, n_appended, with_new_token: bool, out, stream=None):
    np_ = _dev(n_appended, "n_appended", _i32(), numel=plan.B)
    op = _dev(out, "out", _f32(), numel=plan.B * plan.shape.H * 128)
    _check(lib().dkv_decode_combine(plan, int(layer), np_, int(bool(with_new_token)), op, _stream(stream)),
           "dkv_decode_combine")


def dkv_advance(plan: Plan, n_appended, stream=None):
    _check(lib().dkv_advance(plan, _dev(n_appended, "n_appended", _i32(), numel=plan.B), _stream(stream)),
           "dkv_advance")


def dkv_plan_status(plan: Plan, clear: bool = False, stream=None) -> int:
    w = ctypes.c_int32()
    _check(lib().dkv_plan_status(plan, ctypes.byref(w), int(bool(clear)), _stream(stream)), "dkv_plan_status")
    return w.value


def dkv_free(plan: Plan):
    plan.close()


def dkv_budget(rho: float, L: int, H: int, D: int) -> int:
    """K_rho = round(rho L H D) (App. A.3); raises on bad arguments."""
    k = lib().dkv_budget(float(rho), int(L), int(H), int(D))
    if k < 0:
        raise DkvError(1, "dkv_budget", f"rho={rho} L={L} H={H} D={D}")
    return int(k)


def dkv_topk_workspace_bytes() -> int:
    return int(lib().dkv_topk_workspace_bytes())


def dkv_topk_mask(P, K: int, M, workspace, stream=None):
    """M (device uint8, same element count as P) = TopKMask(P, K) of Eq. 3."""
    import torch
    n = P.numel()
    pp = _dev(P, "P", _f32())
    mp = _dev(M, "M", (torch.uint8,), numel=n)
    wp = _dev(workspace, "workspace")
    nbytes = workspace.numel() * workspace.element_size()
    _check(lib().dkv_topk_mask(pp, int(n), int(K), mp, wp, int(nbytes), _stream(stream)), "dkv_topk_mask")


def dkv_decode_attn_noalloc(shape: Shape, B: int, layer: int, reserve_rows: int, d_len, d_off, d_ioff, q, k_new,
                            v_new, n_appended, Kc, Vc, out, scale: float = 0.0, status=None, stream=None):
    """Decode attention that allocates no device memory; d_len/d_off/d_ioff are
    device addresses (ints) or tensors of the plan metadata."""
    T = _torch()
    _check(lib().dkv_decode_attn_noalloc(
        ctypes.byref(shape.c()), int(B), int(layer), int(reserve_rows), _dev(d_len, "d_len"), _dev(d_off, "d_off"),
        _dev(d_ioff, "d_ioff"), _dev(q, "q", T.bf16, B * shape.H * 128),
        _dev(k_new, "k_new", T.bf16, B * shape.H_kv * 128), _dev(v_new, "v_new", T.bf16, B * shape.H_kv * 128),
        _dev(n_appended, "n_appended", T.i32, B), _dev(Kc, "Kc", T.bf16), _dev(Vc, "Vc", T.bf16),
        scale, _dev(out, "out", _f32(), numel=B * shape.H * 128), _dev(status, "status", _i32()),
        _stream(stream)), "dkv_decode_attn_noalloc")


def dkv_plan_read(plan: Plan, stream=None):
    """Host copies (numpy) of the plan's len, off, ioff and idx arrays."""
    info = dkv_plan_query(plan)
    NH = plan.shape.L * plan.B * plan.shape.H_kv
    ln = np.zeros(NH, np.int32)
    off = np.zeros(NH + 1, np.int64)
    ioff = np.zeros(NH + 1, np.int64)
    idx = np.zeros(max(info.kept_rows, 1), np.int32)
    _check(lib().dkv_plan_read(plan, _ptr(ln), _ptr(off), _ptr(ioff), _ptr(idx), _stream(stream)),
           "dkv_plan_read")
    if plan.dense:
        return ln, off, None, None
    return ln, off, ioff, idx[: info.kept_rows]


def _bad(why):
    raise DkvError(DKV_ERR_INVALID_ARG, "argument check", why)


def _where(stream):
    """The current device, where a call's buffers lie, and the stream it runs on."""
    T = _torch()
    if T.raw_stream is not None and T.device is not None and T.torch.cuda.is_initialized():
        at = T.device()
        return at, T.raw_stream(at) if stream is None else _stream(stream)
    return (T.torch.cuda.current_device() if T.torch.cuda.is_available() else 0), _stream(stream)


def _device_of(t, name):
    """The device of a tensor (-1: the host); what is none is refused."""
    try:
        return t.get_device()
    except AttributeError:
        _bad(f"{name} must be a CUDA tensor, not {type(t).__name__}")


def _on(t, name, at, dtypes, numel=None):
    """_dev for a buffer of the paged cache, which must lie on device `at` (the look-ups of t are the binding's time)."""
    if t is None or isinstance(t, int):
        return t
    try:
        if t.get_device() == at and t.is_contiguous() and t.dtype in dtypes and (numel is None or t.numel() == numel):
            return t.data_ptr()
    except AttributeError:
        pass
    if _device_of(t, name) != at and t.is_cuda:
        _bad(f"{name} lies on {t.device}, the current device is cuda:{at}")
    return _dev(t, name, dtypes, numel)


def _work(workspace, at):
    """Address and bytes (so an address alone will not do)."""
    if _device_of(workspace, "workspace") != at or not workspace.is_contiguous():
        _bad(f"workspace must be a contiguous tensor on cuda:{at}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _word(status, at):
    if status is None or isinstance(status, int):
        return status
    try:
        if status.get_device() == at and status.dtype is _T.torch.int32 and status.numel() == 1:
            return status.data_ptr()
    except AttributeError:
        pass
    _device_of(status, "status")
    if status.numel() < 1:
        _bad("status has no element")
    return _on(status, "status", at, _torch().i32)


def _one_type(names, *tensors):
    """Refuses tensors of 16-bit rows that are not of one type (int16, an address and None say nothing of it)."""
    types = {t.dtype for t in tensors if hasattr(t, "dtype")} - {_torch().torch.int16}
    if len(types) > 1:
        _bad(f"{names} are of different types: {sorted(map(str, types))}")


def _page_args(p: Pages, at, len, new_len, table, free_pages, free_count, new_count, workspace, status):
    i32, n = _torch().i32, p.slabs
    return ((_on(len, "len", at, i32, n), _on(new_len, "new_len", at, i32, n), _on(table, "table", at, i32, n * p.max_pages),
             _on(free_pages, "free_pages", at, i32, p.num_pages), _on(free_count, "free_count", at, i32, 1),
             _on(new_count, "new_count", at, i32, 1)), _work(workspace, at), _word(status, at))


def dkv_page_workspace_bytes(pages: Pages) -> int:
    n = int(lib().dkv_page_workspace_bytes(ctypes.byref(pages.c)))
    if n < 0:
        _check(DKV_ERR_INVALID_ARG, "dkv_page_workspace_bytes")
    return n


def dkv_page_tables(pages: Pages, len, new_len, table, free_pages, free_count, new_count, workspace, tokens=None,
                    plan: Plan | None = None, seq=None, cu_tokens=None, slots=None, status=None, stream=None):
    """Pages for tokens[b] new rows of every slab of slot b, or for a plan's kept rows (its sequence i to slot seq[i]);
    slots int32 [L][max_tokens][H_kv] receives the slot map, cu_tokens int32 [B + 1] the token offsets."""
    i32 = _torch().i32
    at, queue = _where(stream)
    (ln, nl, tb, fp, fc, nc), (wp, wb), st = _page_args(pages, at, len, new_len, table, free_pages, free_count, new_count,
                                                        workspace, status)
    most = 0
    if slots is not None:
        if isinstance(slots, int):
            _bad("slots must be a tensor: its size is the most tokens")
        most, rest = divmod(slots.numel(), pages.L * pages.H_kv)
        if rest:
            _bad(f"slots has {slots.numel()} elements, not a multiple of L*H_kv={pages.L * pages.H_kv}")
    _check(lib().dkv_page_tables(
        pages.ref, _on(tokens, "tokens", at, i32, pages.B), None if plan is None else plan.address,
        _on(seq, "seq", at, i32, None if plan is None else plan.B), ln, nl, tb, fp, fc, nc,
        _on(cu_tokens, "cu_tokens", at, i32, pages.B + 1), _on(slots, "slots", at, i32), most, wp, wb, st, queue),
        "dkv_page_tables")


def dkv_page_release(pages: Pages, ended, len, new_len, table, free_pages, free_count, new_count, workspace,
                     status=None, stream=None):
    """The pages of the slots with ended[b] != 0 go back to the free list."""
    at, queue = _where(stream)
    (ln, nl, tb, fp, fc, nc), (wp, wb), st = _page_args(pages, at, len, new_len, table, free_pages, free_count, new_count,
                                                        workspace, status)
    _check(lib().dkv_page_release(pages.ref, _on(ended, "ended", at, _torch().i32, pages.B), ln, nl, tb, fp, fc, nc, wp, wb,
                                  st, queue), "dkv_page_release")


def dkv_page_compact(pages: Pages, plan: Plan, K, V, table, len, Kp, Vp, seq=None, T_stride: int | None = None,
                     status=None, stream=None):
    """The kept rows of plan sequence i become the last rows of slot seq[i]'s slabs. Bytes are copied, so K, V, Kp and Vp
    are of one type (int16, like an address, says nothing of it)."""
    if T_stride is None:
        _device_of(K, "K (without T_stride)")
        T_stride = K.shape[-2]
    T, sh = _torch(), plan.shape
    at, queue = _where(stream)
    r16 = (*T.bf16, T.torch.float16)
    handle = plan.address
    dense = sh.L * plan.B * sh.H_kv * int(T_stride) * 128
    pool = pages.num_pages * pages.page_rows * 128
    for t, name in ((K, "K"), (V, "V")):
        if t is None or isinstance(t, int):
            continue
        _device_of(t, name)
        if t.numel() < dense:
            _bad(f"{name} has {t.numel()} elements, needs at least {dense}")
    _one_type("K, V, Kp and Vp", K, V, Kp, Vp)
    _check(lib().dkv_page_compact(
        pages.ref, handle, _on(seq, "seq", at, T.i32, plan.B), _on(K, "K", at, r16), _on(V, "V", at, r16), int(T_stride),
        _on(table, "table", at, T.i32, pages.slabs * pages.max_pages), _on(len, "len", at, T.i32, pages.slabs),
        _on(Kp, "Kp", at, r16, pool), _on(Vp, "Vp", at, r16, pool), _word(status, at), queue), "dkv_page_compact")


def dkv_chunk_workspace_bytes(pages: Pages) -> int:
    n = int(lib().dkv_chunk_workspace_bytes(ctypes.byref(pages.c)))
    if n < 0:
        _check(DKV_ERR_INVALID_ARG, "dkv_chunk_workspace_bytes")
    return n


def _token_rows(t, name, at, dtype, tokens, heads):
    """Address and token stride (elements) of a [tokens][heads][128] tensor whose tokens may lie apart (a slice of a
    projection); heads and elements are contiguous."""
    try:  # (what is right is found so; what is not is named below)
        if t.get_device() == at and t.dtype is dtype and t.shape == (tokens, heads, 128):
            stride = t.stride()
            if stride[2] == 1 and (stride[1] == 128 or heads == 1):
                return t.data_ptr(), stride[0] if tokens > 1 else heads * 128
    except AttributeError:
        pass
    if _device_of(t, name) != at:
        _bad(f"{name} must be a CUDA tensor on cuda:{at}")
    if t.dtype != dtype or t.shape != (tokens, heads, 128):
        _bad(f"{name} is {t.dtype} {tuple(t.shape)}, expected {dtype} {(tokens, heads, 128)}")
    stride = t.stride()
    if stride[2] != 1 or (heads > 1 and stride[1] != 128):
        _bad(f"{name}: heads and elements of a token must be contiguous")
    return t.data_ptr(), stride[0] if tokens > 1 else heads * 128


def dkv_chunk_attn(pages: Pages, layer: int, q, k_new, v_new, cu_tokens, table, len, Kp, Vp, out, workspace,
                   causal: bool = True, scale: float = 0.0, status=None, stream=None):
    """One layer's new tokens: k_new and v_new [T][H_kv][128] appended to their slabs' pages (None: they are there), and
    the attention of q [T][H][128] -> out [T][H][128], all of q's type (bf16 or fp16). q, k_new and v_new may be slices of
    one projection; k_new and v_new have the same token stride."""
    _device_of(q, "q")
    T, dtype = _torch(), q.dtype
    at, queue = _where(stream)
    half = dtype == T.torch.float16
    if not (half or dtype == T.torch.bfloat16) or q.dim() != 3:
        _bad(f"q is {dtype} of {q.dim()} dimensions, expected bfloat16 or float16 [T][H][128]")
    tokens, one = q.shape[0], (dtype,)
    qp, qs = _token_rows(q, "q", at, dtype, tokens, pages.H)
    kp = vp = None
    ks = 0
    if k_new is not None and v_new is not None:
        kp, ks = _token_rows(k_new, "k_new", at, dtype, tokens, pages.H_kv)
        vp, vs = _token_rows(v_new, "v_new", at, dtype, tokens, pages.H_kv)
        if ks != vs:
            _bad(f"k_new and v_new have token strides {ks} and {vs}")
    elif k_new is not None or v_new is not None:
        _bad("k_new and v_new must both be given or both be None")
    pool = pages.num_pages * pages.page_rows * 128
    wp, wb = _work(workspace, at)
    _check(lib().dkv_chunk_attn(
        pages.ref, int(layer), DKV_FP16 if half else DKV_BF16, tokens, qp, qs, kp, vp, ks,
        _on(cu_tokens, "cu_tokens", at, T.i32, pages.B + 1), _on(table, "table", at, T.i32, pages.slabs * pages.max_pages),
        _on(len, "len", at, T.i32, pages.slabs), _on(Kp, "Kp", at, one, pool), _on(Vp, "Vp", at, one, pool),
        1 if causal else 0, scale, _on(out, "out", at, one, tokens * pages.H * 128), wp, wb, _word(status, at),
        queue), "dkv_chunk_attn")


_SCALINGS = {"none": DKV_ROPE_NONE, "linear": DKV_ROPE_LINEAR, "ntk": DKV_ROPE_NTK, "bands": DKV_ROPE_BANDS, "yarn": DKV_ROPE_YARN}


def dkv_rotary_make(rot_dim: int = 128, theta: float = 10000.0, interleaved: bool = False, scaling: str = "none",
                    factor: float = 1.0, context: int = 0, low: float = 0.0, high: float = 0.0) -> Rotary:
    """Rotary positions of the first rot_dim elements, f_i = theta^(-2i / rot_dim), scaled for a long context: "none",
    "linear", "ntk", "bands" or "yarn"."""
    if scaling not in _SCALINGS:
        _bad(f"scaling is {scaling!r}, expected one of {sorted(_SCALINGS)}")
    r = Rotary()
    _check(lib().dkv_rotary_make(r.ref, int(rot_dim), 1 if interleaved else 0, float(theta), _SCALINGS[scaling], float(factor),
                                 int(context), float(low), float(high)), "dkv_rotary_make")
    return r


def dkv_rotary_custom(freq, interleaved: bool = False, magnitude: float = 1.0) -> Rotary:
    """Rotary positions with these frequencies (radians a position, one a pair)."""
    f = np.ascontiguousarray(freq, dtype=np.float64).reshape(-1)
    r = Rotary()
    _check(lib().dkv_rotary_custom(r.ref, 2 * f.size, 1 if interleaved else 0, _ptr(f), float(magnitude)), "dkv_rotary_custom")
    return r


def _rows16(x, name):
    """Whether x, of [tokens][heads][128] rows, is fp16; what is neither that nor bf16 is refused."""
    T = _torch().torch
    _device_of(x, name)
    dtype = x.dtype
    half = dtype is T.float16
    if not (half or dtype is T.bfloat16) or x.dim() != 3:
        _bad(f"{name} is {x.dtype} of {x.dim()} dimensions, expected bfloat16 or float16 [T][heads][128]")
    return half


def _rotary_ref(rotary):
    if not isinstance(rotary, Rotary):
        _bad(f"rotary must be a Rotary, not {type(rotary).__name__}")
    return rotary.ref


def dkv_rope(x, positions, rotary: Rotary, out, status=None, stream=None):
    """Rows x [T][heads][128] turned by their positions (int32 [T]) -> out, of x's type and shape. Either may be a slice of a
    projection; out may be x."""
    at, queue = _where(stream)
    if _T.calls is not None and isinstance(rotary, Rotary):
        done = _T.calls.rope(_entry.get("dkv_rope") or _address("dkv_rope"), at, queue, rotary.at, x, positions, out, status)
        if done is not None:
            return _check(done, "dkv_rope")
    half = _rows16(x, "x")
    tokens, heads = x.shape[:2]
    xp, xs = _token_rows(x, "x", at, x.dtype, tokens, heads)
    op, os_ = _token_rows(out, "out", at, x.dtype, tokens, heads)
    _check(lib().dkv_rope(_rotary_ref(rotary), DKV_FP16 if half else DKV_BF16, tokens, heads, xp, xs,
                          _on(positions, "positions", at, _torch().i32, tokens), op, os_, _word(status, at), queue), "dkv_rope")


def _scales(pages, at, Ks, Vs):
    n = pages.num_pages * pages.page_rows
    return _on(Ks, "Ks", at, _torch().e8m0, n), _on(Vs, "Vs", at, _torch().e8m0, n)


def dkv_rope_append(pages: Pages, layer: int, q, k_new, v_new, positions, cu_tokens, table, len, Kp, Vp, q_out, Ks=None, Vs=None,
                    rotary: Rotary | None = None, status=None, stream=None):
    """One layer's new tokens: q [T][H][128] turned by their positions (int32 [T]) -> q_out, k_new turned and with v_new
    [T][H_kv][128] written to their slabs' pages, which are of their type, or 8-bit where the scales Ks and Vs are given. q and
    q_out, or k_new and v_new, may be None; without a rotary nothing is turned (and positions is not used)."""
    at, queue = _where(stream)
    if _T.calls is not None and (rotary is None or isinstance(rotary, Rotary)):
        done = _T.calls.rope_append(
            _entry.get("dkv_rope_append") or _address("dkv_rope_append"), at, queue, pages.at, layer, None if rotary is None else rotary.at, q,
            k_new, v_new, positions, cu_tokens, table, len, Kp, Vp, q_out, Ks, Vs, status)
        if done is not None:
            return _check(done, "dkv_rope_append")
    first, name = (q, "q") if q is not None else (k_new, "k_new (without q)")
    half, T = _rows16(first, name), _torch()
    tokens, dtype = first.shape[0], first.dtype
    qp = op = kp = vp = None
    qs = os_ = ks = 0
    if (q is None) != (q_out is None):
        _bad("q and q_out must both be given or both be None")
    if q is not None:
        qp, qs = _token_rows(q, "q", at, dtype, tokens, pages.H)
        op, os_ = _token_rows(q_out, "q_out", at, dtype, tokens, pages.H)
    if (k_new is None) != (v_new is None):
        _bad("k_new and v_new must both be given or both be None")
    if (Ks is None) != (Vs is None):
        _bad("Ks and Vs must both be given or both be None")
    if k_new is not None:
        kp, ks = _token_rows(k_new, "k_new", at, dtype, tokens, pages.H_kv)
        vp, vs = _token_rows(v_new, "v_new", at, dtype, tokens, pages.H_kv)
        if ks != vs:
            _bad(f"k_new and v_new have token strides {ks} and {vs}")
    pool, types = pages.num_pages * pages.page_rows * 128, (dtype,) if Ks is None else T.e4m3
    ksp, vsp = _scales(pages, at, Ks, Vs)
    turn = rotary is not None
    _check(lib().dkv_rope_append(
        pages.ref, int(layer), _rotary_ref(rotary) if turn else None, DKV_FP16 if half else DKV_BF16, tokens,
        _on(positions, "positions", at, T.i32, tokens) if turn else None, qp, qs, op, os_, kp, vp, ks,
        _on(cu_tokens, "cu_tokens", at, T.i32, pages.B + 1), _on(table, "table", at, T.i32, pages.slabs * pages.max_pages),
        _on(len, "len", at, T.i32, pages.slabs), _on(Kp, "Kp", at, types, pool), _on(Vp, "Vp", at, types, pool), ksp, vsp,
        _word(status, at), queue), "dkv_rope_append")


def dkv_quant_compact(pages: Pages, plan: Plan, K, V, table, len, Kp, Vp, Ks, Vs, seq=None, T_stride: int | None = None,
                      status=None, stream=None):
    """The kept rows of plan sequence i become the last rows of slot seq[i]'s slabs, in 8-bit pages with their scales. K and V
    are bfloat16 or float16 [L][plan B][H_kv][T_stride][128]."""
    T, sh = _torch(), plan.shape
    if T.calls is not None:
        at, queue = _where(stream)
        done = T.calls.quant_compact(_entry.get("dkv_quant_compact") or _address("dkv_quant_compact"), at, queue, pages.at, plan.address, seq, sh.L,
                                     plan.B, sh.H_kv, K, V, T_stride, table, len, Kp, Vp, Ks, Vs, status)
        if done is not None:
            return _check(done, "dkv_quant_compact")
    for t, name in ((K, "K"), (V, "V")):
        _device_of(t, name)
        if t.dtype not in (T.torch.bfloat16, T.torch.float16):
            _bad(f"{name} is {t.dtype}, expected bfloat16 or float16")
    _one_type("K and V", K, V)
    if T_stride is None:
        T_stride = K.shape[-2]
    at, queue = _where(stream)
    handle = plan.address
    dense = sh.L * plan.B * sh.H_kv * int(T_stride) * 128
    pool = pages.num_pages * pages.page_rows * 128
    for t, name in ((K, "K"), (V, "V")):
        if t.numel() < dense:
            _bad(f"{name} has {t.numel()} elements, needs at least {dense}")
    ksp, vsp = _scales(pages, at, Ks, Vs)
    _check(lib().dkv_quant_compact(
        pages.ref, handle, _on(seq, "seq", at, T.i32, plan.B), DKV_FP16 if K.dtype == T.torch.float16 else DKV_BF16,
        _on(K, "K", at, (K.dtype,)), _on(V, "V", at, (K.dtype,)), int(T_stride),
        _on(table, "table", at, T.i32, pages.slabs * pages.max_pages), _on(len, "len", at, T.i32, pages.slabs),
        _on(Kp, "Kp", at, T.e4m3, pool), _on(Vp, "Vp", at, T.e4m3, pool), ksp, vsp, _word(status, at), queue), "dkv_quant_compact")


def dkv_quant_workspace_bytes(pages: Pages) -> int:
    n = int(lib().dkv_quant_workspace_bytes(ctypes.byref(pages.c)))
    if n < 0:
        _check(DKV_ERR_INVALID_ARG, "dkv_quant_workspace_bytes")
    return n


def dkv_quant_attn(pages: Pages, layer: int, q, cu_tokens, table, len, Kp, Vp, Ks, Vs, out, workspace, causal: bool = True,
                   scale: float = 0.0, max_tokens: int = 0, status=None, stream=None):
    """One layer's attention of q [T][H][128] over 8-bit pages -> out [T][H][128], both bfloat16 or float16. max_tokens: the
    most tokens that one sequence brings (0: not known; a step of next tokens then takes three launches for two)."""
    at, queue = _where(stream)
    if _T.calls is not None:
        done = _T.calls.quant_attn(_entry.get("dkv_quant_attn") or _address("dkv_quant_attn"), at, queue, pages.at, layer, q, cu_tokens, table,
                                   len, Kp, Vp, Ks, Vs, out, workspace, causal, scale, max_tokens, status)
        if done is not None:
            return _check(done, "dkv_quant_attn")
    half, T = _rows16(q, "q"), _torch()
    tokens = q.shape[0]
    qp, qs = _token_rows(q, "q", at, q.dtype, tokens, pages.H)
    pool = pages.num_pages * pages.page_rows * 128
    ksp, vsp = _scales(pages, at, Ks, Vs)
    wp, wb = _work(workspace, at)
    _check(lib().dkv_quant_attn(
        pages.ref, int(layer), DKV_FP16 if half else DKV_BF16, tokens, int(max_tokens), qp, qs,
        _on(cu_tokens, "cu_tokens", at, T.i32, pages.B + 1), _on(table, "table", at, T.i32, pages.slabs * pages.max_pages),
        _on(len, "len", at, T.i32, pages.slabs), _on(Kp, "Kp", at, T.e4m3, pool), _on(Vp, "Vp", at, T.e4m3, pool), ksp, vsp,
        1 if causal else 0, scale, _on(out, "out", at, (q.dtype,), tokens * pages.H * 128), wp, wb, _word(status, at), queue),
        "dkv_quant_attn")
