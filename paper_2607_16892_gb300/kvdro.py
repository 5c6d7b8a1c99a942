"""Python binding of the kvdro C ABI (include/kvdro.h).

Argument marshalling only: every function here converts its arguments to plain
pointers and sizes and calls the entry point of the same name in
``_build/libkvdro.so``.  Every step of the computation runs in that library's
CUDA kernels; there is no CPU or PyTorch path.  If the library is missing or
cannot be loaded, the first call raises.

Array arguments may be NumPy arrays (host memory) or torch tensors (host or
CUDA memory); the library itself tells host from device pointers.  Streams may
be a ``torch.cuda.Stream``, a raw ``cudaStream_t`` integer, or None: the legacy
default stream, except for the page cache's calls, which take torch tensors only and
go to torch's current stream then.
"""

from __future__ import annotations

import ctypes
import functools
import os
import threading
import weakref
from typing import Any

import numpy as np

from . import build as _build

KVDRO_OK = 0
KVDRO_EINVAL = -1
KVDRO_ENOMEM = -2
KVDRO_ECUDA = -3
KVDRO_ESTATE = -4
KVDRO_ETIMEOUT = -5
KVDRO_ERANGE = -6
KVDRO_FP32 = 0
KVDRO_FP64 = 1
KVDRO_EXACT = 2
KVDRO_ENVELOPE = 3
KVDRO_BF16 = 0
KVDRO_FP16 = 1

_STATUS = {0: "KVDRO_OK", -1: "KVDRO_EINVAL", -2: "KVDRO_ENOMEM", -3: "KVDRO_ECUDA", -4: "KVDRO_ESTATE",
           -5: "KVDRO_ETIMEOUT", -6: "KVDRO_ERANGE"}

# Every entry point declared in include/kvdro.h.
SYMBOLS = ("kvdro_create", "kvdro_load_samples", "kvdro_quantiles", "kvdro_eval_grid", "kvdro_sorted_samples",
           "kvdro_eval_dual", "kvdro_last_grid_ms", "kvdro_eval_grid_noalloc", "kvdro_kv_open", "kvdro_kv_close",
           "kvdro_kv_plan", "kvdro_kv_append", "kvdro_kv_attend", "kvdro_kv_open8", "kvdro_kv_read", "kvdro_kv_attend_shared",
           "kvdro_kv_shared_bytes", "kvdro_sync", "kvdro_last_error", "kvdro_destroy")

_lock = threading.Lock()
_lib = None


class KvdroError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


def library_path() -> str:
    return _build.LIB


def load_library(build_if_missing: bool = True) -> ctypes.CDLL:
    """Load libkvdro.so (building it with nvcc first if it is absent)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        path = _build.LIB
        if not os.path.exists(path):
            if not build_if_missing:
                raise RuntimeError(f"kvdro CUDA library not built: {path}")
            _build.build()
        lib = ctypes.CDLL(path)
        P, i32 = ctypes.c_void_p, ctypes.c_int32
        lib.kvdro_create.restype = ctypes.c_int
        lib.kvdro_create.argtypes = [ctypes.POINTER(P), ctypes.c_int]
        lib.kvdro_load_samples.restype = ctypes.c_int
        lib.kvdro_load_samples.argtypes = [P, i32, P, P, P, P, P]
        lib.kvdro_quantiles.restype = ctypes.c_int
        lib.kvdro_quantiles.argtypes = [P, i32, P, P, P]
        lib.kvdro_eval_grid.restype = ctypes.c_int
        lib.kvdro_eval_grid.argtypes = [P, ctypes.c_int, i32, P, i32, P, i32, P, i32, P, P, P, P, P, P, P, P, P]
        lib.kvdro_eval_dual.restype = ctypes.c_int
        lib.kvdro_eval_dual.argtypes = [P, i32, P, i32, P, i32, P, P, P, P, P, P, P, P]
        lib.kvdro_sorted_samples.restype = ctypes.c_int
        lib.kvdro_sorted_samples.argtypes = [P, P, P]
        lib.kvdro_last_grid_ms.restype = ctypes.c_int
        lib.kvdro_last_grid_ms.argtypes = [P, ctypes.POINTER(ctypes.c_float)]
        lib.kvdro_eval_grid_noalloc.restype = ctypes.c_int
        lib.kvdro_eval_grid_noalloc.argtypes = [i32, P, P, P, P, i32, P, i32, P, i32, P, i32, P, P, P, P, P, P, P, P,
                                                ctypes.c_char_p, i32]
        f64 = ctypes.c_double
        lib.kvdro_kv_open.restype = ctypes.c_int
        lib.kvdro_kv_open.argtypes = [P, ctypes.POINTER(P), ctypes.c_int, i32, i32, i32, i32, P, P, P, P]
        lib.kvdro_kv_close.restype = ctypes.c_int
        lib.kvdro_kv_close.argtypes = [P]
        lib.kvdro_kv_plan.restype = ctypes.c_int
        lib.kvdro_kv_plan.argtypes = [P, i32, i32, i32, i32, i32, P, P, P, P, P, P, P, P, P, P, P, P, P, P]
        lib.kvdro_kv_append.restype = ctypes.c_int
        lib.kvdro_kv_append.argtypes = [P, i32, P, P, P, P, P, P]
        lib.kvdro_kv_attend.restype = ctypes.c_int
        lib.kvdro_kv_attend.argtypes = [P, i32, i32, i32, i32, P, P, P, P, P, i32, f64, ctypes.c_int, i32, f64, P, P, P, P]
        lib.kvdro_kv_open8.restype = ctypes.c_int
        lib.kvdro_kv_open8.argtypes = [P, ctypes.POINTER(P), ctypes.c_int, i32, i32, i32, i32, P, P, P, P, P, P]
        lib.kvdro_kv_read.restype = ctypes.c_int
        lib.kvdro_kv_read.argtypes = [P, i32, i32, P, P, P, i32, P, P, P, P, P]
        lib.kvdro_kv_attend_shared.restype = ctypes.c_int
        lib.kvdro_kv_attend_shared.argtypes = [P, i32, i32, i32, i32, P, P, P, P, P, i32, i32, P, P, P, i32, f64, ctypes.c_int, f64, P, P, P, P,
                                               ctypes.c_size_t, P]
        lib.kvdro_kv_shared_bytes.restype = ctypes.c_int
        lib.kvdro_kv_shared_bytes.argtypes = [i32, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
        lib.kvdro_sync.restype = ctypes.c_int
        lib.kvdro_sync.argtypes = [P]
        lib.kvdro_last_error.restype = ctypes.c_char_p
        lib.kvdro_last_error.argtypes = [P]
        lib.kvdro_destroy.restype = ctypes.c_int
        lib.kvdro_destroy.argtypes = [P]
        _lib = lib
        return lib


# ------------------------------------------------------------------ marshalling

# A grid call marshals some twenty arguments; with NumPy's own attribute paths (dtype names, ndarray.ctypes)
# that took 24 us of host time, more than the smallest grid takes on the GPU, and takes 15 with these.
_DTYPES = {d: np.dtype(d) for d in (np.int32, np.int64, np.float32, np.float64)}
_TORCH_DTYPES: dict = {}  # NumPy scalar type -> torch dtype, filled once a tensor is seen


def _np_ptr(a: np.ndarray) -> int:
    return a.__array_interface__["data"][0]


def _torch_dtype(dtype):
    if not _TORCH_DTYPES:
        import torch
        _TORCH_DTYPES.update({np.int32: torch.int32, np.int64: torch.int64, np.float32: torch.float32,
                              np.float64: torch.float64})
    return _TORCH_DTYPES[dtype]


def _ptr(a: Any, dtype=None):
    """Pointer to the data of a NumPy array or torch tensor (None -> NULL)."""
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        if dtype is not None and a.dtype != _DTYPES[dtype]:
            raise TypeError(f"expected dtype {_DTYPES[dtype]}, got {a.dtype}")
        if not a.flags.c_contiguous:
            raise ValueError("array must be C-contiguous")
        return _np_ptr(a)
    if hasattr(a, "data_ptr"):
        if dtype is not None and a.dtype is not _torch_dtype(dtype):
            want = _DTYPES[dtype].name
            got = str(a.dtype).replace("torch.", "")
            if got != want:
                raise TypeError(f"expected dtype {want}, got {got}")
        if not a.is_contiguous():
            raise ValueError("tensor must be contiguous")
        return a.data_ptr()
    raise TypeError(f"unsupported array type {type(a)}")


def _host(a: Any, dtype) -> np.ndarray:
    """Small host-side parameter arrays are converted to contiguous NumPy of the ABI dtype."""
    if type(a) is np.ndarray and a.ndim and a.dtype == _DTYPES[dtype] and a.flags.c_contiguous:
        return a
    if hasattr(a, "detach"):
        a = a.detach().cpu().numpy()
    return np.ascontiguousarray(np.asarray(a), dtype=dtype)


def _stream(s: Any):
    if s is None:
        return None
    if isinstance(s, int):
        return s
    if hasattr(s, "cuda_stream"):
        return s.cuda_stream
    raise TypeError(f"unsupported stream {type(s)}")


def _numel(a: Any) -> int:
    if isinstance(a, np.ndarray):
        return int(a.size)
    if hasattr(a, "numel"):
        return int(a.numel())
    return int(np.asarray(a).size)


def _need(name: str, a: Any, n: int) -> None:
    """Raise ValueError unless array ``a`` (if given) holds exactly ``n`` elements: the library
    reads or writes exactly that many through the pointer, so a shorter buffer would be
    overrun (on the device or on the host)."""
    if a is None:
        return
    if _numel(a) != n:
        raise ValueError(f"{name} has {_numel(a)} elements; the call needs exactly {n}")


def _on_device(name: str, a: Any) -> None:
    if a is not None and not (hasattr(a, "is_cuda") and a.is_cuda):
        raise ValueError(f"{name} must be a CUDA tensor")


# Class count and sample total of each context's loaded samples (keyed by the handle), so
# that outputs sized by them can be checked before a call.
_loaded: dict = {}


def _check(ctx, status: int):
    if status != KVDRO_OK:
        msg = load_library().kvdro_last_error(ctx).decode() if ctx else ""
        raise KvdroError(status, msg)


# ------------------------------------------------------------------ entry points

def kvdro_create(device_ordinal: int = 0) -> ctypes.c_void_p:
    lib = load_library()
    h = ctypes.c_void_p()
    st = lib.kvdro_create(ctypes.byref(h), int(device_ordinal))
    if st != KVDRO_OK:
        raise KvdroError(st, f"kvdro_create(device={device_ordinal}) failed")
    return h


def _check_samples(K: int, off: np.ndarray, lengths, lm: np.ndarray, li) -> None:
    if int(K) < 1:
        raise ValueError(f"K = {K} must be at least 1")
    _need("offsets", off, int(K) + 1)
    _need("L_max", lm, int(K))
    _need("L_in", li, int(K))
    _need("lengths", lengths, int(off[-1]))


def kvdro_load_samples(ctx, K: int, offsets, lengths, L_max, L_in=None, stream=None) -> None:
    off = _host(offsets, np.int64)
    lm = _host(L_max, np.int32)
    li = None if L_in is None else _host(L_in, np.int32)
    _check_samples(K, off, lengths, lm, li)
    key = getattr(ctx, "value", ctx)
    _loaded.pop(key, None)
    _check(ctx, load_library().kvdro_load_samples(ctx, int(K), _np_ptr(off), _ptr(lengths, np.int32), _np_ptr(lm),
                                                  None if li is None else _np_ptr(li), _stream(stream)))
    _loaded[key] = (int(K), int(off[-1]))


def _ctx_K(ctx):
    """Class count of the context's loaded samples (None if unknown here)."""
    got = _loaded.get(getattr(ctx, "value", ctx))
    return None if got is None else got[0]


def kvdro_quantiles(ctx, F: int, fractiles, out, stream=None) -> None:
    fr = _host(fractiles, np.float64)
    _need("fractiles", fr, int(F))
    K = _ctx_K(ctx)
    if K is not None:
        _need("out", out, K * int(F))
    _check(ctx, load_library().kvdro_quantiles(ctx, int(F), _np_ptr(fr), _ptr(out, np.int32), _stream(stream)))


def _check_grid(R, rr, E, ee, M, cp, cw, NL=None, ll=None) -> None:
    _need("r", rr, int(R))
    if NL is not None:
        _need("lam", ll, int(NL))
    _need("eps", ee, int(E))
    _need("c_p", cp, int(M))
    _need("c_w", cw, int(M))


def _check_outputs(K: int, R: int, E: int, M: int, NL=None, **outs) -> None:
    rows = M * E * K
    size = {"S": M * K * R * (NL or 0), "cost": rows * R, "lam_idx": rows * R, "gamma": rows * R, "r_idx": rows,
            "min_cost": rows, "fhat": rows}
    for name, a in outs.items():
        _need(name, a, size[name])


def kvdro_eval_grid(ctx, precision: int, R: int, r, NL: int, lam, E: int, eps, M: int, c_p, c_w, S=None, cost=None,
                    lam_idx=None, r_idx=None, min_cost=None, fhat=None, stream=None) -> None:
    ft = np.float32 if precision == KVDRO_FP32 else np.float64
    rr, ll, ee = _host(r, np.int32), _host(lam, np.float64), _host(eps, np.float64)
    cp, cw = _host(c_p, np.float64), _host(c_w, np.float64)
    _check_grid(R, rr, E, ee, M, cp, cw, NL=NL, ll=ll)
    K = _ctx_K(ctx)
    if K is not None:
        _check_outputs(K, int(R), int(E), int(M), NL=int(NL), S=S, cost=cost, lam_idx=lam_idx, r_idx=r_idx,
                       min_cost=min_cost, fhat=fhat)
    _check(ctx, load_library().kvdro_eval_grid(
        ctx, int(precision), int(R), _np_ptr(rr), int(NL), _np_ptr(ll), int(E), _np_ptr(ee), int(M),
        _np_ptr(cp), _np_ptr(cw), _ptr(S, ft), _ptr(cost, ft), _ptr(lam_idx, np.int32), _ptr(r_idx, np.int32),
        _ptr(min_cost, ft), _ptr(fhat, np.float64), _stream(stream)))


def kvdro_eval_dual(ctx, R: int, r, E: int, eps, M: int, c_p, c_w, cost=None, gamma=None, r_idx=None,
                    min_cost=None, fhat=None, stream=None) -> None:
    rr, ee = _host(r, np.int32), _host(eps, np.float64)
    cp, cw = _host(c_p, np.float64), _host(c_w, np.float64)
    _check_grid(R, rr, E, ee, M, cp, cw)
    K = _ctx_K(ctx)
    if K is not None:
        _check_outputs(K, int(R), int(E), int(M), cost=cost, gamma=gamma, r_idx=r_idx, min_cost=min_cost, fhat=fhat)
    _check(ctx, load_library().kvdro_eval_dual(
        ctx, int(R), _np_ptr(rr), int(E), _np_ptr(ee), int(M), _np_ptr(cp), _np_ptr(cw),
        _ptr(cost, np.float64), _ptr(gamma, np.float64), _ptr(r_idx, np.int32), _ptr(min_cost, np.float64),
        _ptr(fhat, np.float64), _stream(stream)))


def kvdro_sorted_samples(ctx, out, stream=None) -> None:
    got = _loaded.get(getattr(ctx, "value", ctx))
    if got is not None:
        _need("out", out, got[1])
    _check(ctx, load_library().kvdro_sorted_samples(ctx, _ptr(out, np.int32), _stream(stream)))


def kvdro_last_grid_ms(ctx) -> float:
    ms = ctypes.c_float()
    _check(ctx, load_library().kvdro_last_grid_ms(ctx, ctypes.byref(ms)))
    return float(ms.value)


def kvdro_eval_grid_noalloc(K: int, offsets, lengths, L_max, L_in, R: int, r, NL: int, lam, E: int, eps, M: int,
                            c_p, c_w, cost=None, lam_idx=None, r_idx=None, min_cost=None, fhat=None,
                            stream=None) -> None:
    """FP32 grid pass in the library's static scratch (allocates nothing; see include/kvdro.h).
    ``lengths`` and the outputs must be CUDA tensors on the current device."""
    off, lm = _host(offsets, np.int64), _host(L_max, np.int32)
    li = None if L_in is None else _host(L_in, np.int32)
    rr, ll, ee = _host(r, np.int32), _host(lam, np.float64), _host(eps, np.float64)
    cp, cw = _host(c_p, np.float64), _host(c_w, np.float64)
    _check_samples(K, off, lengths, lm, li)
    _check_grid(R, rr, E, ee, M, cp, cw, NL=NL, ll=ll)
    _check_outputs(int(K), int(R), int(E), int(M), cost=cost, lam_idx=lam_idx, r_idx=r_idx, min_cost=min_cost,
                   fhat=fhat)
    for name, a in (("lengths", lengths), ("cost", cost), ("lam_idx", lam_idx), ("r_idx", r_idx),
                    ("min_cost", min_cost), ("fhat", fhat)):
        _on_device(name, a)
    buf = ctypes.create_string_buffer(512)
    st = load_library().kvdro_eval_grid_noalloc(
        int(K), _np_ptr(off), _ptr(lengths, np.int32), _np_ptr(lm), None if li is None else _np_ptr(li),
        int(R), _np_ptr(rr), int(NL), _np_ptr(ll), int(E), _np_ptr(ee), int(M), _np_ptr(cp),
        _np_ptr(cw), _ptr(cost, np.float32), _ptr(lam_idx, np.int32), _ptr(r_idx, np.int32),
        _ptr(min_cost, np.float32), _ptr(fhat, np.float64), _stream(stream), buf, len(buf))
    if st != KVDRO_OK:
        raise KvdroError(st, buf.value.decode())


# ------------------------------------------------------------------ page cache

class KvdroKv:
    """A handle of ``kvdro_kv_open`` or ``kvdro_kv_open8`` and the tensors it describes, which it keeps alive."""

    __slots__ = ("handle", "ctx", "owner", "k", "v", "exps", "dtype", "heads", "head_dim", "__weakref__")

    def __del__(self):
        try:
            kvdro_kv_close(self)
        except (AttributeError, TypeError):  # never opened, or the interpreter is going down
            pass


# A serving step makes these calls once per layer, so their host time counts: the checks of a good argument take few
# attribute reads, and what is wrong with a bad one is found out afterwards.
def _dev(name: str, a: Any, dtype, n=None) -> int:
    """Pointer of a contiguous CUDA tensor of this torch dtype (and of ``n`` elements)."""
    try:
        if a.is_cuda and a.dtype is dtype and a.is_contiguous() and (n is None or a.numel() == n):
            return a.data_ptr()
    except AttributeError:
        pass
    if not getattr(a, "is_cuda", False):
        raise ValueError(f"{name} must be a CUDA tensor")
    if a.dtype is not dtype:
        raise TypeError(f"{name}: expected dtype {dtype}, got {a.dtype}")
    if not a.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    raise ValueError(f"{name} has {a.numel()} elements; the call needs exactly {n}")


_kv_types: dict = {}

class _Owner:
    """What is open in one context: the library's handles, each closed once at most, and the objects that hold them."""

    __slots__ = ("handles", "caches")

    def __init__(self):
        self.handles, self.caches = set(), weakref.WeakSet()


_owners: dict = {}  # handle of a context -> what is open there, which kvdro_destroy closes
# A cache may be closed by its finalizer, on whatever thread drops it and in the middle of any other call: the calls that
# open, close and free handles run one at a time.
_kv_lock = threading.RLock()
_I2, _I3 = ctypes.c_int64 * 2, ctypes.c_int64 * 3


@functools.lru_cache(maxsize=256)
def _two(s0: int, s1: int):
    """Two strides as the library takes them, made once for each pair (a step's calls have the same ones)."""
    return _I2(s0, s1)


_lib_kv = _i32 = _f32 = None  # the loaded library and torch's dtypes
_current_stream = None  # torch's current stream of a device, as a number (its public form takes a microsecond)


def _kv_setup():
    """The library, once loaded."""
    global _lib_kv, _i32, _f32, _current_stream
    if _i32 is None:
        import torch
        _current_stream = torch._C._cuda_getCurrentRawStream
        _i32, _f32 = torch.int32, torch.float32
        _kv_types.update({torch.bfloat16: KVDRO_BF16, torch.float16: KVDRO_FP16})
    _lib_kv = load_library()
    return _lib_kv


def _heads(cache: KvdroKv, name: str, a: Any, T=None, heads=None):
    """Pointer and strides (None if contiguous) of a CUDA tensor [T][heads][head_dim] of the cache's dtype, T and heads."""
    try:
        if a.is_cuda and a.dtype is cache.dtype:
            t, h, d = a.shape
            if d == cache.head_dim and (T is None or t == T) and (heads is None or h == heads):
                if a.is_contiguous():
                    return a.data_ptr(), None, t, h
                s0, s1, s2 = a.stride()
                if s2 == 1:
                    # a dimension of one element has no stride of its own: any that the library takes will do
                    return a.data_ptr(), _two(s0 if t > 1 else 8, s1 if h > 1 else 8), t, h
    except (AttributeError, ValueError):
        pass
    if not getattr(a, "is_cuda", False):
        raise ValueError(f"{name} must be a CUDA tensor")
    if a.dtype is not cache.dtype:
        raise TypeError(f"{name}: expected the cache's dtype {cache.dtype}, got {a.dtype}")
    if a.dim() == 3 and a.stride(2) != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    raise ValueError(f"{name} has shape {tuple(a.shape)}; the call needs "
                     f"({'T' if T is None else T}, {'heads' if heads is None else heads}, {cache.head_dim})")


def kvdro_kv_open(ctx, k, v) -> KvdroKv:
    """Describe a page cache: ``k`` and ``v`` are CUDA tensors [n_pages][page_size][n_kv_heads][head_dim] of
    bfloat16 or float16 whose last dimension is contiguous (other strides as they are)."""
    _kv_setup()
    for name, a in (("k", k), ("v", v)):
        _on_device(name, a)
        if a.dtype not in _kv_types:
            raise TypeError(f"{name}: expected bfloat16 or float16, got {a.dtype}")
        if a.dim() != 4 or (a.shape[3] > 1 and a.stride(3) != 1):
            raise ValueError(f"{name} must be [n_pages][page_size][n_kv_heads][head_dim] with a contiguous last dimension")
    if k.shape != v.shape or k.dtype is not v.dtype:
        raise ValueError("k and v differ in shape or dtype")
    return _open(ctx, k, v, k.dtype, None)


def kvdro_kv_open8(ctx, k, v, k_exp, v_exp, dtype) -> KvdroKv:
    """Describe a page cache of 8 bits: ``k`` and ``v`` are CUDA tensors [n_pages][page_size][n_kv_heads][head_dim] of
    float8_e4m3fn, ``k_exp`` and ``v_exp`` contiguous ones [n_pages][n_kv_heads][page_size] of uint8 or float8_e8m0fnu; rows that
    calls on the handle take and give are of ``dtype``, bfloat16 or float16."""
    import torch

    _kv_setup()
    for name, a in (("k", k), ("v", v), ("k_exp", k_exp), ("v_exp", v_exp)):
        _on_device(name, a)
    for name, a in (("k", k), ("v", v)):
        if a.dtype is not torch.float8_e4m3fn:
            raise TypeError(f"{name}: expected float8_e4m3fn, got {a.dtype}")
        if a.dim() != 4 or (a.shape[3] > 1 and a.stride(3) != 1):
            raise ValueError(f"{name} must be [n_pages][page_size][n_kv_heads][head_dim] with a contiguous last dimension")
    if k.shape != v.shape:
        raise ValueError("k and v differ in shape")
    n, page, heads, _ = k.shape
    for name, a in (("k_exp", k_exp), ("v_exp", v_exp)):
        if a.dtype not in (torch.uint8, torch.float8_e8m0fnu):
            raise TypeError(f"{name}: expected uint8 or float8_e8m0fnu, got {a.dtype}")
        if a.shape != (n, heads, page) or not a.is_contiguous():
            raise ValueError(f"{name} must be a contiguous tensor [n_pages][n_kv_heads][page_size]")
    if dtype not in _kv_types:
        raise TypeError(f"dtype must be bfloat16 or float16, got {dtype}")
    return _open(ctx, k, v, dtype, (k_exp, v_exp))


def _open(ctx, k, v, dtype, exps) -> KvdroKv:
    n, page, heads, d = k.shape
    strides = [_I3(*(t.stride(i) if t.shape[i] > 1 else 16 for i in range(3))) for t in (k, v)]
    lib, h = load_library(), ctypes.c_void_p()
    with _kv_lock:
        if exps is None:
            _check(ctx, lib.kvdro_kv_open(ctx, ctypes.byref(h), _kv_types[dtype], n, page, heads, d, k.data_ptr(), strides[0], v.data_ptr(),
                                          strides[1]))
        else:
            _check(ctx, lib.kvdro_kv_open8(ctx, ctypes.byref(h), _kv_types[dtype], n, page, heads, d, k.data_ptr(), strides[0],
                                           exps[0].data_ptr(), v.data_ptr(), strides[1], exps[1].data_ptr()))
        c = KvdroKv()
        c.owner = _owners.setdefault(getattr(ctx, "value", ctx), _Owner())
        c.owner.handles.add(h.value)
        c.handle, c.ctx, c.k, c.v, c.exps, c.dtype, c.heads, c.head_dim = h, ctx, k, v, exps, dtype, heads, d
        c.owner.caches.add(c)
    return c


def kvdro_kv_close(cache: KvdroKv) -> None:
    with _kv_lock:
        handle, cache.handle = cache.handle, None
        if handle:
            cache.k = cache.v = cache.exps = None
            if handle.value in cache.owner.handles:  # else freed with its context
                cache.owner.handles.remove(handle.value)
                load_library().kvdro_kv_close(handle)


def kvdro_kv_plan(ctx, page_size: int, cached, new_len, held, table, ring, pool, held_out, pool_out, q_off, kv_len,
                  slot, pos=None, reserve=None, stream=None) -> None:
    """Pages and slots of one step (include/kvdro.h): int32 CUDA tensors; ``table`` is [B][max_pages], ``ring`` holds
    one element per page and ``slot`` one per new token."""
    lib = _lib_kv or _kv_setup()
    B, max_pages = _table(table)
    T, i32 = _numel(slot), _i32
    st = lib.kvdro_kv_plan(
        ctx, page_size, _numel(ring), B, max_pages, T, _dev("cached", cached, i32, B), _dev("new_len", new_len, i32, B),
        None if reserve is None else _dev("reserve", reserve, i32, B), _dev("held", held, i32, B), _dev("table", table, i32),
        _dev("ring", ring, i32), _dev("pool", pool, i32, 2), _dev("held_out", held_out, i32, B),
        _dev("pool_out", pool_out, i32, 2), _dev("q_off", q_off, i32, B + 1), _dev("kv_len", kv_len, i32, B),
        _dev("slot", slot, i32), None if pos is None else _dev("pos", pos, i32, T),
        _current_stream(cached.get_device()) if stream is None else _stream(stream))
    if st:
        _check(ctx, st)


def _table(table, name="table", rows="B", pages="max_pages"):
    try:
        B, max_pages = table.shape
    except (AttributeError, ValueError):
        raise ValueError(f"{name} must be [{rows}][{pages}]") from None
    return B, max_pages


def _open_handle(cache: KvdroKv):
    if not cache.handle:
        raise ValueError("the page cache is closed")
    return cache.handle


def kvdro_kv_append(cache: KvdroKv, k, v, slot, stream=None) -> None:
    """Write the new tokens' keys and values, [T][n_kv_heads][head_dim] (last dimension contiguous), into their slots."""
    lib = _lib_kv or _kv_setup()
    kp, ks, T, heads = _heads(cache, "k", k, None, cache.heads)
    vp, vs, T, heads = _heads(cache, "v", v, T, heads)
    st = lib.kvdro_kv_append(_open_handle(cache), T, kp, ks, vp, vs, _dev("slot", slot, _i32, T),
                             _current_stream(k.get_device()) if stream is None else _stream(stream))
    if st:
        _check(cache.ctx, st)


def kvdro_kv_attend(cache: KvdroKv, q, q_off, kv_len, table, out, lse=None, scale=None, causal: bool = True,
                    window: int = 0, softcap: float = 0.0, max_q: int = 0, stream=None) -> None:
    """Attention of the new tokens ``q`` [T][n_heads][head_dim] over their requests' pages into ``out`` (and ``lse``
    [T][n_heads] float32); ``scale`` defaults to head_dim ** -0.5."""
    lib = _lib_kv or _kv_setup()
    qp, qs, T, heads = _heads(cache, "q", q)
    op, os_, _, _ = _heads(cache, "out", out, T, heads)
    B, max_pages = _table(table)
    st = lib.kvdro_kv_attend(
        _open_handle(cache), B, T, heads, max_q, qp, qs, _dev("q_off", q_off, _i32, B + 1), _dev("kv_len", kv_len, _i32, B),
        _dev("table", table, _i32), max_pages, cache.head_dim ** -0.5 if scale is None else scale, 1 if causal else 0, window,
        softcap, op, os_, None if lse is None else _dev("lse", lse, _f32, T * heads),
        _current_stream(q.get_device()) if stream is None else _stream(stream))
    if st:
        _check(cache.ctx, st)


def kvdro_kv_read(cache: KvdroKv, q_off, kv_len, table, k, v, stream=None) -> None:
    """Keys and values of the requests' last tokens (as many as ``q_off`` says) out of their pages into ``k`` and ``v``,
    [T][n_kv_heads][head_dim] of the cache's dtype (last dimension contiguous)."""
    lib = _lib_kv or _kv_setup()
    kp, ks, T, heads = _heads(cache, "k", k, None, cache.heads)
    vp, vs, T, heads = _heads(cache, "v", v, T, heads)
    B, max_pages = _table(table)
    st = lib.kvdro_kv_read(
        _open_handle(cache), B, T, _dev("q_off", q_off, _i32, B + 1), _dev("kv_len", kv_len, _i32, B), _dev("table", table, _i32), max_pages,
        kp, ks, vp, vs, _current_stream(k.get_device()) if stream is None else _stream(stream))
    if st:
        _check(cache.ctx, st)


def kvdro_kv_shared_bytes(T: int, n_heads: int, head_dim: int) -> int:
    """Bytes of workspace that ``kvdro_kv_attend_shared`` needs for T tokens."""
    n = ctypes.c_size_t()
    st = (_lib_kv or _kv_setup()).kvdro_kv_shared_bytes(T, n_heads, head_dim, ctypes.byref(n))
    if st:
        raise KvdroError(st, f"no workspace for T = {T}, n_heads = {n_heads}, head_dim = {head_dim}")
    return n.value


def kvdro_kv_attend_shared(cache: KvdroKv, q, q_off, kv_len, table, share_off, prefix_len, prefix_table, out, lse=None, scale=None,
                           causal: bool = True, softcap: float = 0.0, max_q: int = 0, work=None, stream=None) -> None:
    """``kvdro_kv_attend`` where requests share_off[g] .. share_off[g + 1] - 1 stand behind the prefix_len[g] tokens of the pages
    ``prefix_table`` [G][prefix_pages]; ``work`` is a CUDA tensor of at least ``kvdro_kv_shared_bytes`` bytes (None: one of torch's allocator,
    on the call's stream)."""
    lib = _lib_kv or _kv_setup()
    qp, qs, T, heads = _heads(cache, "q", q)
    op, os_, _, _ = _heads(cache, "out", out, T, heads)
    B, max_pages = _table(table)
    G, prefix_pages = _table(prefix_table, "prefix_table", "G", "prefix_pages")
    at = _current_stream(q.get_device()) if stream is None else _stream(stream)
    if work is None:
        work = _workspace(kvdro_kv_shared_bytes(T, heads, cache.head_dim), q.device, at)
    elif not (getattr(work, "is_cuda", False) and work.is_contiguous()):
        raise ValueError("work must be a contiguous CUDA tensor")
    st = lib.kvdro_kv_attend_shared(
        _open_handle(cache), B, T, heads, max_q, qp, qs, _dev("q_off", q_off, _i32, B + 1), _dev("kv_len", kv_len, _i32, B),
        _dev("table", table, _i32), max_pages, G, _dev("share_off", share_off, _i32, G + 1), _dev("prefix_len", prefix_len, _i32, G),
        _dev("prefix_table", prefix_table, _i32), prefix_pages, cache.head_dim ** -0.5 if scale is None else scale, 1 if causal else 0, softcap,
        op, os_, None if lse is None else _dev("lse", lse, _f32, T * heads), work.data_ptr(), work.numel() * work.element_size(), at)
    if st:
        _check(cache.ctx, st)


def _workspace(n: int, device, stream: int):
    """Bytes of torch's allocator that are the stream's until it is done with them."""
    import torch

    with torch.cuda.device(device):
        if stream == _current_stream(device.index):
            return torch.empty(n, dtype=torch.uint8, device=device)
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device)):
            return torch.empty(n, dtype=torch.uint8, device=device)


def kvdro_sync(ctx) -> None:
    _check(ctx, load_library().kvdro_sync(ctx))


def kvdro_last_error(ctx) -> str:
    return load_library().kvdro_last_error(ctx).decode()


def kvdro_destroy(ctx) -> None:
    if ctx:
        _loaded.pop(getattr(ctx, "value", ctx), None)
        with _kv_lock:
            owner = _owners.pop(getattr(ctx, "value", ctx), None)
            if owner is not None:
                for cache in list(owner.caches):
                    kvdro_kv_close(cache)
                owner.handles.clear()  # of caches about to be finalized: the library frees them
            load_library().kvdro_destroy(ctx)
