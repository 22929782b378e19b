"""ctypes binding of libflashkm.so: same names as include/flashkm.h, argument marshalling only.

Tensors are torch tensors (device memory, streams); every step of the path runs inside the
library's HIP kernels.  There is no fallback: if the library has not been built, or a call
fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import torch

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libflashkm.so"

FK_F32, FK_F16, FK_BF16 = 0, 1, 2
_DTYPE = {torch.float32: FK_F32, torch.float16: FK_F16, torch.bfloat16: FK_BF16}
_STATUS = {0: "FK_OK", 1: "FK_EINVAL", 2: "FK_EUNSUPPORTED", 3: "FK_EWORKSPACE", 4: "FK_EHIP"}

# every symbol include/flashkm.h declares
EXPORTS = ("fk_last_error", "fk_workspace_bytes", "fk_assign", "fk_sort_inverse", "fk_update",
           "fk_lloyd_iter", "fk_lloyd_ooc", "fk_ooc_workspace_bytes", "fk_stage_timer_start",
           "fk_stage_timer_stop", "fk_plan", "fk_set_option", "fk_standard_assign",
           "fk_standard_update", "fk_assign_static", "fk_assign_static_limit", "fk_kv_append", "fk_kv_read",
           "fk_kv_attend", "fk_kv_workspace_bytes", "fk_kv_plan", "fk_kv_attend_tree", "fk_kv_weigh", "fk_kv_weigh_workspace_bytes", "fk_kv_choose",
           "fk_kv_choose_workspace_bytes", "fk_kv_compact", "fk_kv_plan_tree")
STAGES = ("assign", "sort", "reduce", "finalize")


class _KVCacheStruct(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_codes", "v_codes", "k_scale", "v_scale", "k_levels", "v_levels")] + [
        ("pages", ctypes.c_int64), ("page_size", ctypes.c_int), ("heads", ctypes.c_int), ("d", ctypes.c_int), ("t", ctypes.c_int)]


class FlashKMError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """Open libflashkm.so (built by paper_2603_09229_amd.build); fail loudly if absent."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2603_09229_amd.build` "
                "(or __graft_entry__.build()); there is no fallback path")
        L = ctypes.CDLL(str(LIB_PATH))
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
        L.fk_last_error.restype = ctypes.c_char_p
        L.fk_last_error.argtypes = []
        L.fk_workspace_bytes.restype = sz
        L.fk_workspace_bytes.argtypes = [i32, i64, i32, i32, i32]
        L.fk_ooc_workspace_bytes.restype = sz
        L.fk_ooc_workspace_bytes.argtypes = [i64, i32, i32, i32]
        L.fk_assign.restype = i32
        L.fk_assign.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, vp, sz, vp]
        L.fk_assign_static.restype = i32
        L.fk_assign_static.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, vp]
        L.fk_assign_static_limit.restype = sz
        L.fk_assign_static_limit.argtypes = []
        L.fk_sort_inverse.restype = i32
        L.fk_sort_inverse.argtypes = [vp, vp, vp, i32, i64, i32, vp, sz, vp]
        L.fk_update.restype = i32
        L.fk_update.argtypes = [vp, vp, vp, vp, vp, vp, i32, i64, i32, i32, i32, vp, sz, vp]
        L.fk_lloyd_iter.restype = i32
        L.fk_lloyd_iter.argtypes = [vp, vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, vp, sz, vp]
        L.fk_lloyd_ooc.restype = i32
        L.fk_lloyd_ooc.argtypes = [vp, vp, vp, vp, i64, i32, i32, i32, i32, i64, vp, sz, vp]
        L.fk_standard_assign.restype = i32
        L.fk_standard_assign.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, vp, sz, vp]
        L.fk_standard_update.restype = i32
        L.fk_standard_update.argtypes = [vp, vp, vp, vp, vp, vp, i32, i64, i32, i32, i32, vp]
        cache = ctypes.POINTER(_KVCacheStruct)
        L.fk_kv_append.restype = i32
        L.fk_kv_append.argtypes = [cache, vp, i64, i64, vp, i64, i64, vp, i64, vp, vp, i64, i32, i32, vp, i64, i64, i32, vp, vp]
        L.fk_kv_read.restype = i32
        L.fk_kv_read.argtypes = [cache, vp, i64, vp, vp, vp]
        L.fk_kv_attend.restype = i32
        L.fk_kv_attend.argtypes = [cache, vp, i64, i64, i32, i64, vp, i32, vp, vp, i32, i32, i64, ctypes.c_float, i32, i32, vp, vp,
                                   vp, sz, vp]
        L.fk_kv_workspace_bytes.restype = sz
        L.fk_kv_workspace_bytes.argtypes = [cache, i32, i64, i32, i32, i64]
        f32 = ctypes.c_float
        L.fk_kv_attend_tree.restype = i32
        L.fk_kv_attend_tree.argtypes = [cache, vp, i64, i64, i32, i64, vp, i32, vp, vp, i32, i32, i64, f32, i32, vp, i32, vp, vp, vp, sz, vp]
        L.fk_kv_weigh.restype = i32
        L.fk_kv_weigh.argtypes = [cache, vp, i64, i64, i32, i64, vp, vp, i32, vp, vp, i32, i32, i64, f32, i32, i32, vp, f32, vp, vp, vp, sz, vp]
        L.fk_kv_weigh_workspace_bytes.restype = sz
        L.fk_kv_weigh_workspace_bytes.argtypes = [cache, i32, i64, i32, i32, i64]
        L.fk_kv_choose.restype = i32
        L.fk_kv_choose.argtypes = [cache, vp, vp, i32, vp, i32, i64, i32, i32, i32, vp, vp, vp, sz, vp]
        L.fk_kv_choose_workspace_bytes.restype = sz
        L.fk_kv_choose_workspace_bytes.argtypes = [cache, i32, i64]
        L.fk_kv_compact.restype = i32
        L.fk_kv_compact.argtypes = [cache, vp, i32, vp, i32, i32, vp, vp, vp, i32, i32, vp, vp]
        L.fk_kv_plan.restype = i32
        L.fk_kv_plan.argtypes = [cache, i32, i32, i32, i64, i32, ctypes.c_char_p, sz]
        L.fk_kv_plan_tree.restype = i32
        L.fk_kv_plan_tree.argtypes = L.fk_kv_plan.argtypes
        L.fk_plan.restype = i32
        L.fk_plan.argtypes = [i32, i64, i32, i32, i32, ctypes.c_char_p, sz]
        L.fk_set_option.restype = i32
        L.fk_set_option.argtypes = [ctypes.c_char_p, i32]
        L.fk_stage_timer_start.restype = None
        L.fk_stage_timer_start.argtypes = []
        L.fk_stage_timer_stop.restype = i32
        L.fk_stage_timer_stop.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i32)]
        _lib = L
    return _lib


def _check(status: int):
    if status != 0:
        raise FlashKMError(status, lib().fk_last_error().decode())


def _ptr(t: torch.Tensor | None):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(device) -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _dev(t: torch.Tensor, name: str, dtype=None, shape=None) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t


def _shape3(X: torch.Tensor, C: torch.Tensor):
    if X.dim() != 3 or C.dim() != 3 or X.shape[0] != C.shape[0] or X.shape[2] != C.shape[2]:
        raise ValueError("X must be [B,N,d] and C [B,K,d]")
    return X.shape[0], X.shape[1], X.shape[2], C.shape[1]


def fk_workspace_bytes(B: int, N: int, d: int, K: int, dtype: torch.dtype) -> int:
    return int(lib().fk_workspace_bytes(B, N, d, K, _DTYPE[dtype]))


def fk_ooc_workspace_bytes(chunk_rows: int, d: int, K: int, dtype: torch.dtype) -> int:
    return int(lib().fk_ooc_workspace_bytes(chunk_rows, d, K, _DTYPE[dtype]))


def make_workspace(B: int, N: int, d: int, K: int, dtype: torch.dtype, device) -> torch.Tensor:
    n = fk_workspace_bytes(B, N, d, K, dtype)
    if n == 0:
        raise FlashKMError(2, f"unsupported shape B={B} N={N} d={d} K={K} {dtype}")
    return torch.empty(n, dtype=torch.uint8, device=device)


def fk_assign(X, C, *, min_dist: bool = False, ws=None, out=None):
    """X [B,N,d], C [B,K,d] (same dtype) -> assign [B,N] int32 (and min_dist [B,N] float32)."""
    B, N, d, K = _shape3(X, C)
    _dev(X, "X"); _dev(C, "C", X.dtype)
    ws = ws if ws is not None else make_workspace(B, N, d, K, X.dtype, X.device)
    a = out if out is not None else torch.empty((B, N), dtype=torch.int32, device=X.device)
    _dev(a, "out", torch.int32, (B, N))
    md = torch.empty((B, N), dtype=torch.float32, device=X.device) if min_dist else None
    _check(lib().fk_assign(_ptr(X), _ptr(C), _ptr(a), _ptr(md), B, N, d, K, _DTYPE[X.dtype],
                           _ptr(ws), ws.numel(), _stream(X.device)))
    return (a, md) if min_dist else a


def fk_assign_static(X, C, *, min_dist: bool = False, out=None):
    """fk_assign without a workspace: the library's static scratch holds the centroid layout.
    The outputs are the caller's (allocated here when not passed in)."""
    B, N, d, K = _shape3(X, C)
    _dev(X, "X"); _dev(C, "C", X.dtype)
    a = out if out is not None else torch.empty((B, N), dtype=torch.int32, device=X.device)
    _dev(a, "out", torch.int32, (B, N))
    md = torch.empty((B, N), dtype=torch.float32, device=X.device) if min_dist else None
    _check(lib().fk_assign_static(_ptr(X), _ptr(C), _ptr(a), _ptr(md), B, N, d, K,
                                  _DTYPE[X.dtype], _stream(X.device)))
    return (a, md) if min_dist else a


def fk_sort_inverse(assign, K: int, *, ws=None):
    """assign [B,N] int32 -> (sorted_idx [B,N] int32, seg_offsets [B,K+1] int32)."""
    _dev(assign, "assign", torch.int32)
    B, N = assign.shape
    ws = ws if ws is not None else make_workspace(B, N, 8, K, torch.float32, assign.device)
    si = torch.empty((B, N), dtype=torch.int32, device=assign.device)
    so = torch.empty((B, K + 1), dtype=torch.int32, device=assign.device)
    _check(lib().fk_sort_inverse(_ptr(assign), _ptr(si), _ptr(so), B, N, K, _ptr(ws), ws.numel(),
                                 _stream(assign.device)))
    return si, so


def fk_update(X, assign, C_prev_f32, *, ws=None):
    """-> (C_f32 [B,K,d] float32, C_lp [B,K,d] in X's dtype, counts [B,K] int32)."""
    B, N, d, K = _shape3(X, C_prev_f32)
    _dev(X, "X"); _dev(assign, "assign", torch.int32, (B, N))
    _dev(C_prev_f32, "C_prev_f32", torch.float32)
    ws = ws if ws is not None else make_workspace(B, N, d, K, X.dtype, X.device)
    C_out = torch.empty_like(C_prev_f32)
    C_lp = torch.empty((B, K, d), dtype=X.dtype, device=X.device)
    counts = torch.empty((B, K), dtype=torch.int32, device=X.device)
    _check(lib().fk_update(_ptr(X), _ptr(assign), _ptr(C_prev_f32), _ptr(C_out), _ptr(C_lp),
                           _ptr(counts), B, N, d, K, _DTYPE[X.dtype], _ptr(ws), ws.numel(),
                           _stream(X.device)))
    return C_out, C_lp, counts


def fk_lloyd_iter(X, C_f32, iters: int, *, ws=None, C_lp=None, assign=None, counts=None):
    """`iters` Lloyd iterations in place on C_f32.  -> (assign, counts, C_lp)."""
    B, N, d, K = _shape3(X, C_f32)
    _dev(X, "X"); _dev(C_f32, "C_f32", torch.float32)
    ws = ws if ws is not None else make_workspace(B, N, d, K, X.dtype, X.device)
    if C_lp is None:
        C_lp = torch.empty((B, K, d), dtype=X.dtype, device=X.device)
    if assign is None:
        assign = torch.empty((B, N), dtype=torch.int32, device=X.device)
    if counts is None:
        counts = torch.empty((B, K), dtype=torch.int32, device=X.device)
    _dev(C_lp, "C_lp", X.dtype, (B, K, d))
    _dev(assign, "assign", torch.int32, (B, N)); _dev(counts, "counts", torch.int32, (B, K))
    _check(lib().fk_lloyd_iter(_ptr(X), _ptr(C_f32), _ptr(C_lp), _ptr(assign), _ptr(counts), B, N,
                               d, K, _DTYPE[X.dtype], iters, _ptr(ws), ws.numel(),
                               _stream(X.device)))
    return assign, counts, C_lp


def fk_lloyd_ooc(X_host, C_f32, iters: int, *, dev_ws, chunk_rows: int = 0, keep_assign=True):
    """X_host: pinned CPU tensor [N,d]; C_f32: device [K,d] float32, updated in place.

    -> (assign [N] int32 device or None, counts [K] int32 device).  Blocks until done.
    """
    if X_host.is_cuda or not X_host.is_pinned() or not X_host.is_contiguous() or X_host.dim() != 2:
        raise ValueError("X_host must be a contiguous pinned host tensor [N,d]")
    N, d = X_host.shape
    _dev(C_f32, "C_f32", torch.float32)
    if C_f32.dim() != 2 or C_f32.shape[1] != d:
        raise ValueError("C_f32 must be [K,d]")
    K = C_f32.shape[0]
    _dev(dev_ws, "dev_ws", torch.uint8)
    dev = C_f32.device
    a = torch.empty((N,), dtype=torch.int32, device=dev) if keep_assign else None
    counts = torch.empty((K,), dtype=torch.int32, device=dev)
    _check(lib().fk_lloyd_ooc(_ptr(X_host), _ptr(C_f32), _ptr(a), _ptr(counts), N, d, K,
                              _DTYPE[X_host.dtype], iters, chunk_rows, _ptr(dev_ws),
                              dev_ws.numel(), _stream(dev)))
    return a, counts


def fk_stage_timer_start() -> None:
    lib().fk_stage_timer_start()


def fk_stage_timer_stop() -> dict:
    """-> {stage: (total_ms, intervals)} for the stages recorded since the start call."""
    ms = (ctypes.c_double * 4)()
    n = (ctypes.c_int * 4)()
    rc = lib().fk_stage_timer_stop(ms, n)
    if rc < 0:
        raise FlashKMError(4, "stage timer: HIP event error")
    return {STAGES[i]: (float(ms[i]), int(n[i])) for i in range(4)}


def fk_plan(B: int, N: int, d: int, K: int, dtype: torch.dtype) -> str:
    """One-line description of the kernels and tilings chosen for this shape."""
    buf = ctypes.create_string_buffer(512)
    st = lib().fk_plan(B, N, d, K, _DTYPE[dtype], buf, len(buf))
    if st not in (0, 2):
        _check(st)
    return buf.value.decode()


def fk_set_option(name: str, value: int) -> None:
    _check(lib().fk_set_option(name.encode(), int(value)))


def fk_standard_assign(X, C, *, D=None, ws=None):
    """Comparator (paper Algorithm 1, kernels 1-2): materialises D [B,N,K] float32, then argmin.

    -> (assign [B,N] int32, D)."""
    B, N, d, K = _shape3(X, C)
    _dev(X, "X"); _dev(C, "C", X.dtype)
    ws = ws if ws is not None else make_workspace(B, N, d, K, X.dtype, X.device)
    if D is None:
        D = torch.empty((B, N, K), dtype=torch.float32, device=X.device)
    _dev(D, "D", torch.float32, (B, N, K))
    a = torch.empty((B, N), dtype=torch.int32, device=X.device)
    _check(lib().fk_standard_assign(_ptr(X), _ptr(C), _ptr(D), _ptr(a), B, N, d, K, _DTYPE[X.dtype],
                                    _ptr(ws), ws.numel(), _stream(X.device)))
    return a, D


def fk_standard_update(X, assign, C_prev_f32, *, sums=None):
    """Comparator (paper Algorithm 1, kernels 3-4): atomic scatter, then normalise.

    -> (C_f32 [B,K,d], counts [B,K] int32)."""
    B, N, d, K = _shape3(X, C_prev_f32)
    _dev(X, "X"); _dev(assign, "assign", torch.int32, (B, N))
    _dev(C_prev_f32, "C_prev_f32", torch.float32)
    if sums is None:
        sums = torch.empty((B, K, d), dtype=torch.float32, device=X.device)
    C_out = torch.empty_like(C_prev_f32)
    counts = torch.empty((B, K), dtype=torch.int32, device=X.device)
    _check(lib().fk_standard_update(_ptr(X), _ptr(assign), _ptr(C_prev_f32), _ptr(C_out),
                                    _ptr(counts), _ptr(sums), B, N, d, K, _DTYPE[X.dtype],
                                    _stream(X.device)))
    return C_out, counts


def _int32(**values):
    """ctypes cuts an integer down to the bits that the library takes: what does not fit is refused here."""
    for name, x in values.items():
        if not -2 ** 31 <= x < 2 ** 31:
            raise ValueError(f"{name}={x} is beyond 32 bits")


class KVCache:
    """A paged key/value cache in 4 bits over the caller's tensors (see fk_kv_cache in include/flashkm.h).

    codes [pages, heads, page_size, d/2] uint8, scales [pages, heads, page_size] and levels [heads, 16] of one 16-bit type, the
    levels ascending.  `KVCache.empty` allocates the codes and scales.  The tensors are attributes of these names; they may be replaced or
    moved in memory, every call asks where they are.

    The cache is for inference: results of fk_kv_append, fk_kv_read and fk_kv_attend carry no gradient, whether their inputs ask for one or not."""

    _TENSORS = ("k_codes", "v_codes", "k_scale", "v_scale", "k_levels", "v_levels")

    def __init__(self, k_codes, v_codes, k_scale, v_scale, k_levels, v_levels):
        self.k_codes, self.v_codes, self.k_scale, self.v_scale, self.k_levels, self.v_levels = (
            k_codes, v_codes, k_scale, v_scale, k_levels, v_levels)
        self._bind()

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        if name in self._TENSORS:
            object.__setattr__(self, "_at", None)                     # looked at anew by the next call

    def _bind(self):
        """Checks the tensors and lays down their sizes and places for the library."""
        k_codes, v_codes, k_scale, v_scale, k_levels, v_levels = tensors = [getattr(self, n) for n in self._TENSORS]
        if k_codes.dim() != 4:
            raise ValueError("k_codes must be [pages, heads, page_size, d/2]")
        P, H, S, half = k_codes.shape
        _int32(page_size=S, heads=H, d=2 * half)
        t = k_scale.dtype
        if t not in _DTYPE:
            raise ValueError(f"k_scale must be a type of the library, got {t}")
        _dev(k_codes, "k_codes", torch.uint8)
        _dev(v_codes, "v_codes", torch.uint8, k_codes.shape)
        _dev(k_scale, "k_scale", t, (P, H, S)); _dev(v_scale, "v_scale", t, (P, H, S))
        _dev(k_levels, "k_levels", t, (H, 16)); _dev(v_levels, "v_levels", t, (H, 16))
        if any(x.device != k_codes.device for x in tensors):
            raise ValueError("the cache's tensors must be on one device")
        self.pages, self.heads, self.page_size, self.d, self.dtype, self.device = P, H, S, 2 * half, t, k_codes.device
        at = tuple(x.data_ptr() for x in tensors)
        self._struct = _KVCacheStruct(*at, P, S, H, 2 * half, _DTYPE[t])
        self._ref, self._index, self._at = ctypes.byref(self._struct), k_codes.get_device(), at

    def _here(self):
        """The struct, with the tensors where they are now."""
        if self._at != (self.k_codes.data_ptr(), self.v_codes.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(),
                        self.k_levels.data_ptr(), self.v_levels.data_ptr()):
            self._bind()
        return self._ref

    @classmethod
    def empty(cls, pages: int, page_size: int, k_levels, v_levels, d: int) -> "KVCache":
        H, dev, t = k_levels.shape[0], k_levels.device, k_levels.dtype
        codes = [torch.zeros((pages, H, page_size, d // 2), dtype=torch.uint8, device=dev) for _ in range(2)]
        scale = [torch.zeros((pages, H, page_size), dtype=t, device=dev) for _ in range(2)]
        return cls(*codes, *scale, k_levels, v_levels)


# A call that serves one token is over on the GPU in a few microseconds, so that the checks below count: each asks a tensor's
# properties in one expression (pointers go to ctypes as plain numbers), and only a tensor that fails is looked at closer.
def _rows(t: torch.Tensor, name: str, cache: KVCache, T, heads):
    """Rows [T, heads, d] whose channels are contiguous -> (pointer, token stride, head stride)."""
    if t.dtype is cache.dtype and t.get_device() == cache._index and t.shape == (T, heads, cache.d):
        a, b, c = t.stride()
        if c == 1:
            return t.data_ptr(), a, b
        raise ValueError(f"{name}: the channels of a row must be contiguous")
    if t.dtype != cache.dtype:
        raise ValueError(f"{name} must be {cache.dtype}, got {t.dtype}")
    if t.get_device() != cache._index:
        raise ValueError(f"{name} must be on the cache's device")
    raise ValueError(f"{name} must have shape {(T, heads, cache.d)}, got {tuple(t.shape)}")


def _array(t: torch.Tensor, name: str, cache: KVCache, dtype, shape) -> int:
    """A contiguous tensor on the cache's device -> pointer."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == cache._index and t.is_contiguous():
        return t.data_ptr()
    if t.get_device() != cache._index:
        raise ValueError(f"{name} must be on the cache's device")
    return _dev(t, name, dtype, shape).data_ptr()


def _result(t, name: str, cache: KVCache, like: torch.Tensor, shape):
    """The caller's tensor for a result, or a new one with the rows of `like` -> (tensor, pointer)."""
    if t is not None:
        return t, _array(t, name, cache, cache.dtype, shape)
    t = torch.empty_like(like)                   # (half a microsecond less than torch.empty with a type and a device)
    if not t.is_contiguous():
        t = torch.empty(shape, dtype=cache.dtype, device=cache.device)
    return t, t.data_ptr()


def _raw_stream(cache: KVCache) -> int:
    return torch._C._cuda_getCurrentRawStream(cache._index)


def fk_kv_append(cache: KVCache, k, v, slots, *, positions=None, cos_sin=None, interleaved: bool = False, q=None, q_out=None):
    """k, v [T, heads, d] into the slots [T] int64 of the cache, keys turned by the angles of positions [T] int32 (cos_sin
    [max_pos, rot] float32: cosines, then sines); q [T, q_heads, d] is turned likewise and returned (None without q)."""
    ref = cache._here()
    T, H, d = k.shape[0], cache.heads, cache.d
    kp, kt, kh = _rows(k, "k", cache, T, H)
    vp, vt, vh = _rows(v, "v", cache, T, H)
    rot = max_pos = cs = ps = 0
    if cos_sin is not None:
        if cos_sin.dim() != 2:
            raise ValueError("cos_sin must be [max_pos, rot]")
        max_pos, rot = cos_sin.shape
        if rot:
            if positions is None:
                raise ValueError("cos_sin needs positions")
            cs = _array(cos_sin, "cos_sin", cache, torch.float32, cos_sin.shape)
            ps = _array(positions, "positions", cache, torch.int32, (T,))
    qp = qt = qh = heads = qo = 0
    if q is not None:
        heads = q.shape[1]
        qp, qt, qh = _rows(q, "q", cache, T, heads)
        q_out, qo = _result(q_out, "q_out", cache, q, (T, heads, d))
    _check(lib().fk_kv_append(ref, kp, kt, kh, vp, vt, vh, _array(slots, "slots", cache, torch.int64, (T,)), T, cs, ps,
                              max_pos, rot, interleaved, qp, qt, qh, heads, qo, _raw_stream(cache)))
    return q_out if q is not None else None


def fk_kv_read(cache: KVCache, slots, *, k_out=None, v_out=None):
    """The rows at slots [T] int64 as the values they stand for -> (k, v) [T, heads, d]."""
    ref = cache._here()
    T = slots.shape[0]
    shape = (T, cache.heads, cache.d)
    if k_out is None:
        k_out = cache.k_scale.new_empty(shape)
        kp = k_out.data_ptr()
    else:
        kp = _array(k_out, "k_out", cache, cache.dtype, shape)
    v_out, vp = _result(v_out, "v_out", cache, k_out, shape)
    _check(lib().fk_kv_read(ref, _array(slots, "slots", cache, torch.int64, (T,)), T, kp, vp, _raw_stream(cache)))
    return k_out, v_out


def fk_kv_workspace_bytes(cache: KVCache, B: int, q_heads: int, Tq: int, max_q: int, max_len: int) -> int:
    _int32(B=B, q_heads=q_heads, max_q=max_q)
    return int(lib().fk_kv_workspace_bytes(cache._here(), q_heads, Tq, B, max_q, max_len))


def make_kv_workspace(cache: KVCache, B: int, q_heads: int, Tq: int, max_q: int, max_len: int) -> torch.Tensor:
    """Workspace of fk_kv_attend for these sizes.  Fewer sequences or queries may need more (256 (d + 2) bytes a compute unit and 512
    are enough for any)."""
    n = fk_kv_workspace_bytes(cache, B, q_heads, Tq, max_q, max_len)
    if n == 0:
        raise FlashKMError(2, f"unsupported attention: {lib().fk_last_error().decode()}")
    return torch.empty(n, dtype=torch.uint8, device=cache.device)


def _plan(call, cache: KVCache, B: int, q_heads: int, max_q: int, max_len: int, window: int) -> str:
    _int32(B=B, q_heads=q_heads, max_q=max_q)
    buf = ctypes.create_string_buffer(256)
    window = min(window, 2 ** 31 - 1)                                 # as in fk_kv_attend
    _int32(window=window)
    _check(call(cache._here(), q_heads, B, max_q, max_len, window, buf, len(buf)))
    return buf.value.decode()


def fk_kv_plan(cache: KVCache, B: int, q_heads: int, max_q: int, max_len: int, window: int = 0) -> str:
    """One-line description of what fk_kv_attend would launch for these sizes."""
    return _plan(lib().fk_kv_plan, cache, B, q_heads, max_q, max_len, window)


def fk_kv_plan_tree(cache: KVCache, B: int, q_heads: int, max_q: int, max_len: int, window: int = 0) -> str:
    """One-line description of what fk_kv_attend_tree would launch for these sizes."""
    return _plan(lib().fk_kv_plan_tree, cache, B, q_heads, max_q, max_len, window)


_EWORKSPACE = 3


def _workspace(cache: KVCache, n: int) -> torch.Tensor:
    return torch.empty(n, dtype=torch.uint8, device=cache.device)


def _queries(cache: KVCache, q, pages, q_start, max_q, window):
    """What the queries' arguments come to -> (B, max_pages, pointer of q_start, max_q, window)."""
    B, max_pages = pages.shape
    qs = 0
    if max_q is None:
        if q_start is not None:
            raise ValueError("q_start needs max_q")
        max_q = max(1, q.shape[0] // max(1, B))                       # (no sequence: the library refuses it)
    if q_start is not None:
        qs = _array(q_start, "q_start", cache, torch.int32, (B + 1,))
    if max_q >> 31 or window >> 31:                                   # below 0, which the library refuses, or beyond it
        window = min(window, 2 ** 31 - 1)                             # (no sequence is that long)
        _int32(max_q=max_q, window=window)
    return B, max_pages, qs, max_q, window


def fk_kv_attend(cache: KVCache, q, pages, lens, *, q_start=None, max_q=None, max_len: int = 0, scale=None, causal: bool = True,
                 window: int = 0, lse: bool = False, ws=None, out=None):
    """q [Tq, q_heads, d] against the cached sequences: pages [B, max_pages] int32, lens [B] int32.  The queries of sequence b are
    q[q_start[b] : q_start[b+1]] (q_start [B+1] int32 with the most of a sequence in max_q; without it max_q each, one by default), the
    last tokens of the sequence.  -> out [Tq, q_heads, d] (and the logarithm of the sums [Tq, q_heads] float32)."""
    ref = cache._here()
    Tq, heads, _ = q.shape
    qp, qt, qh = _rows(q, "q", cache, Tq, heads)
    B, max_pages, qs, max_q, window = _queries(cache, q, pages, q_start, max_q, window)
    if not max_len:
        max_len = max_pages * cache.page_size
    if ws is None:
        ws = make_kv_workspace(cache, B, heads, Tq, max_q, max_len)
    out, op = _result(out, "out", cache, q, (Tq, heads, cache.d))
    le = torch.empty((Tq, heads), dtype=torch.float32, device=cache.device) if lse else None
    _check(lib().fk_kv_attend(ref, qp, qt, qh, heads, Tq, _array(pages, "pages", cache, torch.int32, (B, max_pages)), max_pages,
                              _array(lens, "lens", cache, torch.int32, (B,)), qs, B, max_q, max_len,
                              cache.d ** -0.5 if scale is None else scale, causal, window,
                              op, le.data_ptr() if lse else 0,
                              _array(ws, "ws", cache, torch.uint8, ws.shape), ws.numel(), _raw_stream(cache)))
    return (out, le) if lse else out


def fk_kv_attend_tree(cache: KVCache, q, pages, lens, tree, *, q_start=None, max_q=None, max_len: int = 0, scale=None, window: int = 0,
                      lse: bool = False, ws=None, out=None):
    """fk_kv_attend for a tree of drafted tokens, the last ones of each sequence: query i sees what lies before the tree and the
    tree's tokens j whose bit j % 64 of tree[i, j // 64] is set (tree [Tq, words] int64; kv_cache.tree_masks makes it)."""
    ref = cache._here()
    Tq, heads, _ = q.shape
    qp, qt, qh = _rows(q, "q", cache, Tq, heads)
    B, max_pages, qs, max_q, window = _queries(cache, q, pages, q_start, max_q, window)
    if tree.dim() != 2:
        raise ValueError("tree must be [Tq, words]")
    words = tree.shape[1]
    _int32(words=words)
    if not max_len:
        max_len = max_pages * cache.page_size
    if ws is None:
        ws = make_kv_workspace(cache, B, heads, Tq, max_q, max_len)
    out, op = _result(out, "out", cache, q, (Tq, heads, cache.d))
    le = torch.empty((Tq, heads), dtype=torch.float32, device=cache.device) if lse else None
    _check(lib().fk_kv_attend_tree(ref, qp, qt, qh, heads, Tq, _array(pages, "pages", cache, torch.int32, (B, max_pages)), max_pages,
                                   _array(lens, "lens", cache, torch.int32, (B,)), qs, B, max_q, max_len,
                                   cache.d ** -0.5 if scale is None else scale, window,
                                   _array(tree, "tree", cache, torch.int64, (Tq, words)), words, op, le.data_ptr() if lse else 0,
                                   _array(ws, "ws", cache, torch.uint8, ws.shape), ws.numel(), _raw_stream(cache)))
    return (out, le) if lse else out


def fk_kv_weigh(cache: KVCache, q, lse, pages, lens, mass, *, q_start=None, max_q=None, max_len: int = 0, scale=None, causal: bool = True,
                window: int = 0, known=None, decay: float = 1.0, ws=None, out=None):
    """The attention weights of q [Tq, q_heads, d], whose softmax sums have the logarithms lse [Tq, q_heads] float32 (fk_kv_attend gives
    them), added up for every token and cache head into mass [pages, heads, page_size] float32, or into `out` beside it.  Tokens from
    place known[b] on ([B] int32) have no weights yet; older ones fade by `decay`.  -> mass, or out"""
    ref = cache._here()
    Tq, heads, _ = q.shape
    qp, qt, qh = _rows(q, "q", cache, Tq, heads)
    B, max_pages, qs, max_q, window = _queries(cache, q, pages, q_start, max_q, window)
    shape = (cache.pages, cache.heads, cache.page_size)
    mp = _array(mass, "mass", cache, torch.float32, shape)
    op = mp if out is None else _array(out, "out", cache, torch.float32, shape)
    L = lib()
    args = (ref, qp, qt, qh, heads, Tq, _array(lse, "lse", cache, torch.float32, (Tq, heads)),
            _array(pages, "pages", cache, torch.int32, (B, max_pages)), max_pages, _array(lens, "lens", cache, torch.int32, (B,)), qs, B, max_q,
            max_len, cache.d ** -0.5 if scale is None else scale, causal, window,
            0 if known is None else _array(known, "known", cache, torch.int32, (B,)), decay, mp, op)
    if ws is not None:
        _check(L.fk_kv_weigh(*args, _array(ws, "ws", cache, torch.uint8, ws.shape), ws.numel(), _raw_stream(cache)))
    else:
        status = L.fk_kv_weigh(*args, 0, 0, _raw_stream(cache))       # few queries need no workspace, and their calls are the short ones
        if status == _EWORKSPACE:
            room = max_pages * cache.page_size
            ws = _workspace(cache, fk_kv_weigh_workspace_bytes(cache, B, heads, Tq, max_q, min(max_len or room, room)))
            status = L.fk_kv_weigh(*args, ws.data_ptr(), ws.numel(), _raw_stream(cache))
        _check(status)
    return mass if out is None else out


def fk_kv_weigh_workspace_bytes(cache: KVCache, B: int, q_heads: int, Tq: int, max_q: int, max_len: int) -> int:
    """Bytes of `ws` for fk_kv_weigh of these sizes, and of these alone; 0 where it needs none.  max_len: at most what the page table has room for."""
    _int32(B=B, q_heads=q_heads, max_q=max_q)
    return int(lib().fk_kv_weigh_workspace_bytes(cache._here(), q_heads, Tq, B, max_q, max_len))


def fk_kv_choose_workspace_bytes(cache: KVCache, B: int, max_len: int) -> int:
    """Bytes of `ws` for fk_kv_choose; 0 where it needs none.  max_len: at most what the page table has room for."""
    _int32(B=B)
    return int(lib().fk_kv_choose_workspace_bytes(cache._here(), B, max_len))


def fk_kv_choose(cache: KVCache, mass, pages, lens, keep: int, *, first: int = 0, last: int = 0, max_len: int = 0, kept=None, counts=None,
                 ws=None):
    """The places that stay when sequences are cut down to `keep` tokens: the first ones, the last ones, and those with the largest weights
    mass [pages, heads, page_size] float32, for each head -> (kept [B, heads, keep] int32, ascending, -1 behind them; counts [B] int32)."""
    ref = cache._here()
    B, max_pages = pages.shape
    _int32(keep=keep, first=first, last=last)
    L = lib()
    if kept is None:
        kept = torch.empty((B, cache.heads, max(keep, 0)), dtype=torch.int32, device=cache.device)
    if counts is None:
        counts = torch.empty_like(lens)
    args = (ref, _array(mass, "mass", cache, torch.float32, (cache.pages, cache.heads, cache.page_size)),
            _array(pages, "pages", cache, torch.int32, (B, max_pages)), max_pages, _array(lens, "lens", cache, torch.int32, (B,)), B, max_len, keep,
            first, last, _array(kept, "kept", cache, torch.int32, (B, cache.heads, keep)), _array(counts, "counts", cache, torch.int32, (B,)))
    if ws is not None:
        _check(L.fk_kv_choose(*args, _array(ws, "ws", cache, torch.uint8, ws.shape), ws.numel(), _raw_stream(cache)))
    else:
        status = L.fk_kv_choose(*args, 0, 0, _raw_stream(cache))      # (as in fk_kv_weigh)
        if status == _EWORKSPACE:
            room = max_pages * cache.page_size
            ws = _workspace(cache, fk_kv_choose_workspace_bytes(cache, B, min(max_len or room, room)))
            status = L.fk_kv_choose(*args, ws.data_ptr(), ws.numel(), _raw_stream(cache))
        _check(status)
    return kept, counts


def fk_kv_compact(cache: KVCache, pages, kept, counts, *, start=None, to_pages=None, mass=None):
    """Moves rows to the front of their sequences: place start[b] + j gets the row of place start[b] + kept[b, h, j], for j < counts[b]
    (kept [B, heads or 1, most] int32, ascending; counts, start [B] int32), and mass [pages, heads, page_size] float32 likewise; in place, or
    into the pages of to_pages [B, max_pages] int32."""
    ref = cache._here()
    B, max_pages = pages.shape
    if kept.dim() != 3:
        raise ValueError("kept must be [B, heads or 1, places]")
    _, heads, most = kept.shape
    to, to_max = 0, 0
    if to_pages is not None:
        if to_pages.dim() != 2:
            raise ValueError("to_pages must be [B, max_pages]")
        to_max = to_pages.shape[1]
        to = _array(to_pages, "to_pages", cache, torch.int32, (B, to_max))
    _check(lib().fk_kv_compact(ref, _array(pages, "pages", cache, torch.int32, (B, max_pages)), max_pages,
                               _array(kept, "kept", cache, torch.int32, (B, heads, most)), heads, most,
                               _array(counts, "counts", cache, torch.int32, (B,)),
                               0 if start is None else _array(start, "start", cache, torch.int32, (B,)), to, to_max, B,
                               0 if mass is None else _array(mass, "mass", cache, torch.float32,
                                                             (cache.pages, cache.heads, cache.page_size)), _raw_stream(cache)))
