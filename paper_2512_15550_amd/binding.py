"""ctypes binding of ``libctkvr.so`` -- argument marshalling only.

Device arguments are torch tensors (used for their memory and for the current
HIP stream); host arguments are numpy arrays.  Function names are the C ABI's.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libctkvr.so")

F32, BF16 = 0, 1
LAST_C, KMEANS = 0, 1
BUILD_EXACT, BUILD_MFMA = 0, 1

_STATUS = {0: "OK", -1: "EINVAL", -2: "ENOMEM", -3: "EHIP", -4: "EUNSUPPORTED"}


class CtkvrError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ctkvr: {_STATUS.get(code, code)}: {msg}")
        self.code = code


class _CParams(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("n_centroids", ctypes.c_int32), ("centroid_div", ctypes.c_int32), ("list_len", ctypes.c_int32),
                ("n_probe", ctypes.c_int32), ("top_k", ctypes.c_int32), ("sm_scale", ctypes.c_float),
                ("centroid_mode", ctypes.c_int32), ("kmeans_iters", ctypes.c_int32), ("build_algo", ctypes.c_int32),
                ("n_init", ctypes.c_int32), ("n_local", ctypes.c_int32)]


class _CInfo(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("c_max", ctypes.c_int32),
                ("list_len", ctypes.c_int32), ("n_probe", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("l_stride", ctypes.c_int32), ("index_bytes", ctypes.c_int64), ("device_bytes", ctypes.c_int64)]


class _CCacheParams(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("num_pages", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("sm_scale", ctypes.c_float), ("softcap", ctypes.c_float), ("rope_base", ctypes.c_double),
                ("rope_freq", ctypes.c_void_p), ("rope_axis", ctypes.c_void_p)]


@dataclass
class Params:
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int = 128
    page_size: int = 16
    dtype: int = BF16
    n_centroids: int = 0
    centroid_div: int = 0
    list_len: int = 0
    n_probe: int = 0
    top_k: int = 0
    sm_scale: float = 0.0
    centroid_mode: int = LAST_C
    kmeans_iters: int = 0
    build_algo: int = BUILD_EXACT
    n_init: int = 0
    n_local: int = 0

    def c(self) -> _CParams:
        return _CParams(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.page_size, self.dtype,
                        self.n_centroids, self.centroid_div, self.list_len, self.n_probe, self.top_k,
                        float(self.sm_scale), self.centroid_mode, self.kmeans_iters, self.build_algo, self.n_init,
                        self.n_local)


_lib = None

EXPORTS = ["ctkvr_build_index", "ctkvr_index_load", "ctkvr_decode_step", "ctkvr_free", "ctkvr_last_error",
           "ctkvr_index_info", "ctkvr_index_lists", "ctkvr_index_centroids", "ctkvr_index_last_candidates",
           "ctkvr_profile_enable", "ctkvr_profile_collect", "ctkvr_centroid_update", "ctkvr_decode_step_window",
           "ctkvr_selftest_exp", "ctkvr_decode_step_static", "ctkvr_index_set_decode_path", "ctkvr_index_decode_path",
           "ctkvr_index_check", "ctkvr_profile_phases", "ctkvr_measure_dispatch_floor", "ctkvr_index_build_route", "ctkvr_release_scratch",
           "ctkvr_cache_create", "ctkvr_cache_free", "ctkvr_cache_append", "ctkvr_cache_attn", "ctkvr_cache_weights", "ctkvr_cache_evict"]
PATH_AUTO, PATH_STAGED, PATH_FUSED = 0, 1, 2
N_STAGES = 9
STAGE_NAMES = ["centroid_cos", "recall_gather", "score", "denom", "keyhist", "classify",
               "rerank_select", "sparse_attn", "null"]


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load ``libctkvr.so``; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2512_15550_amd.build` "
                          "(or __graft_entry__.build()); there is no fallback path")
    L = ctypes.CDLL(_LIB_PATH)
    vp, ip, fp = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
    L.ctkvr_last_error.restype = ctypes.c_char_p
    L.ctkvr_build_index.restype = ctypes.c_int
    L.ctkvr_build_index.argtypes = [ctypes.POINTER(_CParams), vp, ip, ctypes.c_int32, vp, ip, ctypes.c_int32, ip, ip,
                                    vp, ctypes.POINTER(ctypes.c_void_p)]
    L.ctkvr_index_load.restype = ctypes.c_int
    L.ctkvr_index_load.argtypes = [ctypes.POINTER(_CParams), ip, vp, ip, vp, ctypes.POINTER(ctypes.c_void_p)]
    L.ctkvr_decode_step.restype = ctypes.c_int
    L.ctkvr_decode_step.argtypes = [vp, vp, vp, vp, ip, ctypes.c_int32, fp, fp, ip, ip, ip, vp]
    L.ctkvr_decode_step_static.restype = ctypes.c_int
    L.ctkvr_decode_step_static.argtypes = L.ctkvr_decode_step.argtypes
    L.ctkvr_decode_step_window.restype = ctypes.c_int
    L.ctkvr_decode_step_window.argtypes = [vp, vp, vp, vp, ip, ctypes.c_int32, ip, fp, fp, ip, ip, ip, vp]
    L.ctkvr_centroid_update.restype = ctypes.c_int
    L.ctkvr_centroid_update.argtypes = [vp, vp, vp]
    L.ctkvr_free.restype = None
    L.ctkvr_free.argtypes = [vp]
    L.ctkvr_index_info.restype = ctypes.c_int
    L.ctkvr_index_info.argtypes = [vp, ctypes.POINTER(_CInfo)]
    for name in ("ctkvr_index_lists", "ctkvr_index_centroids", "ctkvr_index_last_candidates"):
        getattr(L, name).restype = ctypes.c_int
        getattr(L, name).argtypes = [vp, vp]
    L.ctkvr_profile_enable.restype = ctypes.c_int
    L.ctkvr_profile_enable.argtypes = [vp, ctypes.c_int32]
    L.ctkvr_profile_collect.restype = ctypes.c_int
    L.ctkvr_profile_collect.argtypes = [vp, vp, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]
    L.ctkvr_index_set_decode_path.restype = ctypes.c_int
    L.ctkvr_index_set_decode_path.argtypes = [vp, ctypes.c_int32]
    L.ctkvr_index_decode_path.restype = ctypes.c_int
    L.ctkvr_index_decode_path.argtypes = [vp]
    L.ctkvr_index_check.restype = ctypes.c_int
    L.ctkvr_index_check.argtypes = [vp]
    L.ctkvr_release_scratch.restype = ctypes.c_int
    L.ctkvr_release_scratch.argtypes = []
    L.ctkvr_index_build_route.restype = ctypes.c_int
    L.ctkvr_index_build_route.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]
    L.ctkvr_profile_phases.restype = ctypes.c_int
    L.ctkvr_profile_phases.argtypes = [vp, ctypes.c_int32, vp]
    L.ctkvr_measure_dispatch_floor.restype = ctypes.c_int
    L.ctkvr_measure_dispatch_floor.argtypes = [ctypes.c_int32, ctypes.POINTER(ctypes.c_float), vp]
    L.ctkvr_selftest_exp.restype = ctypes.c_int
    L.ctkvr_selftest_exp.argtypes = [ctypes.POINTER(ctypes.c_uint64), vp]
    i32, i64, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    L.ctkvr_cache_create.restype = ctypes.c_int
    L.ctkvr_cache_create.argtypes = [ctypes.POINTER(_CCacheParams), vp, ctypes.POINTER(ctypes.c_void_p)]
    L.ctkvr_cache_free.restype = None
    L.ctkvr_cache_free.argtypes = [vp]
    L.ctkvr_cache_append.restype = ctypes.c_int
    L.ctkvr_cache_append.argtypes = [vp, vp, i64, vp, i64, vp, i64, ip, ip, ip, ip, i32, vp, vp, vp, vp]
    L.ctkvr_cache_attn.restype = ctypes.c_int
    L.ctkvr_cache_attn.argtypes = [vp, vp, i64, vp, vp, ip, ip, ip, i32, fp, ip, ip, vp, fp, vp]
    L.ctkvr_cache_weights.restype = ctypes.c_int
    L.ctkvr_cache_weights.argtypes = [vp, vp, i64, fp, vp, ip, ip, ip, i32, fp, ip, ip, f32, fp, fp, i32, vp]
    L.ctkvr_cache_evict.restype = ctypes.c_int
    L.ctkvr_cache_evict.argtypes = [vp, fp, i32, ip, ip, i32, i32, i32, vp, vp, fp, ip, ip, vp]
    _lib = L
    return L


def ctkvr_last_error() -> str:
    return load_library().ctkvr_last_error().decode()


def _check(rc: int) -> None:
    if rc != 0:
        raise CtkvrError(rc, ctkvr_last_error())


def _dev(t, dtype=None) -> Optional[int]:
    """Device pointer of a contiguous CUDA/HIP torch tensor (None passes NULL)."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected dtype {dtype}, got {t.dtype}")
    return t.data_ptr()


def _host_i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a), dtype=np.int32)


def _stream() -> int:
    import torch
    return torch.cuda.current_stream().cuda_stream


def _torch_dtype(dtype: int):
    import torch
    return torch.bfloat16 if dtype == BF16 else torch.float32


class Index:
    """Owner of a ``ctkvr_index*``; freed on ``ctkvr_free`` or garbage collection."""

    def __init__(self, handle: int, params: Params):
        self.handle = handle
        self.params = params

    def __del__(self):
        try:
            ctkvr_free(self)
        except Exception:
            pass


def ctkvr_build_index(params: Params, q_prefill, cu_seqlens, q_is_tail: bool, k_pages, block_table, ctx_lens,
                      init_pos=None) -> Index:
    import torch
    L = load_library()
    cu = _host_i32(cu_seqlens)
    cl = _host_i32(ctx_lens)
    td = _torch_dtype(params.dtype)
    out = ctypes.c_void_p()
    cp = params.c()
    rc = L.ctkvr_build_index(ctypes.byref(cp), _dev(q_prefill, td), cu.ctypes.data, int(bool(q_is_tail)),
                             _dev(k_pages, td), _dev(block_table, torch.int32), int(block_table.shape[1]),
                             cl.ctypes.data, _dev(init_pos, torch.int32) if init_pos is not None else None, _stream(),
                             ctypes.byref(out))
    _check(rc)
    return Index(out.value, params)


def ctkvr_index_load(params: Params, ctx_lens, centroids: np.ndarray, lists: np.ndarray) -> Index:
    """centroids: host array [batch][h][C_max][d], uint16 bit patterns for bf16 or float32; lists int32."""
    L = load_library()
    cl = _host_i32(ctx_lens)
    want = np.uint16 if params.dtype == BF16 else np.float32
    cen = np.ascontiguousarray(centroids)
    if cen.dtype != want:
        raise ValueError(f"centroids must be {want}")
    li = _host_i32(lists)
    out = ctypes.c_void_p()
    cp = params.c()
    rc = L.ctkvr_index_load(ctypes.byref(cp), cl.ctypes.data, cen.ctypes.data, li.ctypes.data, _stream(),
                            ctypes.byref(out))
    _check(rc)
    return Index(out.value, params)


def ctkvr_decode_step(idx: Index, q, k_pages, v_pages, block_table, out, out_lse=None, out_sel=None, out_ncand=None,
                      out_probe=None) -> None:
    import torch
    L = load_library()
    td = _torch_dtype(idx.params.dtype)
    rc = L.ctkvr_decode_step(idx.handle, _dev(q, td), _dev(k_pages, td), _dev(v_pages, td),
                             _dev(block_table, torch.int32), int(block_table.shape[1]), _dev(out, torch.float32),
                             _dev(out_lse, torch.float32), _dev(out_sel, torch.int32), _dev(out_ncand, torch.int32),
                             _dev(out_probe, torch.int32), _stream())
    _check(rc)


def ctkvr_decode_step_static(idx: Index, q, k_pages, v_pages, block_table, out, out_lse=None, out_sel=None,
                             out_ncand=None, out_probe=None) -> None:
    """The decode step on the library's static scratch array (allocates nothing)."""
    import torch
    L = load_library()
    td = _torch_dtype(idx.params.dtype)
    rc = L.ctkvr_decode_step_static(idx.handle, _dev(q, td), _dev(k_pages, td), _dev(v_pages, td),
                                    _dev(block_table, torch.int32), int(block_table.shape[1]), _dev(out, torch.float32),
                                    _dev(out_lse, torch.float32), _dev(out_sel, torch.int32),
                                    _dev(out_ncand, torch.int32), _dev(out_probe, torch.int32), _stream())
    _check(rc)


def ctkvr_decode_step_window(idx: Index, q, k_pages, v_pages, block_table, cur_lens, out, out_lse=None, out_sel=None,
                             out_ncand=None, out_probe=None) -> None:
    """cur_lens: device int32 [batch] (tokens now in the cache) or None."""
    import torch
    L = load_library()
    td = _torch_dtype(idx.params.dtype)
    rc = L.ctkvr_decode_step_window(idx.handle, _dev(q, td), _dev(k_pages, td), _dev(v_pages, td),
                                    _dev(block_table, torch.int32), int(block_table.shape[1]),
                                    _dev(cur_lens, torch.int32), _dev(out, torch.float32), _dev(out_lse, torch.float32),
                                    _dev(out_sel, torch.int32), _dev(out_ncand, torch.int32),
                                    _dev(out_probe, torch.int32), _stream())
    _check(rc)


def ctkvr_centroid_update(idx: Index, q) -> None:
    td = _torch_dtype(idx.params.dtype)
    _check(load_library().ctkvr_centroid_update(idx.handle, _dev(q, td), _stream()))


def ctkvr_free(idx: Optional[Index]) -> None:
    if idx is not None and idx.handle:
        load_library().ctkvr_free(idx.handle)
        idx.handle = 0


def ctkvr_index_info(idx: Index) -> dict:
    info = _CInfo()
    _check(load_library().ctkvr_index_info(idx.handle, ctypes.byref(info)))
    return {name: getattr(info, name) for name, _ in _CInfo._fields_}


def ctkvr_index_lists(idx: Index) -> np.ndarray:
    i = ctkvr_index_info(idx)
    out = np.empty((i["batch"], i["n_kv_heads"], i["c_max"], i["list_len"]), np.int32)
    _check(load_library().ctkvr_index_lists(idx.handle, out.ctypes.data))
    return out


def ctkvr_index_centroids(idx: Index) -> np.ndarray:
    i = ctkvr_index_info(idx)
    out = np.empty((i["batch"], i["n_q_heads"], i["c_max"], i["head_dim"]),
                   np.uint16 if i["dtype"] == BF16 else np.float32)
    _check(load_library().ctkvr_index_centroids(idx.handle, out.ctypes.data))
    return out


def ctkvr_index_last_candidates(idx: Index) -> np.ndarray:
    i = ctkvr_index_info(idx)
    out = np.empty((i["batch"], i["n_kv_heads"], i["l_stride"]), np.int32)
    _check(load_library().ctkvr_index_last_candidates(idx.handle, out.ctypes.data))
    return out


def ctkvr_profile_enable(idx: Index, max_steps: int) -> None:
    _check(load_library().ctkvr_profile_enable(idx.handle, int(max_steps)))


def ctkvr_profile_collect(idx: Index, capacity_steps: int) -> np.ndarray:
    """ms per (step, stage) for the steps recorded since the last collect."""
    out = np.zeros((capacity_steps, N_STAGES), np.float32)
    n = ctypes.c_int32(0)
    _check(load_library().ctkvr_profile_collect(idx.handle, out.ctypes.data, int(capacity_steps), ctypes.byref(n)))
    return out[:n.value]


def ctkvr_selftest_exp() -> int:
    """Number of fp32 inputs in [-32, 0] on which the library's two forms of the fixed-point exponential differ."""
    n = ctypes.c_uint64(0)
    _check(load_library().ctkvr_selftest_exp(ctypes.byref(n), _stream()))
    return int(n.value)


def ctkvr_index_set_decode_path(idx: Index, path: int) -> None:
    """PATH_AUTO, PATH_STAGED (one launch per stage) or PATH_FUSED (the whole step in one launch)."""
    _check(load_library().ctkvr_index_set_decode_path(idx.handle, int(path)))


def ctkvr_index_decode_path(idx: Index) -> int:
    rc = load_library().ctkvr_index_decode_path(idx.handle)
    if rc < 0:
        _check(rc)
    return rc


def ctkvr_index_build_route(idx: Index):
    """(built by the candidate route?, chunks it handed back to the route that ranks every key)."""
    a, b = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(load_library().ctkvr_index_build_route(idx.handle, ctypes.byref(a), ctypes.byref(b)))
    return bool(a.value), int(b.value)


def ctkvr_release_scratch() -> None:
    """Frees the current device's memory kept between indexes and builds, and the pinned memory of list and centroid copies."""
    _check(load_library().ctkvr_release_scratch())


def ctkvr_index_check(idx: Index) -> None:
    """Synchronises; raises if a single-launch step on this index gave up a wait."""
    _check(load_library().ctkvr_index_check(idx.handle))


def ctkvr_profile_phases(idx: Index, enable: bool = True) -> np.ndarray:
    """The 16 wall-clock stamps (100 MHz ticks) of the last single-launch step's first block (0-7 leaving each
    phase, 8-13 arriving at each barrier); sets stamping on or off."""
    out = np.zeros(64, np.int64)
    _check(load_library().ctkvr_profile_phases(idx.handle, int(bool(enable)), out.ctypes.data))
    return out


def ctkvr_measure_dispatch_floor(n_launches: int = 200) -> float:
    """Microseconds per launch of a graph of empty kernels launched one behind the other."""
    us = ctypes.c_float(0.0)
    _check(load_library().ctkvr_measure_dispatch_floor(int(n_launches), ctypes.byref(us), _stream()))
    return float(us.value)


# ---- the paged KV cache ------------------------------------------------------
@dataclass
class CacheParams:
    """Geometry of a paged KV cache and of the calls on it; ``rope_freq`` (64 float64) and ``rope_axis`` (64 uint8) are
    host arrays or None."""
    batch: int
    n_q_heads: int
    n_kv_heads: int
    num_pages: int
    max_pages: int
    max_new: int
    head_dim: int = 128
    page_size: int = 16
    dtype: int = BF16
    sm_scale: float = 0.0
    softcap: float = 0.0
    rope_base: float = 10000.0
    rope_freq: Optional[np.ndarray] = None
    rope_axis: Optional[np.ndarray] = None


class Cache:
    """Owner of a ``ctkvr_cache*`` on one device; freed on ``ctkvr_cache_free`` or garbage collection."""

    def __init__(self, handle: int, params: CacheParams, device: int):
        import torch
        p = params
        self.handle = handle
        self.params = p
        self.device = device
        self.torch_dtype = _torch_dtype(p.dtype)
        self.n_axes = 1 if p.rope_axis is None else int(np.max(p.rope_axis)) + 1
        # what every call asks for; a step of one token is a few microseconds, of which looking these up again would be a fair part
        self._lib = load_library()
        self._int, self._float = torch.int32, torch.float32
        self._shapes = {"pages": (p.num_pages, p.n_kv_heads, p.page_size, 128), "cu": (p.batch + 1,), "batch": (p.batch,),
                        "table": (p.batch, p.max_pages), "heads": (p.n_q_heads,)}
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self._stream = raw if raw is not None else (lambda d: torch.cuda.current_stream(d).cuda_stream)

    def stream(self) -> int:
        """The current stream of the cache's device."""
        return self._stream(self.device)

    def __del__(self):
        try:
            ctkvr_cache_free(self)
        except Exception:
            pass


def _on(cache: Cache, name, t, dtype, shape):
    """Device pointer of a contiguous tensor of this type and shape on the cache's device (None passes NULL)."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == cache.device:
        return t.data_ptr()
    raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on device {cache.device}, got "
                     f"{t.dtype}, {tuple(t.shape)}, strides {t.stride()}, {t.device}")


def _rows_on(cache: Cache, name, t, total, heads):
    """Device pointer and token stride of [total][heads][128], the heads of a token contiguous."""
    if t is None:
        return None, 0
    if t.dtype is cache.torch_dtype and t.shape == (total, heads, 128) and t.get_device() == cache.device:
        token, head, element = t.stride()
        if total == 0 or (element == 1 and (heads == 1 or head == 128)):
            return t.data_ptr(), (token if total > 1 else heads * 128)
    raise ValueError(f"{name}: expected a {cache.torch_dtype} tensor of shape {(total, heads, 128)} on device {cache.device}, a token's heads "
                     f"contiguous, got {t.dtype}, {tuple(t.shape)}, strides {t.stride()}, {t.device}")


def _pages_on(cache: Cache, name, t):
    return _on(cache, name, t, cache.torch_dtype, cache._shapes["pages"])


def _batch_on(cache: Cache, cu_new, cur_lens, block_table):
    s, i32 = cache._shapes, cache._int
    return (_on(cache, "cu_new", cu_new, i32, s["cu"]), _on(cache, "cur_lens", cur_lens, i32, s["batch"]),
            _on(cache, "block_table", block_table, i32, s["table"]))


def ctkvr_cache_create(params: CacheParams) -> Cache:
    import torch
    L = load_library()
    freq = None if params.rope_freq is None else np.ascontiguousarray(params.rope_freq, np.float64)
    axis = None if params.rope_axis is None else np.ascontiguousarray(params.rope_axis, np.uint8)
    for name, a in (("rope_freq", freq), ("rope_axis", axis)):
        if a is not None and a.shape != (64,):
            raise ValueError(f"{name}: expected 64 values, got shape {a.shape}")
    cp = _CCacheParams(params.batch, params.n_q_heads, params.n_kv_heads, params.head_dim, params.page_size, params.dtype,
                       params.num_pages, params.max_pages, params.max_new, float(params.sm_scale), float(params.softcap),
                       float(params.rope_base), None if freq is None else freq.ctypes.data, None if axis is None else axis.ctypes.data)
    out = ctypes.c_void_p()
    _check(L.ctkvr_cache_create(ctypes.byref(cp), _stream(), ctypes.byref(out)))
    return Cache(out.value, params, torch.cuda.current_device())


def ctkvr_cache_free(cache: Optional[Cache]) -> None:
    if cache is not None and cache.handle:
        load_library().ctkvr_cache_free(cache.handle)
        cache.handle = 0


def ctkvr_cache_append(cache: Cache, q, k, v, cu_new, cur_lens, block_table, q_out, k_pages, v_pages, positions=None) -> None:
    """q, k and v may be views of a fused projection; q and q_out, or k and v, may be None."""
    p = cache.params
    total = (q if q is not None else k).shape[0]
    cu, cur, table = _batch_on(cache, cu_new, cur_lens, block_table)
    (qp, qs), (kp, ks) = _rows_on(cache, "q", q, total, p.n_q_heads), _rows_on(cache, "k", k, total, p.n_kv_heads)
    vp, vs = _rows_on(cache, "v", v, total, p.n_kv_heads)
    _check(cache._lib.ctkvr_cache_append(
        cache.handle, qp, qs, kp, ks, vp, vs, _on(cache, "positions", positions, cache._int, (cache.n_axes, total)), cu, cur, table, total,
        _on(cache, "q_out", q_out, cache.torch_dtype, (total, p.n_q_heads, 128)), _pages_on(cache, "k_pages", k_pages),
        _pages_on(cache, "v_pages", v_pages), cache.stream()))


def _masks_on(cache: Cache, total, slopes, prefix_lens, first_key):
    return (_on(cache, "slopes", slopes, cache._float, cache._shapes["heads"]),
            _on(cache, "prefix_lens", prefix_lens, cache._int, cache._shapes["batch"]),
            _on(cache, "first_key", first_key, cache._int, (total,)))


def ctkvr_cache_attn(cache: Cache, q, k_pages, v_pages, cu_new, cur_lens, block_table, out, out_lse=None, slopes=None, prefix_lens=None,
                     first_key=None) -> None:
    h, total = cache.params.n_q_heads, q.shape[0]
    cu, cur, table = _batch_on(cache, cu_new, cur_lens, block_table)
    qp, qs = _rows_on(cache, "q", q, total, h)
    _check(cache._lib.ctkvr_cache_attn(
        cache.handle, qp, qs, _pages_on(cache, "k_pages", k_pages), _pages_on(cache, "v_pages", v_pages), cu, cur, table, total,
        *_masks_on(cache, total, slopes, prefix_lens, first_key), _on(cache, "out", out, cache.torch_dtype, (total, h, 128)),
        _on(cache, "out_lse", out_lse, cache._float, (total, h)), cache.stream()))


def ctkvr_cache_weights(cache: Cache, q, lse, k_pages, cu_new, cur_lens, block_table, weights_in, weights_out, decay=1.0, slopes=None,
                        prefix_lens=None, first_key=None) -> None:
    """weights_in (None: zeros) and weights_out: fp32 [batch][g][weights_stride]."""
    p, total = cache.params, q.shape[0]
    cu, cur, table = _batch_on(cache, cu_new, cur_lens, block_table)
    qp, qs = _rows_on(cache, "q", q, total, p.n_q_heads)
    shape = (p.batch, p.n_kv_heads, weights_out.shape[-1])
    _check(cache._lib.ctkvr_cache_weights(
        cache.handle, qp, qs, _on(cache, "lse", lse, cache._float, (total, p.n_q_heads)), _pages_on(cache, "k_pages", k_pages), cu, cur,
        table, total, *_masks_on(cache, total, slopes, prefix_lens, first_key), float(decay),
        _on(cache, "weights_in", weights_in, cache._float, shape), _on(cache, "weights_out", weights_out, cache._float, shape), shape[2],
        cache.stream()))


def ctkvr_cache_evict(cache: Cache, weights_in, k_pages, v_pages, cur_lens, block_table, budget, out_ids, n_init=0, n_local=0,
                      weights_out=None, out_lens=None) -> None:
    """out_ids: int32 [batch][g][budget]; out_lens: int32 [batch], cur_lens itself or None."""
    p = cache.params
    shape = (p.batch, p.n_kv_heads, weights_in.shape[-1])
    _check(cache._lib.ctkvr_cache_evict(
        cache.handle, _on(cache, "weights_in", weights_in, cache._float, shape), shape[2],
        _on(cache, "cur_lens", cur_lens, cache._int, cache._shapes["batch"]), _on(cache, "block_table", block_table, cache._int, cache._shapes["table"]),
        int(budget), int(n_init), int(n_local), _pages_on(cache, "k_pages", k_pages), _pages_on(cache, "v_pages", v_pages),
        _on(cache, "weights_out", weights_out, cache._float, shape),
        _on(cache, "out_ids", out_ids, cache._int, (p.batch, p.n_kv_heads, int(budget))),
        _on(cache, "out_lens", out_lens, cache._int, cache._shapes["batch"]), cache.stream()))
