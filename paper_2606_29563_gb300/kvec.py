"""Python binding of libkvec (include/kvec.h): ctypes marshalling only.

Every function here forwards to the C ABI entry point of the same name.  All
computation happens in the CUDA kernels of libkvec; there is no Python or CPU
fallback.  If the library is missing, importing this module still works but the
first call raises ``KvecUnavailable`` (build it with ``build.build()``).
"""
from __future__ import annotations

import ctypes
import os
import threading
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libkvec.so")

KVEC_OK = 0
KVEC_ERR_INVALID_ARG = 1
KVEC_ERR_UNSUPPORTED = 2
KVEC_ERR_CUDA = 3
KVEC_ERR_DEVICE_TIMEOUT = 4
KVEC_ERR_OOM = 5

# kernel ids of kvec_kernel_time
KERNEL_NAMES = ("score", "window", "heads", "select", "gather")

EXPORTED = ("kvec_create", "kvec_destroy", "kvec_state_bytes", "kvec_reset", "kvec_select_layer",
            "kvec_select_layers", "kvec_debug_scores", "kvec_sync_status", "kvec_set_profiling",
            "kvec_kernel_time", "kvec_status_string", "kvec_last_error", "kvec_select_layer_noalloc",
            "kvec_select_layer_lse", "kvec_select_layers_lse", "kvec_decode_attention",
            "kvec_noalloc_sync_status", "kvec_set_test_fault", "kvec_output_capacity",
            "kvec_rotate_append", "kvec_paged_decode_bytes", "kvec_paged_decode_window_bytes", "kvec_paged_decode",
            "kvec_paged_evict", "kvec_prefill_bytes", "kvec_prefill_attention", "kvec_rotate_append_quant",
            "kvec_paged_decode_quant", "kvec_paged_evict_quant", "kvec_paged_read", "kvec_shared_decode_bytes",
            "kvec_shared_decode", "kvec_paged_decode_quant_bytes", "kvec_shared_decode_quant_bytes",
            "kvec_shared_decode_quant")

KVEC_BF16 = 0
KVEC_FP16 = 1


class KvecUnavailable(ImportError):
    pass


class KvecError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"kvec status {status}: {message}")
        self.status = status


class kvec_params(ctypes.Structure):
    _fields_ = [
        ("num_q_heads", ctypes.c_int), ("num_kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
        ("window", ctypes.c_int), ("obs_window", ctypes.c_int), ("ext_window", ctypes.c_int),
        ("pool_kernel", ctypes.c_int), ("num_ext_heads", ctypes.c_int),
        ("lam", ctypes.c_float), ("beta", ctypes.c_float), ("softmax_scale", ctypes.c_float),
        ("max_batch", ctypes.c_int), ("max_seqlen", ctypes.c_int), ("max_layers", ctypes.c_int),
        ("pool_mode", ctypes.c_int), ("head_criterion", ctypes.c_int), ("all_positions", ctypes.c_int),
        ("head_budget", ctypes.c_int), ("ada_floor", ctypes.c_float),
    ]


class kvec_debug_view(ctypes.Structure):
    _fields_ = [
        ("P_O", ctypes.c_void_p), ("P_Oext", ctypes.c_void_p), ("I", ctypes.c_void_p),
        ("sigma", ctypes.c_void_p), ("htop", ctypes.c_void_p), ("pres_bits", ctypes.c_void_p),
        ("Pprime", ctypes.c_void_p), ("row_stats", ctypes.c_void_p),
        ("max_seqlen", ctypes.c_int), ("words_per_row", ctypes.c_int),
    ]


class kvec_paged_cache(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int), ("page_size", ctypes.c_int), ("num_pages", ctypes.c_int), ("max_pages", ctypes.c_int),
        ("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p), ("weights", ctypes.c_void_p),
        ("page_table", ctypes.c_void_p), ("lens", ctypes.c_void_p),
    ]


class kvec_paged_scales(ctypes.Structure):
    _fields_ = [("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p)]


class kvec_shared_prefix(ctypes.Structure):
    _fields_ = [
        ("num_groups", ctypes.c_int), ("max_pages", ctypes.c_int),
        ("page_table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("cu_seqs", ctypes.c_void_p),
    ]


class kvec_rotate_args(ctypes.Structure):
    _fields_ = [
        ("dtype", ctypes.c_int), ("num_tokens", ctypes.c_int),
        ("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
        ("q_norm", ctypes.c_void_p), ("k_norm", ctypes.c_void_p), ("eps", ctypes.c_float),
        ("rot_dim", ctypes.c_int), ("interleaved", ctypes.c_int), ("max_positions", ctypes.c_int),
        ("rot_table", ctypes.c_void_p), ("positions", ctypes.c_void_p),
        ("q_out", ctypes.c_void_p), ("k_out", ctypes.c_void_p),
    ]


_lib = None
_lock = threading.Lock()
_vp = ctypes.c_void_p
_pp = ctypes.POINTER(ctypes.c_void_p)


def load() -> ctypes.CDLL:
    """Loads libkvec.so once; raises KvecUnavailable when it has not been built."""
    global _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(LIB_PATH):
            raise KvecUnavailable(f"{LIB_PATH} is missing: build the CUDA library first "
                                  "(python -c 'import __graft_entry__ as g; g.build()')")
        lib = ctypes.CDLL(LIB_PATH)
        i, st = ctypes.c_int, ctypes.c_int
        sig = {
            "kvec_create": ([ctypes.POINTER(kvec_params), ctypes.POINTER(_vp)], st),
            "kvec_destroy": ([_vp], st),
            "kvec_state_bytes": ([i], ctypes.c_size_t),
            "kvec_reset": ([_vp, _vp, i, _vp], st),
            "kvec_select_layer": ([_vp, i, _vp, _vp, _vp, _vp, _vp, _vp, i, _vp, _vp, _vp, _vp], st),
            "kvec_select_layers": ([_vp, i, i, _vp, _vp, _pp, _pp, _pp, _vp, i, _pp, _pp, _pp, _vp], st),
            "kvec_debug_scores": ([_vp, ctypes.POINTER(kvec_debug_view)], st),
            "kvec_sync_status": ([_vp], st),
            "kvec_set_profiling": ([_vp, i], st),
            "kvec_kernel_time": ([_vp, i, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int)], st),
            "kvec_status_string": ([i], ctypes.c_char_p),
            "kvec_last_error": ([], ctypes.c_char_p),
            "kvec_select_layer_noalloc": ([ctypes.POINTER(kvec_params), i, _vp, _vp, _vp, _vp, _vp, _vp, i, _vp,
                                           _vp, _vp, _vp], st),
            "kvec_select_layer_lse": ([_vp, i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, i, _vp, _vp, _vp, _vp], st),
            "kvec_select_layers_lse": ([_vp, i, i, _vp, _vp, _pp, _pp, _pp, _pp, _vp, i, _pp, _pp, _pp, _vp], st),
            "kvec_decode_attention": ([_vp, i, _vp, _vp, _vp, _vp, i, _vp, _vp], st),
            "kvec_noalloc_sync_status": ([_vp], st),
            "kvec_set_test_fault": ([i], None),
            "kvec_output_capacity": ([ctypes.POINTER(kvec_params), i], i),
            "kvec_rotate_append": ([_vp, ctypes.POINTER(kvec_rotate_args), i, _vp, ctypes.POINTER(kvec_paged_cache),
                                    _vp], st),
            "kvec_paged_decode_bytes": ([_vp, i, i, i], ctypes.c_size_t),
            "kvec_paged_decode_window_bytes": ([_vp, i, i, i, i, i], ctypes.c_size_t),
            "kvec_paged_decode": ([_vp, i, _vp, ctypes.POINTER(kvec_paged_cache), i, i, i, _vp, _vp, ctypes.c_size_t,
                                   _vp], st),
            "kvec_prefill_bytes": ([_vp, i, _vp, _vp, i, i], ctypes.c_size_t),
            "kvec_prefill_attention": ([_vp, i, i, _vp, _vp, _vp, _vp, _vp, _vp, _vp, i, i, _vp, _vp, _vp,
                                        ctypes.c_size_t, _vp], st),
            "kvec_paged_evict": ([_vp, i, ctypes.POINTER(kvec_paged_cache), _vp, i, i, i, i, i, _vp, _vp, _vp], st),
            "kvec_rotate_append_quant": ([_vp, ctypes.POINTER(kvec_rotate_args), i, _vp, ctypes.POINTER(kvec_paged_cache),
                                          ctypes.POINTER(kvec_paged_scales), _vp], st),
            "kvec_paged_decode_quant": ([_vp, i, _vp, ctypes.POINTER(kvec_paged_cache), ctypes.POINTER(kvec_paged_scales),
                                         i, i, i, _vp, _vp, ctypes.c_size_t, _vp], st),
            "kvec_paged_evict_quant": ([_vp, i, ctypes.POINTER(kvec_paged_cache), ctypes.POINTER(kvec_paged_scales), _vp,
                                        i, i, i, i, i, _vp, _vp, _vp], st),
            "kvec_paged_decode_quant_bytes": ([_vp, i, i, i, i, i], ctypes.c_size_t),
            "kvec_shared_decode_bytes": ([_vp, i, i, i], ctypes.c_size_t),
            "kvec_shared_decode_quant_bytes": ([_vp, i, i, i], ctypes.c_size_t),
            "kvec_shared_decode_quant": ([_vp, i, _vp, ctypes.POINTER(kvec_paged_cache), ctypes.POINTER(kvec_paged_scales),
                                          ctypes.POINTER(kvec_paged_cache), ctypes.POINTER(kvec_shared_prefix), i, i, _vp,
                                          _vp, ctypes.c_size_t, _vp], st),
            "kvec_shared_decode": ([_vp, i, _vp, ctypes.POINTER(kvec_paged_cache), ctypes.POINTER(kvec_shared_prefix), i, i,
                                    _vp, _vp, ctypes.c_size_t, _vp], st),
            "kvec_paged_read": ([_vp, i, ctypes.POINTER(kvec_paged_cache), ctypes.POINTER(kvec_paged_scales), _vp, _vp, i,
                                 _vp, _vp, _vp], st),
        }
        for name, (args, res) in sig.items():
            fn = getattr(lib, name)
            fn.argtypes = args
            fn.restype = res
        _lib = lib
        return lib


def _check(status: int) -> None:
    if status != KVEC_OK:
        msg = load().kvec_last_error().decode(errors="replace")
        raise KvecError(status, msg)


def _arr(ptrs: Sequence[int]):
    return (ctypes.c_void_p * len(ptrs))(*[ctypes.c_void_p(int(p)) for p in ptrs])


def kvec_create(params: kvec_params) -> int:
    h = ctypes.c_void_p()
    _check(load().kvec_create(ctypes.byref(params), ctypes.byref(h)))
    return h.value


def kvec_destroy(handle: int) -> None:
    _check(load().kvec_destroy(handle))


def kvec_state_bytes(max_seqlen: int) -> int:
    return int(load().kvec_state_bytes(int(max_seqlen)))


def kvec_reset(handle: int, state_ptr: int, batch: int, stream: int = 0) -> None:
    _check(load().kvec_reset(handle, state_ptr, int(batch), stream))


def kvec_select_layer(handle: int, batch: int, cu_host_ptr: int, cu_dev_ptr: int, q_obs: int, k: int, v: int,
                      state: int, budget: int, out_idx: int, out_k: int, out_v: int, stream: int = 0) -> None:
    _check(load().kvec_select_layer(handle, int(batch), cu_host_ptr, cu_dev_ptr, q_obs, k, v, state, int(budget),
                                    out_idx, out_k, out_v, stream))


def kvec_select_layers(handle: int, batch: int, cu_host_ptr: int, cu_dev_ptr: int, q_obs: Sequence[int],
                       k: Sequence[int], v: Sequence[int], state: int, budget: int, out_idx: Sequence[int],
                       out_k: Sequence[int], out_v: Sequence[int], stream: int = 0) -> None:
    n = len(q_obs)
    _check(load().kvec_select_layers(handle, n, int(batch), cu_host_ptr, cu_dev_ptr, _arr(q_obs), _arr(k), _arr(v),
                                     state, int(budget), _arr(out_idx), _arr(out_k), _arr(out_v), stream))


def kvec_select_layer_lse(handle: int, batch: int, cu_host_ptr: int, cu_dev_ptr: int, q_obs: int, k: int, v: int,
                          lse: int, state: int, budget: int, out_idx: int, out_k: int, out_v: int,
                          stream: int = 0) -> None:
    _check(load().kvec_select_layer_lse(handle, int(batch), cu_host_ptr, cu_dev_ptr, q_obs, k, v, lse, state,
                                        int(budget), out_idx, out_k, out_v, stream))


def kvec_select_layers_lse(handle: int, batch: int, cu_host_ptr: int, cu_dev_ptr: int, q_obs: Sequence[int],
                           k: Sequence[int], v: Sequence[int], lse: Sequence[int], state: int, budget: int,
                           out_idx: Sequence[int], out_k: Sequence[int], out_v: Sequence[int],
                           stream: int = 0) -> None:
    n = len(q_obs)
    _check(load().kvec_select_layers_lse(handle, n, int(batch), cu_host_ptr, cu_dev_ptr, _arr(q_obs), _arr(k),
                                         _arr(v), _arr(lse), state, int(budget), _arr(out_idx), _arr(out_k),
                                         _arr(out_v), stream))


def kvec_select_layer_noalloc(params: kvec_params, batch: int, cu_host_ptr: int, cu_dev_ptr: int, q_obs: int,
                              k: int, v: int, state: int, budget: int, out_idx: int, out_k: int, out_v: int,
                              stream: int = 0) -> None:
    """kvec_select_layer without a handle; scratch comes from the library's static device array."""
    _check(load().kvec_select_layer_noalloc(ctypes.byref(params), int(batch), cu_host_ptr, cu_dev_ptr, q_obs, k, v,
                                            state, int(budget), out_idx, out_k, out_v, stream))


def kvec_noalloc_sync_status(stream: int = 0) -> None:
    """Raises KvecError for a device-side error recorded by kvec_select_layer_noalloc calls."""
    _check(load().kvec_noalloc_sync_status(stream))


def kvec_output_capacity(params: kvec_params, budget: int) -> int:
    """Rows per KV head of the selection outputs (the budget for the uniform fill)."""
    cap = int(load().kvec_output_capacity(ctypes.byref(params), int(budget)))
    if cap < 1:
        raise KvecError(KVEC_ERR_INVALID_ARG, "invalid parameters or budget for the output capacity")
    return cap


def kvec_set_test_fault(fault: int) -> None:
    """Test hook of the error path (1: window kernels give up on a withheld accumulator;
    2: a warp of the score and general window kernels gives up on a wait; 3: kvec_create's larger
    allocations fail; 4: prefill attention and paged decode wait for what does not come; 0: off)."""
    load().kvec_set_test_fault(int(fault))


def kvec_decode_attention(handle: int, batch: int, q: int, k_cache: int, v_cache: int, lens: int, cap: int,
                          out: int, stream: int = 0) -> None:
    _check(load().kvec_decode_attention(handle, int(batch), q, k_cache, v_cache, lens, int(cap), out, stream))


def kvec_rotate_append(handle: int, args: kvec_rotate_args, batch: int, cu_tokens: Optional[int] = None,
                       cache: Optional[kvec_paged_cache] = None, stream: int = 0) -> None:
    _check(load().kvec_rotate_append(handle, args, batch, cu_tokens, cache, stream))


def kvec_paged_decode_bytes(handle: int, batch: int, max_len: int, with_weights: bool) -> int:
    return int(load().kvec_paged_decode_bytes(handle, batch, max_len, 1 if with_weights else 0))


def kvec_paged_decode_window_bytes(handle: int, batch: int, max_len: int, window: int, sinks: int, with_weights: bool) -> int:
    return int(load().kvec_paged_decode_window_bytes(handle, batch, max_len, window, sinks, 1 if with_weights else 0))


def kvec_paged_decode(handle: int, batch: int, q: int, cache: kvec_paged_cache, max_len: int, window: int, sinks: int,
                      out: int, scratch: int, scratch_bytes: int, stream: int = 0) -> None:
    _check(load().kvec_paged_decode(handle, batch, q, cache, max_len, window, sinks, out, scratch, scratch_bytes,
                                    stream))


def kvec_paged_evict(handle: int, batch: int, cache: kvec_paged_cache, new_table: int, new_max_pages: int, max_len: int,
                     budget: int, sinks: int, recent: int, new_lens: int, kept: int, stream: int = 0) -> None:
    _check(load().kvec_paged_evict(handle, batch, cache, new_table, new_max_pages, max_len, budget, sinks, recent,
                                   new_lens, kept, stream))


def kvec_paged_decode_quant_bytes(handle: int, batch: int, max_len: int, window: int, sinks: int, with_weights: bool) -> int:
    return int(load().kvec_paged_decode_quant_bytes(handle, batch, max_len, window, sinks, 1 if with_weights else 0))


def kvec_shared_decode_bytes(handle: int, batch: int, max_len: int, with_weights: bool) -> int:
    return int(load().kvec_shared_decode_bytes(handle, batch, max_len, 1 if with_weights else 0))


def kvec_shared_decode(handle: int, batch: int, q: int, cache: kvec_paged_cache, prefix: kvec_shared_prefix, max_len: int,
                       max_prefix: int, out: int, scratch: int, scratch_bytes: int, stream: int = 0) -> None:
    _check(load().kvec_shared_decode(handle, batch, q, cache, prefix, max_len, max_prefix, out, scratch, scratch_bytes,
                                     stream))


def kvec_shared_decode_quant_bytes(handle: int, batch: int, max_len: int, with_weights: bool) -> int:
    return int(load().kvec_shared_decode_quant_bytes(handle, batch, max_len, 1 if with_weights else 0))


def kvec_shared_decode_quant(handle: int, batch: int, q: int, cache: kvec_paged_cache, scales: kvec_paged_scales,
                             pool: kvec_paged_cache, prefix: kvec_shared_prefix, max_len: int, max_prefix: int, out: int,
                             scratch: int, scratch_bytes: int, stream: int = 0) -> None:
    _check(load().kvec_shared_decode_quant(handle, batch, q, cache, scales, pool, prefix, max_len, max_prefix, out, scratch,
                                           scratch_bytes, stream))


def kvec_rotate_append_quant(handle: int, args: kvec_rotate_args, batch: int, cu_tokens: Optional[int],
                             cache: kvec_paged_cache, scales: kvec_paged_scales, stream: int = 0) -> None:
    _check(load().kvec_rotate_append_quant(handle, args, batch, cu_tokens, cache, scales, stream))


def kvec_paged_decode_quant(handle: int, batch: int, q: int, cache: kvec_paged_cache, scales: kvec_paged_scales,
                            max_len: int, window: int, sinks: int, out: int, scratch: int, scratch_bytes: int,
                            stream: int = 0) -> None:
    _check(load().kvec_paged_decode_quant(handle, batch, q, cache, scales, max_len, window, sinks, out, scratch,
                                          scratch_bytes, stream))


def kvec_paged_evict_quant(handle: int, batch: int, cache: kvec_paged_cache, scales: kvec_paged_scales, new_table: int,
                           new_max_pages: int, max_len: int, budget: int, sinks: int, recent: int, new_lens: int,
                           kept: int, stream: int = 0) -> None:
    _check(load().kvec_paged_evict_quant(handle, batch, cache, scales, new_table, new_max_pages, max_len, budget, sinks,
                                         recent, new_lens, kept, stream))


def kvec_paged_read(handle: int, batch: int, cache: kvec_paged_cache, scales: Optional[kvec_paged_scales],
                    first: Optional[int], cu_rows: int, num_rows: int, k_out: int, v_out: int, stream: int = 0) -> None:
    _check(load().kvec_paged_read(handle, batch, cache, scales, first, cu_rows, num_rows, k_out, v_out, stream))


def kvec_prefill_attention(handle: int, dtype: int, batch: int, cu_q_host: int, cu_q_dev: int, cu_k_host: int,
                           cu_k_dev: int, q: int, k: int, v: int, window: int, sinks: int, out: int,
                           lse: Optional[int] = None, scratch: Optional[int] = None, scratch_bytes: int = 0,
                           stream: int = 0) -> None:
    _check(load().kvec_prefill_attention(handle, dtype, batch, cu_q_host, cu_q_dev, cu_k_host, cu_k_dev, q, k, v,
                                         window, sinks, out, lse, scratch, scratch_bytes, stream))


def kvec_prefill_bytes(handle: int, batch: int, cu_q_host: int, cu_k_host: int, window: int = 0, sinks: int = 0) -> int:
    return int(load().kvec_prefill_bytes(handle, batch, cu_q_host, cu_k_host, window, sinks))


def kvec_debug_scores(handle: int) -> kvec_debug_view:
    view = kvec_debug_view()
    _check(load().kvec_debug_scores(handle, ctypes.byref(view)))
    return view


def kvec_sync_status(handle: int) -> None:
    _check(load().kvec_sync_status(handle))


def kvec_set_profiling(handle: int, enable: bool) -> None:
    _check(load().kvec_set_profiling(handle, 1 if enable else 0))


def kvec_kernel_time(handle: int, kernel: int):
    ms, n = ctypes.c_double(), ctypes.c_int()
    _check(load().kvec_kernel_time(handle, int(kernel), ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def kvec_status_string(status: int) -> str:
    return load().kvec_status_string(int(status)).decode()


def make_params(num_q_heads: int, num_kv_heads: int, head_dim: int = 128, window: int = 32, obs_window: int = 16,
                ext_window: int = 32, pool_kernel: int = 7, num_ext_heads: int = 3, lam: float = 1.0,
                beta: float = 0.25, softmax_scale: float = 0.0, max_batch: int = 1, max_seqlen: int = 8192,
                max_layers: int = 32, pool_mode: int = 0, head_criterion: int = 0,
                all_positions: int = 0, head_budget: int = 0, ada_floor: float = 1.0) -> kvec_params:
    return kvec_params(num_q_heads, num_kv_heads, head_dim, window, obs_window, ext_window, pool_kernel,
                       num_ext_heads, lam, beta, softmax_scale, max_batch, max_seqlen, max_layers, pool_mode,
                       head_criterion, all_positions, head_budget, ada_floor)


def params_from_workload(wl, max_batch: Optional[int] = None, max_seqlen: Optional[int] = None,
                         max_layers: Optional[int] = None) -> kvec_params:
    return make_params(wl.num_q_heads, wl.num_kv_heads, wl.head_dim, wl.window, wl.obs_window, wl.ext_window,
                       wl.pool_kernel, wl.num_ext_heads, wl.lam, wl.beta, 0.0,
                       max_batch or wl.batch, max_seqlen or wl.max_seqlen, max_layers or max(wl.layers, 1),
                       getattr(wl, "pool_mode", 0), getattr(wl, "head_criterion", 0),
                       getattr(wl, "all_positions", 0), getattr(wl, "head_budget", 0),
                       getattr(wl, "ada_floor", 1.0))


class _DeviceArray:
    """Exposes a raw device pointer through __cuda_array_interface__ (zero copy)."""

    def __init__(self, ptr: int, shape, typestr: str):
        self.__cuda_array_interface__ = {"shape": tuple(shape), "typestr": typestr, "data": (int(ptr), False),
                                         "version": 3, "strides": None}


def _dtype_code(t, dtype) -> int:
    if dtype is t.bfloat16:
        return KVEC_BF16
    if dtype is t.float16:
        return KVEC_FP16
    raise KvecError(KVEC_ERR_INVALID_ARG, f"dtype {dtype} is neither bfloat16 nor float16")


def _want(ok: bool, message: str) -> None:
    if not ok:
        raise KvecError(KVEC_ERR_INVALID_ARG, message)


class PagedCache:
    """A paged cache (kvec_paged_cache): holds its tensors, computes nothing.

    k_pages, v_pages bf16 or fp16 [num_pages][H_kv][page_size][d]; page_table int32 [batch][max_pages];
    lens int32 [batch]; weights fp32 [num_pages][H_kv][page_size] or None.  All contiguous, on one device.  Their
    contents may change between calls; other tensors need another PagedCache.

    A cache of 8 bits has float8_e4m3fn pages, k_scales and v_scales fp32 [num_pages][H_kv][page_size] and dtype, the
    type of the queries that go with it and of rows that are read back; the same methods take it."""

    def __init__(self, k_pages, v_pages, page_table, lens, weights=None, k_scales=None, v_scales=None, dtype=None):
        import torch as t
        self.eight = k_pages.dtype is t.float8_e4m3fn
        if self.eight:
            _want(dtype is not None and k_scales is not None and v_scales is not None,
                  "a cache of 8 bits needs k_scales, v_scales and dtype")
        else:
            _want(k_scales is None and v_scales is None, "k_scales and v_scales go with float8_e4m3fn pages")
            _want(dtype is None or dtype is k_pages.dtype, "dtype is the pages' where these are of 16 bits")
            dtype = k_pages.dtype
        self.dtype_code = _dtype_code(t, dtype)
        _want(k_pages.dim() == 4 and v_pages.shape == k_pages.shape and v_pages.dtype == k_pages.dtype,
              "k_pages and v_pages must be [num_pages][H_kv][page_size][d], of one type")
        _want(page_table.dim() == 2 and page_table.dtype == t.int32 and page_table.shape[1] >= 1,
              "page_table must be int32 [batch][max_pages]")
        _want(lens.dtype == t.int32 and tuple(lens.shape) == (page_table.shape[0],), "lens must be int32 [batch]")
        for name, x in (("weights", weights), ("k_scales", k_scales), ("v_scales", v_scales)):
            _want(x is None or (x.dtype == t.float32 and x.shape == k_pages.shape[:3]),
                  f"{name} must be fp32 [num_pages][H_kv][page_size]")
        parts = [x for x in (k_pages, v_pages, page_table, lens, weights, k_scales, v_scales) if x is not None]
        _want(all(x.is_contiguous() for x in parts), "a cache's tensors must be contiguous")
        _want(all(x.device == k_pages.device for x in parts), "a cache's tensors must be on one device")
        self.k_pages, self.v_pages, self.page_table, self.lens, self.weights = k_pages, v_pages, page_table, lens, weights
        self.k_scales, self.v_scales = k_scales, v_scales
        self.batch, self.max_pages = page_table.shape
        self.page_size = k_pages.shape[2]
        self.capacity = self.max_pages * self.page_size
        self.dtype, self.device = dtype, k_pages.device
        self.kv_heads, self.head_dim = k_pages.shape[1], k_pages.shape[3]
        self.c = kvec_paged_cache(self.dtype_code, self.page_size, k_pages.shape[0], self.max_pages,
                                  k_pages.data_ptr(), v_pages.data_ptr(),
                                  None if weights is None else weights.data_ptr(), page_table.data_ptr(), lens.data_ptr())
        self.scales = kvec_paged_scales(k_scales.data_ptr(), v_scales.data_ptr()) if self.eight else None


class SharedPrefix:
    """Prefixes that groups of consecutive sequences share (kvec_shared_prefix): holds its tensors, computes nothing.

    page_table int32 [num_groups][max_pages] of pages of the cache's pool; lens int32 [num_groups]; cu_seqs int32
    [num_groups + 1]: group r's sequences are cu_seqs[r] .. cu_seqs[r + 1] - 1.  All contiguous, on the cache's device.

    pool: for a cache of 8 bits, the PagedCache of 16 bits whose pages page_table means (None: the cache's own pages)."""

    def __init__(self, page_table, lens, cu_seqs, pool=None):
        import torch as t
        _want(pool is None or not pool.eight, "a prefix's pool must be a cache of 16 bits")
        _want(page_table.dim() == 2 and page_table.dtype == t.int32 and page_table.shape[1] >= 1,
              "page_table must be int32 [num_groups][max_pages]")
        groups = page_table.shape[0]
        _want(lens.dtype == t.int32 and tuple(lens.shape) == (groups,), "lens must be int32 [num_groups]")
        _want(cu_seqs.dtype == t.int32 and tuple(cu_seqs.shape) == (groups + 1,), "cu_seqs must be int32 [num_groups + 1]")
        parts = (page_table, lens, cu_seqs)
        _want(all(x.is_contiguous() for x in parts), "a prefix's tensors must be contiguous")
        _want(all(x.device == lens.device for x in parts), "a prefix's tensors must be on one device")
        self.pool = pool
        self.page_table, self.lens, self.cu_seqs = parts
        self.max_pages, self.device = page_table.shape[1], lens.device
        self.c = kvec_shared_prefix(groups, self.max_pages, page_table.data_ptr(), lens.data_ptr(), cu_seqs.data_ptr())


class KvecSelector:
    """Owns a kvec handle; torch tensors in, torch tensors out.  Marshalling only.

    torch provides device memory and streams; every step runs in libkvec.
    """

    def __init__(self, params: kvec_params):
        import torch
        self._torch = torch
        self.params = params
        self.handle = None
        self.handle = kvec_create(params)
        self.device = torch.device("cuda", torch.cuda.current_device())
        self._current = torch._C._cuda_getCurrentRawStream   # torch.cuda.current_stream makes an object, 2 us
        self._lib = load()
        self._decode_bytes = {}      # the bytes of scratch by function and sizes
        self.state_bytes = kvec_state_bytes(params.max_seqlen)

    def close(self) -> None:
        if self.handle:
            kvec_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def new_state(self, batch: int, device="cuda"):
        t = self._torch
        st = t.empty((batch, self.state_bytes), dtype=t.uint8, device=device)
        kvec_reset(self.handle, st.data_ptr(), batch, t.cuda.current_stream(st.device).cuda_stream)
        return st

    def alloc_outputs(self, batch: int, budget: int, device="cuda"):
        """out_idx, out_k, out_v with kvec_output_capacity rows per head."""
        t = self._torch
        p = self.params
        cap = kvec_output_capacity(p, budget)
        return (t.empty((batch, p.num_kv_heads, cap), dtype=t.int32, device=device),
                t.empty((batch, p.num_kv_heads, cap, p.head_dim), dtype=t.bfloat16, device=device),
                t.empty((batch, p.num_kv_heads, cap, p.head_dim), dtype=t.bfloat16, device=device))

    def select_layer(self, cu_host, cu_dev, q_obs, k, v, state, budget: int, outs=None, stream=None, lse=None):
        """lse: optional fp32 [batch][w][H_q] window-row log-sum-exp (kvec_select_layer_lse)."""
        t = self._torch
        batch = cu_host.numel() - 1
        if outs is None:
            outs = self.alloc_outputs(batch, budget, q_obs.device)
        s = stream if stream is not None else t.cuda.current_stream(q_obs.device)
        if lse is None:
            kvec_select_layer(self.handle, batch, cu_host.data_ptr(), cu_dev.data_ptr(), q_obs.data_ptr(),
                              k.data_ptr(), v.data_ptr(), state.data_ptr(), budget, outs[0].data_ptr(),
                              outs[1].data_ptr(), outs[2].data_ptr(), s.cuda_stream)
        else:
            kvec_select_layer_lse(self.handle, batch, cu_host.data_ptr(), cu_dev.data_ptr(), q_obs.data_ptr(),
                                  k.data_ptr(), v.data_ptr(), lse.data_ptr(), state.data_ptr(), budget,
                                  outs[0].data_ptr(), outs[1].data_ptr(), outs[2].data_ptr(), s.cuda_stream)
        return outs

    def select_layers(self, cu_host, cu_dev, qs, ks, vs, state, budget: int, outs, stream=None, lses=None):
        """lses: optional per-layer fp32 [batch][w][H_q] window-row log-sum-exp (kvec_select_layers_lse)."""
        t = self._torch
        batch = cu_host.numel() - 1
        s = stream if stream is not None else t.cuda.current_stream(qs[0].device)
        common = ([x.data_ptr() for x in qs], [x.data_ptr() for x in ks], [x.data_ptr() for x in vs])
        tail = ([o[0].data_ptr() for o in outs], [o[1].data_ptr() for o in outs], [o[2].data_ptr() for o in outs],
                s.cuda_stream)
        if lses is None:
            kvec_select_layers(self.handle, batch, cu_host.data_ptr(), cu_dev.data_ptr(), *common, state.data_ptr(),
                               budget, *tail)
        else:
            kvec_select_layers_lse(self.handle, batch, cu_host.data_ptr(), cu_dev.data_ptr(), *common,
                                   [x.data_ptr() for x in lses], state.data_ptr(), budget, *tail)
        return outs

    def decode_attention(self, q, k_cache, v_cache, lens, out=None, stream=None):
        """One decoding step over a compacted cache (kvec_decode_attention).

        q bf16 [batch][H_q][d]; k_cache, v_cache bf16 [batch][H_kv][cap][d];
        lens int32 [batch] on the device.  Returns fp32 [batch][H_q][d]."""
        t = self._torch
        batch, cap = q.shape[0], k_cache.shape[2]
        if out is None:
            out = t.empty((batch, q.shape[1], q.shape[2]), dtype=t.float32, device=q.device)
        s = stream if stream is not None else t.cuda.current_stream(q.device)
        kvec_decode_attention(self.handle, batch, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                              lens.data_ptr(), cap, out.data_ptr(), s.cuda_stream)
        return out

    # ------------------------------------------------------------ decoding over pages
    # A small call is bound by its host time: messages are formed only where a check fails.
    # stream: the call's (None: the current one); what it reads must be ready there, and what is made
    # for it comes from that stream's memory.  What is given to a call on another stream than the current one may be
    # let go at once: its memory is not used again before that stream's work so far is done.  (A stream that torch did
    # not make has to live until they are let go.)

    def _empty(self, shape, dtype, stream):
        """Memory that work on `stream` (None: the current one) may use at once, from that stream's pool."""
        t = self._torch
        if stream is None or stream.cuda_stream == self._current(self.device.index):
            return t.empty(shape, dtype=dtype, device=self.device)
        with t.cuda.stream(stream):
            return t.empty(shape, dtype=dtype, device=self.device)

    def _raw(self, stream):
        return self._current(self.device.index) if stream is None else stream.cuda_stream

    def _used(self, stream, cache, *tensors):
        """After a call on `stream`: tells the allocator of its tensors, which came from other streams' memory."""
        if stream.cuda_stream == self._current(self.device.index):
            return
        if cache is not None:
            tensors += (cache.k_pages, cache.v_pages, cache.page_table, cache.lens, cache.weights, cache.k_scales,
                        cache.v_scales)
        for x in tensors:
            if x is not None:
                x.record_stream(stream)

    def _check(self, name, x, shape, dtype):
        """A contiguous tensor of the handle's device."""
        if x.shape != shape or x.dtype is not dtype or x.device != self.device or not x.is_contiguous():
            raise KvecError(KVEC_ERR_INVALID_ARG, f"{name} must be contiguous {dtype} {list(shape)} on {self.device}, "
                                                  f"not {x.dtype} {list(x.shape)} on {x.device}")

    def _rows(self, name, x, T, heads, dtype):
        """Token rows [T][heads][d], heads side by side; the elements from a token to the next."""
        d = self.params.head_dim
        if x.shape != (T, heads, d) or x.dtype is not dtype or x.device != self.device:
            raise KvecError(KVEC_ERR_INVALID_ARG, f"{name} must be {dtype} {[T, heads, d]} on {self.device}, "
                                                  f"not {x.dtype} {list(x.shape)} on {x.device}")
        st = x.stride()
        if T and (st[2] != 1 or (st[1] != d and heads > 1)):
            raise KvecError(KVEC_ERR_INVALID_ARG, f"{name}'s heads must lie side by side")
        return st[0] if T > 1 else heads * d

    def _check_cache(self, cache):
        p = self.params
        if cache.kv_heads != p.num_kv_heads or cache.head_dim != p.head_dim or cache.device != self.device:
            raise KvecError(KVEC_ERR_INVALID_ARG, f"the cache's pages must have {p.num_kv_heads} KV heads of "
                                                  f"{p.head_dim}, on {self.device}")

    def rotate_append(self, q, k, v, positions, rot_table=None, cache=None, cu_tokens=None, q_norm=None, k_norm=None,
                      eps: float = 1e-6, interleaved: bool = False, q_out=None, k_out=None, stream=None):
        """Norms of new tokens' queries and keys, rotation, and the store into the cache (kvec_rotate_append, or
        kvec_rotate_append_quant for one of 8 bits).

        q [T][H_q][d], k, v [T][H_kv][d], tokens any multiple of 8 elements apart; positions int32 [T];
        rot_table fp32 [max_positions][rot_dim]; cu_tokens int32 [batch + 1] on the device (None: a token a sequence).
        Without a cache k_out is made and (q_out, k_out) returned; with one q_out, or both where k_out is given."""
        t, p = self._torch, self.params
        T, dtype, Hq, Hkv, d = q.shape[0], q.dtype, p.num_q_heads, p.num_kv_heads, p.head_dim
        code = _dtype_code(t, dtype)
        q_stride = self._rows("q", q, T, Hq, dtype)
        k_stride = self._rows("k", k, T, Hkv, dtype)
        v_stride = 0 if v is None else self._rows("v", v, T, Hkv, dtype)
        self._check("positions", positions, (T,), t.int32)
        rot = most = 0
        if rot_table is not None:
            _want(rot_table.dim() == 2, "rot_table must be [max_positions][rot_dim]")
            most, rot = rot_table.shape
            self._check("rot_table", rot_table, (most, rot), t.float32)
        if q_norm is not None:
            self._check("q_norm", q_norm, (d,), dtype)
        if k_norm is not None:
            self._check("k_norm", k_norm, (d,), dtype)
        batch = T
        if cu_tokens is not None:
            batch = cu_tokens.shape[0] - 1
            self._check("cu_tokens", cu_tokens, (batch + 1,), t.int32)
        if cache is not None:
            self._check_cache(cache)
            if cache.batch != batch:
                raise KvecError(KVEC_ERR_INVALID_ARG, f"the cache has {cache.batch} sequences, the call {batch}")
        want_k = cache is None or k_out is not None
        if q_out is None:
            q_out = self._empty((T, Hq, d), dtype, stream)
        else:
            self._check("q_out", q_out, (T, Hq, d), dtype)
        if k_out is not None:
            self._check("k_out", k_out, (T, Hkv, d), dtype)
        elif cache is None:
            k_out = self._empty((T, Hkv, d), dtype, stream)
        if T:
            a = kvec_rotate_args(code, T, q.data_ptr(), k.data_ptr(), None if v is None else v.data_ptr(), q_stride,
                                 k_stride, v_stride, None if q_norm is None else q_norm.data_ptr(),
                                 None if k_norm is None else k_norm.data_ptr(), eps, rot, 1 if interleaved else 0, most,
                                 None if rot_table is None else rot_table.data_ptr(), positions.data_ptr(),
                                 q_out.data_ptr(), None if k_out is None else k_out.data_ptr())
            cu = None if cu_tokens is None else cu_tokens.data_ptr()
            if cache is not None and cache.eight:
                st = self._lib.kvec_rotate_append_quant(self.handle, a, batch, cu, cache.c, cache.scales, self._raw(stream))
            else:
                st = self._lib.kvec_rotate_append(self.handle, a, batch, cu, None if cache is None else cache.c,
                                                  self._raw(stream))
            if st:
                _check(st)
            if stream is not None:
                self._used(stream, cache, q, k, v, positions, rot_table, cu_tokens, q_norm, k_norm, q_out, k_out)
        return (q_out, k_out) if want_k else q_out

    def _scratch_bytes(self, of, *sizes):
        need = self._decode_bytes.get((of, sizes))
        if need is None:
            if len(self._decode_bytes) >= 256:   # a loop's bounds may grow with every step
                self._decode_bytes.clear()
            need = self._decode_bytes[of, sizes] = of(self.handle, *sizes)
        return need

    def paged_decode(self, q, cache, max_len: Optional[int] = None, window: int = 0, sinks: int = 0, out=None,
                     stream=None):
        """One new token per sequence over a paged cache (kvec_paged_decode, or kvec_paged_decode_quant over one of 8 bits);
        adds to cache.weights where it has them.

        q [batch][H_q][d] of the cache's type, contiguous; max_len: a bound on the lengths (the capacity).  Scratch
        (kvec_paged_decode_window_bytes) and, with weights, part of the time go by max_len or the window: give the least
        bound that is known."""
        p = self.params
        batch, dtype = cache.batch, cache.dtype
        shape = (batch, p.num_q_heads, p.head_dim)
        self._check_cache(cache)
        self._check("q", q, shape, dtype)
        if out is None:
            out = self._empty(shape, dtype, stream)
        else:
            self._check("out", out, shape, dtype)
        if max_len is None:
            max_len = cache.capacity
        if (max_len | window | sinks) >> 31:   # ctypes would pass their lower 32 bits
            raise KvecError(KVEC_ERR_INVALID_ARG, "max_len, window and sinks must be in [0, 2^31)")
        need = self._scratch_bytes(kvec_paged_decode_quant_bytes if cache.eight else kvec_paged_decode_window_bytes, batch,
                                   max_len, window, sinks, cache.weights is not None)
        scratch = self._empty(max(need, 16), self._torch.uint8, stream)
        if cache.eight:
            st = self._lib.kvec_paged_decode_quant(self.handle, batch, q.data_ptr(), cache.c, cache.scales, max_len, window,
                                                   sinks, out.data_ptr(), scratch.data_ptr(), need, self._raw(stream))
        else:
            st = self._lib.kvec_paged_decode(self.handle, batch, q.data_ptr(), cache.c, max_len, window, sinks,
                                             out.data_ptr(), scratch.data_ptr(), need, self._raw(stream))
        if st:
            _check(st)
        if stream is not None:
            self._used(stream, cache, q, out)
        return out

    def shared_decode(self, q, cache, prefix, max_len: Optional[int] = None, max_prefix: Optional[int] = None, out=None,
                      stream=None):
        """One new token per sequence where groups of sequences share a prefix (kvec_shared_decode, or kvec_shared_decode_quant
        where cache is one of 8 bits); adds to cache.weights, where it has them, for the sequences' own slots.

        q [batch][H_q][d] of the cache's dtype, contiguous; cache: the sequences' own slots, prefix a SharedPrefix of
        pages of the same pool, or with a cache of 8 bits of its own pool's.  max_len bounds the own lengths, max_prefix
        those of the prefixes (the capacities): give the least bounds that are known."""
        p = self.params
        batch, dtype = cache.batch, cache.dtype
        shape = (batch, p.num_q_heads, p.head_dim)
        self._check_cache(cache)
        pool = prefix.pool
        if cache.eight:
            if pool is None:
                raise KvecError(KVEC_ERR_UNSUPPORTED, "behind a cache of 8 bits a prefix needs a pool of 16 bits")
            self._check_cache(pool)
        else:
            _want(pool is None or (pool.k_pages is cache.k_pages and pool.v_pages is cache.v_pages),
                  "a prefix before a cache of 16 bits lies in the same pages")
            pool = cache
        _want(prefix.device == self.device, "the prefix must be on the handle's device")
        self._check("q", q, shape, dtype)
        if out is None:
            out = self._empty(shape, dtype, stream)
        else:
            self._check("out", out, shape, dtype)
        if max_len is None:
            max_len = cache.capacity
        if max_prefix is None:
            max_prefix = prefix.max_pages * pool.page_size
        if (max_len | max_prefix) >> 31:
            raise KvecError(KVEC_ERR_INVALID_ARG, "max_len and max_prefix must be in [0, 2^31)")
        need = self._scratch_bytes(kvec_shared_decode_quant_bytes if cache.eight else kvec_shared_decode_bytes, batch, max_len,
                                   cache.weights is not None)
        scratch = self._empty(max(need, 16), self._torch.uint8, stream)
        tail = (prefix.c, max_len, max_prefix, out.data_ptr(), scratch.data_ptr(), need, self._raw(stream))
        if cache.eight:
            st = self._lib.kvec_shared_decode_quant(self.handle, batch, q.data_ptr(), cache.c, cache.scales, pool.c, *tail)
        else:
            st = self._lib.kvec_shared_decode(self.handle, batch, q.data_ptr(), cache.c, *tail)
        if st:
            _check(st)
        if stream is not None:
            self._used(stream, cache, q, out, prefix.page_table, prefix.lens, prefix.cu_seqs)
            self._used(stream, pool)
        return out

    def paged_evict(self, cache, new_table, budget: int, sinks: int = 0, recent: int = 0, max_len: Optional[int] = None,
                    new_lens=None, kept=None, stream=None):
        """Eviction by accumulated weight to the pages of new_table (kvec_paged_evict, or kvec_paged_evict_quant).

        cache.weights hold what paged_decode added since rotate_append set a slot's to 0; a prompt's slots count with
        its own attention only where the caller has written it there.
        new_table int32 [batch][pages], contiguous, of pages that page_table does not use.  Returns (new_lens int32
        [batch], kept int32 [batch][H_kv][budget])."""
        t, p = self._torch, self.params
        batch, Hkv = cache.batch, p.num_kv_heads
        self._check_cache(cache)
        _want(new_table.dim() == 2, "new_table must be int32 [batch][pages]")
        self._check("new_table", new_table, (batch, new_table.shape[1]), t.int32)
        _want(1 <= budget <= 1 << 20, "budget must be in [1, 2^20]")
        if max_len is None:
            max_len = cache.capacity
        if (max_len | sinks | recent) >> 31:
            raise KvecError(KVEC_ERR_INVALID_ARG, "max_len, sinks and recent must be in [0, 2^31)")
        if new_lens is None:
            new_lens = self._empty((batch,), t.int32, stream)
        else:
            self._check("new_lens", new_lens, (batch,), t.int32)
        if kept is None:
            kept = self._empty((batch, Hkv, budget), t.int32, stream)
        else:
            self._check("kept", kept, (batch, Hkv, budget), t.int32)
        tail = (new_table.data_ptr(), new_table.shape[1], max_len, budget, sinks, recent, new_lens.data_ptr(),
                kept.data_ptr(), self._raw(stream))
        if cache.eight:
            st = self._lib.kvec_paged_evict_quant(self.handle, batch, cache.c, cache.scales, *tail)
        else:
            st = self._lib.kvec_paged_evict(self.handle, batch, cache.c, *tail)
        if st:
            _check(st)
        if stream is not None:
            self._used(stream, cache, new_table, new_lens, kept)
        return new_lens, kept

    def paged_read(self, cache, cu_rows, num_rows: int, first=None, k_out=None, v_out=None, stream=None):
        """A paged cache's slots as packed rows of its dtype, as prefill_attention takes keys and values (kvec_paged_read).

        cu_rows int32 [batch + 1] on the device, num_rows its last entry, which the host knows; first int32 [batch] (None:
        0): the slots that the sequences' rows begin with.  Returns (k, v) [num_rows][H_kv][d]."""
        t, p = self._torch, self.params
        batch, shape = cache.batch, (num_rows, p.num_kv_heads, p.head_dim)
        self._check_cache(cache)
        _want(0 <= num_rows < 1 << 31, "num_rows must be in [0, 2^31)")
        self._check("cu_rows", cu_rows, (batch + 1,), t.int32)
        if first is not None:
            self._check("first", first, (batch,), t.int32)
        if k_out is None:
            k_out = self._empty(shape, cache.dtype, stream)
        else:
            self._check("k_out", k_out, shape, cache.dtype)
        if v_out is None:
            v_out = self._empty(shape, cache.dtype, stream)
        else:
            self._check("v_out", v_out, shape, cache.dtype)
        st = self._lib.kvec_paged_read(self.handle, batch, cache.c, cache.scales, None if first is None else first.data_ptr(),
                                       cu_rows.data_ptr(), num_rows, k_out.data_ptr(), v_out.data_ptr(), self._raw(stream))
        if st:
            _check(st)
        if stream is not None:
            self._used(stream, cache, cu_rows, first, k_out, v_out)
        return k_out, v_out

    def prefill_attention(self, q, k, v, cu_q_host, cu_q_dev, cu_k_host=None, cu_k_dev=None, window: int = 0,
                          sinks: int = 0, out=None, lse=None, stream=None):
        """Causal attention of packed sequences (kvec_prefill_attention).

        q [T_q][H_q][d], k, v [T_k][H_kv][d] bf16 or fp16, contiguous; cu_* int32 [batch + 1], host and device copies
        (cu_k: cu_q).  Returns (out as q, lse fp32 [T_q][H_q])."""
        t, p = self._torch, self.params
        dtype, Tq, Hq, Hkv, d = q.dtype, q.shape[0], p.num_q_heads, p.num_kv_heads, p.head_dim
        code = _dtype_code(t, dtype)
        if cu_k_host is None:
            cu_k_host, cu_k_dev = cu_q_host, cu_q_dev
        Tk, batch = k.shape[0], cu_q_host.shape[0] - 1
        self._check("q", q, (Tq, Hq, d), dtype)
        self._check("k", k, (Tk, Hkv, d), dtype)
        self._check("v", v, (Tk, Hkv, d), dtype)
        self._check("cu_q_dev", cu_q_dev, (batch + 1,), t.int32)
        self._check("cu_k_dev", cu_k_dev, (batch + 1,), t.int32)
        for x in (cu_q_host, cu_k_host):
            _want(x.dtype is t.int32 and x.shape == (batch + 1,) and x.device.type == "cpu" and x.is_contiguous(),
                  "cu_q_host and cu_k_host must be contiguous int32 [batch + 1] on the host")
        if (window | sinks) >> 31:
            raise KvecError(KVEC_ERR_INVALID_ARG, "window and sinks must be in [0, 2^31)")
        cu_q, cu_k = cu_q_host.data_ptr(), cu_k_host.data_ptr()
        last = ctypes.c_int32.from_address   # the host copies' last entries (a tensor's item takes 2 us)
        _want(batch >= 1 and last(cu_q + 4 * batch).value <= Tq and last(cu_k + 4 * batch).value <= Tk,
              "cu_q_host or cu_k_host passes the rows given")
        if out is None:
            out = self._empty((Tq, Hq, d), dtype, stream)
        else:
            self._check("out", out, (Tq, Hq, d), dtype)
        if lse is None:
            lse = self._empty((Tq, Hq), t.float32, stream)
        else:
            self._check("lse", lse, (Tq, Hq), t.float32)
        need = self._lib.kvec_prefill_bytes(self.handle, batch, cu_q, cu_k, window, sinks)
        scratch = self._empty(need, t.uint8, stream) if need else None
        st = self._lib.kvec_prefill_attention(self.handle, code, batch, cu_q, cu_q_dev.data_ptr(), cu_k, cu_k_dev.data_ptr(),
                                              q.data_ptr(), k.data_ptr(), v.data_ptr(), window, sinks, out.data_ptr(),
                                              lse.data_ptr(), scratch.data_ptr() if need else None, need, self._raw(stream))
        if st:
            _check(st)
        if stream is not None:
            self._used(stream, None, q, k, v, cu_q_dev, cu_k_dev, out, lse)
        return out, lse

    def debug(self, device="cuda"):
        """Copies of the last layer's intermediates (see kvec_debug_view)."""
        t = self._torch
        p = self.params
        v = kvec_debug_scores(self.handle)
        MB, H, ML, W = p.max_batch, p.num_kv_heads, v.max_seqlen, v.words_per_row
        R = (p.num_q_heads // p.num_kv_heads) * p.window

        def grab(ptr, shape, typestr):
            return t.as_tensor(_DeviceArray(ptr, shape, typestr), device=device).clone()

        return {
            "P_O": grab(v.P_O, (MB, H, ML), "<f4"), "P_Oext": grab(v.P_Oext, (MB, H, ML), "<f4"),
            "I": grab(v.I, (MB, ML), "<f4"), "sigma": grab(v.sigma, (MB, H), "<f4"),
            "htop": grab(v.htop, (MB, H), "<i4"), "pres_bits": grab(v.pres_bits, (MB, H, W), "<u4"),
            "Pprime": grab(v.Pprime, (MB, H, ML), "<f4"), "row_stats": grab(v.row_stats, (MB, H, R, 2), "<f4"),
        }
