"""ctypes binding of include/kvfold.h: same names, argument marshalling only.

The library must have been built (``python -m paper_2605_12471_amd.build`` or
``__graft_entry__.build()``); loading fails loudly otherwise -- there is no
fallback path.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import threading
from typing import Optional

KVFOLD_F32 = 0
KVFOLD_BF16 = 1
TUNE_SPLITS = 0
TUNE_UNITS_PER_WAVE = 1
TUNE_PAIR_UNITS = 2
TUNE_FUSED_APPEND = 3

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.environ.get("KVFOLD_LIB_PATH") or os.path.join(_HERE, "_lib", "libkvfold.so")
_lib = None


class kvfold_config_t(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("n_layers", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("chunk_tokens", ctypes.c_int32),
        ("capacity_tokens", ctypes.c_int64),
        ("dtype", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float),
        ("device", ctypes.c_int32),
        ("kv_buffer", ctypes.c_void_p),
        ("kv_buffer_bytes", ctypes.c_size_t),
    ]


class kvfold_pcache_config_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in (
        "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "page_tokens", "n_pages", "dtype")] + [
        ("softmax_scale", ctypes.c_float), ("device", ctypes.c_int32), ("kv_buffer", ctypes.c_void_p), ("kv_buffer_bytes", ctypes.c_size_t)]


class kvfold_batch_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("n_seqs", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("max_len", ctypes.c_int64), ("tables", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("lens", ctypes.c_void_p),
                ("cu_new", ctypes.c_void_p), ("slots", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("kv_stride", ctypes.c_int64)]


class kvfold_plan_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_workgroups", "n_splits", "units_per_wave", "tiles_per_split",
                                              "fused_append", "pair_units", "pair_order")]


class KvFoldError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {kvfold_status_string(status)} (status {status}, hip error {kvfold_last_hip_error()})")


def lib_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load libkvfold.so and declare the prototypes of every exported entry point."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2605_12471_amd.build` "
            "(there is no non-HIP fallback)")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    cfgp = ctypes.POINTER(kvfold_config_t)
    lib.kvfold_cache_bytes_required.argtypes = [cfgp]
    lib.kvfold_cache_bytes_required.restype = ctypes.c_size_t
    lib.kvfold_cache_create.argtypes = [cfgp, ctypes.POINTER(vp)]
    lib.kvfold_cache_create.restype = ctypes.c_int
    lib.kvfold_step.argtypes = [vp, ctypes.c_int, vp, vp, vp, i64, vp, vp]
    lib.kvfold_step.restype = ctypes.c_int
    lib.kvfold_step_ex.argtypes = [vp, ctypes.c_int, vp, vp, vp, i32, i64, vp, vp, vp]
    lib.kvfold_step_ex.restype = ctypes.c_int
    lib.kvfold_step_rope.argtypes = [vp, ctypes.c_int, vp, vp, vp, i32, i64, vp, vp, vp, vp, vp]
    lib.kvfold_step_rope.restype = ctypes.c_int
    lib.kvfold_step_window.argtypes = [vp, ctypes.c_int, vp, vp, vp, i32, i64, i32, i64, vp, vp, vp]
    lib.kvfold_step_window.restype = ctypes.c_int
    lib.kvfold_step_noalloc.argtypes = [vp, ctypes.c_int, vp, vp, vp, i32, i64, vp, vp, vp]
    lib.kvfold_step_noalloc.restype = ctypes.c_int
    lib.kvfold_cache_destroy.argtypes = [vp]
    lib.kvfold_cache_destroy.restype = ctypes.c_int
    lib.kvfold_cache_length.argtypes = [vp, ctypes.c_int]
    lib.kvfold_cache_length.restype = i64
    lib.kvfold_cache_view.argtypes = [vp, ctypes.c_int, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                      ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.kvfold_cache_view.restype = ctypes.c_int
    lib.kvfold_cache_truncate.argtypes = [vp, ctypes.c_int, i64]
    lib.kvfold_cache_truncate.restype = ctypes.c_int
    lib.kvfold_cache_set_length.argtypes = [vp, ctypes.c_int, i64]
    lib.kvfold_cache_set_length.restype = ctypes.c_int
    lib.kvfold_cache_set_storage_roundtrip.argtypes = [vp, i32]
    lib.kvfold_cache_set_storage_roundtrip.restype = ctypes.c_int
    lib.kvfold_cache_set_tuning.argtypes = [vp, i32, i32]
    lib.kvfold_cache_set_tuning.restype = ctypes.c_int
    lib.kvfold_cache_plan.argtypes = [vp, i32, i64, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    lib.kvfold_cache_plan.restype = ctypes.c_int
    lib.kvfold_plan_for.argtypes = [ctypes.POINTER(kvfold_config_t), i32, i32, i64, i32, i64, ctypes.POINTER(kvfold_plan_t)]
    lib.kvfold_plan_for.restype = ctypes.c_int
    lib.kvfold_cache_profile_begin.argtypes = [vp, i32]
    lib.kvfold_cache_profile_begin.restype = ctypes.c_int
    dp = ctypes.POINTER(ctypes.c_double)
    lib.kvfold_cache_profile_end.argtypes = [vp, ctypes.POINTER(i32), dp, dp, dp]
    lib.kvfold_cache_profile_end.restype = ctypes.c_int
    lib.kvfold_status_string.argtypes = [ctypes.c_int]
    lib.kvfold_status_string.restype = ctypes.c_char_p
    lib.kvfold_measure_peaks.argtypes = [i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    lib.kvfold_measure_peaks.restype = ctypes.c_int
    lib.kvfold_qcache_bytes_required.argtypes = [cfgp]
    lib.kvfold_qcache_bytes_required.restype = ctypes.c_size_t
    lib.kvfold_qcache_create.argtypes = [cfgp, ctypes.POINTER(vp)]
    lib.kvfold_qcache_create.restype = ctypes.c_int
    lib.kvfold_qcache_destroy.argtypes = [vp]
    lib.kvfold_qcache_destroy.restype = ctypes.c_int
    lib.kvfold_qcache_step.argtypes = [vp, ctypes.c_int, vp, vp, vp, i32, i64, vp, vp, vp, vp, vp]
    lib.kvfold_qcache_step.restype = ctypes.c_int
    lib.kvfold_qcache_append.argtypes = [vp, ctypes.c_int, vp, vp, i64, i64, i64, i64, vp, vp, vp]
    lib.kvfold_qcache_append.restype = ctypes.c_int
    lib.kvfold_qcache_read.argtypes = [vp, ctypes.c_int, i64, i64, vp, vp, vp]
    lib.kvfold_qcache_read.restype = ctypes.c_int
    lib.kvfold_qcache_length.argtypes = [vp, ctypes.c_int]
    lib.kvfold_qcache_length.restype = i64
    lib.kvfold_qcache_truncate.argtypes = [vp, ctypes.c_int, i64]
    lib.kvfold_qcache_truncate.restype = ctypes.c_int
    lib.kvfold_cache_weigh.argtypes = [vp, ctypes.c_int, vp, i32, vp, vp, vp, vp, i32, vp]
    lib.kvfold_cache_weigh.restype = ctypes.c_int
    lib.kvfold_evict_workspace_bytes.argtypes = [vp, i64]
    lib.kvfold_evict_workspace_bytes.restype = ctypes.c_size_t
    lib.kvfold_cache_evict.argtypes = [vp, ctypes.c_int, vp, i64, i64, i64, vp, ctypes.c_int, vp, vp, vp, ctypes.c_size_t, vp]
    lib.kvfold_cache_evict.restype = ctypes.c_int
    pcfgp, batchp = ctypes.POINTER(kvfold_pcache_config_t), ctypes.POINTER(kvfold_batch_t)
    lib.kvfold_pcache_bytes_required.argtypes = [pcfgp]
    lib.kvfold_pcache_bytes_required.restype = ctypes.c_size_t
    lib.kvfold_pcache_create.argtypes = [pcfgp, ctypes.POINTER(vp)]
    lib.kvfold_pcache_create.restype = ctypes.c_int
    lib.kvfold_pcache_destroy.argtypes = [vp]
    lib.kvfold_pcache_destroy.restype = ctypes.c_int
    lib.kvfold_pcache_view.argtypes = [vp, ctypes.c_int, ctypes.POINTER(vp), ctypes.POINTER(vp)]
    lib.kvfold_pcache_view.restype = ctypes.c_int
    lib.kvfold_pcache_assign.argtypes = [vp, i32, vp, vp, vp, vp, vp, i64, vp, vp, vp, vp, i64, vp, vp, vp]
    lib.kvfold_pcache_assign.restype = ctypes.c_int
    lib.kvfold_pcache_workspace_bytes.argtypes = [vp, batchp]
    lib.kvfold_pcache_workspace_bytes.restype = ctypes.c_size_t
    lib.kvfold_pcache_step.argtypes = [vp, ctypes.c_int, batchp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.kvfold_pcache_step.restype = ctypes.c_int
    lib.kvfold_pcache_append.argtypes = [vp, ctypes.c_int, vp, vp, i64, vp, i32, vp]
    lib.kvfold_pcache_append.restype = ctypes.c_int
    lib.kvfold_last_hip_error.argtypes = []
    lib.kvfold_last_hip_error.restype = ctypes.c_int
    _lib = lib
    return lib


# ---------------------------------------------------------------------------------------------
# Functions with the header's names.  Pointers are plain integers (e.g. torch's data_ptr()).
# Each returns the library's status code (or value) untouched.
# ---------------------------------------------------------------------------------------------
def make_config(n_layers, n_q_heads, n_kv_heads, head_dim, chunk_tokens, capacity_tokens, dtype,
                softmax_scale=0.0, device=0, kv_buffer=None, kv_buffer_bytes=0) -> kvfold_config_t:
    return kvfold_config_t(ctypes.sizeof(kvfold_config_t), n_layers, n_q_heads, n_kv_heads, head_dim, chunk_tokens,
                           capacity_tokens, dtype, softmax_scale, device, kv_buffer, kv_buffer_bytes)


def kvfold_cache_bytes_required(cfg: kvfold_config_t) -> int:
    return int(load_library().kvfold_cache_bytes_required(ctypes.byref(cfg)))


def kvfold_cache_create(cfg: Optional[kvfold_config_t]):
    """Returns (status, handle); handle is None on error."""
    h = ctypes.c_void_p()
    rc = load_library().kvfold_cache_create(ctypes.byref(cfg) if cfg is not None else None, ctypes.byref(h))
    return rc, (h if rc == 0 else None)


def kvfold_step(cache, layer, q, k_new, v_new, pos_offset, out, stream=0) -> int:
    return load_library().kvfold_step(cache, layer, q, k_new, v_new, pos_offset, out, stream)


def kvfold_step_ex(cache, layer, q, k_new, v_new, n_tokens, pos_offset, out, lse=None, stream=0) -> int:
    return load_library().kvfold_step_ex(cache, layer, q, k_new, v_new, n_tokens, pos_offset, out, lse, stream)


def kvfold_step_rope(cache, layer, q, k_new, v_new, n_tokens, pos_offset, rope_cos, rope_sin, out, lse=None,
                     stream=0) -> int:
    return load_library().kvfold_step_rope(cache, layer, q, k_new, v_new, n_tokens, pos_offset, rope_cos, rope_sin,
                                           out, lse, stream)


def kvfold_step_window(cache, layer, q, k_new, v_new, n_tokens, pos_offset, n_sink, window, out, lse=None, stream=0) -> int:
    return load_library().kvfold_step_window(cache, layer, q, k_new, v_new, n_tokens, pos_offset, n_sink, window,
                                             out, lse, stream)


def kvfold_step_noalloc(cache, layer, q, k_new, v_new, n_tokens, pos_offset, out, lse=None, stream=0) -> int:
    return load_library().kvfold_step_noalloc(cache, layer, q, k_new, v_new, n_tokens, pos_offset, out, lse, stream)


def kvfold_cache_destroy(cache) -> int:
    return load_library().kvfold_cache_destroy(cache)


def kvfold_cache_length(cache, layer) -> int:
    return int(load_library().kvfold_cache_length(cache, layer))


def kvfold_cache_view(cache, layer):
    """Returns (status, k_ptr, v_ptr, row_stride_elems, head_stride_elems)."""
    k, v = ctypes.c_void_p(), ctypes.c_void_p()
    rs, hs = ctypes.c_int64(), ctypes.c_int64()
    rc = load_library().kvfold_cache_view(cache, layer, ctypes.byref(k), ctypes.byref(v), ctypes.byref(rs),
                                          ctypes.byref(hs))
    return rc, k.value, v.value, rs.value, hs.value


def kvfold_cache_truncate(cache, layer, new_len) -> int:
    return load_library().kvfold_cache_truncate(cache, layer, new_len)


def kvfold_cache_set_length(cache, layer, new_len) -> int:
    return load_library().kvfold_cache_set_length(cache, layer, new_len)


def kvfold_cache_set_storage_roundtrip(cache, n_bits) -> int:
    return load_library().kvfold_cache_set_storage_roundtrip(cache, n_bits)


def kvfold_cache_set_tuning(cache, knob, value) -> int:
    return load_library().kvfold_cache_set_tuning(cache, knob, value)


def kvfold_cache_plan(cache, n_tokens, len_after):
    """Returns (status, n_workgroups, n_splits)."""
    w, s = ctypes.c_int32(), ctypes.c_int32()
    rc = load_library().kvfold_cache_plan(cache, n_tokens, len_after, ctypes.byref(w), ctypes.byref(s))
    return rc, w.value, s.value


def kvfold_plan_for(cfg, n_compute_units, n_tokens, len_after, n_sink=0, window=0):
    """Host-only.  Returns (status, kvfold_plan_t)."""
    pl = kvfold_plan_t()
    rc = load_library().kvfold_plan_for(ctypes.byref(cfg) if cfg is not None else None, n_compute_units, n_tokens, len_after,
                                        n_sink, window, ctypes.byref(pl))
    return rc, pl


def kvfold_cache_profile_begin(cache, max_steps) -> int:
    return load_library().kvfold_cache_profile_begin(cache, max_steps)


def kvfold_cache_profile_end(cache):
    """Returns (status, n_steps, append_ms, attention_ms, merge_ms)."""
    n = ctypes.c_int32()
    a, t, m = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
    rc = load_library().kvfold_cache_profile_end(cache, ctypes.byref(n), ctypes.byref(a), ctypes.byref(t),
                                                 ctypes.byref(m))
    return rc, n.value, a.value, t.value, m.value


def kvfold_cache_weigh(cache, layer, q, n_tokens, rope_cos, rope_sin, lse, weights, add=0, stream=0) -> int:
    return load_library().kvfold_cache_weigh(cache, layer, q, n_tokens, rope_cos, rope_sin, lse, weights, add, stream)


def kvfold_evict_workspace_bytes(cache, n_keep) -> int:
    return int(load_library().kvfold_evict_workspace_bytes(cache, n_keep))


def kvfold_cache_evict(cache, layer, weights, n_keep, n_sink, n_recent, to, to_layer, to_weights, kept, workspace, workspace_bytes, stream=0) -> int:
    return load_library().kvfold_cache_evict(cache, layer, weights, n_keep, n_sink, n_recent, to, to_layer, to_weights, kept, workspace, workspace_bytes, stream)


def kvfold_qcache_bytes_required(cfg: kvfold_config_t) -> int:
    return int(load_library().kvfold_qcache_bytes_required(ctypes.byref(cfg)))


def kvfold_qcache_create(cfg: Optional[kvfold_config_t]):
    """Returns (status, handle); handle is None on error."""
    h = ctypes.c_void_p()
    rc = load_library().kvfold_qcache_create(ctypes.byref(cfg) if cfg is not None else None, ctypes.byref(h))
    return rc, (h if rc == 0 else None)


def kvfold_qcache_destroy(cache) -> int:
    return load_library().kvfold_qcache_destroy(cache)


def kvfold_qcache_step(cache, layer, q, k_new, v_new, n_tokens, pos_offset, rope_cos, rope_sin, out, lse=None, stream=0) -> int:
    return load_library().kvfold_qcache_step(cache, layer, q, k_new, v_new, n_tokens, pos_offset, rope_cos, rope_sin, out, lse, stream)


def kvfold_qcache_append(cache, layer, k, v, token_stride, head_stride, n_tokens, pos_offset, rope_cos=None, rope_sin=None, stream=0) -> int:
    return load_library().kvfold_qcache_append(cache, layer, k, v, token_stride, head_stride, n_tokens, pos_offset, rope_cos, rope_sin, stream)


def kvfold_qcache_read(cache, layer, first, n_tokens, k_out, v_out, stream=0) -> int:
    return load_library().kvfold_qcache_read(cache, layer, first, n_tokens, k_out, v_out, stream)


def kvfold_qcache_length(cache, layer) -> int:
    return int(load_library().kvfold_qcache_length(cache, layer))


def kvfold_qcache_truncate(cache, layer, new_len) -> int:
    return load_library().kvfold_qcache_truncate(cache, layer, new_len)


def make_pconfig(n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages, dtype, softmax_scale=0.0, device=0, kv_buffer=None, kv_buffer_bytes=0):
    return kvfold_pcache_config_t(ctypes.sizeof(kvfold_pcache_config_t), n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages, dtype, softmax_scale,
                                  device, kv_buffer, kv_buffer_bytes)


def make_batch(n_seqs, n_tokens, max_new, max_len, tables=None, table_stride=1, lens=None, cu_new=None, slots=None, q_stride=0, kv_stride=0):
    return kvfold_batch_t(ctypes.sizeof(kvfold_batch_t), n_seqs, n_tokens, max_new, max_len, tables, table_stride, lens, cu_new, slots, q_stride, kv_stride)


def kvfold_pcache_bytes_required(cfg) -> int:
    return int(load_library().kvfold_pcache_bytes_required(ctypes.byref(cfg)))


def kvfold_pcache_create(cfg):
    h = ctypes.c_void_p()
    rc = load_library().kvfold_pcache_create(ctypes.byref(cfg) if cfg is not None else None, ctypes.byref(h))
    return rc, (h if rc == 0 else None)


def kvfold_pcache_destroy(cache) -> int:
    return load_library().kvfold_pcache_destroy(cache)


def kvfold_pcache_view(cache, layer):
    k, v = ctypes.c_void_p(), ctypes.c_void_p()
    return load_library().kvfold_pcache_view(cache, layer, ctypes.byref(k), ctypes.byref(v)), k.value, v.value


def kvfold_pcache_assign(cache, n_seqs, lens, n_new, free_pages, n_free, tables, table_stride, lens_after, cu_new, slots, positions, n_slots, n_free_after, status,
                         stream=0) -> int:
    return load_library().kvfold_pcache_assign(cache, n_seqs, lens, n_new, free_pages, n_free, tables, table_stride, lens_after, cu_new, slots, positions, n_slots,
                                               n_free_after, status, stream)


def kvfold_pcache_workspace_bytes(cache, batch) -> int:
    return int(load_library().kvfold_pcache_workspace_bytes(cache, ctypes.byref(batch) if batch is not None else None))


def kvfold_pcache_step(cache, layer, batch, q, k_new, v_new, out, lse, workspace, workspace_bytes, stream=0) -> int:
    return load_library().kvfold_pcache_step(cache, layer, ctypes.byref(batch) if batch is not None else None, q, k_new, v_new, out, lse, workspace, workspace_bytes, stream)


def kvfold_pcache_append(cache, layer, k, v, kv_stride, slots, n_tokens, stream=0) -> int:
    return load_library().kvfold_pcache_append(cache, layer, k, v, kv_stride, slots, n_tokens, stream)


def kvfold_status_string(status: int) -> str:
    return load_library().kvfold_status_string(status).decode()


def kvfold_measure_peaks(device=0, mfma=True, hbm=True):
    """(status, bf16 matrix-instruction TFLOP/s or None, HBM read GB/s or None) of the GPU `device`."""
    t, g = ctypes.c_double(0.0), ctypes.c_double(0.0)
    rc = load_library().kvfold_measure_peaks(device, ctypes.byref(t) if mfma else None, ctypes.byref(g) if hbm else None)
    return rc, (t.value if mfma and rc == 0 else None), (g.value if hbm and rc == 0 else None)


def kvfold_last_hip_error() -> int:
    return int(load_library().kvfold_last_hip_error())


# ---------------------------------------------------------------------------------------------
# Convenience wrapper for torch callers (still marshalling only).
# ---------------------------------------------------------------------------------------------
def _current_stream(device) -> int:
    """Handle of the calling thread's current stream on the device, what torch.cuda.current_stream(device).cuda_stream
    is, without the object in between (0.3 us of host time instead of 1.4)."""
    import torch
    try:
        return torch._C._cuda_getCurrentRawStream(device)
    except AttributeError:
        return torch.cuda.current_stream(device).cuda_stream


_native = False  # module of csrc/py_step.cpp; None: not there, or built for another torch; False: not looked for yet
_native_lock = threading.Lock()


def _native_step():
    global _native
    if _native is False:
        with _native_lock:  # (a thread that finds another one looking waits for what it finds)
            if _native is False:
                _native = _load_native()
    return _native


def _load_native():
    import importlib.util

    import torch
    spec = importlib.util.spec_from_file_location("kvfold_py_step", os.path.join(_HERE, "_lib", "kvfold_py_step.so"))
    try:
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError:  # (also: no such file)
        return None
    return module if module.torch_version == torch.__version__.split("+")[0] else None


class KvFoldCache:
    """Owns one library cache handle; ``step`` takes torch tensors on the cache's device."""

    def __init__(self, n_layers, n_q_heads, n_kv_heads, head_dim, chunk_tokens, capacity_tokens, dtype="bf16",
                 softmax_scale=0.0, device=0):
        self.dtype_name = dtype
        self.cfg = make_config(n_layers, n_q_heads, n_kv_heads, head_dim, chunk_tokens, capacity_tokens,
                               {"f32": KVFOLD_F32, "bf16": KVFOLD_BF16}[dtype], softmax_scale, device)
        rc, self.handle = kvfold_cache_create(self.cfg)
        if rc:
            raise KvFoldError(rc, "kvfold_cache_create")
        # what every step needs, as plain Python values: fields of a ctypes structure are slow to read
        self._device, self._hq, self._hkv, self._d, self._capacity = device, n_q_heads, n_kv_heads, head_dim, capacity_tokens
        self._lib = load_library()
        self._bound = self._bound_weights = False  # what the native step, and the calls beside it, know of this cache; None: there is none

    def _bind(self):
        native, lib = _native_step(), self._lib
        if native is None or self.handle is None:
            self._bound = None
        else:
            address = [ctypes.cast(f, ctypes.c_void_p).value
                       for f in (lib.kvfold_step_ex, lib.kvfold_step_noalloc, lib.kvfold_step_rope, lib.kvfold_step_window)]
            self._bound = native.bind(*address, self.handle.value, self._device, self._hq, self._hkv, self._d, self.dtype_name != "f32")
        return self._bound

    def _bind_weights(self):
        native, lib = _native_step(), self._lib
        if native is None or self.handle is None:
            self._bound_weights = None
        else:
            address = [ctypes.cast(f, ctypes.c_void_p).value for f in (lib.kvfold_cache_weigh, lib.kvfold_cache_evict)]
            self._bound_weights = native.bind_weights(*address, self.handle.value, self._device, self._hq, self._hkv, self._d, self._capacity,
                                                      self.dtype_name != "f32")
        return self._bound_weights

    def close(self):
        self._bound = self._bound_weights = None
        if getattr(self, "handle", None) is not None:
            rc = kvfold_cache_destroy(self.handle)
            self.handle = None
            if rc:
                raise KvFoldError(rc, "kvfold_cache_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _stream(self, stream):
        return _current_stream(self._device) if stream is None else stream

    def _check(self, name, t, shape, dtype=None):
        """Marshalling validation: the kernels trust shapes and element types, so a mismatch must stop here."""
        import torch
        want = dtype or (torch.float32 if self.dtype_name == "f32" else torch.bfloat16)
        if t.dtype == want and t.shape == shape and t.is_cuda and t.get_device() == self._device and t.is_contiguous():
            return
        if not (t.is_cuda and t.device.index == self.cfg.device):
            raise ValueError(f"{name}: expected a tensor on cuda:{self.cfg.device}, got {t.device}")
        if t.dtype != want:
            raise ValueError(f"{name}: expected dtype {want}, got {t.dtype}")
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
        if not t.is_contiguous():
            raise ValueError(f"{name}: expected a contiguous tensor")

    def step(self, layer, q, k_new, v_new, out, pos_offset=None, lse=None, stream=None, rope=None, window=None,
             noalloc=False):
        """Enqueue one fold step; q/k_new/v_new/out (and lse) are contiguous device tensors.  rope = (cos, sin),
        fp32 device tensors [n][head_dim/2]: q and k_new are unrotated and the step rotates them.  window =
        (n_sink, window): the sink + sliding-window step.  noalloc: through kvfold_step_noalloc."""
        pos = self.length(layer) if pos_offset is None else pos_offset
        bound = self._bound
        if bound is False:
            bound = self._bind()
        if bound is not None:
            rc = _native.step(bound, layer, q, k_new, v_new, out, pos, lse, stream, rope, window, noalloc)
            if rc == 0:
                return out
            if rc is not None:
                raise KvFoldError(rc, "kvfold_step_window" if window is not None else "kvfold_step_rope" if rope is not None
                                  else "kvfold_step_noalloc" if noalloc else "kvfold_step_ex")
        shape = q.shape
        n = shape[0] if len(shape) == 3 else -1
        wide, narrow = (n, self._hq, self._d), (n, self._hkv, self._d)
        self._check("q", q, wide)
        self._check("out", out, wide)
        self._check("k_new", k_new, narrow)
        self._check("v_new", v_new, narrow)
        lse_ptr = None
        if lse is not None:
            import torch
            self._check("lse", lse, (self._hq, n), torch.float32)
            lse_ptr = lse.data_ptr()
        if ((rope is not None and rope is not False) + (window is not None and window is not False) +
                (noalloc is not None and noalloc is not False)) > 1:
            raise ValueError("rope, window and noalloc are separate entry points")
        if window is not None:
            n_sink, win = window
            rc = self._lib.kvfold_step_window(self.handle, layer, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), n, pos,
                                              n_sink, win, out.data_ptr(), lse_ptr, self._stream(stream))
            if rc:
                raise KvFoldError(rc, "kvfold_step_window")
            return out
        if rope is None:
            fn, name = ((self._lib.kvfold_step_noalloc, "kvfold_step_noalloc") if noalloc
                        else (self._lib.kvfold_step_ex, "kvfold_step_ex"))
            rc = fn(self.handle, layer, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), n, pos,
                    out.data_ptr(), lse_ptr, self._stream(stream))
            if rc:
                raise KvFoldError(rc, name)
            return out
        import torch
        cos, sin = rope
        self._check("rope cos", cos, (n, self._d // 2), torch.float32)
        self._check("rope sin", sin, (n, self._d // 2), torch.float32)
        rc = self._lib.kvfold_step_rope(self.handle, layer, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), n, pos,
                                        cos.data_ptr(), sin.data_ptr(), out.data_ptr(), lse_ptr, self._stream(stream))
        if rc:
            raise KvFoldError(rc, "kvfold_step_rope")
        return out

    def weigh(self, layer, q, lse, weights, add=True, rope=None, stream=None):
        """Enqueue kvfold_cache_weigh behind a step: its q [n][Hq][d] and the lse [Hq][n] that it left; weights fp32 [Hkv][capacity], added to or
        (add=False) set.  rope = (cos, sin), fp32 [n][d/2]: q is unrotated.  Returns weights."""
        bound = self._bound_weights
        if bound is False:
            bound = self._bind_weights()
        if bound is not None:
            rc = _native.weigh(bound, layer, q, lse, weights, add, rope, stream)
            if rc == 0:
                return weights
            if rc is not None:
                raise KvFoldError(rc, "kvfold_cache_weigh")
        import torch
        f32, shape = torch.float32, q.shape
        n = shape[0] if len(shape) == 3 else -1
        self._check("q", q, (n, self._hq, self._d))
        self._check("lse", lse, (self._hq, n), f32)
        self._check("weights", weights, (self._hkv, self._capacity), f32)
        cos = sin = None
        if rope is not None:
            cos, sin = rope
            self._check("rope cos", cos, (n, self._d // 2), f32)
            self._check("rope sin", sin, (n, self._d // 2), f32)
            cos, sin = cos.data_ptr(), sin.data_ptr()
        rc = self._lib.kvfold_cache_weigh(self.handle, layer, q.data_ptr(), n, cos, sin, lse.data_ptr(), weights.data_ptr(), 1 if add else 0, self._stream(stream))
        if rc:
            raise KvFoldError(rc, "kvfold_cache_weigh")
        return weights

    def evict(self, layer, weights, n_keep, n_sink=0, n_recent=0, to=None, to_layer=0, to_weights=None, kept=None, workspace=None, stream=None):
        """Enqueue kvfold_cache_evict: per KV head the first n_sink rows, the last n_recent and the heaviest between them, n_keep in all, move
        to the front of this layer or to layer to_layer of the cache `to`.  weights fp32 [Hkv][capacity]; to_weights fp32 [Hkv][capacity of the
        target]; kept int32 [Hkv][n_keep], made here if not given, and returned.  workspace: a uint8 tensor of evict_workspace_bytes(n_keep), else one
        is made.  What is made here is of the pool of the stream that the call runs on, `stream` or torch's current one; `kept` may be used, behind the
        call, and let go on either."""
        import torch
        target = self if to is None else to
        if not isinstance(target, KvFoldCache):
            raise TypeError(f"to: expected a KvFoldCache, got {type(to).__name__}")
        if target.handle is None:
            raise ValueError("to: the cache is closed")
        bound = self._bound_weights
        if bound is False:
            bound = self._bind_weights()
        if bound is not None and to is not None:
            into = to._bound_weights
            if into is False:
                into = to._bind_weights()
        else:
            into = None
        if bound is not None and (to is None or into is not None) and type(n_keep) is int and 0 < n_keep <= self._capacity and type(weights) is torch.Tensor:
            rows, space = self._evict_memory(weights, n_keep, kept, workspace, stream)
            rc = _native.evict(bound, layer, weights, n_keep, n_sink, n_recent, into, to_layer, to_weights, rows, space, stream)
            if rc == 0:
                return rows
            if rc is not None:
                raise KvFoldError(rc, "kvfold_cache_evict")
        self._check("weights", weights, (self._hkv, self._capacity), torch.float32)
        if to_weights is not None:
            self._check("to_weights", to_weights, (self._hkv, target._capacity), torch.float32)
        if workspace is not None:
            self._check("workspace", workspace, (workspace.numel(),), torch.uint8)
        if kept is not None:
            self._check("kept", kept, (self._hkv, n_keep), torch.int32)
        kept, workspace = self._evict_memory(weights, n_keep if 0 < n_keep <= self._capacity else 0, kept, workspace, stream)
        rc = self._lib.kvfold_cache_evict(self.handle, layer, weights.data_ptr(), n_keep, n_sink, n_recent, None if to is None else to.handle, to_layer,
                                          None if to_weights is None else to_weights.data_ptr(), kept.data_ptr(), workspace.data_ptr(),
                                          workspace.numel(), self._stream(stream))
        if rc:
            raise KvFoldError(rc, "kvfold_cache_evict")
        return kept

    def _evict_memory(self, weights, n_keep, kept, workspace, stream):
        """kept and workspace, made if they are not given."""
        import torch
        if (kept is None or workspace is None) and stream is not None and stream != self._stream(None):
            made = kept is None
            with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=self._device)):
                kept, workspace = self._evict_memory(weights, n_keep, kept, workspace, None)
            if made and kept.is_cuda:
                kept.record_stream(torch.cuda.current_stream(self._device))
        if kept is None:
            kept = torch.empty((self._hkv, n_keep), dtype=torch.int32, device=weights.device)
        if workspace is None:
            workspace = torch.empty((max(kvfold_evict_workspace_bytes(self.handle, n_keep), 4),), dtype=torch.uint8, device=weights.device)
        return kept, workspace

    def evict_workspace_bytes(self, n_keep) -> int:
        return kvfold_evict_workspace_bytes(self.handle, n_keep)

    def bytes_required(self) -> int:
        return kvfold_cache_bytes_required(self.cfg)

    def length(self, layer=0) -> int:
        n = kvfold_cache_length(self.handle, layer)
        if n < 0:
            raise KvFoldError(n, "kvfold_cache_length")
        return n

    def truncate(self, layer, new_len):
        rc = kvfold_cache_truncate(self.handle, layer, new_len)
        if rc:
            raise KvFoldError(rc, "kvfold_cache_truncate")

    def set_length(self, layer, new_len):
        rc = kvfold_cache_set_length(self.handle, layer, new_len)
        if rc:
            raise KvFoldError(rc, "kvfold_cache_set_length")

    def set_storage_roundtrip(self, n_bits):
        rc = kvfold_cache_set_storage_roundtrip(self.handle, n_bits)
        if rc:
            raise KvFoldError(rc, "kvfold_cache_set_storage_roundtrip")

    def set_tuning(self, knob, value):
        rc = kvfold_cache_set_tuning(self.handle, knob, value)
        if rc:
            raise KvFoldError(rc, "kvfold_cache_set_tuning")

    def plan(self, n_tokens, len_after):
        rc, w, s = kvfold_cache_plan(self.handle, n_tokens, len_after)
        if rc:
            raise KvFoldError(rc, "kvfold_cache_plan")
        return w, s

    def profile_begin(self, max_steps):
        rc = kvfold_cache_profile_begin(self.handle, max_steps)
        if rc:
            raise KvFoldError(rc, "kvfold_cache_profile_begin")

    def profile_end(self):
        """(n_steps, append_ms, attention_ms, merge_ms) summed over the profiled steps."""
        rc, n, a, t, m = kvfold_cache_profile_end(self.handle)
        if rc:
            raise KvFoldError(rc, "kvfold_cache_profile_end")
        return n, a, t, m

    def view(self, layer=0):
        """(K, V) device tensors [Hkv][capacity][d] aliasing the cache rows of ``layer`` (no copy).  They keep the cache from being collected; ``close()``
        frees their memory all the same."""
        import torch
        rc, k, v, rs, hs = kvfold_cache_view(self.handle, layer)
        if rc:
            raise KvFoldError(rc, "kvfold_cache_view")
        c = self.cfg
        es = 4 if self.dtype_name == "f32" else 2

        def wrap(ptr):
            class _Holder:  # device memory described by pointer + shape; torch aliases it, nothing is copied
                __cuda_array_interface__ = {"shape": (c.n_kv_heads, c.capacity_tokens, c.head_dim),
                                            "typestr": "<f4" if es == 4 else "<i2", "data": (ptr, False),
                                            "version": 3}
            holder = _Holder()
            holder.owner = self  # (torch holds on to the holder as long as there is a tensor on the memory)
            t = torch.as_tensor(holder, device=f"cuda:{c.device}")
            return t if es == 4 else t.view(torch.bfloat16)

        return wrap(k), wrap(v)


def _expect(name, t, dtype, device, shape=None, contiguous=True):
    if not (t.is_cuda and t.get_device() == device):
        raise ValueError(f"{name}: expected a tensor on cuda:{device}, got {t.device}")
    if t.dtype != dtype:
        raise ValueError(f"{name}: expected dtype {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor")
    return t.data_ptr()


class KvFoldQuantCache:
    """Owns one cache held in 8 bits (``kvfold_qcache_*``); bf16 torch tensors on the cache's device."""

    def __init__(self, n_layers, n_q_heads, n_kv_heads, head_dim, chunk_tokens, capacity_tokens, softmax_scale=0.0, device=0):
        import torch
        self._bf16, self._f32 = torch.bfloat16, torch.float32
        self.cfg = make_config(n_layers, n_q_heads, n_kv_heads, head_dim, chunk_tokens, capacity_tokens, KVFOLD_BF16, softmax_scale, device)
        self.handle = None
        rc, self.handle = kvfold_qcache_create(self.cfg)
        if rc:
            raise KvFoldError(rc, "kvfold_qcache_create")
        self._device, self._hq, self._hkv, self._d = device, n_q_heads, n_kv_heads, head_dim
        self._lib = load_library()
        self._bound = False  # what the native calls know of this cache; None: there are none

    def _bind(self):
        native, lib = _native_step(), self._lib
        if native is None or self.handle is None:
            self._bound = None
        else:
            address = [ctypes.cast(f, ctypes.c_void_p).value for f in (lib.kvfold_qcache_step, lib.kvfold_qcache_read)]
            self._bound = native.bind_quant(*address, self.handle.value, self._device, self._hq, self._hkv, self._d)
        return self._bound

    def close(self):
        self._bound = None
        if getattr(self, "handle", None) is not None:
            rc = kvfold_qcache_destroy(self.handle)
            self.handle = None
            if rc:
                raise KvFoldError(rc, "kvfold_qcache_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _stream(self, stream):
        if stream is not None:
            return stream
        import torch
        return torch.cuda.current_stream(self._device).cuda_stream

    def _angles(self, rope, n):
        if rope is None:
            return None, None
        cos, sin = rope
        return (_expect("rope cos", cos, self._f32, self._device, (n, self._d // 2)), _expect("rope sin", sin, self._f32, self._device, (n, self._d // 2)))

    def step(self, layer, q, k_new, v_new, out, pos_offset=None, lse=None, stream=None, rope=None):
        """Enqueue one fold step: q, out [n][Hq][d], k_new, v_new [n][Hkv][d], lse fp32 [Hq][n], all contiguous.  rope = (cos, sin), fp32
        [n][d/2]: q and k_new are unrotated and the step rotates them."""
        pos = self.length(layer) if pos_offset is None else pos_offset
        bound = self._bound
        if bound is False:
            bound = self._bind()
        if bound is not None:
            rc = _native.quant_step(bound, layer, q, k_new, v_new, out, pos, lse, stream, rope)
            if rc == 0:
                return out
            if rc is not None:
                raise KvFoldError(rc, "kvfold_qcache_step")
        n = q.shape[0] if q.dim() == 3 else -1
        wide, narrow = (n, self._hq, self._d), (n, self._hkv, self._d)
        args = [_expect("q", q, self._bf16, self._device, wide), _expect("k_new", k_new, self._bf16, self._device, narrow),
                _expect("v_new", v_new, self._bf16, self._device, narrow)]
        cos, sin = self._angles(rope, n)
        rc = self._lib.kvfold_qcache_step(self.handle, layer, *args, n, pos, cos, sin,
                                          _expect("out", out, self._bf16, self._device, wide),
                                          None if lse is None else _expect("lse", lse, self._f32, self._device, (self._hq, n)), self._stream(stream))
        if rc:
            raise KvFoldError(rc, "kvfold_qcache_step")
        return out

    def append(self, layer, k, v, pos_offset=None, stream=None, rope=None):
        """Append rows without attention: k, v [n][Hkv][d], any strides alike of both that are multiples of 8 elements, rows themselves
        contiguous (``KvFoldCache.view(...)[:, :n].transpose(0, 1)``, say)."""
        n = k.shape[0] if k.dim() == 3 else -1
        strides = []
        for name, t in (("k", k), ("v", v)):
            _expect(name, t, self._bf16, self._device, (n, self._hkv, self._d), contiguous=False)
            strides.append((t.stride(0) if n > 1 else 0, t.stride(1) if self._hkv > 1 else 0))  # (of one row, or one head, a stride means nothing)
            if strides[-1] != strides[0] or (n and t.stride(2) != 1):
                raise ValueError(f"{name}: expected rows of stride 1 and the same strides for k and v, got {t.stride()}")
        cos, sin = self._angles(rope, n)
        rc = self._lib.kvfold_qcache_append(self.handle, layer, k.data_ptr(), v.data_ptr(), *strides[0], n,
                                            self.length(layer) if pos_offset is None else pos_offset, cos, sin, self._stream(stream))
        if rc:
            raise KvFoldError(rc, "kvfold_qcache_append")

    def read(self, layer, first, k_out, v_out, stream=None):
        """Rows [first, first + n) as the fp32 numbers they stand for: k_out, v_out [n][Hkv][d] (either may be None)."""
        given = [t for t in (k_out, v_out) if t is not None]
        if not given:
            return
        bound = self._bound
        if bound is False:
            bound = self._bind()
        if bound is not None:
            rc = _native.quant_read(bound, layer, first, k_out, v_out, stream)
            if rc == 0:
                return
            if rc is not None:
                raise KvFoldError(rc, "kvfold_qcache_read")
        n = given[0].shape[0] if given[0].dim() == 3 else -1
        ptr = [None if t is None else _expect(name, t, self._f32, self._device, (n, self._hkv, self._d)) for name, t in (("k_out", k_out), ("v_out", v_out))]
        rc = self._lib.kvfold_qcache_read(self.handle, layer, first, n, *ptr, self._stream(stream))
        if rc:
            raise KvFoldError(rc, "kvfold_qcache_read")

    def bytes_required(self) -> int:
        return kvfold_qcache_bytes_required(self.cfg)

    def length(self, layer=0) -> int:
        n = self._lib.kvfold_qcache_length(self.handle, layer)
        if n < 0:
            raise KvFoldError(n, "kvfold_qcache_length")
        return n

    def truncate(self, layer, new_len):
        rc = self._lib.kvfold_qcache_truncate(self.handle, layer, new_len)
        if rc:
            raise KvFoldError(rc, "kvfold_qcache_truncate")


class KvFoldPagedCache:
    """Owns one cache in pages (``kvfold_pcache_*``), which sequences share; tables, lengths and places are tensors of the caller's, in a ``KvFoldBatch``."""

    def __init__(self, n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages, dtype="bf16", softmax_scale=0.0, device=0):
        import torch
        self.dtype_name = dtype
        self.cfg = make_pconfig(n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages, {"f32": KVFOLD_F32, "bf16": KVFOLD_BF16}[dtype], softmax_scale,
                                device)
        self.handle = None
        rc, self.handle = kvfold_pcache_create(self.cfg)
        if rc:
            raise KvFoldError(rc, "kvfold_pcache_create")
        self._dtype, self._f32, self._i32, self._i64, self._u8 = torch.float32 if dtype == "f32" else torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.uint8
        self._device, self._hq, self._hkv, self._d, self._page, self._n_pages, self._n_layers = device, n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages, n_layers
        self._lib = load_library()
        self._bound = False  # as in KvFoldCache

    def _bind(self):
        native, lib = _native_step(), self._lib
        if native is None or self.handle is None:
            self._bound = None
        else:
            address = [ctypes.cast(f, ctypes.c_void_p).value for f in (lib.kvfold_pcache_step, lib.kvfold_pcache_assign)]
            self._bound = native.bind_paged(*address, self.handle.value, self._device, self._hq, self._hkv, self._d, self._n_pages, self.dtype_name != "f32")
        return self._bound

    def close(self):
        self._bound = None
        if getattr(self, "handle", None) is not None:
            rc = kvfold_pcache_destroy(self.handle)
            self.handle = None
            if rc:
                raise KvFoldError(rc, "kvfold_pcache_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _stream(self, stream):
        return _current_stream(self._device) if stream is None else stream

    def _rows(self, name, t, n, heads):
        """Address and token stride of [n][heads][d] rows whose heads lie side by side, as parts of a fused projection's result do."""
        _expect(name, t, self._dtype, self._device, (n, heads, self._d), contiguous=False)
        if n and ((heads > 1 and t.stride(1) != self._d) or t.stride(2) != 1 or (n > 1 and t.stride(0) < heads * self._d)):
            raise ValueError(f"{name}: expected a token's heads side by side, got strides {t.stride()}")
        return t.data_ptr(), t.stride(0) if n > 1 else heads * self._d

    def assign(self, batch, lens, n_new, free_pages, n_free, stream=None):
        """Where the new tokens of the batch's sequences go, into the batch's own tensors (tables, lens, cu_new, slots, positions, n_free, status): lens, n_new int32
        [n_seqs], free_pages int32 [n_pages], n_free int32 [1].  Nothing is synchronised: status says on the device whether there was room."""
        bound = self._bound
        if bound is False:
            bound = self._bind()
        if bound is not None:
            rc = _native.paged_assign(bound, lens, n_new, free_pages, n_free, batch.tables, batch.lens, batch.cu_new, batch.slots, batch.positions, batch.n_free,
                                      batch.status, stream)
            if rc == 0:
                return batch
            if rc is not None:
                raise KvFoldError(rc, "kvfold_pcache_assign")
        s = batch.n_seqs
        tables, lens_after, cu_new, slots, positions, n_free_after, status = self._expect_batch(batch)
        rc = self._lib.kvfold_pcache_assign(
            self.handle, s, _expect("lens", lens, self._i32, self._device, (s,)), _expect("n_new", n_new, self._i32, self._device, (s,)),
            _expect("free_pages", free_pages, self._i32, self._device, (self._n_pages,)), _expect("n_free", n_free, self._i32, self._device, (1,)),
            tables, batch.tables.shape[1], lens_after, cu_new, slots, positions, batch.n_tokens, n_free_after, status, self._stream(stream))
        if rc:
            raise KvFoldError(rc, "kvfold_pcache_assign")
        return batch

    def _expect_batch(self, batch):
        """Addresses of the batch's tables, lens, cu_new, slots, positions, n_free and status, which have to be what they were made as."""
        s, n, i32 = batch.n_seqs, batch.n_tokens, self._i32
        return [_expect(f"batch.{name}", getattr(batch, name), dtype, self._device, shape) for name, dtype, shape in (
            ("tables", i32, (s, batch.tables.shape[-1])), ("lens", i32, (s,)), ("cu_new", i32, (s + 1,)), ("slots", self._i64, (n,)), ("positions", i32, (n,)),
            ("n_free", i32, (1,)), ("status", i32, (1,)))]

    def step(self, layer, batch, q, k_new, v_new, out, lse=None, stream=None):
        """Enqueue one fold step of every sequence of the batch: q, out [n_tokens][Hq][d], k_new, v_new [n_tokens][Hkv][d], lse fp32 [Hq][n_tokens].  q, k_new and v_new
        may be parts of one tensor.  k_new = v_new = None: the new rows are in the pages already (``append``)."""
        n = batch.n_tokens
        if batch.cache is not self and batch.cache._hkv != self._hkv:  # (its workspace has a counter for each sequence and KV head)
            raise ValueError(f"batch: made for {batch.cache._hkv} KV heads, the cache has {self._hkv}")
        bound = self._bound
        if bound is False:
            bound = self._bind()
        if bound is not None:
            rc = _native.paged_step(bound, layer, batch.n_seqs, batch.tables, batch.lens, None if batch.one_each else batch.cu_new, batch.slots, batch.workspace, n,
                                    batch.max_new, batch.max_len, q, k_new, v_new, out, lse, stream)
            if rc == 0:
                return out
            if rc is not None:
                raise KvFoldError(rc, "kvfold_pcache_step")
        q_at, q_stride = self._rows("q", q, n, self._hq)
        k_at = v_at = None
        kv_stride = 0
        if (k_new is None) != (v_new is None):
            raise ValueError("k_new and v_new: both or neither")
        if k_new is not None:
            (k_at, kv_stride), (v_at, v_stride) = self._rows("k_new", k_new, n, self._hkv), self._rows("v_new", v_new, n, self._hkv)
            if v_stride != kv_stride:
                raise ValueError(f"v_new: expected the strides of k_new, got {v_new.stride()} beside {k_new.stride()}")
        tables, lens, cu_new, slots = self._expect_batch(batch)[:4]
        desc = make_batch(batch.n_seqs, n, batch.max_new, batch.max_len, tables, batch.tables.shape[1], lens, None if batch.one_each else cu_new,
                          None if k_new is None else slots)
        desc.q_stride, desc.kv_stride = q_stride, kv_stride
        rc = self._lib.kvfold_pcache_step(
            self.handle, layer, ctypes.byref(desc), q_at, k_at, v_at, _expect("out", out, self._dtype, self._device, (n, self._hq, self._d)),
            None if lse is None else _expect("lse", lse, self._f32, self._device, (self._hq, n)),
            _expect("batch.workspace", batch.workspace, self._u8, self._device, (batch.workspace.numel(),)), batch.workspace.numel(), self._stream(stream))
        if rc:
            raise KvFoldError(rc, "kvfold_pcache_step")
        return out

    def append(self, layer, k, v, slots, stream=None):
        """Rows k, v [n][Hkv][d] to their places, slots int64 [n], without attention; a place outside the cache (-1) is passed over."""
        n = k.shape[0] if k.dim() == 3 else -1
        (k_at, stride), (v_at, v_stride) = self._rows("k", k, n, self._hkv), self._rows("v", v, n, self._hkv)
        if v_stride != stride:
            raise ValueError(f"v: expected the strides of k, got {v.stride()} beside {k.stride()}")
        rc = self._lib.kvfold_pcache_append(self.handle, layer, k_at, v_at, stride, _expect("slots", slots, self._i64, self._device, (n,)), n, self._stream(stream))
        if rc:
            raise KvFoldError(rc, "kvfold_pcache_append")

    def bytes_required(self) -> int:
        return kvfold_pcache_bytes_required(self.cfg)

    def view(self, layer=0):
        """Torch tensors aliasing the layer's K and V pages, [n_pages][Hkv][page_tokens][d] each; they keep the cache."""
        import torch
        rc, k, v = kvfold_pcache_view(self.handle, layer)
        if rc:
            raise KvFoldError(rc, "kvfold_pcache_view")
        shape = (self._n_pages, self._hkv, self._page, self._d)
        return tuple(_alias(self, at, shape, self._dtype, f"cuda:{self._device}", torch) for at in (k, v))


def _alias(owner, at, shape, dtype, device, torch):
    class Memory:  # (no bf16 in this protocol: 16-bit whole numbers, then viewed)
        __cuda_array_interface__ = {"shape": shape, "typestr": "<i2" if dtype == torch.bfloat16 else "<f4", "data": (at, False), "version": 3, "strides": None}
    memory = Memory()
    memory.owner = owner
    t = torch.as_tensor(memory, device=device)
    return t.view(dtype) if t.dtype != dtype else t


class KvFoldBatch:
    """A batch of sequences for ``KvFoldPagedCache``: the tables [n_seqs][pages] int32, which are the caller's, and what goes with them, made here where not
    given: lens int32 [n_seqs] (the new tokens among them), cu_new int32 [n_seqs + 1], slots int64 [n_tokens], and the workspace of its steps.

    n_tokens rows are packed in a step's tensors; max_new and max_len bound the new tokens and the tokens of any sequence.  one_each: every sequence has
    exactly one new token, and n_tokens = n_seqs (a sequence whose place is none, as after an assign whose status is not 0, has no new token; a step without k_new and
    v_new does not look at places).  A batch is good for one step at a time: steps that may overlap (on streams of their own) have a batch each.
    Its workspace is for its number of sequences and its cache's of KV heads: a step on another cache has to have as many.
    What is made here is made on the current stream: a step on another one waits for it."""

    def __init__(self, cache, tables, n_tokens, max_new, max_len, lens=None, cu_new=None, slots=None, one_each=False):
        import torch
        dev = cache._device
        _expect("tables", tables, torch.int32, dev)
        if tables.dim() != 2 or not tables.shape[1]:
            raise ValueError(f"tables: expected [n_seqs][pages], got {tuple(tables.shape)}")
        self.cache, self.tables, self.n_seqs, self.n_tokens, self.one_each = cache, tables, tables.shape[0], n_tokens, one_each
        self.max_new, self.max_len = max_new, max_len
        where = f"cuda:{dev}"

        def mine(name, given, shape, dtype, value=0):
            if given is None:
                return torch.full(shape, value, dtype=dtype, device=where)
            _expect(name, given, dtype, dev, shape)
            return given
        if not (0 <= n_tokens < 1 << 31 and 1 <= max_new < 1 << 31 and 1 <= max_len <= 1 << 30):
            raise ValueError(f"a batch of {n_tokens} tokens, max_new {max_new}, max_len {max_len} is none")
        self.lens = mine("lens", lens, (self.n_seqs,), torch.int32)
        self.cu_new = mine("cu_new", cu_new, (self.n_seqs + 1,), torch.int32)
        self.slots = mine("slots", slots, (n_tokens,), torch.int64, -1)  # (no place, until one is given)
        self.positions, self.n_free, self.status = (torch.zeros(shape, dtype=torch.int32, device=where) for shape in ((n_tokens,), (1,), (1,)))
        need = kvfold_pcache_workspace_bytes(cache.handle, make_batch(self.n_seqs, n_tokens, max_new, max_len, tables.data_ptr(), tables.shape[1], None, None, None))
        if not need:
            raise ValueError(f"a batch of {self.n_seqs} sequences, {n_tokens} tokens, max_new {max_new}, max_len {max_len} is none")
        self.workspace = torch.zeros((need,), dtype=torch.uint8, device=where)
