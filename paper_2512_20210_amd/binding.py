"""ctypes binding of include/plora.h: same names, argument marshalling only.

Functions return the library's status code (and outputs where the C call has out-parameters).
Device buffers are passed as integers (tensor.data_ptr()), streams as integers
(torch.cuda.current_stream().cuda_stream).  PagedLoraPool is a convenience wrapper that raises
PloraError on a negative status and keeps the objects it must keep alive.
"""
import ctypes as C
import os
import sys

import numpy as np

__all__ = ["PLORA_OK", "PLORA_ERR_INVAL", "PLORA_ERR_NOMEM", "PLORA_ERR_EXISTS", "PLORA_ERR_NOTFOUND",
           "PLORA_ERR_BUSY", "PLORA_ERR_HIP", "PLORA_ERR_LIMIT", "PLORA_F16", "PLORA_BF16", "PLORA_F32", "PLORA_POOL_PLACEMENT_ONLY",
           "plora_pool_create", "plora_pool_destroy", "plora_adapter_bytes", "plora_load_adapter",
           "plora_adapter_ready", "plora_wait_adapter", "plora_sync_adapter", "plora_evict", "plora_adapter_pages", "plora_compact", "plora_batch_begin", "plora_batch_info",
           "plora_shrink", "plora_expand", "plora_delta", "plora_delta_static", "plora_batch_end", "plora_pool_stats", "plora_pool_set_option",
           "plora_profile", "plora_profile_read", "plora_probe_stream", "plora_probe_h2d", "plora_last_hip", "plora_version", "PloraError", "PagedLoraPool", "lib", "LIB_PATH",
           "plora_predictor_create", "plora_predictor_destroy", "plora_predictor_observe", "plora_predictor_observed",
           "plora_predictor_predict", "plora_predictor_train", "plora_predictor_train_batch",
           "plora_predictor_param_count", "plora_predictor_get_params", "plora_predictor_set_params",
           "plora_predictor_loss_grad", "plora_predictor_set_threads", "LstmPredictor",
           "plora_manager_create", "plora_manager_destroy", "plora_manager_set_adapter", "plora_manager_set_prediction",
           "plora_manager_request", "plora_manager_prefetch", "plora_manager_scores", "plora_manager_residents",
           "plora_manager_state", "plora_manager_get_stats", "plora_manager_log", "ResidencyManager",
           "plora_suggest_page_bytes",
           "PLORA_ROTARY_NONE", "PLORA_ROTARY_LINEAR", "PLORA_ROTARY_NTK", "PLORA_ROTARY_TURNS",
           "plora_rotary_table", "plora_rotate", "plora_kv_page_bytes", "plora_kv_append", "plora_kv_read", "plora_kv_attend",
           "RotaryConfig", "RotaryStruct", "RowsStruct", "KvCacheStruct", "KvBatchStruct", "Rotary", "KvBatch", "PagedKvCache",
           "PLORA_ACT_NONE", "PLORA_ACT_SILU", "PLORA_ACT_GELU",
           "plora_norm", "plora_fp8_quantise", "plora_fp8_quantise_weights", "plora_fp8_matmul", "plora_fp8_grouped", "plora_fp8_tile_of", "plora_route",
           "plora_route_workspace_bytes", "MatrixStruct", "Fp8RowsStruct", "Fp8WeightsStruct", "NormWeightsStruct", "BlockNormStruct",
           "Fp8Rows", "Fp8Weights", "Routing", "NormWeights", "BlockNorm"]

PLORA_OK, PLORA_ERR_INVAL, PLORA_ERR_NOMEM, PLORA_ERR_EXISTS = 0, -1, -2, -3
PLORA_ERR_NOTFOUND, PLORA_ERR_BUSY, PLORA_ERR_HIP, PLORA_ERR_LIMIT = -4, -5, -6, -7
PLORA_F16, PLORA_BF16, PLORA_F32 = 0, 1, 2
PLORA_POOL_PLACEMENT_ONLY = 1
PLORA_ROTARY_NONE, PLORA_ROTARY_LINEAR, PLORA_ROTARY_NTK, PLORA_ROTARY_TURNS = 0, 1, 2, 3
PLORA_ACT_NONE, PLORA_ACT_SILU, PLORA_ACT_GELU = 0, 1, 2
_STATUS = {0: "OK", -1: "INVAL", -2: "NOMEM", -3: "EXISTS", -4: "NOTFOUND", -5: "BUSY", -6: "HIP", -7: "LIMIT"}

LIB_PATH = os.environ.get("PLORA_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libplora.so")
if not os.path.exists(LIB_PATH):
    raise ImportError("libplora.so is not built: run `python paper_2512_20210_amd/build.py` "
                      "(or __graft_entry__.build()); there is no fallback implementation")
lib = C.CDLL(LIB_PATH)


class _Layout(C.Structure):
    _fields_ = [("n_slots", C.c_int32), ("d_in", C.POINTER(C.c_int32)), ("d_out", C.POINTER(C.c_int32)),
                ("dtype", C.c_int32), ("max_adapters", C.c_int32), ("max_rank", C.c_int32)]


class _Stats(C.Structure):
    _fields_ = [(k, C.c_uint64) for k in ("page_bytes", "n_pages", "used_pages", "free_pages", "resident_adapters",
                                          "resident_bytes", "internal_frag_bytes", "loads", "evictions",
                                          "nomem_failures", "h2d_bytes", "h2d_copies")] + [("h2d_ms", C.c_double), ("staged_loads", C.c_uint64), ("fused_launches", C.c_uint64),
                                                                                        ("fused_timeouts", C.c_uint64), ("compacted_adapters", C.c_uint64),
                                                                                        ("compacted_pages", C.c_uint64), ("compact_ms", C.c_double)]


_vp, _i32, _u32, _u64, _f32 = C.c_void_p, C.c_int32, C.c_uint32, C.c_uint64, C.c_float
lib.plora_pool_create.argtypes = [C.c_size_t, _u32, C.POINTER(_Layout), _vp, _u32, C.POINTER(_vp)]
lib.plora_pool_destroy.argtypes = [_vp]
lib.plora_adapter_bytes.argtypes = [_vp, _i32]
lib.plora_adapter_bytes.restype = _u64
lib.plora_load_adapter.argtypes = [_vp, _i32, _i32, _f32, _vp, _vp, C.POINTER(C.POINTER(_i32)), C.POINTER(_u32)]
lib.plora_adapter_ready.argtypes = [_vp, _i32]
lib.plora_wait_adapter.argtypes = [_vp, _i32, _vp]
lib.plora_evict.argtypes = [_vp, _i32]
lib.plora_compact.argtypes = [_vp, _vp, _u32, C.POINTER(_u32), C.POINTER(_u32)]
lib.plora_adapter_pages.argtypes = [_vp, _i32, C.POINTER(C.POINTER(_i32)), C.POINTER(_u32)]
lib.plora_sync_adapter.argtypes = [_vp, _i32]
lib.plora_batch_begin.argtypes = [_vp, _vp, _i32, _vp, C.POINTER(_vp)]
lib.plora_batch_info.argtypes = [_vp, C.POINTER(_i32), C.POINTER(_i32), C.POINTER(C.POINTER(_i32)),
                                 C.POINTER(C.POINTER(_i32)), C.POINTER(C.POINTER(_i32))]
lib.plora_shrink.argtypes = [_vp, _vp, _i32, _i32, _vp, _vp, _vp]
lib.plora_expand.argtypes = [_vp, _vp, _i32, _i32, _vp, _vp, _vp]
lib.plora_delta.argtypes = [_vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp]
lib.plora_delta_static.argtypes = [_vp, _vp, _i32, _i32, _vp, _vp, _vp]
lib.plora_batch_end.argtypes = [_vp, _vp]
lib.plora_pool_stats.argtypes = [_vp, C.POINTER(_Stats)]
lib.plora_pool_set_option.argtypes = [_vp, C.c_char_p, C.c_int64]
lib.plora_profile.argtypes = [_vp, C.c_int]
lib.plora_profile_read.argtypes = [_vp, C.POINTER(C.c_double), C.POINTER(C.c_uint64)]
lib.plora_probe_stream.argtypes = [_u64, _u64, _u32, _u32, _i32, _vp, C.POINTER(C.c_double)]
lib.plora_probe_h2d.argtypes = [_u64, _i32, _vp, C.POINTER(C.c_double)]
lib.plora_last_hip.argtypes = []
lib.plora_version.argtypes = []


class _ManagerConfig(C.Structure):
    _fields_ = [("alpha", C.c_double), ("beta", C.c_double), ("gamma", C.c_double), ("theta", C.c_double), ("window", C.c_int32)]


class _ManagerStats(C.Structure):
    _fields_ = [(k, C.c_uint64) for k in ("hits", "misses", "loads", "evictions", "failed_loads", "skipped_busy", "waited_for_busy",
                                          "prefetch_loads", "useful_prefetches", "wasted_prefetches", "prefetch_no_room",
                                          "util_samples")] + [(k, C.c_double) for k in ("page_util_sum", "page_util_min",
                                                                                         "byte_util_sum", "byte_util_min")]


lib.plora_manager_create.argtypes = [_vp, _i32, C.POINTER(_ManagerConfig), C.POINTER(_vp)]
lib.plora_manager_destroy.argtypes = [_vp]
lib.plora_manager_set_adapter.argtypes = [_vp, _i32, _i32, _f32, _vp]
lib.plora_manager_set_prediction.argtypes = [_vp, _vp]
lib.plora_manager_request.argtypes = [_vp, _i32, _vp, C.POINTER(_i32)]
lib.plora_manager_prefetch.argtypes = [_vp, _vp, _vp, C.POINTER(_i32)]
lib.plora_manager_scores.argtypes = [_vp, _vp, _vp, _i32, C.POINTER(_i32)]
lib.plora_manager_residents.argtypes = [_vp, _vp, _i32, C.POINTER(_i32)]
lib.plora_manager_state.argtypes = [_vp, _i32]
lib.plora_manager_get_stats.argtypes = [_vp, C.POINTER(_ManagerStats)]
lib.plora_manager_log.argtypes = [_vp, _vp, C.c_int64, C.POINTER(C.c_int64), _i32]
lib.plora_suggest_page_bytes.argtypes = [C.POINTER(_Layout), _vp, _vp, _i32, C.c_double, C.c_size_t, C.c_size_t,
                                         C.POINTER(C.c_size_t), C.POINTER(C.c_double)]


class _PredictorConfig(C.Structure):
    _fields_ = [("n_adapters", C.c_int32), ("window", C.c_int32), ("hidden", C.c_int32), ("layers", C.c_int32),
                ("replay", C.c_int32), ("batch", C.c_int32), ("lr", C.c_float), ("beta1", C.c_float),
                ("beta2", C.c_float), ("eps", C.c_float), ("seed", C.c_uint64)]


_fp = C.POINTER(C.c_float)
lib.plora_predictor_create.argtypes = [C.POINTER(_PredictorConfig), C.POINTER(_vp)]
lib.plora_predictor_destroy.argtypes = [_vp]
lib.plora_predictor_observe.argtypes = [_vp, _vp, _i32]
lib.plora_predictor_observed.argtypes = [_vp]
lib.plora_predictor_observed.restype = C.c_int64
lib.plora_predictor_predict.argtypes = [_vp, _vp]
lib.plora_predictor_train.argtypes = [_vp, _i32, _fp]
lib.plora_predictor_train_batch.argtypes = [_vp, _vp, _i32, _fp]
lib.plora_predictor_param_count.argtypes = [_vp]
lib.plora_predictor_param_count.restype = C.c_int64
lib.plora_predictor_get_params.argtypes = [_vp, _vp]
lib.plora_predictor_set_params.argtypes = [_vp, _vp]
lib.plora_predictor_loss_grad.argtypes = [_vp, _vp, _vp, _fp, _vp]
lib.plora_predictor_set_threads.argtypes = [_vp, _i32]


def _ptr_array(ptrs):
    return (C.c_void_p * len(ptrs))(*[int(p) for p in ptrs])


def plora_pool_create(page_bytes, n_pages, d_in, d_out, dtype, max_adapters, max_rank, slab_ptr=None, flags=0):
    """-> (status, pool handle)."""
    di = np.ascontiguousarray(d_in, dtype=np.int32)
    do = np.ascontiguousarray(d_out, dtype=np.int32)
    lay = _Layout(len(di), di.ctypes.data_as(C.POINTER(C.c_int32)), do.ctypes.data_as(C.POINTER(C.c_int32)),
                  dtype, max_adapters, max_rank)
    h = C.c_void_p()
    rc = lib.plora_pool_create(page_bytes, n_pages, C.byref(lay), slab_ptr, flags, C.byref(h))
    return rc, h


def plora_pool_destroy(pool):
    return lib.plora_pool_destroy(pool)


def plora_adapter_bytes(pool, rank):
    return lib.plora_adapter_bytes(pool, rank)


def plora_load_adapter(pool, aid, rank, scale, pinned_host_ptr, copy_stream=None):
    """-> (status, page table as an int32 numpy copy or None)."""
    pt = C.POINTER(C.c_int32)()
    n = C.c_uint32(0)
    rc = lib.plora_load_adapter(pool, aid, rank, scale, pinned_host_ptr, copy_stream, C.byref(pt), C.byref(n))
    if rc:
        return rc, None
    return rc, np.ctypeslib.as_array(pt, shape=(n.value,)).copy()


def plora_adapter_ready(pool, aid):
    return lib.plora_adapter_ready(pool, aid)


def plora_wait_adapter(pool, aid, stream=None):
    return lib.plora_wait_adapter(pool, aid, stream)


def plora_sync_adapter(pool, aid):
    return lib.plora_sync_adapter(pool, aid)


def plora_evict(pool, aid):
    return lib.plora_evict(pool, aid)


def plora_adapter_pages(pool, aid):
    """-> (status, copy of the adapter's page table as an int32 array)."""
    pt, n = C.POINTER(_i32)(), _u32(0)
    rc = lib.plora_adapter_pages(pool, aid, C.byref(pt), C.byref(n))
    if rc != PLORA_OK:
        return rc, None
    return rc, np.ctypeslib.as_array(pt, shape=(n.value,)).copy() if n.value else np.empty(0, np.int32)


def plora_compact(pool, stream=None, max_pages=0):
    """-> (status, pages moved, adapters moved)."""
    pages, adapters = _u32(0), _u32(0)
    rc = lib.plora_compact(pool, stream, max_pages, C.byref(pages), C.byref(adapters))
    return rc, pages.value, adapters.value


def plora_batch_begin(pool, tok2adapter, stream=None):
    """tok2adapter: host int32 array. -> (status, batch handle)."""
    t2a = np.ascontiguousarray(tok2adapter, dtype=np.int32)
    b = C.c_void_p()
    rc = lib.plora_batch_begin(pool, t2a.ctypes.data_as(C.c_void_p), len(t2a), stream, C.byref(b))
    return rc, b


def plora_batch_info(batch):
    """-> (status, perm, seg_adapter, seg_start) as numpy copies."""
    ns, npm = C.c_int32(0), C.c_int32(0)
    perm, sa, ss = C.POINTER(C.c_int32)(), C.POINTER(C.c_int32)(), C.POINTER(C.c_int32)()
    rc = lib.plora_batch_info(batch, C.byref(ns), C.byref(npm), C.byref(perm), C.byref(sa), C.byref(ss))
    if rc:
        return rc, None, None, None

    def arr(p, n):
        return np.ctypeslib.as_array(p, shape=(n,)).copy() if n else np.zeros(0, np.int32)
    return rc, arr(perm, npm.value), arr(sa, ns.value), arr(ss, ns.value + 1)


def plora_shrink(pool, batch, slot0, n_slots, x_ptrs, v_ptrs, stream=None):
    return lib.plora_shrink(pool, batch, slot0, n_slots, _ptr_array(x_ptrs), _ptr_array(v_ptrs), stream)


def plora_expand(pool, batch, slot0, n_slots, v_ptrs, y_ptrs, stream=None):
    return lib.plora_expand(pool, batch, slot0, n_slots, _ptr_array(v_ptrs), _ptr_array(y_ptrs), stream)


def plora_delta(pool, batch, slot0, n_slots, x_ptrs, v_ptrs, y_ptrs, stream=None):
    return lib.plora_delta(pool, batch, slot0, n_slots, _ptr_array(x_ptrs), _ptr_array(v_ptrs), _ptr_array(y_ptrs), stream)


def plora_delta_static(pool, batch, slot0, n_slots, x_ptrs, y_ptrs, stream=None):
    return lib.plora_delta_static(pool, batch, slot0, n_slots, _ptr_array(x_ptrs), _ptr_array(y_ptrs), stream)


def plora_batch_end(pool, batch):
    return lib.plora_batch_end(pool, batch)


def plora_pool_stats(pool):
    """-> (status, dict)."""
    st = _Stats()
    rc = lib.plora_pool_stats(pool, C.byref(st))
    return rc, {k: getattr(st, k) for k, _ in _Stats._fields_}


def plora_pool_set_option(pool, key, value):
    return lib.plora_pool_set_option(pool, key.encode(), int(value))


def plora_profile(pool, enable):
    return lib.plora_profile(pool, int(enable))


def plora_profile_read(pool):
    """-> (status, ms[3], launches[3]) for the shrink kernels, the expand kernels and the one-launch form."""
    ms = (C.c_double * 3)()
    n = (C.c_uint64 * 3)()
    rc = lib.plora_profile_read(pool, ms, n)
    return rc, list(ms), list(n)


def plora_probe_stream(w_bytes, y_bytes, w_tile, y_tile, iters, stream=None):
    """-> (status, ms per launch)."""
    ms = C.c_double(0.0)
    rc = lib.plora_probe_stream(w_bytes, y_bytes, w_tile, y_tile, iters, stream, C.byref(ms))
    return rc, ms.value


def plora_probe_h2d(nbytes, iters, stream=None):
    """-> (status, ms per copy)."""
    ms = C.c_double(0.0)
    rc = lib.plora_probe_h2d(nbytes, iters, stream, C.byref(ms))
    return rc, ms.value


def plora_last_hip():
    return lib.plora_last_hip()


def plora_version():
    return lib.plora_version()


class PloraError(RuntimeError):
    def __init__(self, call, code):
        extra = " (hipError %d)" % plora_last_hip() if code == PLORA_ERR_HIP else ""
        super().__init__("%s -> %s%s" % (call, _STATUS.get(code, code), extra))
        self.code = code


def _check(call, rc):
    if rc < 0:
        raise PloraError(call, rc)
    return rc


class PagedLoraPool:
    """Raises on errors, keeps host blobs and pointer arrays alive; no arithmetic of its own."""

    def __init__(self, page_bytes, n_pages, d_in, d_out, dtype, max_adapters, max_rank, slab=None,
                 placement_only=False):
        self.d_in, self.d_out = list(d_in), list(d_out)
        self.dtype, self.max_rank, self.max_adapters = dtype, max_rank, max_adapters
        self.page_bytes, self.n_pages = page_bytes, n_pages
        self._slab = slab  # a torch tensor, kept alive
        rc, self.h = plora_pool_create(page_bytes, n_pages, d_in, d_out, dtype, max_adapters, max_rank,
                                       None if slab is None else slab.data_ptr(),
                                       PLORA_POOL_PLACEMENT_ONLY if placement_only else 0)
        _check("plora_pool_create", rc)
        self._blobs = {}

    def close(self):
        if self.h:
            _check("plora_pool_destroy", plora_pool_destroy(self.h))
            self.h = None

    def adapter_bytes(self, rank):
        return plora_adapter_bytes(self.h, rank)

    def load(self, aid, rank, scale, pinned_blob=None, copy_stream=None):
        """pinned_blob: page-locked torch tensor (or None for a placement-only pool)."""
        ptr = None if pinned_blob is None else pinned_blob.data_ptr()
        rc, pt = plora_load_adapter(self.h, aid, rank, scale, ptr, copy_stream)
        _check("plora_load_adapter", rc)
        self._blobs[aid] = pinned_blob
        return pt

    def ready(self, aid):
        return _check("plora_adapter_ready", plora_adapter_ready(self.h, aid)) == 1

    def wait(self, aid, stream=None):
        _check("plora_wait_adapter", plora_wait_adapter(self.h, aid, stream))

    def evict(self, aid):
        _check("plora_evict", plora_evict(self.h, aid))
        self._blobs.pop(aid, None)

    def page_table(self, aid):
        rc, pt = plora_adapter_pages(self.h, aid)
        _check("plora_adapter_pages", rc)
        return pt

    def compact(self, stream=None, max_pages=0):
        rc, pages, adapters = plora_compact(self.h, stream, max_pages)
        _check("plora_compact", rc)
        return pages, adapters

    def batch_begin(self, tok2adapter, stream=None):
        rc, b = plora_batch_begin(self.h, tok2adapter, stream)
        _check("plora_batch_begin", rc)
        return b

    def batch_info(self, batch):
        rc, perm, sa, ss = plora_batch_info(batch)
        _check("plora_batch_info", rc)
        return perm, sa, ss

    def shrink(self, batch, slot0, x_tensors, v_tensors, stream=None):
        _check("plora_shrink", plora_shrink(self.h, batch, slot0, len(x_tensors), [t.data_ptr() for t in x_tensors],
                                            [t.data_ptr() for t in v_tensors], stream))

    def expand(self, batch, slot0, v_tensors, y_tensors, stream=None):
        _check("plora_expand", plora_expand(self.h, batch, slot0, len(y_tensors), [t.data_ptr() for t in v_tensors],
                                            [t.data_ptr() for t in y_tensors], stream))

    def delta(self, batch, slot0, x_tensors, v_tensors, y_tensors, stream=None):
        _check("plora_delta", plora_delta(self.h, batch, slot0, len(x_tensors), [t.data_ptr() for t in x_tensors],
                                          [t.data_ptr() for t in v_tensors], [t.data_ptr() for t in y_tensors], stream))

    def delta_static(self, batch, slot0, x_tensors, y_tensors, stream=None):
        _check("plora_delta_static", plora_delta_static(self.h, batch, slot0, len(x_tensors), [t.data_ptr() for t in x_tensors],
                                                        [t.data_ptr() for t in y_tensors], stream))

    def batch_end(self, batch):
        _check("plora_batch_end", plora_batch_end(self.h, batch))

    def stats(self):
        rc, st = plora_pool_stats(self.h)
        _check("plora_pool_stats", rc)
        return st

    def profile(self, enable):
        _check("plora_profile", plora_profile(self.h, enable))

    def profile_read(self):
        rc, ms, n = plora_profile_read(self.h)
        _check("plora_profile_read", rc)
        return ms, n

    def set_option(self, key, value):
        _check("plora_pool_set_option", plora_pool_set_option(self.h, key, value))


# ---------------------------------------------------------------------------------------------
# traffic predictor (host only)
# ---------------------------------------------------------------------------------------------
def plora_predictor_create(n_adapters, window=8, hidden=64, layers=2, replay=10000, batch=64, lr=1e-3, beta1=0.9,
                           beta2=0.999, eps=1e-8, seed=0):
    cfg = _PredictorConfig(n_adapters, window, hidden, layers, replay, batch, lr, beta1, beta2, eps, seed)
    out = C.c_void_p()
    rc = lib.plora_predictor_create(C.byref(cfg), C.byref(out))
    return rc, out.value


def plora_predictor_destroy(pred):
    return lib.plora_predictor_destroy(pred)


def plora_predictor_observe(pred, ids):
    a = np.ascontiguousarray(ids, dtype=np.int32)
    return lib.plora_predictor_observe(pred, a.ctypes.data, len(a))


def plora_predictor_observed(pred):
    return lib.plora_predictor_observed(pred)


def plora_predictor_predict(pred, n_adapters):
    out = np.empty(n_adapters, np.float32)
    rc = lib.plora_predictor_predict(pred, out.ctypes.data)
    return rc, out


def plora_predictor_train(pred, steps):
    loss = C.c_float()
    rc = lib.plora_predictor_train(pred, steps, C.byref(loss))
    return rc, loss.value


def plora_predictor_train_batch(pred, target_pos):
    a = np.ascontiguousarray(target_pos, dtype=np.int32)
    loss = C.c_float()
    rc = lib.plora_predictor_train_batch(pred, a.ctypes.data, len(a), C.byref(loss))
    return rc, loss.value


def plora_predictor_set_threads(pred, threads):
    return lib.plora_predictor_set_threads(pred, threads)


def plora_predictor_param_count(pred):
    return lib.plora_predictor_param_count(pred)


def plora_predictor_get_params(pred):
    out = np.empty(lib.plora_predictor_param_count(pred), np.float32)
    rc = lib.plora_predictor_get_params(pred, out.ctypes.data)
    return rc, out


def plora_predictor_set_params(pred, params):
    a = np.ascontiguousarray(params, dtype=np.float32)
    if a.size != lib.plora_predictor_param_count(pred):
        return PLORA_ERR_INVAL
    return lib.plora_predictor_set_params(pred, a.ctypes.data)


def plora_predictor_loss_grad(pred, seq, target, want_grad=True):
    s = np.ascontiguousarray(seq, dtype=np.float32)
    t = np.ascontiguousarray(target, dtype=np.float32)
    loss = C.c_float()
    grad = np.empty(lib.plora_predictor_param_count(pred), np.float32) if want_grad else None
    rc = lib.plora_predictor_loss_grad(pred, s.ctypes.data, t.ctypes.data, C.byref(loss), None if grad is None else grad.ctypes.data)
    return rc, loss.value, grad


class LstmPredictor:
    """The library's predictor behind the interface the prefetch manager expects: predict(ids of the
    coming interval) returns p_hat computed from the intervals seen so far, and only then records the
    coming interval's requests (they become history once the interval is over) and trains."""

    def __init__(self, n_adapters, window=8, hidden=64, layers=2, replay=10000, batch=64, lr=1e-3, seed=0,
                 train_steps=1, threads=1):
        self.n, self.train_steps = int(n_adapters), int(train_steps)
        rc, self.h = plora_predictor_create(n_adapters, window, hidden, layers, replay, batch, lr, seed=seed)
        _check("plora_predictor_create", rc)
        _check("plora_predictor_set_threads", plora_predictor_set_threads(self.h, threads))
        self.last_loss = None

    def predict(self, next_interval_ids):
        rc, p_hat = plora_predictor_predict(self.h, self.n)
        _check("plora_predictor_predict", rc)
        _check("plora_predictor_observe", plora_predictor_observe(self.h, next_interval_ids))
        if self.train_steps:
            rc, self.last_loss = plora_predictor_train(self.h, self.train_steps)
            _check("plora_predictor_train", rc)
        return p_hat

    def close(self):
        if self.h:
            plora_predictor_destroy(self.h)
            self.h = None


# ---------------------------------------------------------------------------------------------
# residency policy (host only)
# ---------------------------------------------------------------------------------------------
def plora_manager_create(pool, n_adapters, alpha=0.4, beta=0.3, gamma=0.3, theta=0.5, window=1000):
    cfg = _ManagerConfig(alpha, beta, gamma, theta, window)
    out = C.c_void_p()
    rc = lib.plora_manager_create(pool, n_adapters, C.byref(cfg), C.byref(out))
    return rc, out.value


def plora_manager_destroy(mgr):
    return lib.plora_manager_destroy(mgr)


def plora_manager_set_adapter(mgr, aid, rank, scale, pinned_host_ptr=None):
    return lib.plora_manager_set_adapter(mgr, aid, rank, scale, pinned_host_ptr)


def plora_manager_set_prediction(mgr, p_hat):
    if p_hat is None:
        return lib.plora_manager_set_prediction(mgr, None)
    a = np.ascontiguousarray(p_hat, dtype=np.float32)
    return lib.plora_manager_set_prediction(mgr, a.ctypes.data)


def plora_manager_request(mgr, aid, copy_stream=None):
    """-> (status, hit)."""
    hit = C.c_int32(0)
    rc = lib.plora_manager_request(mgr, aid, copy_stream, C.byref(hit))
    return rc, hit.value


def plora_manager_prefetch(mgr, p_hat, prefetch_stream=None):
    """-> (status, number of loads started)."""
    a = np.ascontiguousarray(p_hat, dtype=np.float32)
    n = C.c_int32(0)
    rc = lib.plora_manager_prefetch(mgr, a.ctypes.data, prefetch_stream, C.byref(n))
    return rc, n.value


def plora_manager_residents(mgr):
    n = C.c_int32(0)
    rc = lib.plora_manager_residents(mgr, None, 0, C.byref(n))
    ids = np.empty(n.value, np.int32)
    if rc == 0 and n.value:
        rc = lib.plora_manager_residents(mgr, ids.ctypes.data, n.value, C.byref(n))
    return rc, ids


def plora_manager_scores(mgr):
    """-> (status, ids ascending, scores)."""
    n = C.c_int32(0)
    rc = lib.plora_manager_scores(mgr, None, None, 0, C.byref(n))
    ids, sc = np.empty(n.value, np.int32), np.empty(n.value, np.float64)
    if rc == 0 and n.value:
        rc = lib.plora_manager_scores(mgr, ids.ctypes.data, sc.ctypes.data, n.value, C.byref(n))
    return rc, ids, sc


def plora_manager_state(mgr, aid):
    return lib.plora_manager_state(mgr, aid)


def plora_manager_get_stats(mgr):
    st = _ManagerStats()
    rc = lib.plora_manager_get_stats(mgr, C.byref(st))
    return rc, {k: getattr(st, k) for k, _ in _ManagerStats._fields_}


def plora_manager_log(mgr, clear=False):
    """-> (status, int32 array of (kind, id) pairs; kind 0 = load, 1 = evict)."""
    n = C.c_int64(0)
    rc = lib.plora_manager_log(mgr, None, 0, C.byref(n), 0)
    out = np.empty((n.value, 2), np.int32)
    if rc == 0:
        rc = lib.plora_manager_log(mgr, out.ctypes.data if n.value else None, n.value, C.byref(n), int(clear))
    return rc, out


class ResidencyManager:
    """The library's residency policy (load on demand, eviction by score, threshold prefetching) with
    errors raised; no arithmetic of its own."""

    def __init__(self, pool, ranks, scales, blob_of=None, alpha=0.4, beta=0.3, gamma=0.3, theta=0.5, window=1000,
                 copy_stream=None, prefetch_stream=None):
        """pool: PagedLoraPool; ranks / scales: per adapter id; blob_of(id) -> page-locked torch tensor (None for
        a placement-only pool)."""
        self.pool, self.theta = pool, theta
        self.copy_stream, self.prefetch_stream = copy_stream, prefetch_stream
        rc, self.h = plora_manager_create(pool.h, len(ranks), alpha, beta, gamma, theta, window)
        _check("plora_manager_create", rc)
        self._blobs = []
        for i, (r, sc) in enumerate(zip(ranks, scales)):
            blob = blob_of(i) if blob_of is not None else None
            self._blobs.append(blob)
            _check("plora_manager_set_adapter", plora_manager_set_adapter(self.h, i, int(r), float(sc), None if blob is None else blob.data_ptr()))

    def close(self):
        if self.h:
            plora_manager_destroy(self.h)
            self.h = None

    def request(self, aid):
        rc, hit = plora_manager_request(self.h, int(aid), self.copy_stream)
        _check("plora_manager_request", rc)
        return bool(hit)

    def prefetch(self, p_hat):
        rc, n = plora_manager_prefetch(self.h, p_hat, self.prefetch_stream)
        _check("plora_manager_prefetch", rc)
        return n

    def set_prediction(self, p_hat):
        _check("plora_manager_set_prediction", plora_manager_set_prediction(self.h, p_hat))

    def residents(self):
        rc, ids = plora_manager_residents(self.h)
        _check("plora_manager_residents", rc)
        return ids

    def scores(self):
        rc, ids, sc = plora_manager_scores(self.h)
        _check("plora_manager_scores", rc)
        return dict(zip(ids.tolist(), sc.tolist()))

    def state(self, aid):
        return _check("plora_manager_state", plora_manager_state(self.h, int(aid)))

    def stats(self):
        rc, st = plora_manager_get_stats(self.h)
        _check("plora_manager_get_stats", rc)
        return st

    def log(self, clear=False):
        rc, a = plora_manager_log(self.h, clear)
        _check("plora_manager_log", rc)
        return [tuple(x) for x in a.tolist()]


def plora_suggest_page_bytes(d_in, d_out, dtype, ranks, weights, max_internal_frag=0.02, min_page=4096, max_page=2 << 20):
    """-> (status, page_bytes, expected internal fragmentation at that page size)."""
    di = np.ascontiguousarray(d_in, dtype=np.int32)
    do = np.ascontiguousarray(d_out, dtype=np.int32)
    lay = _Layout(len(di), di.ctypes.data_as(C.POINTER(C.c_int32)), do.ctypes.data_as(C.POINTER(C.c_int32)), dtype, 1, 1)
    r = np.ascontiguousarray(ranks, dtype=np.int32)
    w = np.ascontiguousarray(weights, dtype=np.float64)
    if len(r) != len(w):
        return PLORA_ERR_INVAL, 0, 0.0
    page, frag = C.c_size_t(0), C.c_double(0.0)
    rc = lib.plora_suggest_page_bytes(C.byref(lay), r.ctypes.data, w.ctypes.data, len(r), max_internal_frag, min_page, max_page,
                                      C.byref(page), C.byref(frag))
    return rc, page.value, frag.value


# ---------------------------------------------------------------------------------------------
# rotary positions, the paged 4-bit KV cache, attention
# ---------------------------------------------------------------------------------------------
class RowsStruct(C.Structure):
    """plora_rows; strides in elements."""
    _fields_ = [("data", _vp), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class RotaryStruct(C.Structure):
    _fields_ = [("table", _vp), ("max_pos", _i32), ("rot_dim", _i32), ("interleaved", _i32)]


class RotaryConfig(C.Structure):
    """plora_rotary_config."""
    _fields_ = [(k, C.c_double) for k in ("base", "factor", "low", "high", "magnitude")] + [("scaling", _i32), ("original_len", _i32)]

    def __init__(self, base=10000.0, factor=1.0, low=0.0, high=0.0, magnitude=1.0, scaling=PLORA_ROTARY_NONE, original_len=0):
        super().__init__(base, factor, low, high, magnitude, scaling, original_len)


class KvCacheStruct(C.Structure):
    _fields_ = [(k, _i32) for k in ("dtype", "n_kv_heads", "head_dim", "page_tokens", "n_pages")] + [("pages", _vp)]


class KvBatchStruct(C.Structure):
    _fields_ = [(k, _i32) for k in ("n_seqs", "n_tokens", "max_new", "max_len", "table_stride")] + [
        (k, _vp) for k in ("tok_start", "kv_len", "page_table", "positions")]


_rows_p, _rotary_p, _cache_p, _batch_p = C.POINTER(RowsStruct), C.POINTER(RotaryStruct), C.POINTER(KvCacheStruct), C.POINTER(KvBatchStruct)
lib.plora_rotary_table.argtypes = [C.POINTER(RotaryConfig), _i32, _i32, _vp, _vp]
lib.plora_rotate.argtypes = [_rotary_p, _i32, _i32, _i32, _i32, _vp, _rows_p, _rows_p, _i32, _vp]
lib.plora_kv_page_bytes.argtypes = [_cache_p]
lib.plora_kv_page_bytes.restype = _u64
lib.plora_kv_append.argtypes = [_cache_p, _batch_p, _rows_p, _rows_p, _rotary_p, _vp]
lib.plora_kv_read.argtypes = [_cache_p, _batch_p, _rows_p, _rows_p, _vp]
lib.plora_kv_attend.argtypes = [_cache_p, _batch_p, _i32, _rows_p, _rows_p, _f32, _i32, _i32, _rotary_p, _vp, _u64, _vp]


def plora_rotary_table(config, rot_dim, max_pos, table_ptr, stream=None):
    return lib.plora_rotary_table(C.byref(config), rot_dim, max_pos, table_ptr, stream)


def plora_rotate(rotary, dtype, n_tokens, n_heads, head_dim, positions_ptr, x, y, inverse=0, stream=None):
    """rotary: RotaryStruct; x, y: RowsStruct."""
    return lib.plora_rotate(rotary, dtype, n_tokens, n_heads, head_dim, positions_ptr, x, y, int(inverse), stream)


def plora_kv_page_bytes(cache):
    return lib.plora_kv_page_bytes(cache)


def plora_kv_append(cache, batch, k, v, rotary=None, stream=None):
    """cache: KvCacheStruct, batch: KvBatchStruct, k, v: RowsStruct, rotary: RotaryStruct or None."""
    return lib.plora_kv_append(cache, batch, k, v, rotary, stream)


def plora_kv_read(cache, batch, k, v, stream=None):
    return lib.plora_kv_read(cache, batch, k, v, stream)


def plora_kv_attend(cache, batch, n_heads, q, out, scale, causal=1, window=0, rotary=None, workspace_ptr=None, workspace_bytes=0, stream=None):
    return lib.plora_kv_attend(cache, batch, n_heads, q, out, scale, int(causal), int(window), rotary, workspace_ptr, workspace_bytes, stream)


_INT32 = 100
_DTYPE_NAMES = {"torch.float16": PLORA_F16, "torch.bfloat16": PLORA_BF16, "torch.float32": PLORA_F32, "torch.int32": _INT32}
_dtypes = {}  # torch dtype object -> plora_dtype, _INT32, or -1 for others (filled as they are met: this module does without torch)


def _dtype_of(t):
    d = t.dtype
    code = _dtypes.get(d)
    if code is None:
        code = _dtypes[d] = _DTYPE_NAMES.get(str(d), -1)
    return code


def _device():
    """The GPU that this thread's kernels run on: these calls have no pool that would know theirs."""
    global _device
    _device = sys.modules["torch"].cuda.current_device  # (from now on; torch is there, for its tensors are)
    return _device()


def _rows_of(call, t, n_tokens, heads, head_dim, dtype, device):
    """plora_rows of a torch tensor [tokens, heads, head_dim] (any strides the library takes, the last one 1)."""
    st = t.stride()
    if t.shape != (n_tokens, heads, head_dim) or st[2] != 1 or _dtype_of(t) != dtype or t.get_device() != device:
        raise PloraError(call, PLORA_ERR_INVAL)
    return RowsStruct(t.data_ptr(), st[0], st[1])


def _ints_of(call, t, least, device):
    """Device pointer of a contiguous int32 torch tensor of at least that many entries."""
    if _dtype_of(t) != _INT32 or not t.is_contiguous() or t.numel() < least or t.get_device() != device:
        raise PloraError(call, PLORA_ERR_INVAL)
    return t.data_ptr()


def _three(call, t):
    if t.dim() != 3:
        raise PloraError(call, PLORA_ERR_INVAL)
    return t.shape


# Rotary, KvBatch and PagedKvCache take torch tensors, all of the GPU that is torch's current one at the call (others are refused: the
# kernels would run elsewhere).  stream: a hipStream_t as a number; None is the null stream, not torch's current one, so a program
# that works on a stream of its own passes torch.cuda.current_stream().cuda_stream.
class Rotary:
    """A table of angles (torch float32 tensor [positions, rot_dim/2, 2] on the GPU) and how a head is rotated by it."""

    def __init__(self, table, rot_dim, interleaved=False):
        if str(table.dtype) != "torch.float32" or not table.is_contiguous() or table.dim() != 3 or table.shape[1] * 2 != rot_dim or \
                table.shape[2] != 2 or not table.is_cuda:
            raise PloraError("Rotary", PLORA_ERR_INVAL)
        self.table = table  # kept alive
        self.device = table.get_device()
        self.c = RotaryStruct(table.data_ptr(), table.shape[0], rot_dim, int(interleaved))

    @classmethod
    def make(cls, table, config=None, interleaved=False, stream=None):
        """Fills `table` by `config` (a RotaryConfig) first."""
        if table.dim() != 3:
            raise PloraError("Rotary", PLORA_ERR_INVAL)
        out = cls(table, table.shape[1] * 2, interleaved)
        if out.device != _device():
            raise PloraError("plora_rotary_table", PLORA_ERR_INVAL)
        _check("plora_rotary_table", plora_rotary_table(config or RotaryConfig(), out.c.rot_dim, out.c.max_pos, table.data_ptr(), stream))
        return out

    def rotate(self, positions, x, out, inverse=False, stream=None):
        """out = x [tokens, heads, head_dim] rotated by positions (int32 [tokens]); out may be x."""
        call = "plora_rotate"
        device = _device()
        if self.device != device:
            raise PloraError(call, PLORA_ERR_INVAL)
        n, heads, d = _three(call, x)
        dtype = _dtype_of(x)
        rows = _rows_of(call, x, n, heads, d, dtype, device)
        rc = lib.plora_rotate(self.c, dtype, n, heads, d, _ints_of(call, positions, n, device), rows,
                              rows if out is x else _rows_of(call, out, n, heads, d, dtype, device), inverse, stream)
        if rc:
            _check("plora_rotate", rc)
        return out


class KvBatch:
    """The sequences of a step (int32 tensors on the GPU): tok_start [n + 1], kv_len [n], page_table [n, columns], positions
    [n_tokens] or None; max_new / max_len: most tokens of a sequence in this step / in the cache."""

    def __init__(self, tok_start, kv_len, page_table, n_tokens, max_new, max_len, positions=None):
        n = kv_len.numel()
        call = "KvBatch"
        if page_table.dim() != 2 or page_table.shape[0] != n:
            raise PloraError(call, PLORA_ERR_INVAL)
        self.kept = (tok_start, kv_len, page_table, positions)
        self.n_tokens = n_tokens
        self.device = dev = kv_len.get_device()
        if dev < 0:  # not on a GPU
            raise PloraError(call, PLORA_ERR_INVAL)
        self.c = KvBatchStruct(n, n_tokens, max_new, max_len, page_table.shape[1], _ints_of(call, tok_start, n + 1, dev), _ints_of(call, kv_len, n, dev),
                               _ints_of(call, page_table, n, dev), None if positions is None else _ints_of(call, positions, n_tokens, dev))


class PagedKvCache:
    """One layer's keys and values in 4 bits, on pages of a caller's tensor (uint8 [pages, page bytes] on the GPU)."""

    def __init__(self, dtype, n_kv_heads, head_dim, page_tokens, pages):
        if pages.dim() != 2:
            raise PloraError("PagedKvCache", PLORA_ERR_INVAL)
        self.pages = pages  # kept alive
        self.device = pages.get_device()
        self.dtype, self.heads, self.head_dim = dtype, n_kv_heads, head_dim
        self.c = KvCacheStruct(dtype, n_kv_heads, head_dim, page_tokens, pages.shape[0], pages.data_ptr())
        page = plora_kv_page_bytes(self.c)
        if not page or pages.shape[1] != page or not pages.is_contiguous() or str(pages.dtype) != "torch.uint8" or not pages.is_cuda:
            raise PloraError("PagedKvCache", PLORA_ERR_INVAL)

    @staticmethod
    def page_bytes(n_kv_heads, head_dim, page_tokens):
        return plora_kv_page_bytes(KvCacheStruct(PLORA_F16, n_kv_heads, head_dim, page_tokens, 1, None))

    def _rows(self, call, batch, t, device):
        return _rows_of(call, t, batch.n_tokens, self.heads, self.head_dim, self.dtype, device)

    def append(self, batch, k, v, rotary=None, stream=None):
        """k, v: [tokens, kv heads, head_dim]; rotary: applied to k."""
        call = "plora_kv_append"
        device = _device()
        if self.device != device or batch.device != device or (rotary is not None and rotary.device != device):
            raise PloraError(call, PLORA_ERR_INVAL)
        rc = lib.plora_kv_append(self.c, batch.c, self._rows(call, batch, k, device), self._rows(call, batch, v, device),
                                 None if rotary is None else rotary.c, stream)
        if rc:
            _check(call, rc)

    def read(self, batch, k, v, stream=None):
        call = "plora_kv_read"
        device = _device()
        if self.device != device or batch.device != device:
            raise PloraError(call, PLORA_ERR_INVAL)
        rc = lib.plora_kv_read(self.c, batch.c, self._rows(call, batch, k, device), self._rows(call, batch, v, device), stream)
        if rc:
            _check(call, rc)

    def attend(self, batch, q, out, scale, workspace=None, causal=True, window=0, rotary=None, stream=None):
        """q, out: [tokens, heads, head_dim]; workspace: any contiguous tensor on the GPU, or None; rotary: applied to q."""
        call = "plora_kv_attend"
        device = _device()
        if self.device != device or batch.device != device or (rotary is not None and rotary.device != device):
            raise PloraError(call, PLORA_ERR_INVAL)
        n, heads, d = _three(call, q)
        if d != self.head_dim or n != batch.n_tokens:
            raise PloraError(call, PLORA_ERR_INVAL)
        ws, size = None, 0
        if workspace is not None:
            if not workspace.is_contiguous() or workspace.get_device() != device:
                raise PloraError(call, PLORA_ERR_INVAL)
            size = workspace.nbytes
            ws = workspace.data_ptr() if size else None
        rc = lib.plora_kv_attend(self.c, batch.c, heads, _rows_of(call, q, n, heads, d, self.dtype, device),
                                 _rows_of(call, out, n, heads, d, self.dtype, device), scale,
                                 causal, window, None if rotary is None else rotary.c, ws, size, stream)
        if rc:
            _check(call, rc)
        return out


# ---------------------------------------------------------------------------------------------
# the base layer: norms between blocks, rows and weights in 8 bits, their products, routing
# ---------------------------------------------------------------------------------------------
class MatrixStruct(C.Structure):
    """plora_matrix; stride in elements."""
    _fields_ = [("data", _vp), ("stride", C.c_int64)]


class Fp8RowsStruct(C.Structure):
    _fields_ = [("codes", _vp), ("scales", _vp), ("code_stride", C.c_int64), ("scale_stride", C.c_int64)]


class Fp8WeightsStruct(C.Structure):
    _fields_ = [("n_experts", _i32), ("n", _i32), ("k", _i32), ("codes", _vp), ("scales", _vp)]


class NormWeightsStruct(C.Structure):
    _fields_ = [("weight", _vp), ("bias", _vp), ("eps", _f32), ("offset", _f32), ("center", _i32)]


_matrix_p, _fp8_rows_p, _fp8_weights_p = (C.POINTER(t) for t in (MatrixStruct, Fp8RowsStruct, Fp8WeightsStruct))


class BlockNormStruct(C.Structure):
    """plora_block_norm; its matrices' fields one by one."""
    _fields_ = [("dtype", _i32), ("n_tokens", _i32), ("dim", _i32), ("scale", _f32), ("block", _vp), ("block_stride", C.c_int64), ("places", _vp),
                ("place_weights", _vp), ("top_k", _i32), ("n_block_rows", _i32), ("post", _vp), ("pre", _vp)] + [
                    f for m in ("gate", "residual", "hidden", "out") for f in ((m, _vp), (m + "_stride", C.c_int64))] + [
                        ("codes", _vp), ("scales", _vp), ("code_stride", C.c_int64), ("scale_stride", C.c_int64)]


lib.plora_norm.argtypes = [C.POINTER(BlockNormStruct), _vp]
lib.plora_fp8_quantise.argtypes = [_i32, _i32, _i32, _matrix_p, _i32, _fp8_rows_p, _vp]
lib.plora_fp8_quantise_weights.argtypes = [_i32, _matrix_p, _fp8_weights_p, _vp]
lib.plora_fp8_matmul.argtypes = [_fp8_rows_p, _fp8_weights_p, _i32, _i32, _matrix_p, _vp]
lib.plora_fp8_grouped.argtypes = [_fp8_rows_p, _i32, _fp8_weights_p, _vp, _vp, _i32, _i32, _matrix_p, _vp]
lib.plora_fp8_tile_of.argtypes = [_fp8_rows_p, _i32, _fp8_weights_p, _i32, _i32, _i32, _i32, _vp]
lib.plora_route.argtypes = [_i32, _i32, _i32, _i32, _matrix_p, _i32, _f32, _vp, _vp, _vp, _vp, _vp, _vp, _u64, _vp]
lib.plora_route_workspace_bytes.argtypes = [_i32, _i32]
lib.plora_route_workspace_bytes.restype = _u64


def plora_norm(args, stream=None):
    """args: BlockNormStruct."""
    return lib.plora_norm(args, stream)


def plora_fp8_quantise(dtype, n_rows, k, x, activation, out, stream=None):
    """x: MatrixStruct, out: Fp8RowsStruct."""
    return lib.plora_fp8_quantise(dtype, n_rows, k, x, activation, out, stream)


def plora_fp8_quantise_weights(dtype, w, out, stream=None):
    """w: MatrixStruct, out: Fp8WeightsStruct."""
    return lib.plora_fp8_quantise_weights(dtype, w, out, stream)


def plora_fp8_matmul(x, w, dtype, n_rows, out, stream=None):
    """x: Fp8RowsStruct, w: Fp8WeightsStruct, out: MatrixStruct."""
    return lib.plora_fp8_matmul(x, w, dtype, n_rows, out, stream)


def plora_fp8_grouped(x, n_x_rows, w, offsets_ptr, rows_ptr, dtype, n_rows, out, stream=None):
    return lib.plora_fp8_grouped(x, n_x_rows, w, offsets_ptr, rows_ptr, dtype, n_rows, out, stream)


def plora_fp8_tile_of(x, n_x_rows, w, dtype, n_rows, grouped=False, gathered=False):
    """-> (status, (rows, channels, parts)) of the kernel that the product of these sizes runs on; x: Fp8RowsStruct, w: Fp8WeightsStruct."""
    tile = (_i32 * 3)()
    rc = lib.plora_fp8_tile_of(x, n_x_rows, w, dtype, n_rows, int(grouped), int(gathered), tile)
    return rc, tuple(tile)


def plora_route_workspace_bytes(n_tokens, n_experts):
    return lib.plora_route_workspace_bytes(n_tokens, n_experts)


def plora_route(dtype, n_tokens, n_experts, top_k, logits, renormalise, scale, experts_ptr, weights_ptr, offsets_ptr, rows_ptr, places_ptr,
                workspace_ptr=None, workspace_bytes=0, stream=None):
    """logits: MatrixStruct."""
    return lib.plora_route(dtype, n_tokens, n_experts, top_k, logits, int(renormalise), scale, experts_ptr, weights_ptr, offsets_ptr, rows_ptr, places_ptr,
                           workspace_ptr, workspace_bytes, stream)


_ELEMENTS = (PLORA_F16, PLORA_BF16, PLORA_F32)
_EIGHT = ("torch.float8_e4m3fn", "torch.uint8")
_NO_ROWS = (None, None, 0, 0)
_MOST = 0x7fffffff  # the library's counts have 32 bits; ctypes would take larger ones modulo 2^32


def _place_of(call, t, n_rows, width, dtype, device):
    """(pointer, row stride) of a torch tensor [rows, width] (a row's elements one behind the other)."""
    if t.shape != (n_rows, width) or _dtype_of(t) != dtype or t.get_device() != device:
        raise PloraError(call, PLORA_ERR_INVAL)
    row, element = t.stride()
    if element != 1 and width > 1:
        raise PloraError(call, PLORA_ERR_INVAL)
    return t.data_ptr(), row if n_rows > 1 else -(-width // 8) * 8  # (one row may have any stride)


def _matrix_of(call, t, n_rows, width, dtype, device):
    """plora_matrix of such a tensor."""
    return MatrixStruct(*_place_of(call, t, n_rows, width, dtype, device))


def _two(call, t):
    if t.dim() != 2:
        raise PloraError(call, PLORA_ERR_INVAL)
    a, b = t.shape
    if a > _MOST or b > _MOST:
        raise PloraError(call, PLORA_ERR_LIMIT)
    return a, b


# The classes below take torch tensors as those above do: all of the GPU that is torch's current one at the call; stream None is the null stream.
class Fp8Rows:
    """Rows of k values in 8 bits: codes [rows, k] (float8_e4m3fn, or uint8 with the same bytes) and scales [ceil(k / 128), rows] (float32)."""

    def __init__(self, codes, scales):
        call = "Fp8Rows"
        n, k = _two(call, codes)
        blocks, rows = _two(call, scales)
        self.device = codes.get_device()
        if self.device < 0 or scales.get_device() != self.device or str(codes.dtype) not in _EIGHT or str(scales.dtype) != "torch.float32" or rows != n or \
                blocks != -(-k // 128) or (k > 1 and codes.stride(1) != 1) or (n > 1 and scales.stride(1) != 1):
            raise PloraError(call, PLORA_ERR_INVAL)
        self.codes, self.scales = codes, scales  # kept alive
        self.n, self.k = n, k
        # (a tensor of one row or one block may have any stride there)
        self.fields = (codes.data_ptr(), scales.data_ptr(), codes.stride(0) if n > 1 else -(-k // 16) * 16, scales.stride(0) if blocks > 1 else n)
        self.c = Fp8RowsStruct(*self.fields)

    def quantise(self, x, activation=PLORA_ACT_NONE, stream=None):
        """Becomes x [rows, k]; with an activation x is [rows, 2k], the gate's half first."""
        call = "plora_fp8_quantise"
        device = _device()
        dtype = _dtype_of(x)
        if self.device != device or dtype not in _ELEMENTS:
            raise PloraError(call, PLORA_ERR_INVAL)
        rc = lib.plora_fp8_quantise(dtype, self.n, self.k, _matrix_of(call, x, self.n, self.k if activation == PLORA_ACT_NONE else 2 * self.k, dtype, device),
                                    activation, self.c, stream)
        if rc:
            _check(call, rc)
        return self


class Fp8Weights:
    """Weights in 8 bits: codes [n, k], or [experts, n, k] for grouped products, and scales [.., ceil(n / 128), ceil(k / 128)], contiguous."""

    def __init__(self, codes, scales):
        call = "Fp8Weights"
        if codes.dim() not in (2, 3) or scales.dim() != codes.dim():
            raise PloraError(call, PLORA_ERR_INVAL)
        n, k = codes.shape[-2:]
        experts = codes.shape[0] if codes.dim() == 3 else 1
        if max(codes.shape) > _MOST:
            raise PloraError(call, PLORA_ERR_LIMIT)
        self.device = codes.get_device()
        if self.device < 0 or scales.get_device() != self.device or str(codes.dtype) not in _EIGHT or str(scales.dtype) != "torch.float32" or \
                scales.shape != (*codes.shape[:-2], -(-n // 128), -(-k // 128)) or not codes.is_contiguous() or not scales.is_contiguous():
            raise PloraError(call, PLORA_ERR_INVAL)
        self.codes, self.scales = codes, scales  # kept alive
        self.n, self.k = n, k
        self.c = Fp8WeightsStruct(experts, n, k, codes.data_ptr(), scales.data_ptr())

    def quantise(self, w, stream=None):
        """Becomes w, of the codes' shape and contiguous."""
        call = "plora_fp8_quantise_weights"
        dtype = _dtype_of(w)
        if self.device != _device() or w.get_device() != self.device or dtype not in _ELEMENTS or w.shape != self.codes.shape or not w.is_contiguous():
            raise PloraError(call, PLORA_ERR_INVAL)
        rc = lib.plora_fp8_quantise_weights(dtype, MatrixStruct(w.data_ptr(), self.k), self.c, stream)
        if rc:
            _check(call, rc)
        return self

    def matmul(self, x, out, stream=None):
        """out [rows, n] = x (Fp8Rows) times the weights."""
        call = "plora_fp8_matmul"
        device = _device()
        dtype = _dtype_of(out)
        if self.device != device or x.device != device or x.k != self.k or dtype not in _ELEMENTS:
            raise PloraError(call, PLORA_ERR_INVAL)
        rc = lib.plora_fp8_matmul(x.c, self.c, dtype, x.n, _matrix_of(call, out, x.n, self.n, dtype, device), stream)
        if rc:
            _check(call, rc)
        return out

    def grouped(self, x, offsets, out, rows=None, stream=None):
        """Out rows offsets[e] .. offsets[e + 1] - 1 = their x rows times expert e's weights; rows (int32): the x row of every out row."""
        call = "plora_fp8_grouped"
        device = _device()
        dtype = _dtype_of(out)
        if self.device != device or x.device != device or x.k != self.k or dtype not in _ELEMENTS:
            raise PloraError(call, PLORA_ERR_INVAL)
        n = _two(call, out)[0]
        rc = lib.plora_fp8_grouped(x.c, x.n, self.c, _ints_of(call, offsets, self.c.n_experts + 1, device),
                                   None if rows is None else _ints_of(call, rows, n, device), dtype, n,
                                   _matrix_of(call, out, n, self.n, dtype, device), stream)
        if rc:
            _check(call, rc)
        return out


class Routing:
    """What routing writes (int32 tensors but for weights, float32; contiguous, on the GPU): experts, weights and places [tokens, top_k],
    offsets [n_experts + 1], rows [tokens * top_k]; workspace: a contiguous tensor of at least workspace_bytes(tokens, n_experts), or None."""

    def __init__(self, experts, weights, offsets, rows, places, workspace=None):
        call = "Routing"
        n, k = _two(call, experts)
        self.device = dev = offsets.get_device()
        if dev < 0 or str(weights.dtype) != "torch.float32" or not weights.is_contiguous() or weights.get_device() != dev or weights.shape != (n, k) or \
                places.shape != (n, k) or (workspace is not None and (not workspace.is_contiguous() or workspace.get_device() != dev)):
            raise PloraError(call, PLORA_ERR_INVAL)
        self.experts, self.weights, self.offsets, self.rows, self.places, self.workspace = experts, weights, offsets, rows, places, workspace
        self.n, self.k, self.n_experts = n, k, offsets.numel() - 1
        if self.n_experts > _MOST:
            raise PloraError(call, PLORA_ERR_LIMIT)
        size = 0 if workspace is None else workspace.nbytes
        self.at = (_ints_of(call, experts, n * k, dev), weights.data_ptr(), _ints_of(call, offsets, 2, dev), _ints_of(call, rows, n * k, dev),
                   _ints_of(call, places, n * k, dev), workspace.data_ptr() if size else None, size)

    @staticmethod
    def workspace_bytes(n_tokens, n_experts):
        return plora_route_workspace_bytes(n_tokens, n_experts)

    def route(self, logits, renormalise=True, scale=1.0, stream=None):
        """Chooses by logits [tokens, n_experts] and sorts."""
        call = "plora_route"
        device = _device()
        dtype = _dtype_of(logits)
        if self.device != device or dtype not in _ELEMENTS:
            raise PloraError(call, PLORA_ERR_INVAL)
        rc = lib.plora_route(dtype, self.n, self.n_experts, self.k, _matrix_of(call, logits, self.n, self.n_experts, dtype, device), int(renormalise), scale,
                             *self.at, stream)
        if rc:
            _check(call, rc)
        return self


class NormWeights:
    """A norm's parameters: weight and bias [dim] (or None), eps; center: the mean is taken off first; offset: added to the weight."""

    def __init__(self, weight=None, bias=None, eps=1e-6, center=False, offset=0.0):
        call = "NormWeights"
        self.kept = [t for t in (weight, bias) if t is not None]
        for t in self.kept:
            if t.dim() != 1 or not t.is_contiguous() or t.get_device() < 0 or t.shape != self.kept[0].shape or t.dtype != self.kept[0].dtype or \
                    t.get_device() != self.kept[0].get_device():
                raise PloraError(call, PLORA_ERR_INVAL)
        self.c = NormWeightsStruct(None if weight is None else weight.data_ptr(), None if bias is None else bias.data_ptr(), eps, offset, int(center))
        self.at = C.addressof(self.c)
        self.of = (self.kept[0].numel(), _dtype_of(self.kept[0]), self.kept[0].get_device()) if self.kept else None

    def fits(self, dim, dtype, device):
        return self.of is None or self.of == (dim, dtype, device)


class BlockNorm:
    """What lies between two blocks: hidden = residual + scale * gate * post(block), result = pre(hidden); pre, post: NormWeights or None."""

    def __init__(self, pre=None, post=None, scale=1.0):
        self.pre, self.post, self.scale = pre, post, scale

    def run(self, block, residual=None, hidden=None, out=None, out8=None, gate=None, places=None, place_weights=None, stream=None):
        """block, residual, hidden, out, gate: [tokens, dim]; gate may be [dim], one for all tokens; out8: Fp8Rows in place of out.
        places (int32 [tokens, top_k], as Routing has them) and place_weights: block's rows are the experts', and a token takes the weighted sum of its own."""
        call = "plora_norm"
        device = _device()
        dtype = _dtype_of(block)
        rows, dim = _two(call, block)
        n, top_k, block_rows, at, weights_at = rows, 0, 0, None, None
        if places is not None:
            n, top_k = _two(call, places)
            block_rows, at = rows, _ints_of(call, places, n * top_k, device)
            if place_weights is None or place_weights.shape != (n, top_k) or str(place_weights.dtype) != "torch.float32" or \
                    not place_weights.is_contiguous() or place_weights.get_device() != device:
                raise PloraError(call, PLORA_ERR_INVAL)
            weights_at = place_weights.data_ptr()
        elif place_weights is not None:
            raise PloraError(call, PLORA_ERR_INVAL)
        pre, post = self.pre, self.post
        if dtype not in _ELEMENTS or (pre is not None and not pre.fits(dim, dtype, device)) or (post is not None and not post.fits(dim, dtype, device)) or \
                (out8 is not None and (out8.device != device or out8.n != n or out8.k != dim)):
            raise PloraError(call, PLORA_ERR_INVAL)
        if gate is not None and gate.dim() == 1:
            if gate.shape[0] != dim:
                raise PloraError(call, PLORA_ERR_INVAL)
            gate = gate.expand(n, dim)
        b, bs = _place_of(call, block, rows, dim, dtype, device)
        g, gs = (None, 0) if gate is None else _place_of(call, gate, n, dim, dtype, device)
        r, rs = (None, 0) if residual is None else _place_of(call, residual, n, dim, dtype, device)
        h, hs = (None, 0) if hidden is None else _place_of(call, hidden, n, dim, dtype, device)
        o, os_ = (None, 0) if out is None else _place_of(call, out, n, dim, dtype, device)
        c, s, cs, ss = _NO_ROWS if out8 is None else out8.fields
        args = BlockNormStruct(dtype, n, dim, self.scale, b, bs, at, weights_at, top_k, block_rows, None if post is None else post.at,
                               None if pre is None else pre.at, g, gs, r, rs, h, hs, o, os_, c, s, cs, ss)
        rc = lib.plora_norm(args, stream)
        if rc:
            _check(call, rc)
