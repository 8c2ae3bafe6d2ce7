"""Thin ctypes binding of libstca.so (the C ABI in include/stca.h).

Argument marshalling only: torch tensors supply device memory and the stream;
every step of the computation runs in the library's HIP kernels.  There is no
fallback: if the library is missing, loading it raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libstca.so")

STCA_OK, STCA_ERR_INVALID_ARG, STCA_ERR_UNSUPPORTED, STCA_ERR_WORKSPACE, STCA_ERR_HIP = 0, -1, -2, -3, -4
STCA_ERR_RANGE = -5
STCA_F32, STCA_BF16 = 0, 1
# execution forms (stca_dims_t.kv_form / attn_form / bwd_form); 0 = automatic
STCA_KV_AUTO, STCA_KV_FUSED, STCA_KV_MATERIALIZE = 0, 1, 2
STCA_ATTN_AUTO, STCA_ATTN_STANDARD, STCA_ATTN_REORDERED = 0, 1, 2
STCA_BWD_AUTO, STCA_BWD_FUSED, STCA_BWD_GENERIC, STCA_BWD_REORDERED = 0, 1, 2, 3
FORMS = {
    "kv": {"auto": STCA_KV_AUTO, "fused": STCA_KV_FUSED, "materialize": STCA_KV_MATERIALIZE},
    "attn": {"auto": STCA_ATTN_AUTO, "standard": STCA_ATTN_STANDARD, "reordered": STCA_ATTN_REORDERED},
    "bwd": {"auto": STCA_BWD_AUTO, "fused": STCA_BWD_FUSED, "generic": STCA_BWD_GENERIC,
            "reordered": STCA_BWD_REORDERED},
}

EXPORTED = ("stca_workspace_size", "stca_saved_size", "stca_saved_layout", "stca_forward", "stca_backward",
            "stca_device_status", "stca_status_string", "stca_path", "stca_forward_launch_count",
            "stca_forward_profiled", "stca_backward_launch_count", "stca_backward_profiled",
            "stca_sl_beta", "stca_sl_sample", "stca_sl_allocate", "stca_sl_pack",
            "stca_paper_workspace_size", "stca_paper_saved_size", "stca_paper_saved_layout", "stca_forward_paper",
            "stca_paper_launch_count", "stca_forward_paper_profiled", "stca_train_record_size", "stca_forward_train",
            "stca_backward_record", "stca_forward_noalloc", "stca_attn_workspace_size", "stca_attn_saved_size",
            "stca_attn_saved_layout", "stca_attn_forward", "stca_attn_backward", "stca_bias_edges",
            "stca_cache_write", "stca_cache_read", "stca_cache_attn_workspace_size", "stca_cache_attn")
STCA_CACHE_BF16, STCA_CACHE_INT8 = 0, 1
CACHE_WS_BYTES = 256  # STCA_CACHE_WS_BYTES
NOALLOC_SCRATCH_BYTES = 256 << 20  # STCA_NOALLOC_SCRATCH_BYTES
PAPER_WEIGHT_FIELDS = ("ffn_u", "ffn_v", "ffn_o", "wq", "wk", "wv", "wo", "wc", "wz", "z_u", "z_v", "z_o")


class stca_dims_t(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("ffn_hidden", ctypes.c_int32), ("dtype", ctypes.c_int32), ("kv_form", ctypes.c_int32),
                ("attn_form", ctypes.c_int32), ("bwd_form", ctypes.c_int32), ("chunk_blocks", ctypes.c_int32)]


class stca_batch_t(ctypes.Structure):
    _fields_ = [("n_requests", ctypes.c_int32), ("n_hist", ctypes.c_int64), ("n_tgt", ctypes.c_int64),
                ("hist_off", ctypes.c_void_p), ("tgt_off", ctypes.c_void_p),
                ("hist_off_host", ctypes.c_void_p), ("tgt_off_host", ctypes.c_void_p)]


class stca_weights_t(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("wq", "wk", "wv", "wo", "w1", "w2")]


class stca_wgrads_t(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("dwq", "dwk", "dwv", "dwo", "dw1", "dw2")]


class stca_saved_layout_t(ctypes.Structure):
    _fields_ = [(k, ctypes.c_size_t) for k in ("s", "a", "u", "lse", "total")]


class stca_paper_weights_t(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in PAPER_WEIGHT_FIELDS]


class stca_paper_saved_layout_t(ctypes.Structure):
    _fields_ = [(k, ctypes.c_size_t) for k in ("q", "a", "o", "lse", "xt", "total")]


class stca_attn_t(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("d_head", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("softcap", ctypes.c_float),
                ("masked", ctypes.c_int32), ("n_buckets", ctypes.c_int32), ("edges_host", ctypes.c_void_p)]


class stca_attn_in_t(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("ldq", ctypes.c_int64),
                ("ldk", ctypes.c_int64), ("ldv", ctypes.c_int64), ("tgt_pos", ctypes.c_void_p),
                ("hist_pos", ctypes.c_void_p), ("bias", ctypes.c_void_p)]


class stca_attn_grads_t(ctypes.Structure):
    _fields_ = [("dq", ctypes.c_void_p), ("dk", ctypes.c_void_p), ("dv", ctypes.c_void_p), ("lddq", ctypes.c_int64),
                ("lddk", ctypes.c_int64), ("lddv", ctypes.c_int64), ("dbias", ctypes.c_void_p)]


class stca_attn_saved_layout_t(ctypes.Structure):
    _fields_ = [(k, ctypes.c_size_t) for k in ("a", "max", "sum", "total")]


class stca_cache_t(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("d_head", ctypes.c_int32), ("format", ctypes.c_int32), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("pos", ctypes.c_void_p)]


class stca_cache_rows_t(ctypes.Structure):
    _fields_ = [("n_requests", ctypes.c_int32), ("n_rows", ctypes.c_int64), ("row_off", ctypes.c_void_p),
                ("start", ctypes.c_void_p), ("table", ctypes.c_void_p), ("table_ld", ctypes.c_int32)]


class stca_cache_batch_t(ctypes.Structure):
    _fields_ = [("n_requests", ctypes.c_int32), ("n_tgt", ctypes.c_int64), ("tgt_off", ctypes.c_void_p),
                ("tgt_off_host", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("max_len", ctypes.c_int32),
                ("table", ctypes.c_void_p), ("table_ld", ctypes.c_int32)]


class StcaError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {status_string(status)} ({status})")
        self.status = status


_lib = None


def lib():
    """Load libstca.so (built in-tree by paper_2511_06077_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2511_06077_amd.build`")
        # torch ships its own HIP runtime (soname libamdhip64.so.7, needed by
        # torch as libamdhip64.so): load it first so that libstca binds to the
        # same runtime instead of pulling in a second copy.
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.POINTER
        L.stca_workspace_size.restype = ctypes.c_size_t
        L.stca_workspace_size.argtypes = [P(stca_dims_t), P(stca_batch_t), ctypes.c_int]
        L.stca_saved_size.restype = ctypes.c_size_t
        L.stca_saved_size.argtypes = [P(stca_dims_t), P(stca_batch_t)]
        L.stca_saved_layout.restype = ctypes.c_int
        L.stca_saved_layout.argtypes = [P(stca_dims_t), P(stca_batch_t), P(stca_saved_layout_t)]
        L.stca_forward.restype = ctypes.c_int
        L.stca_forward.argtypes = [P(stca_dims_t), P(stca_batch_t), ctypes.c_void_p, ctypes.c_void_p,
                                   P(stca_weights_t), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                   ctypes.c_size_t, ctypes.c_void_p]
        L.stca_backward.restype = ctypes.c_int
        L.stca_backward.argtypes = [P(stca_dims_t), P(stca_batch_t), ctypes.c_void_p, ctypes.c_void_p,
                                    P(stca_weights_t), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                    P(stca_wgrads_t), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
        L.stca_device_status.restype = ctypes.c_int
        L.stca_device_status.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
        L.stca_status_string.restype = ctypes.c_char_p
        L.stca_status_string.argtypes = [ctypes.c_int]
        L.stca_path.restype = ctypes.c_int
        L.stca_path.argtypes = [P(stca_dims_t)]
        L.stca_forward_launch_count.restype = ctypes.c_int
        L.stca_forward_launch_count.argtypes = [P(stca_dims_t), P(stca_batch_t)]
        L.stca_forward_profiled.restype = ctypes.c_int
        L.stca_forward_profiled.argtypes = [P(stca_dims_t), P(stca_batch_t), ctypes.c_void_p, ctypes.c_void_p,
                                            P(stca_weights_t), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                            ctypes.c_size_t, ctypes.c_void_p, P(ctypes.c_void_p), ctypes.c_int,
                                            P(ctypes.c_char_p)]
        L.stca_backward_launch_count.restype = ctypes.c_int
        L.stca_backward_launch_count.argtypes = [P(stca_dims_t), P(stca_batch_t)]
        L.stca_backward_profiled.restype = ctypes.c_int
        L.stca_backward_profiled.argtypes = [P(stca_dims_t), P(stca_batch_t), ctypes.c_void_p, ctypes.c_void_p,
                                             P(stca_weights_t), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                             P(stca_wgrads_t), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                                             P(ctypes.c_void_p), ctypes.c_int, P(ctypes.c_char_p)]
        L.stca_train_record_size.restype = ctypes.c_size_t
        L.stca_train_record_size.argtypes = [P(stca_dims_t), P(stca_batch_t)]
        L.stca_forward_train.restype = ctypes.c_int
        L.stca_forward_train.argtypes = [P(stca_dims_t), P(stca_batch_t), ctypes.c_void_p, ctypes.c_void_p,
                                         P(stca_weights_t), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_size_t, ctypes.c_void_p]
        L.stca_backward_record.restype = ctypes.c_int
        L.stca_backward_record.argtypes = [P(stca_dims_t), P(stca_batch_t), ctypes.c_void_p, ctypes.c_void_p,
                                           P(stca_weights_t), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                           ctypes.c_void_p, P(stca_wgrads_t), ctypes.c_void_p, ctypes.c_size_t,
                                           ctypes.c_void_p]
        L.stca_forward_noalloc.restype = ctypes.c_int
        L.stca_forward_noalloc.argtypes = [P(stca_dims_t), P(stca_batch_t), ctypes.c_void_p, ctypes.c_void_p,
                                           P(stca_weights_t), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        I32P = P(ctypes.c_int32)
        L.stca_sl_beta.restype = ctypes.c_double
        L.stca_sl_beta.argtypes = [ctypes.c_double, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        L.stca_sl_sample.restype = ctypes.c_int
        L.stca_sl_sample.argtypes = [ctypes.c_uint64, ctypes.c_int32, ctypes.c_double, ctypes.c_int32, ctypes.c_int32,
                                     ctypes.c_int32, P(ctypes.c_double), I32P]
        L.stca_sl_allocate.restype = ctypes.c_int
        L.stca_sl_allocate.argtypes = [ctypes.c_int32, I32P, I32P, ctypes.c_int64, I32P]
        L.stca_sl_pack.restype = ctypes.c_int
        L.stca_sl_pack.argtypes = [ctypes.c_int32, I32P, I32P, I32P, I32P]
        L.stca_paper_workspace_size.restype = ctypes.c_size_t
        L.stca_paper_workspace_size.argtypes = [P(stca_dims_t), P(stca_batch_t)]
        L.stca_paper_saved_size.restype = ctypes.c_size_t
        L.stca_paper_saved_size.argtypes = [P(stca_dims_t), P(stca_batch_t)]
        L.stca_paper_saved_layout.restype = ctypes.c_int
        L.stca_paper_saved_layout.argtypes = [P(stca_dims_t), P(stca_batch_t), P(stca_paper_saved_layout_t)]
        L.stca_forward_paper.restype = ctypes.c_int
        L.stca_forward_paper.argtypes = [P(stca_dims_t), P(stca_batch_t), ctypes.c_void_p, ctypes.c_void_p,
                                         P(stca_paper_weights_t), ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_size_t, ctypes.c_void_p]
        L.stca_paper_launch_count.restype = ctypes.c_int
        L.stca_paper_launch_count.argtypes = [P(stca_dims_t), P(stca_batch_t)]
        L.stca_forward_paper_profiled.restype = ctypes.c_int
        L.stca_forward_paper_profiled.argtypes = [P(stca_dims_t), P(stca_batch_t), ctypes.c_void_p, ctypes.c_void_p,
                                                  P(stca_paper_weights_t), ctypes.c_void_p, ctypes.c_void_p,
                                                  ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                                                  P(ctypes.c_void_p), ctypes.c_int, P(ctypes.c_char_p)]
        V, SZ, I64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64
        A, B = P(stca_attn_t), P(stca_batch_t)
        for name, res, args in (
                ("stca_attn_workspace_size", SZ, [A, B, ctypes.c_int]),
                ("stca_attn_saved_size", SZ, [A, B]),
                ("stca_attn_saved_layout", ctypes.c_int, [A, B, P(stca_attn_saved_layout_t)]),
                ("stca_attn_forward", ctypes.c_int, [A, B, P(stca_attn_in_t), V, V, V, SZ, V]),
                ("stca_attn_backward", ctypes.c_int, [A, B, P(stca_attn_in_t), V, V, P(stca_attn_grads_t), V, SZ, V]),
                ("stca_bias_edges", ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, I32P]),
                ("stca_cache_write", ctypes.c_int,
                 [P(stca_cache_t), P(stca_cache_rows_t), ctypes.c_int32, V, V, I64, I64, V, V, V]),
                ("stca_cache_read", ctypes.c_int,
                 [P(stca_cache_t), P(stca_cache_rows_t), ctypes.c_int32, V, V, I64, I64, V, V, V]),
                ("stca_cache_attn_workspace_size", SZ, [A, P(stca_cache_t), P(stca_cache_batch_t)]),
                ("stca_cache_attn", ctypes.c_int,
                 [A, P(stca_cache_t), P(stca_cache_batch_t), V, I64, V, V, V, V, SZ, V])):
            getattr(L, name).restype, getattr(L, name).argtypes = res, args
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().stca_status_string(int(status)).decode()


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def dims(d_model: int, n_heads: int, n_layers: int, ffn_hidden: int, dtype: int, kv: str = "auto",
         attn: str = "auto", bwd: str = "auto", chunk_blocks: int = 0) -> stca_dims_t:
    """Model shape and execution forms (names as in FORMS; chunk_blocks 0 =
    automatic)."""
    return stca_dims_t(d_model, n_heads, n_layers, ffn_hidden, dtype, FORMS["kv"][kv], FORMS["attn"][attn],
                       FORMS["bwd"][bwd], chunk_blocks)


def batch(n_requests: int, n_hist: int, n_tgt: int, hist_off, tgt_off, hist_off_host=None,
          tgt_off_host=None) -> stca_batch_t:
    """hist_off / tgt_off: device int32 tensors; *_host: optional contiguous
    int32 numpy arrays (kept alive by the caller)."""
    def host(a):
        return None if a is None else a.ctypes.data
    return stca_batch_t(n_requests, n_hist, n_tgt, _ptr(hist_off), _ptr(tgt_off), host(hist_off_host),
                        host(tgt_off_host))


def weights(wq, wk, wv, wo, w1, w2) -> stca_weights_t:
    return stca_weights_t(*(_ptr(t) for t in (wq, wk, wv, wo, w1, w2)))


def wgrads(dwq, dwk, dwv, dwo, dw1, dw2) -> stca_wgrads_t:
    return stca_wgrads_t(*(_ptr(t) for t in (dwq, dwk, dwv, dwo, dw1, dw2)))


def stca_path(d: stca_dims_t) -> int:
    return lib().stca_path(ctypes.byref(d))


def stca_workspace_size(d: stca_dims_t, b: stca_batch_t, with_backward: bool = False) -> int:
    return lib().stca_workspace_size(ctypes.byref(d), ctypes.byref(b), int(with_backward))


def stca_saved_size(d: stca_dims_t, b: stca_batch_t) -> int:
    return lib().stca_saved_size(ctypes.byref(d), ctypes.byref(b))


def stca_saved_layout(d: stca_dims_t, b: stca_batch_t) -> stca_saved_layout_t:
    out = stca_saved_layout_t()
    st = lib().stca_saved_layout(ctypes.byref(d), ctypes.byref(b), ctypes.byref(out))
    if st != STCA_OK:
        raise StcaError(st, "stca_saved_layout")
    return out


def stca_forward(d, b, hist, tgt, w, out, saved, ws, ws_bytes: int, stream=None, check: bool = True) -> int:
    st = lib().stca_forward(ctypes.byref(d), ctypes.byref(b), _ptr(hist), _ptr(tgt), ctypes.byref(w), _ptr(out),
                            _ptr(saved), _ptr(ws), int(ws_bytes), _ptr(stream))
    if check and st != STCA_OK:
        raise StcaError(st, "stca_forward")
    return st


def stca_backward(d, b, hist, tgt, w, dout, dhist, dtgt, dw, ws, ws_bytes: int, stream=None,
                  check: bool = True) -> int:
    st = lib().stca_backward(ctypes.byref(d), ctypes.byref(b), _ptr(hist), _ptr(tgt), ctypes.byref(w),
                             _ptr(dout), _ptr(dhist), _ptr(dtgt), ctypes.byref(dw), _ptr(ws), int(ws_bytes),
                             _ptr(stream))
    if check and st != STCA_OK:
        raise StcaError(st, "stca_backward")
    return st


def stca_forward_noalloc(d, b, hist, tgt, w, out, saved, stream=None, check: bool = True) -> int:
    """stca_forward with the library's own per-GPU scratch array as the
    workspace (no workspace argument, nothing allocated)."""
    st = lib().stca_forward_noalloc(ctypes.byref(d), ctypes.byref(b), _ptr(hist), _ptr(tgt), ctypes.byref(w),
                                    _ptr(out), _ptr(saved), _ptr(stream))
    if check and st != STCA_OK:
        raise StcaError(st, "stca_forward_noalloc")
    return st


def stca_train_record_size(d: stca_dims_t, b: stca_batch_t) -> int:
    return lib().stca_train_record_size(ctypes.byref(d), ctypes.byref(b))


def stca_forward_train(d, b, hist, tgt, w, out, record, ws, ws_bytes: int, stream=None, check: bool = True) -> int:
    st = lib().stca_forward_train(ctypes.byref(d), ctypes.byref(b), _ptr(hist), _ptr(tgt), ctypes.byref(w),
                                  _ptr(out), _ptr(record), _ptr(ws), int(ws_bytes), _ptr(stream))
    if check and st != STCA_OK:
        raise StcaError(st, "stca_forward_train")
    return st


def stca_backward_record(d, b, hist, tgt, w, record, dout, dhist, dtgt, dw, ws, ws_bytes: int, stream=None,
                         check: bool = True) -> int:
    st = lib().stca_backward_record(ctypes.byref(d), ctypes.byref(b), _ptr(hist), _ptr(tgt), ctypes.byref(w),
                                    _ptr(record), _ptr(dout), _ptr(dhist), _ptr(dtgt), ctypes.byref(dw), _ptr(ws),
                                    int(ws_bytes), _ptr(stream))
    if check and st != STCA_OK:
        raise StcaError(st, "stca_backward_record")
    return st


def stca_device_status(ws, stream=None) -> int:
    return lib().stca_device_status(_ptr(ws), _ptr(stream))


def stca_forward_launch_count(d: stca_dims_t, b: stca_batch_t) -> int:
    return lib().stca_forward_launch_count(ctypes.byref(d), ctypes.byref(b))


def stca_forward_profiled(d, b, hist, tgt, w, out, saved, ws, ws_bytes: int, stream, events, labels=None) -> int:
    """events: a ctypes array of hipEvent_t (see HipEvents); labels: optional
    ctypes array of c_char_p receiving kernel names."""
    st = lib().stca_forward_profiled(ctypes.byref(d), ctypes.byref(b), _ptr(hist), _ptr(tgt), ctypes.byref(w),
                                     _ptr(out), _ptr(saved), _ptr(ws), int(ws_bytes), _ptr(stream), events,
                                     len(events), labels)
    if st != STCA_OK:
        raise StcaError(st, "stca_forward_profiled")
    return st


def stca_backward_launch_count(d: stca_dims_t, b: stca_batch_t) -> int:
    return lib().stca_backward_launch_count(ctypes.byref(d), ctypes.byref(b))


def stca_backward_profiled(d, b, hist, tgt, w, dout, dhist, dtgt, dw, ws, ws_bytes: int, stream, events,
                           labels=None) -> int:
    """As stca_backward, with events recorded at phase boundaries (see HipEvents)."""
    st = lib().stca_backward_profiled(ctypes.byref(d), ctypes.byref(b), _ptr(hist), _ptr(tgt), ctypes.byref(w),
                                      _ptr(dout), _ptr(dhist), _ptr(dtgt), ctypes.byref(dw), _ptr(ws), int(ws_bytes),
                                      _ptr(stream), events, len(events), labels)
    if st != STCA_OK:
        raise StcaError(st, "stca_backward_profiled")
    return st


# ---- paper-exact stack
def paper_weights(**w) -> stca_paper_weights_t:
    """Keyword arguments named as PAPER_WEIGHT_FIELDS (wc may be None for one layer)."""
    return stca_paper_weights_t(*(_ptr(w.get(k)) for k in PAPER_WEIGHT_FIELDS))


def stca_paper_workspace_size(d: stca_dims_t, b: stca_batch_t) -> int:
    return lib().stca_paper_workspace_size(ctypes.byref(d), ctypes.byref(b))


def stca_paper_saved_size(d: stca_dims_t, b: stca_batch_t) -> int:
    return lib().stca_paper_saved_size(ctypes.byref(d), ctypes.byref(b))


def stca_paper_saved_layout(d: stca_dims_t, b: stca_batch_t) -> stca_paper_saved_layout_t:
    out = stca_paper_saved_layout_t()
    st = lib().stca_paper_saved_layout(ctypes.byref(d), ctypes.byref(b), ctypes.byref(out))
    if st != STCA_OK:
        raise StcaError(st, "stca_paper_saved_layout")
    return out


def stca_forward_paper(d, b, hist, tgt, w, z, saved, ws, ws_bytes: int, stream=None, check: bool = True) -> int:
    st = lib().stca_forward_paper(ctypes.byref(d), ctypes.byref(b), _ptr(hist), _ptr(tgt), ctypes.byref(w), _ptr(z),
                                  _ptr(saved), _ptr(ws), int(ws_bytes), _ptr(stream))
    if check and st != STCA_OK:
        raise StcaError(st, "stca_forward_paper")
    return st


def stca_paper_launch_count(d: stca_dims_t, b: stca_batch_t) -> int:
    return lib().stca_paper_launch_count(ctypes.byref(d), ctypes.byref(b))


def stca_forward_paper_profiled(d, b, hist, tgt, w, z, saved, ws, ws_bytes: int, stream, events, labels=None) -> int:
    st = lib().stca_forward_paper_profiled(ctypes.byref(d), ctypes.byref(b), _ptr(hist), _ptr(tgt), ctypes.byref(w),
                                           _ptr(z), _ptr(saved), _ptr(ws), int(ws_bytes), _ptr(stream), events,
                                           len(events), labels)
    if st != STCA_OK:
        raise StcaError(st, "stca_forward_paper_profiled")
    return st


# ---- stand-alone attention and paged history cache
def _checked(name: str, check: bool, *args) -> int:
    st = getattr(lib(), name)(*args)
    if check and st != STCA_OK:
        raise StcaError(st, name)
    return st


def attn(n_heads: int, n_kv_heads: int, d_head: int, dtype: int, scale: float, softcap: float = 0.0,
         masked: bool = False, n_buckets: int = 0, edges=None) -> stca_attn_t:
    """edges: contiguous int32 numpy array [n_buckets - 1], kept alive by the caller."""
    return stca_attn_t(n_heads, n_kv_heads, d_head, dtype, scale, softcap, int(masked), n_buckets,
                       None if edges is None else edges.ctypes.data)


def attn_in(q, k, v, ldq: int = 0, ldk: int = 0, ldv: int = 0, tgt_pos=None, hist_pos=None,
            bias=None) -> stca_attn_in_t:
    return stca_attn_in_t(_ptr(q), _ptr(k), _ptr(v), ldq, ldk, ldv, _ptr(tgt_pos), _ptr(hist_pos), _ptr(bias))


def attn_grads(dq, dk, dv, lddq: int = 0, lddk: int = 0, lddv: int = 0, dbias=None) -> stca_attn_grads_t:
    return stca_attn_grads_t(_ptr(dq), _ptr(dk), _ptr(dv), lddq, lddk, lddv, _ptr(dbias))


def cache(n_pages: int, page_size: int, n_kv_heads: int, d_head: int, fmt: int, k, v, k_exp=None, v_exp=None,
          pos=None) -> stca_cache_t:
    return stca_cache_t(n_pages, page_size, n_kv_heads, d_head, fmt, _ptr(k), _ptr(v), _ptr(k_exp), _ptr(v_exp),
                        _ptr(pos))


def cache_rows(n_requests: int, n_rows: int, row_off, start, table, table_ld: int) -> stca_cache_rows_t:
    return stca_cache_rows_t(n_requests, n_rows, _ptr(row_off), _ptr(start), _ptr(table), table_ld)


def cache_batch(n_requests: int, n_tgt: int, tgt_off, lens, max_len: int, table, table_ld: int,
                tgt_off_host=None) -> stca_cache_batch_t:
    """tgt_off_host: optional contiguous int32 numpy array, kept alive by the caller."""
    return stca_cache_batch_t(n_requests, n_tgt, _ptr(tgt_off), None if tgt_off_host is None else
                              tgt_off_host.ctypes.data, _ptr(lens), max_len, _ptr(table), table_ld)


def stca_attn_workspace_size(a: stca_attn_t, b: stca_batch_t, with_backward: bool = False) -> int:
    return lib().stca_attn_workspace_size(ctypes.byref(a), ctypes.byref(b), int(with_backward))


def stca_attn_saved_size(a: stca_attn_t, b: stca_batch_t) -> int:
    return lib().stca_attn_saved_size(ctypes.byref(a), ctypes.byref(b))


def stca_attn_saved_layout(a: stca_attn_t, b: stca_batch_t) -> stca_attn_saved_layout_t:
    out = stca_attn_saved_layout_t()
    _checked("stca_attn_saved_layout", True, ctypes.byref(a), ctypes.byref(b), ctypes.byref(out))
    return out


def stca_attn_forward(a, b, given, out, saved, ws, ws_bytes: int, stream=None, check: bool = True) -> int:
    return _checked("stca_attn_forward", check, ctypes.byref(a), ctypes.byref(b), ctypes.byref(given), _ptr(out),
                    _ptr(saved), _ptr(ws), int(ws_bytes), _ptr(stream))


def stca_attn_backward(a, b, given, saved, dout, grads, ws, ws_bytes: int, stream=None, check: bool = True) -> int:
    return _checked("stca_attn_backward", check, ctypes.byref(a), ctypes.byref(b), ctypes.byref(given), _ptr(saved),
                    _ptr(dout), ctypes.byref(grads), _ptr(ws), int(ws_bytes), _ptr(stream))


def bias_edges(n_buckets: int, n_exact: int, max_distance: int):
    """Edges [n_buckets - 1] (int32): 1 .. n_exact, then a geometric series to max_distance."""
    import numpy as np
    out = np.empty(max(0, n_buckets - 1), dtype=np.int32)
    _checked("stca_bias_edges", True, n_buckets, n_exact, max_distance, _i32p(out))
    return out


def stca_cache_write(c, rows, dtype: int, k, v, ldk: int = 0, ldv: int = 0, pos=None, ws=None, stream=None,
                     check: bool = True) -> int:
    return _checked("stca_cache_write", check, ctypes.byref(c), ctypes.byref(rows), dtype, _ptr(k), _ptr(v), ldk, ldv,
                    _ptr(pos), _ptr(ws), _ptr(stream))


def stca_cache_read(c, rows, dtype: int, k, v, ldk: int = 0, ldv: int = 0, pos=None, ws=None, stream=None,
                    check: bool = True) -> int:
    return _checked("stca_cache_read", check, ctypes.byref(c), ctypes.byref(rows), dtype, _ptr(k), _ptr(v), ldk, ldv,
                    _ptr(pos), _ptr(ws), _ptr(stream))


def stca_cache_attn_workspace_size(a: stca_attn_t, c: stca_cache_t, b: stca_cache_batch_t) -> int:
    return lib().stca_cache_attn_workspace_size(ctypes.byref(a), ctypes.byref(c), ctypes.byref(b))


def stca_cache_attn(a, c, b, q, ldq: int, tgt_pos, bias, out, ws, ws_bytes: int, stream=None,
                    check: bool = True) -> int:
    return _checked("stca_cache_attn", check, ctypes.byref(a), ctypes.byref(c), ctypes.byref(b), _ptr(q), ldq,
                    _ptr(tgt_pos), _ptr(bias), _ptr(out), _ptr(ws), int(ws_bytes), _ptr(stream))


class HipEvents:
    """A set of HIP events created through the HIP runtime (for timing kernels
    on the stream the library launches them on)."""

    def __init__(self, n: int):
        self.hip = ctypes.CDLL("libamdhip64.so")
        self.hip.hipEventCreateWithFlags.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_uint]
        self.hip.hipEventElapsedTime.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.c_void_p, ctypes.c_void_p]
        self.hip.hipEventSynchronize.argtypes = [ctypes.c_void_p]
        self.hip.hipEventDestroy.argtypes = [ctypes.c_void_p]
        self.ev = (ctypes.c_void_p * n)()
        for i in range(n):
            e = ctypes.c_void_p()
            # timing-only events: no system-scope fence (cache writeback and
            # invalidate) when recorded, which would otherwise slow the
            # kernels around every marker
            if self.hip.hipEventCreateWithFlags(ctypes.byref(e), 0x20000000) != 0:  # hipEventDisableSystemFence
                raise RuntimeError("hipEventCreateWithFlags failed")
            self.ev[i] = e
        self.labels = (ctypes.c_char_p * max(1, n - 1))()

    def elapsed_ms(self, i: int, j: int) -> float:
        if self.hip.hipEventSynchronize(self.ev[j]) != 0:
            raise RuntimeError("hipEventSynchronize failed")
        ms = ctypes.c_float()
        if self.hip.hipEventElapsedTime(ctypes.byref(ms), self.ev[i], self.ev[j]) != 0:
            raise RuntimeError("hipEventElapsedTime failed")
        return float(ms.value)

    def label(self, k: int) -> str:
        v = self.labels[k]
        return v.decode() if v else "?"

    def close(self):
        for i in range(len(self.ev)):
            if self.ev[i]:
                self.hip.hipEventDestroy(self.ev[i])
                self.ev[i] = None


# ---- stochastic-length batches (host functions)
def _i32p(a):
    return None if a is None else a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def sl_beta(alpha: float, l_min: int, l_avg: int, l_max: int) -> float:
    return lib().stca_sl_beta(alpha, l_min, l_avg, l_max)


def sl_sample(seed: int, n: int, alpha: float, l_min: int, l_avg: int, l_max: int):
    """(l_raw float64 [n], l_train int32 [n])"""
    import numpy as np
    raw = np.empty(n, dtype=np.float64)
    out = np.empty(n, dtype=np.int32)
    st = lib().stca_sl_sample(seed, n, alpha, l_min, l_avg, l_max,
                              raw.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), _i32p(out))
    if st != STCA_OK:
        raise StcaError(st, "stca_sl_sample")
    return raw, out


def sl_allocate(l_full, l_train, budget: int):
    import numpy as np
    l_full = np.ascontiguousarray(l_full, dtype=np.int32)
    l_train = np.ascontiguousarray(l_train, dtype=np.int32)
    out = np.empty_like(l_full)
    st = lib().stca_sl_allocate(len(l_full), _i32p(l_full), _i32p(l_train), int(budget), _i32p(out))
    if st != STCA_OK:
        raise StcaError(st, "stca_sl_allocate")
    return out


def sl_pack(full_off, l_keep):
    """(hist_off int32 [n+1], src_rows int32 [sum l_keep])"""
    import numpy as np
    full_off = np.ascontiguousarray(full_off, dtype=np.int32)
    l_keep = np.ascontiguousarray(l_keep, dtype=np.int32)
    hoff = np.empty(len(l_keep) + 1, dtype=np.int32)
    src = np.empty(int(l_keep.sum()), dtype=np.int32)
    st = lib().stca_sl_pack(len(l_keep), _i32p(full_off), _i32p(l_keep), _i32p(hoff), _i32p(src))
    if st != STCA_OK:
        raise StcaError(st, "stca_sl_pack")
    return hoff, src
