"""The stand-alone attention and the paged history cache on the GPU: plans that
hold a batch's offsets, workspace and saved buffer, and call the C ABI
(stca_attn_*, stca_cache_*).  Plumbing only, as in device.py: allocation,
checks and pointer marshalling; all computation happens in libstca.so.

    plan = CrossAttention(hist_off, tgt_off, n_heads=8, d_head=32, edges=bias_edges(32, 8, 8192),
                          masked=True, backward=True)
    out = plan.forward(q, k, v, tgt_pos=..., bias=...)
    dq, dk, dv, dbias = plan.backward(dout, q, k, v, tgt_pos=..., bias=...)

    cache = HistoryCache(n_pages=4096, page_size=64, n_kv_heads=8, d_head=32)    # 8 bits
    cache.write(k, v, row_off, start, table)
    serve = CacheAttention(cache, tgt_off, n_heads=8, max_len=10240, edges=..., masked=...)
    out = serve.forward(q, lens, table, tgt_pos=..., bias=...)

A plan's workspace (and what its forward saved) belongs to one stream at a
time: calls, or replays of captured graphs, that may overlap need a plan each.
A forward replaces what the plan's backward reads.  stream= (a handle) is the
stream of a call in place of the current one, as if it were made under
torch.cuda.stream: the inputs have to be ready on it, and results belong to it
(another stream waits for it, and records its use with Tensor.record_stream).
"""
from __future__ import annotations

import math
from typing import Optional

import numpy as np

from . import stca
from .device import launch_on
from .stca import bias_edges  # noqa: F401  (public here too)


def _torch():
    import torch
    return torch


def _dtype_code(dtype):
    torch = _torch()
    if dtype == torch.bfloat16:
        return stca.STCA_BF16
    if dtype == torch.float32:
        return stca.STCA_F32
    raise ValueError(f"dtype {dtype}: bfloat16 or float32")


def _rows(name, t, heads, d_head, dtype, device, n=None):
    """(tensor, row stride) of rows [n][heads][d_head] (or [n][heads * d_head])
    whose heads lie one after the other; rows may be strided."""
    if not hasattr(t, "data_ptr") or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name}: a {dtype} tensor on {device} is needed")
    if t.is_contiguous() and t.shape == (t.shape[0] if n is None else n, heads, d_head):
        return t, 0
    dense = t.numel() == 0  # (no strides to speak of)
    if t.dim() == 3:
        ok = t.shape[1:] == (heads, d_head) and (dense or t.stride(2) == 1 and (heads == 1 or t.stride(1) == d_head))
    else:
        ok = t.dim() == 2 and t.shape[1] == heads * d_head and (dense or t.stride(1) == 1)
    if not ok or (n is not None and t.shape[0] != n):
        raise ValueError(f"{name}: rows [{n}][{heads}][{d_head}] with dense heads are needed, "
                         f"not {tuple(t.shape)} strided {t.stride()}")
    if t.shape[0] <= 1:
        return t, 0
    if t.stride(0) < heads * d_head:
        raise ValueError(f"{name}: rows overlap (stride {t.stride(0)})")
    return t, t.stride(0)


def _flat(name, t, dtype, shape, device):
    if (not hasattr(t, "data_ptr") or t.dtype != dtype or t.device != device or t.shape != shape
            or not t.is_contiguous()):
        raise ValueError(f"{name}: a contiguous {dtype} tensor {tuple(shape)} on {device} is needed")
    return t


def _int32(name, a):
    """a as a contiguous int32 array of the same values."""
    given = np.asarray(a.cpu().numpy() if isinstance(a, _torch().Tensor) else a)
    with np.errstate(invalid="ignore"):
        host = np.ascontiguousarray(given.astype(np.int32))
    if not np.array_equal(host, given):
        raise ValueError(f"{name}: whole numbers of 32 bits are needed")
    return host


def _offsets(off, device):
    torch = _torch()
    host = _int32("offsets", off)
    if host.ndim != 1 or len(host) < 2:
        raise ValueError("offsets: [requests + 1] is needed")
    return host, torch.from_numpy(host.copy()).to(device)


def _device(device):
    torch = _torch()
    d = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if d.type == "cuda" and d.index is None else d


class _Scores:
    """What CrossAttention and CacheAttention share: the scores' form."""

    def _scores(self, n_heads, n_kv_heads, d_head, dtype, scale, softcap, edges, masked):
        self.n_heads, self.n_kv_heads, self.d_head, self.dtype = n_heads, n_kv_heads, d_head, dtype
        self.edges = None if edges is None else _int32("edges", edges)
        if self.edges is not None and self.edges.ndim != 1:
            raise ValueError("edges: one-dimensional")
        self.n_buckets = 0 if self.edges is None else len(self.edges) + 1
        self.masked = bool(masked)
        scale = 1.0 / math.sqrt(d_head) if scale is None else scale
        self.attn = stca.attn(n_heads, n_kv_heads, d_head, _dtype_code(dtype), scale, softcap, masked,
                              self.n_buckets, self.edges)

    def _given(self, tgt_pos, bias, n_tgt):
        torch = _torch()
        if self.masked or self.n_buckets:
            _flat("tgt_pos", tgt_pos, torch.int32, (n_tgt,), self.device)
        if self.n_buckets:
            _flat("bias", bias, torch.float32, (self.n_heads, self.n_buckets), self.device)
        elif bias is not None:
            raise ValueError("bias: given, but the plan has no edges")

    def _workspace(self, nbytes, where):
        if nbytes == 0:
            raise stca.StcaError(stca.STCA_ERR_INVALID_ARG, where)
        self.ws_bytes = nbytes
        return _torch().empty(nbytes, dtype=_torch().uint8, device=self.device)

    def stream(self):
        return _torch().cuda.current_stream(self.device.index).cuda_stream

    def device_status(self, stream: Optional[int] = None) -> int:
        return stca.stca_device_status(self.ws, self.stream() if stream is None else stream)


class CrossAttention(_Scores):
    """Attention of a ragged batch's targets over their request's history:
    capped scores, a learned bias by buckets of distance (edges: int32, see
    bias_edges) and a mask to hist_pos <= tgt_pos; backward=True keeps what the
    gradients need."""

    def __init__(self, hist_off, tgt_off, n_heads: int, d_head: int, *, n_kv_heads: Optional[int] = None, dtype=None,
                 scale: Optional[float] = None, softcap: float = 0.0, edges=None, masked: bool = False,
                 backward: bool = False, device="cuda", host_offsets: bool = True):
        torch = _torch()
        self.device = _device(device)
        self._scores(n_heads, n_kv_heads or n_heads, d_head, dtype or torch.bfloat16, scale, softcap, edges, masked)
        self.hoff_h, self.hoff = _offsets(hist_off, self.device)
        self.toff_h, self.toff = _offsets(tgt_off, self.device)
        if len(self.hoff_h) != len(self.toff_h):
            raise ValueError("hist_off and tgt_off: one entry per request and one more")
        self.n_hist, self.n_tgt = int(self.hoff_h[-1]), int(self.toff_h[-1])
        self.batch = stca.batch(len(self.hoff_h) - 1, self.n_hist, self.n_tgt, self.hoff, self.toff,
                                self.hoff_h if host_offsets else None, self.toff_h if host_offsets else None)
        self.ws = self._workspace(stca.stca_attn_workspace_size(self.attn, self.batch, backward),
                                  "stca_attn_workspace_size")
        self.saved = None
        if backward:
            n = stca.stca_attn_saved_size(self.attn, self.batch)
            self.saved = torch.empty(max(n, 16), dtype=torch.uint8, device=self.device)
        self.has_saved = False

    def _in(self, q, k, v, tgt_pos, hist_pos, bias):
        torch = _torch()
        q, ldq = _rows("q", q, self.n_heads, self.d_head, self.dtype, self.device, self.n_tgt)
        k, ldk = _rows("k", k, self.n_kv_heads, self.d_head, self.dtype, self.device, self.n_hist)
        v, ldv = _rows("v", v, self.n_kv_heads, self.d_head, self.dtype, self.device, self.n_hist)
        self._given(tgt_pos, bias, self.n_tgt)
        if hist_pos is not None:
            _flat("hist_pos", hist_pos, torch.int32, (self.n_hist,), self.device)
        return stca.attn_in(q, k, v, ldq, ldk, ldv, tgt_pos, hist_pos, bias)

    def forward(self, q, k, v, tgt_pos=None, hist_pos=None, bias=None, stream: Optional[int] = None):
        """out [n_tgt][n_heads][d_head]"""
        torch = _torch()
        given = self._in(q, k, v, tgt_pos, hist_pos, bias)
        with launch_on(self.device, stream):
            out = torch.empty((self.n_tgt, self.n_heads, self.d_head), dtype=self.dtype, device=self.device)
            stca.stca_attn_forward(self.attn, self.batch, given, out, self.saved, self.ws, self.ws_bytes,
                                   self.stream() if stream is None else stream)
        self.has_saved = self.saved is not None
        return out

    def backward(self, dout, q, k, v, tgt_pos=None, hist_pos=None, bias=None, stream: Optional[int] = None):
        """(dq, dk, dv, dbias) of sum <dout, out> for the inputs of the last
        forward; dbias is None without edges."""
        torch = _torch()
        if self.saved is None:
            raise ValueError("backward: the plan was made without backward=True")
        if not self.has_saved:
            raise ValueError("backward: no forward before it")
        given = self._in(q, k, v, tgt_pos, hist_pos, bias)
        _flat("dout", dout, self.dtype, (self.n_tgt, self.n_heads, self.d_head), self.device)
        with launch_on(self.device, stream):
            t = dict(dtype=self.dtype, device=self.device)
            dq = torch.empty((self.n_tgt, self.n_heads, self.d_head), **t)
            dk = torch.empty((self.n_hist, self.n_kv_heads, self.d_head), **t)
            dv = torch.empty((self.n_hist, self.n_kv_heads, self.d_head), **t)
            dbias = None
            if self.n_buckets:
                dbias = torch.empty((self.n_heads, self.n_buckets), dtype=torch.float32, device=self.device)
            stca.stca_attn_backward(self.attn, self.batch, given, self.saved, dout,
                                    stca.attn_grads(dq, dk, dv, dbias=dbias), self.ws, self.ws_bytes,
                                    self.stream() if stream is None else stream)
        return dq, dk, dv, dbias


class HistoryCache:
    """Pages of K and V rows, 8-bit ("int8") or bf16 ("bf16"); positions=True
    keeps every row's position beside it.  Pages are handed out by the caller:
    table [requests][..] (int32) lists each request's pages, and its row i is
    slot i % page_size of page table[i // page_size].  Writes to slots of their own
    and reads may overlap on several streams; device_status is then the last one's
    to end.  The pages are cleared on the stream that is current here: other streams
    wait for it before their first write."""

    def __init__(self, n_pages: int, page_size: int, n_kv_heads: int, d_head: int, fmt: str = "int8",
                 positions: bool = False, device="cuda"):
        torch = _torch()
        if fmt not in ("int8", "bf16"):
            raise ValueError(f"fmt {fmt!r}: int8 or bf16")
        self.device = _device(device)
        self.n_pages, self.page_size, self.n_kv_heads, self.d_head, self.fmt = (n_pages, page_size, n_kv_heads,
                                                                                d_head, fmt)
        # zeros, not empty: a page's unwritten slots read as zero
        def pages(*shape, dtype):
            return torch.zeros((n_pages, *shape), dtype=dtype, device=self.device)
        held = torch.int8 if fmt == "int8" else torch.bfloat16
        self.k = pages(n_kv_heads, page_size, d_head, dtype=held)
        self.v = pages(n_kv_heads, d_head, page_size, dtype=held)
        self.k_exp = pages(n_kv_heads, page_size, dtype=torch.uint8) if fmt == "int8" else None
        self.v_exp = pages(n_kv_heads, page_size, dtype=torch.uint8) if fmt == "int8" else None
        self.pos = pages(page_size, dtype=torch.int32) if positions else None
        self.ws = torch.zeros(stca.CACHE_WS_BYTES, dtype=torch.uint8, device=self.device)
        self.cache = stca.cache(n_pages, page_size, n_kv_heads, d_head,
                                stca.STCA_CACHE_INT8 if fmt == "int8" else stca.STCA_CACHE_BF16, self.k, self.v,
                                self.k_exp, self.v_exp, self.pos)

    def _rows(self, row_off, start, table, n_rows):
        torch = _torch()
        R = row_off.shape[0] - 1
        _flat("row_off", row_off, torch.int32, (R + 1,), self.device)
        _flat("start", start, torch.int32, (R,), self.device)
        if table.dim() != 2 or table.shape[0] != R:
            raise ValueError(f"table: [{R}][pages] is needed, not {tuple(table.shape)}")
        _flat("table", table, torch.int32, table.shape, self.device)
        return stca.cache_rows(R, n_rows, row_off, start, table, table.shape[1])

    def stream(self):
        return _torch().cuda.current_stream(self.device.index).cuda_stream

    def device_status(self, stream: Optional[int] = None) -> int:
        """Of the last write or read."""
        return stca.stca_device_status(self.ws, self.stream() if stream is None else stream)

    def write(self, k, v, row_off, start, table, pos=None, stream: Optional[int] = None):
        """Packed rows k, v [n][n_kv_heads][d_head]: request r's rows
        [row_off[r], row_off[r + 1]) become its cache rows from start[r] on."""
        torch = _torch()
        n = k.shape[0]
        k, ldk = _rows("k", k, self.n_kv_heads, self.d_head, k.dtype, self.device, n)
        v, ldv = _rows("v", v, self.n_kv_heads, self.d_head, k.dtype, self.device, n)
        if (pos is not None) != (self.pos is not None):
            raise ValueError("pos: given exactly where the cache keeps positions")
        if pos is not None:
            _flat("pos", pos, torch.int32, (n,), self.device)
        rows = self._rows(row_off, start, table, n)
        with launch_on(self.device, stream):
            stca.stca_cache_write(self.cache, rows, _dtype_code(k.dtype), k, v, ldk, ldv, pos, self.ws,
                                  self.stream() if stream is None else stream)

    def read(self, row_off, start, table, n_rows: int, dtype=None, stream: Optional[int] = None):
        """(k, v) [n_rows][n_kv_heads][d_head], and pos where the cache keeps them.
        Rows without a page are not written, and hold anything (see device_status)."""
        torch = _torch()
        dtype = dtype or torch.bfloat16
        rows = self._rows(row_off, start, table, n_rows)
        with launch_on(self.device, stream):
            k, v = (torch.empty((n_rows, self.n_kv_heads, self.d_head), dtype=dtype, device=self.device)
                    for _ in range(2))
            pos = None if self.pos is None else torch.empty(n_rows, dtype=torch.int32, device=self.device)
            stca.stca_cache_read(self.cache, rows, _dtype_code(dtype), k, v, 0, 0, pos, self.ws,
                                 self.stream() if stream is None else stream)
        return (k, v) if pos is None else (k, v, pos)


class CacheAttention(_Scores):
    """Attention of a batch's new targets over their requests' cached rows.
    tgt_off (host) and max_len fix the plan; the rows in use, lens, and the
    pages, table, are each call's own."""

    def __init__(self, cache: HistoryCache, tgt_off, n_heads: int, max_len: int, *, scale: Optional[float] = None,
                 softcap: float = 0.0, edges=None, masked: bool = False):
        torch = _torch()
        self.cache, self.device, self.max_len = cache, cache.device, int(max_len)
        self._scores(n_heads, cache.n_kv_heads, cache.d_head, torch.bfloat16, scale, softcap, edges, masked)
        self.toff_h, self.toff = _offsets(tgt_off, self.device)
        self.n_requests, self.n_tgt = len(self.toff_h) - 1, int(self.toff_h[-1])
        # (sizes do not depend on where lens and table lie: each call's own are set below)
        self.batch = stca.cache_batch(self.n_requests, self.n_tgt, self.toff, self.toff, self.max_len, self.toff,
                                      -(-self.max_len // cache.page_size), self.toff_h)
        self.ws = self._workspace(stca.stca_cache_attn_workspace_size(self.attn, cache.cache, self.batch),
                                  "stca_cache_attn_workspace_size")

    def forward(self, q, lens, table, tgt_pos=None, bias=None, stream: Optional[int] = None):
        """out [n_tgt][n_heads][d_head] over the first lens[r] rows of each request."""
        torch = _torch()
        q, ldq = _rows("q", q, self.n_heads, self.d_head, self.dtype, self.device, self.n_tgt)
        _flat("lens", lens, torch.int32, (self.n_requests,), self.device)
        if table.dim() != 2 or table.shape[0] != self.n_requests or table.shape[1] * self.cache.page_size < self.max_len:
            raise ValueError(f"table: [{self.n_requests}][pages of {self.max_len} rows] is needed")
        _flat("table", table, torch.int32, table.shape, self.device)
        self._given(tgt_pos, bias, self.n_tgt)
        with launch_on(self.device, stream):
            out = torch.empty((self.n_tgt, self.n_heads, self.d_head), dtype=self.dtype, device=self.device)
            b = self.batch
            b.lens, b.table, b.table_ld = lens.data_ptr(), table.data_ptr(), table.shape[1]
            stca.stca_cache_attn(self.attn, self.cache.cache, b, q, ldq, tgt_pos, bias, out,
                                 self.ws, self.ws_bytes, self.stream() if stream is None else stream)
        return out
