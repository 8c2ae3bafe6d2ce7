"""What stands around the attention in a model, on the GPU: rows from ids and
their tables' gradients, norms around a block with its gate and residual scale,
the norm of all gradients and clipping (stca_embed_*, stca_norm_*, stca_clip).
Plumbing only, as in device.py: allocation, checks and pointer marshalling; all
computation happens in libstca.so.

    embed = EmbeddingSum((n_items, n_actions, n_positions), d, scale=d ** 0.5, dtype=torch.float32)
    hist = embed.forward((items, actions, positions), (item_ids, action_ids, position_ids))

    norm = BlockNorm(d, kind="rms", gate="sigmoid", backward=True)
    _, y = norm.forward(x, pre=(w0,))                                     # in front of the first block
    h, y = norm.forward(x, block=o, gate=g, post=(w1,), layer_scale=s, pre=(w2,))
    grads = norm.backward(dy, x, dh=dh, block=o, gate=g, post=(w1,), layer_scale=s, pre=(w2,))

    table = EmbeddingGradient(n_items, n_hist + n_tgt, d, scale=d ** 0.5)
    rows, values, count = table.sparse([(item_ids, dhist), (target_ids, dtgt)])

    norm = GradientNorm(1.0).clip([dwq, dwk, values], counts=[None, None, count])   # in place

An object's workspace belongs to one stream at a time: calls, or replays of
captured graphs, that may overlap need an object each.  stream= (a handle) is the
stream of a call in place of the current one, as if it were made under
torch.cuda.stream: the inputs have to be ready on it, and so has the object, whose
workspace is made (and cleared, where it holds a status) on the stream that is
current then; results belong to it.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Sequence

from . import stca
from .attention import _device, _dtype_code, _flat, _torch
from .device import launch_on

_KINDS = {"rms": stca.STCA_NORM_RMS, "layer": stca.STCA_NORM_LAYER}
_GATES = {None: stca.STCA_GATE_NONE, "sigmoid": stca.STCA_GATE_SIGMOID, "silu": stca.STCA_GATE_SILU}


def _there(t, device):
    """t lies on `device`.  (get_device is -1 on the host; comparing devices costs a microsecond.)"""
    return t.get_device() == (-1 if device.index is None else device.index)


def _matrix(name, t, d, dtype, device, n=None):
    """(tensor, row stride) of rows [n][d]; rows may be strided."""
    if not hasattr(t, "data_ptr") or t.dtype != dtype or not _there(t, device):
        raise ValueError(f"{name}: a {dtype} tensor on {device} is needed")
    shape = t.shape
    if len(shape) != 2 or shape[1] != d or (n is not None and shape[0] != n):
        raise ValueError(f"{name}: rows [{'n' if n is None else n}][{d}] are needed, not {tuple(shape)}")
    if t.is_contiguous():
        return t, 0
    if t.stride(1) != 1 or (t.shape[0] > 1 and t.stride(0) < d):
        raise ValueError(f"{name}: dense rows that do not overlap are needed, not strides {t.stride()}")
    return (t, t.stride(0)) if t.shape[0] > 1 else (t, 0)


def _vector(name, t, n, dtype, device):
    if not hasattr(t, "data_ptr") or t.dtype != dtype or not _there(t, device) or t.dim() != 1 or not t.is_contiguous() \
            or (n is not None and t.shape[0] != n):
        raise ValueError(f"{name}: a contiguous {dtype} tensor [{'n' if n is None else n}] on {device} is needed")
    return t


def _like(x):
    """Dense rows of x's shape and type."""
    torch = _torch()
    return torch.empty_like(x, memory_format=torch.contiguous_format)


class _Streamed:
    def stream(self):
        return _torch().cuda.current_stream(self.device.index).cuda_stream

    def _at(self, stream):
        return self.stream() if stream is None else stream

    def _on(self, stream):
        """launch_on, for an object whose tensors are the GPU's."""
        if self.device.type != "cuda":
            raise ValueError(f"{self.device}: calls need a GPU")
        return launch_on(self.device, stream)


class EmbeddingSum(_Streamed):
    """Rows from the ids of one or several tables (`rows` of each): their sum, times
    `scale`, in out_dtype.  A negative id is no row."""

    def __init__(self, rows: Sequence[int], d: int, *, scale: float = 1.0, dtype=None, out_dtype=None, device="cuda"):
        torch = _torch()
        self.device = _device(device)
        self.rows = tuple(int(r) for r in ((rows,) if isinstance(rows, int) else rows))
        self.d, self.dtype = int(d), dtype or torch.bfloat16
        self.out_dtype = out_dtype or torch.bfloat16
        if not 1 <= len(self.rows) <= stca.EMBED_FIELDS:
            raise ValueError(f"rows: 1 to {stca.EMBED_FIELDS} tables")
        self.embed = stca.embed(self.d, _dtype_code(self.dtype), _dtype_code(self.out_dtype), float(scale))
        self.ws = torch.zeros(stca.CACHE_WS_BYTES, dtype=torch.uint8, device=self.device)

    def forward(self, tables, ids, out=None, stream: Optional[int] = None):
        """out [n][d]; tables and ids (int32 [n]): one a field (or a tensor each, of one field)."""
        torch = _torch()
        tables = (tables,) if isinstance(tables, torch.Tensor) else tables
        ids = (ids,) if isinstance(ids, torch.Tensor) else ids
        if len(tables) != len(self.rows) or len(ids) != len(self.rows):
            raise ValueError(f"{len(self.rows)} tables and ids are needed")
        n = ids[0].shape[0] if ids[0].dim() == 1 else None
        fields = []
        for f, (t, i, r) in enumerate(zip(tables, ids, self.rows)):
            t, ld = _matrix(f"tables[{f}]", t, self.d, self.dtype, self.device, r)
            fields.append((t, r, ld, _vector(f"ids[{f}]", i, n, torch.int32, self.device)))
        ldo = 0
        if out is not None:
            out, ldo = _matrix("out", out, self.d, self.out_dtype, self.device, n)
        with self._on(stream):
            if out is None:
                out = torch.empty((n, self.d), dtype=self.out_dtype, device=self.device)
            stca.stca_embed_forward(self.embed, stca.embed_fields(fields), n, out, ldo, self.ws, self._at(stream))
        return out

    def device_status(self, stream: Optional[int] = None) -> int:
        """STCA_ERR_INVALID_ARG once a lookup has met an id behind its table (see clear_status)."""
        return stca.stca_device_status(self.ws, self._at(stream))

    def clear_status(self):
        """On the current stream."""
        self.ws.zero_()


class EmbeddingGradient(_Streamed):
    """The gradient of a table of `rows` rows that up to `n` ids look up, from rows
    dout of `dtype`: times `scale`, fp32."""

    def __init__(self, rows: int, n: int, d: int, *, scale: float = 1.0, dtype=None, device="cuda"):
        torch = _torch()
        self.device = _device(device)
        self.rows, self.n, self.d, self.dtype = int(rows), int(n), int(d), dtype or torch.float32
        self.grad = stca.embed_grad(self.d, _dtype_code(self.dtype), self.rows, float(scale))
        self.ws_bytes = stca.stca_embed_grad_workspace_size(self.grad, self.n)
        if self.ws_bytes == 0:
            raise stca.StcaError(stca.STCA_ERR_INVALID_ARG, "stca_embed_grad_workspace_size")
        self.ws = torch.zeros(self.ws_bytes, dtype=torch.uint8, device=self.device)

    def _parts(self, parts):
        torch = _torch()
        if not 1 <= len(parts) <= stca.EMBED_PARTS:
            raise ValueError(f"parts: 1 to {stca.EMBED_PARTS} pairs of ids and dout")
        out, total = [], 0
        for p, (ids, dout) in enumerate(parts):
            ids = _vector(f"parts[{p}]: ids", ids, None, torch.int32, self.device)
            n = ids.shape[0]
            dout, ld = _matrix(f"parts[{p}]: dout", dout, self.d, self.dtype, self.device, n)
            out.append((ids, dout, ld, n))
            total += n
        if total > self.n:
            raise ValueError(f"parts: {total} rows, where the object was made for {self.n}")
        return stca.embed_parts(out), total

    def dense(self, parts, out=None, accumulate: bool = False, stream: Optional[int] = None):
        """[rows][d] fp32 over all parts [(ids, dout), ..]; accumulate adds to `out`."""
        torch = _torch()
        given, _ = self._parts(parts)
        if accumulate and out is None:
            raise ValueError("accumulate: out is needed")
        ld = 0
        if out is not None:
            out, ld = _matrix("out", out, self.d, torch.float32, self.device, self.rows)
        with self._on(stream):
            if out is None:
                out = torch.empty((self.rows, self.d), dtype=torch.float32, device=self.device)
            stca.stca_embed_grad_dense(self.grad, given, out, ld, accumulate, self.ws, self.ws_bytes, self._at(stream))
        return out

    def sparse(self, parts, out=None, stream: Optional[int] = None):
        """(rows int32 [c], values fp32 [c][d], count int32 [1]), c = min(ids, table's
        rows): the distinct ids in ascending order and their gradients; what lies behind
        the count is left as it was.  out: such a triple to be written, of as many rows or more."""
        torch = _torch()
        given, total = self._parts(parts)
        cap = min(total, self.rows)
        if out is not None:
            _vector("out: rows", out[0], None, torch.int32, self.device)
            _matrix("out: values", out[1], self.d, torch.float32, self.device, out[0].shape[0])
            _flat("out: count", out[2], torch.int32, (1,), self.device)
            if out[0].shape[0] < cap or not out[1].is_contiguous():
                raise ValueError(f"out: {cap} contiguous rows are needed")
        with self._on(stream):
            if out is None:
                new = dict(device=self.device)
                out = (torch.empty(cap, dtype=torch.int32, **new), torch.empty((cap, self.d), dtype=torch.float32, **new),
                       torch.empty(1, dtype=torch.int32, **new))
            rows, values, count = out
            # (no ids: there is no row to point at)
            stca.stca_embed_grad_sparse(self.grad, given, rows if cap else self.ws, values if cap else self.ws, count,
                                        self.ws, self.ws_bytes, self._at(stream))
        return out

    def device_status(self, stream: Optional[int] = None) -> int:
        """Of the last call."""
        return stca.stca_device_status(self.ws, self._at(stream))


class BlockNormGrads(NamedTuple):
    """Gradients of what was given, None for the rest: x, block and gate in the rows'
    dtype; pre and post (weight, bias) and layer_scale fp32."""
    x: object
    block: object
    gate: object
    pre: tuple
    post: tuple
    layer_scale: object


def _affine(p):
    """(weight, bias) of None, (weight,), (weight, bias) or a weight."""
    if p is None:
        return None, None
    if not isinstance(p, (tuple, list)):
        return p, None
    if len(p) > 2:
        raise ValueError("a norm's parameters: (weight, bias)")
    return (tuple(p) + (None, None))[:2]


class BlockNorm(_Streamed):
    """t = post(block) act(gate);  h = x + scale layer_scale t;  y = pre(h), with rms or
    layer norms.  forward(x) alone is y = pre(x)."""

    def __init__(self, d: int, *, kind: str = "rms", gate: Optional[str] = None, scale: float = 1.0, eps: float = 1e-6,
                 dtype=None, backward: bool = False, device="cuda"):
        torch = _torch()
        if kind not in _KINDS:
            raise ValueError(f"kind {kind!r}: rms or layer")
        if gate not in _GATES:
            raise ValueError(f"gate {gate!r}: None, sigmoid or silu")
        self.device = _device(device)
        self.d, self.kind, self.gate, self.dtype = int(d), kind, gate, dtype or torch.bfloat16
        self.scale, self.eps, self.has_backward = float(scale), float(eps), bool(backward)
        code = _dtype_code(self.dtype)
        # without a block; with one, by (post, pre)
        def form(gate, post, pre):
            return stca.norm(self.d, code, _KINDS[kind], gate, post, pre, self.scale, self.eps)
        self._alone = form(stca.STCA_GATE_NONE, False, True)
        self._forms = {(post, pre): form(_GATES[gate], post, pre) for post in (False, True) for pre in (False, True)}
        self.ws_bytes = stca.stca_norm_workspace_size(self._alone, 1 << 30)  # (enough for any number of rows)
        if self.ws_bytes == 0:
            raise stca.StcaError(stca.STCA_ERR_INVALID_ARG, "stca_norm_workspace_size")
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device) if backward else None

    def _given(self, x, block, gate, pre, post, layer_scale, want_y):
        torch = _torch()
        x, ldx = _matrix("x", x, self.d, self.dtype, self.device)
        n, ldb, ldg = x.shape[0], 0, 0
        if block is None:
            if gate is not None or post is not None or layer_scale is not None or not want_y:
                raise ValueError("gate, post, layer_scale and pre=False belong to a block")
            form = self._alone
        else:
            block, ldb = _matrix("block", block, self.d, self.dtype, self.device, n)
            if (gate is None) != (self.gate is None):
                raise ValueError(f"gate: given exactly where there is one ({self.gate})")
            if gate is not None:
                gate, ldg = _matrix("gate", gate, self.d, self.dtype, self.device, n)
            form = self._forms[post is not None, want_y]
        params = [*(_affine(pre) if want_y else (None, None)), *_affine(post), layer_scale]
        for name, t in zip(("pre: weight", "pre: bias", "post: weight", "post: bias", "layer_scale"), params):
            if t is not None:
                _vector(name, t, self.d, torch.float32, self.device)
        return form, stca.norm_in(x, block, gate, ldx, ldb, ldg, *params), n, params

    def forward(self, x, *, block=None, gate=None, pre=None, post=None, layer_scale=None, stream: Optional[int] = None):
        """(h, y) of rows [n][d]; h is x where there is no block.  pre, post: (weight,
        bias) or (weight,), fp32 [d]; () for a norm without them.  post=None: the block's
        rows as they are; pre=False: no y (None)."""
        want_y = pre is not False
        form, given, n, _ = self._given(x, block, gate, pre, post, layer_scale, want_y)
        with self._on(stream):
            h = None if block is None else _like(x)
            y = _like(x) if want_y else None
            stca.stca_norm_forward(form, given, n, h, 0, y, 0, self._at(stream))
        return (x if h is None else h), y

    def backward(self, dy, x, *, dh=None, block=None, gate=None, pre=None, post=None, layer_scale=None,
                 stream: Optional[int] = None) -> BlockNormGrads:
        """Gradients of sum <dy, y> + sum <dh, h> for the inputs of a forward; dh=None: h
        is not used but for y; dy=None with pre=False."""
        torch = _torch()
        if not self.has_backward:
            raise ValueError("backward: the object was made without backward=True")
        want_y = pre is not False
        form, given, n, params = self._given(x, block, gate, pre, post, layer_scale, want_y)
        lddy = lddh = 0
        if want_y:
            dy, lddy = _matrix("dy", dy, self.d, self.dtype, self.device, n)
        elif dy is not None:
            raise ValueError("dy: given, but there is no y")
        if dh is not None:
            dh, lddh = _matrix("dh", dh, self.d, self.dtype, self.device, n)
        elif not want_y:
            raise ValueError("dh: needed where there is no y")
        with self._on(stream):
            dx, db, dg = (None if t is None else _like(x) for t in (x, block, gate))
            wanted = sum(t is not None for t in params)
            sums = iter(torch.empty((wanted, self.d), dtype=torch.float32, device=self.device).unbind(0) if wanted else ())
            dp = [None if t is None else next(sums) for t in params]
            out = stca.norm_grads(dx, db, dg, 0, 0, 0, *dp)
            stca.stca_norm_backward(form, given, n, dh, lddh, dy, lddy, out, self.ws, self.ws_bytes, self._at(stream))
        return BlockNormGrads(dx, db, dg, (dp[0], dp[1]), (dp[2], dp[3]), dp[4])


class GradientNorm(_Streamed):
    """The norm of all gradients (at most `most` tensors) together, and clipping to
    max_norm."""

    def __init__(self, max_norm: float = float("inf"), most: int = 1024, device="cuda"):
        self.device, self.max_norm, self.most = _device(device), float(max_norm), int(most)
        if not self.max_norm > 0.0 or self.most < 0:
            raise ValueError("max_norm: above 0; most: at least 0")
        self.ws_bytes = stca.stca_clip_workspace_size(self.most)
        self.ws = _torch().empty(self.ws_bytes, dtype=_torch().uint8, device=self.device)

    def norm(self, grads, counts=None, stream: Optional[int] = None):
        """The norm as an fp32 tensor of no dimensions on the device; the gradients stay as they are."""
        return self._call(grads, [None] * len(grads), counts, stream)

    def clip(self, grads, out=None, counts=None, stream: Optional[int] = None):
        """The norm (as norm()); every gradient times min(1, max_norm / norm), in place or
        into `out` (a tensor of the same size, fp32 or bf16, each).  A norm that is not
        finite changes nothing.  counts: None, or an int32 tensor [1] with the number of
        rows (first dimension) in use, for each; the others are not touched."""
        return self._call(grads, grads if out is None else out, counts, stream)

    def _call(self, grads, out, counts, stream):
        torch = _torch()
        grads, out = list(grads), list(out)
        counts = [None] * len(grads) if counts is None else list(counts)
        if len(out) != len(grads) or len(counts) != len(grads):
            raise ValueError("out and counts: one for every gradient")
        if len(grads) > self.most:
            raise ValueError(f"{len(grads)} gradients, where the object was made for {self.most}")
        codes = {torch.float32: stca.STCA_F32, torch.bfloat16: stca.STCA_BF16}
        at = -1 if self.device.index is None else self.device.index
        items = []
        for i, (g, o, c) in enumerate(zip(grads, out, counts)):
            n, code, row = g.numel(), codes.get(g.dtype), 0
            ok = code is not None and g.get_device() == at and g.is_contiguous()
            p, to = 0, code
            if o is g:
                p = g.data_ptr()
            elif o is not None:
                p, to = o.data_ptr(), codes.get(o.dtype)
                ok = ok and to is not None and o.get_device() == at and o.is_contiguous() and o.numel() == n
            if not ok:
                raise ValueError(f"gradient {i}: contiguous fp32 or bf16 tensors of one size on {self.device} are needed")
            if c is not None:
                _flat(f"counts[{i}]", c, torch.int32, (1,), self.device)
                if g.dim() == 0:
                    raise ValueError(f"counts[{i}]: the gradient has no rows")
                row = max(1, n // max(1, g.shape[0]))
            items.append((g.data_ptr(), p, n, code, to, 0 if c is None else c.data_ptr(), row))
        with self._on(stream):
            norm = torch.empty((), dtype=torch.float32, device=self.device)
            stca.stca_clip(stca.grads(items), self.max_norm, norm, self.ws, self.ws_bytes, self._at(stream))
        return norm
