"""The layers of a sequence surrogate around its attention, on CUDA tensors (gp_norm*, gp_rotate*,
gp_gated* and gp_adamw of include/baco_gp.h): norms, rotary positions, the gated feed-forward block,
each with its gradient, and a step of AdamW over many tensors.

As in ``seq``, this module only marshals arguments. A description is made once, buffers once per
use; the `*_into` calls are asynchronous on the current stream, and the plain calls allocate their
outputs. A call's buffers belong to one stream at a time; threads may share a description, each with
buffers of its own. No call records a graph: gradients have calls of their own, for a
torch.autograd.Function, and the plain calls refuse tensors that ask for one outside of it.
"""
from __future__ import annotations

import ctypes as C
import math
import operator
import threading
from typing import Optional, Sequence

from . import gp
from .gp import _check, _torch
from .seq import Documents, _INVALID, _call, _dtype_code, _stream, _workspace


def _device(device):
    return _torch().cuda.current_device() if device is None else int(device)


def _matrix(x, shape, dtype, device, name):
    """Pointer and row stride of a tensor argument."""
    if x.shape != shape or x.dtype is not dtype or x.get_device() != device:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on cuda:{device}, "
                         f"not {x.dtype} {tuple(x.shape)} on {x.device}")
    row, one = x.stride()
    if one != 1 and shape[1] > 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return x.data_ptr(), row


def _vector(x, shape, dtype, device, name):
    if x is None:
        return None
    if x.shape != shape or x.dtype is not dtype or x.get_device() != device or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on "
                         f"cuda:{device}")
    return x.data_ptr()


def _no_graph(*tensors):
    """For calls whose results have no graph: they would lose a gradient without a word."""
    if _torch().is_grad_enabled() and any(x is not None and x.requires_grad for x in tensors):
        raise ValueError("a tensor requires a gradient, and the result would have no graph: call within a "
                         "torch.autograd.Function, or under torch.no_grad()")


def _workspace_size(n):
    """A size in bytes; raises what the library refused."""
    if n == _INVALID:
        raise gp.GPError(1, gp.load().gp_last_error().decode())
    return n


# ------------------------------------------------------------------ norms
class Norm:
    """A layer norm of rows of `width` (centre False: by the root mean square): their dtype, the
    type of the weight (None: there is none; dtype or torch.float32) and, if there is one, of the
    bias, and eps."""

    def __init__(self, width: int, dtype, weight=None, bias: bool = False, eps: float = 1e-5,
                 centre: bool = True):
        self.width, self.dtype, self.weight_dtype, self.has_bias = int(width), dtype, weight, bool(bias)
        if bias and weight is None:
            raise ValueError("a bias goes with a weight")
        s = gp._Norm()
        s.dtype = _dtype_code(dtype)
        s.weight_dtype = s.dtype if weight is None else _dtype_code(weight)
        s.width, s.centre, s.eps = self.width, int(bool(centre)), float(eps)
        self.struct, self.ref, self.lib = s, C.byref(s), gp.load()
        self.grad_workspace_bytes(0)             # raises if the description is invalid

    def grad_workspace_bytes(self, rows: int) -> int:
        return _workspace_size(gp.load().gp_norm_grad_workspace_bytes(self.ref, int(rows)))


class NormBuffers:
    """Outputs and workspace, on a device (the current one if None), of a norm's calls on `rows`
    rows: out, with residual the sum that was normalised, stats [rows, 2], and with grad dx and
    (with a weight) dweight and dbias."""

    def __init__(self, norm: Norm, rows: int, residual: bool = False, grad: bool = False,
                 device: Optional[int] = None):
        torch = _torch()
        self.norm, self.rows, self.device = norm, int(rows), _device(device)
        self.shape = torch.Size((self.rows, norm.width))
        self.vector = torch.Size((norm.width,))
        dev = torch.device("cuda", self.device)
        rows_of = dict(size=self.shape, dtype=norm.dtype, device=dev)
        self.out = torch.empty(**rows_of)
        self.sum = torch.empty(**rows_of) if residual else None
        self.stats = torch.empty((self.rows, 2), dtype=torch.float32, device=dev) if grad else None
        self.dx = self.dweight = self.dbias = self.workspace = None
        self.workspace_bytes = 0
        if grad:
            self.dx = torch.empty(**rows_of)
            w = dict(size=self.vector, dtype=norm.weight_dtype, device=dev)
            if norm.weight_dtype is not None:
                self.dweight = torch.empty(**w)
                self.dbias = torch.empty(**w) if norm.has_bias else None
            self.workspace, self.workspace_bytes = _workspace(
                norm.grad_workspace_bytes(self.rows), self.device)


def _norm_weights(norm, bufs, weight, bias):
    if (weight is None) != (norm.weight_dtype is None) or (bias is None) == norm.has_bias:
        raise ValueError("weight and bias go with a description that has them")
    return (_vector(weight, bufs.vector, norm.weight_dtype, bufs.device, "weight"),
            _vector(bias, bufs.vector, norm.weight_dtype, bufs.device, "bias"))


def norm_into(norm: Norm, x, bufs: NormBuffers, weight=None, bias=None, residual=None):
    """gp_norm of x [rows, width] (+ residual; the rows' strides are free) into bufs.out, bufs.sum
    and bufs.stats."""
    if bufs.norm is not norm:
        raise ValueError("the buffers are another norm's")
    if (residual is None) != (bufs.sum is None):
        raise ValueError("a residual goes with buffers that have a sum")
    at = bufs.shape, norm.dtype, bufs.device
    w, b = _norm_weights(norm, bufs, weight, bias)
    r, s = (None, 0), (None, 0)
    if residual is not None:
        r, s = _matrix(residual, *at, "residual"), _matrix(bufs.sum, *at, "sum")
    _call(bufs.device, norm.lib.gp_norm, (
        norm.ref, bufs.rows, *_matrix(x, *at, "x"), *r, w, b, *_matrix(bufs.out, *at, "out"), *s,
        None if bufs.stats is None else bufs.stats.data_ptr(), _stream(x)))


def norm(norm: Norm, x, weight=None, bias=None, residual=None) -> dict:
    _no_graph(x, weight, bias, residual)
    bufs = NormBuffers(norm, x.shape[0], residual=residual is not None,
                       device=x.get_device() if x.is_cuda else None)
    norm_into(norm, x, bufs, weight, bias, residual)
    out = {"out": bufs.out, "_buffers": bufs}
    if residual is not None:
        out["sum"] = bufs.sum
    return out


def norm_grad_into(norm: Norm, h, dout, bufs: NormBuffers, weight=None, dsum=None):
    """gp_norm_grad into bufs.dx (the gradient of x, and of the residual), dweight and dbias, from
    dout and, where the sum is used elsewhere too, dsum; h: what was normalised (bufs.sum, or x
    without a residual), with the stats that norm_into left in bufs for it."""
    if bufs.norm is not norm:
        raise ValueError("the buffers are another norm's")
    if bufs.dx is None:
        raise ValueError("the buffers were made without grad")
    at = bufs.shape, norm.dtype, bufs.device
    if (weight is None) != (norm.weight_dtype is None):
        raise ValueError("weight goes with a description that has one")
    w = _vector(weight, bufs.vector, norm.weight_dtype, bufs.device, "weight")
    ws = bufs.workspace
    _call(bufs.device, norm.lib.gp_norm_grad, (
        norm.ref, bufs.rows, *_matrix(h, *at, "h"), bufs.stats.data_ptr(), w,
        *_matrix(dout, *at, "dout"), *((None, 0) if dsum is None else _matrix(dsum, *at, "dsum")),
        *_matrix(bufs.dx, *at, "dx"), None if bufs.dweight is None else bufs.dweight.data_ptr(),
        None if bufs.dbias is None else bufs.dbias.data_ptr(),
        None if ws is None else ws.data_ptr(), bufs.workspace_bytes, _stream(h)))


# ------------------------------------------------------------------ rotary positions
def frequencies(rotated: int, base: float = 10000.0, factor: float = 1.0,
                original: Optional[float] = None, near: float = 1.0, far: float = 32.0):
    """Angles per position of a head's pairs, f_i = base^(-2i / rotated), for runs `factor` times
    as long as trained: divided by it, or by parts where `original`, the trained length, is given:
    pairs that make `far` turns over it or more stay, those of `near` turns or less are divided, and
    between them the share that stays grows with the turns."""
    out = []
    for i in range(rotated // 2):
        f = base ** (-2.0 * i / rotated)
        keep = 0.0
        if original is not None:
            keep = min(1.0, max(0.0, (original * f / (2 * math.pi) - near) / (far - near)))
        out.append(f * (keep + (1.0 - keep) / factor))
    return out


class Rotary:
    """How heads of size dim are rotated, on a device (the current one if None): the first
    `rotated` values (None: all), in pairs (i, i + rotated / 2) or, interleaved, (2i, 2i + 1), by
    `frequencies` of base, factor, original, near and far, or by angles of the caller's own
    (angles: radians per position, one per pair); magnitude: factor of the rotated values."""

    def __init__(self, dim: int, dtype, rotated: Optional[int] = None, base: float = 10000.0,
                 interleaved: bool = False, factor: float = 1.0, original: Optional[float] = None,
                 near: float = 1.0, far: float = 32.0, magnitude: float = 1.0,
                 angles: Optional[Sequence[float]] = None, device: Optional[int] = None):
        torch = _torch()
        self.dim, self.dtype, self.device = int(dim), dtype, _device(device)
        self.rotated = self.dim if rotated is None else int(rotated)
        if not (base > 0 and factor > 0) or (original is not None and not far > near):
            raise ValueError("need base > 0, factor > 0 and far > near")
        if angles is None:
            angles = frequencies(self.rotated, base, factor, original, near, far)
        angles = [float(a) for a in angles]
        if self.rotated % 2 or len(angles) != self.rotated // 2:
            raise ValueError("rotated must be even, with an angle per pair")
        self.turns = torch.tensor([a / (2 * math.pi) for a in angles], dtype=torch.float64,
                                  device=torch.device("cuda", self.device))
        s = gp._Rotary()
        s.dtype, s.dim, s.rotated = _dtype_code(dtype), self.dim, self.rotated
        s.interleaved, s.magnitude = int(bool(interleaved)), float(magnitude)
        s.turns = self.turns.data_ptr()
        self.struct, self.ref, self.lib = s, C.byref(s), gp.load()
        none = C.byref(gp._Heads(0, self.dim, self.dim))
        _check(self.lib.gp_rotate(self.ref, 0, None, 1, none, none, 0, None))   # raises if invalid
        self.slots = _HeadSlots(self)


class _HeadSlot:
    """One tensor argument [rows, heads, dim] of a description's calls: the gp_heads struct that is
    filled for each call."""

    __slots__ = ("name", "of", "struct", "ref")

    def __init__(self, name, of):
        self.name, self.of = name, of
        self.struct = gp._Heads()
        self.ref = C.byref(self.struct)

    def __call__(self, x, rows, heads):
        of = self.of
        if x.shape != (rows, heads, of.dim) or x.dtype is not of.dtype or x.get_device() != of.device:
            raise ValueError(f"{self.name} must be a {of.dtype} tensor of shape "
                             f"{(rows, heads, of.dim)} on cuda:{of.device}, not {x.dtype} "
                             f"{tuple(x.shape)} on {x.device}")
        s = self.struct
        s.row, s.head, one = x.stride()
        if one != 1:
            raise ValueError(f"{self.name}'s last axis must be contiguous")
        s.data = x.data_ptr()
        return self.ref


class _HeadSlots(threading.local):
    """A description's slots, a set per thread: a call releases the interpreter while the library
    reads them."""

    def __init__(self, of):
        for n in ("x", "out", "q", "k", "v", "k_cache", "v_cache"):
            setattr(self, n, _HeadSlot(n, of))


def positions(docs: Documents):
    """int32 [q_rows]: where each query row of the documents stands, pos(i) = i + Lk - Lq as
    attention has it (0 for rows of no document). Nothing is read back."""
    torch = _torch()
    rows = torch.arange(docs.q_rows, dtype=torch.int64, device=docs.q_begin.device)
    if docs.n == 0:
        return rows.int().zero_()
    qb, qe = docs.q_begin.long().clamp(0, docs.q_rows), docs.q_end.long().clamp(0, docs.q_rows)
    kb, ke = docs.k_begin.long().clamp(0, docs.k_rows), docs.k_end.long().clamp(0, docs.k_rows)
    order = torch.argsort(qb * (1 << 31) + qe)       # (of documents at one place, the empty first)
    at = order[(torch.searchsorted(qb[order], rows, right=True) - 1).clamp_min(0)]
    mine = (rows >= qb[at]) & (rows < qe[at])
    pos = rows - qb[at] + (ke - kb).clamp_min(0)[at] - (qe - qb)[at]
    return torch.where(mine, pos, torch.zeros_like(pos)).int()


def _positions(p, rows, device, dtype, name):
    if p.shape != (rows,) or p.dtype is not dtype or p.get_device() != device or not p.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} vector of {rows} on cuda:{device}")
    return p.data_ptr()


def rotate_into(rotary: Rotary, positions, x, out, inverse: bool = False):
    """gp_rotate of x [rows, heads, dim] (strides of rows and heads are free, multiples of 8) by
    positions (int32 [rows]) into out, which may be x; inverse: the opposite way, for a gradient.
    Query and key heads that lie side by side are rotated in one call."""
    rows, heads = x.shape[0], x.shape[1]
    t = rotary.slots
    _call(rotary.device, rotary.lib.gp_rotate, (
        rotary.ref, rows, _positions(positions, rows, rotary.device, _torch().int32, "positions"),
        heads, t.x(x, rows, heads), t.out(out, rows, heads), int(inverse), _stream(x)))


def rotate(rotary: Rotary, positions, x, inverse: bool = False):
    _no_graph(x)
    out = _torch().empty(x.shape, dtype=x.dtype, device=x.device)
    rotate_into(rotary, positions, x, out, inverse)
    return out


def append_into(rotary: Rotary, positions, slots, q, k, v, out, k_cache, v_cache):
    """gp_rotate_append: rotated q [rows, heads, dim] into out, rotated k and v
    [rows, kv_heads, dim] into the rows `slots` (int64 [rows], all different; outside the cache: not
    kept) of k_cache and v_cache [cache_rows, kv_heads, dim]."""
    torch = _torch()
    rows, heads, kv_heads, n = q.shape[0], q.shape[1], k.shape[1], k_cache.shape[0]
    t, dev = rotary.slots, rotary.device
    _call(dev, rotary.lib.gp_rotate_append, (
        rotary.ref, rows, _positions(positions, rows, dev, torch.int32, "positions"),
        _positions(slots, rows, dev, torch.int64, "slots"), heads, t.q(q, rows, heads),
        t.out(out, rows, heads), kv_heads, t.k(k, rows, kv_heads), t.v(v, rows, kv_heads), n,
        t.k_cache(k_cache, n, kv_heads), t.v_cache(v_cache, n, kv_heads), _stream(q)))


# ------------------------------------------------------------------ gated feed-forward block
ACTIVATIONS = {"silu": 0, "gelu": 1}


class Gated:
    """A gated block's sizes (multiples of 8), dtype (torch.bfloat16 or torch.float16) and
    activation ("silu" or "gelu"). Its weights are [hidden, width], rows of any stride."""

    def __init__(self, width: int, hidden: int, dtype, activation: str = "silu"):
        torch = _torch()
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}")
        self.width, self.hidden, self.dtype = int(width), int(hidden), dtype
        s = gp._Gated()
        s.dtype, s.width, s.hidden = _dtype_code(dtype), self.width, self.hidden
        s.activation = ACTIVATIONS[activation]
        self.struct, self.ref, self.lib = s, C.byref(s), gp.load()
        self.weight_shape = torch.Size((self.hidden, self.width))
        none = [C.byref(gp._Matrix(16, self.width))] * 4
        _check(self.lib.gp_gated(self.ref, 0, *none, None))      # raises if invalid

    def grad_workspace_bytes(self, rows: int) -> int:
        n = gp.load().gp_gated_grad_workspace_bytes(self.ref, int(rows))
        if n == _INVALID:
            none = [None] * 7
            _check(gp.load().gp_gated_grad(self.ref, int(rows), *none, None, 0, None))
        return n


class GatedBuffers:
    """Outputs and workspace, on a device (the current one if None), of a block's calls on `rows`
    rows: out [rows, hidden], and with grad dx, dw_gate and dw_up."""

    def __init__(self, gated: Gated, rows: int, grad: bool = False, device: Optional[int] = None):
        torch = _torch()
        self.gated, self.rows, self.device = gated, int(rows), _device(device)
        dev = torch.device("cuda", self.device)
        of = dict(dtype=gated.dtype, device=dev)
        self.x_shape = torch.Size((self.rows, gated.width))
        self.out_shape = torch.Size((self.rows, gated.hidden))
        self.out = torch.empty(self.out_shape, **of)
        self.dx = self.dw_gate = self.dw_up = self.workspace = None
        self.workspace_bytes = 0
        if grad:
            self.dx = torch.empty(self.x_shape, **of)
            self.dw_gate = torch.empty(gated.weight_shape, **of)
            self.dw_up = torch.empty(gated.weight_shape, **of)
            self.workspace, self.workspace_bytes = _workspace(
                gated.grad_workspace_bytes(self.rows), self.device)
        self.slots = _MatrixSlots()


class _MatrixSlots(threading.local):
    def __init__(self):
        self.of = [gp._Matrix() for _ in range(7)]
        self.refs = [C.byref(x) for x in self.of]


def _matrices(bufs, args):
    """References to gp_matrix structs of (tensor, shape, name) arguments."""
    slots, dtype, device = bufs.slots, bufs.gated.dtype, bufs.device
    for s, (x, shape, name) in zip(slots.of, args):
        s.data, s.row = _matrix(x, shape, dtype, device, name)
    return slots.refs[:len(args)]


def gated_into(gated: Gated, x, w_gate, w_up, bufs: GatedBuffers):
    """gp_gated of x [rows, width] into bufs.out."""
    if bufs.gated is not gated:
        raise ValueError("the buffers are another block's")
    w = gated.weight_shape
    _call(bufs.device, gated.lib.gp_gated, (
        gated.ref, bufs.rows, *_matrices(bufs, (
            (x, bufs.x_shape, "x"), (w_gate, w, "w_gate"), (w_up, w, "w_up"),
            (bufs.out, bufs.out_shape, "out"))), _stream(x)))


def gated(gated: Gated, x, w_gate, w_up):
    _no_graph(x, w_gate, w_up)
    bufs = GatedBuffers(gated, x.shape[0], device=x.get_device() if x.is_cuda else None)
    gated_into(gated, x, w_gate, w_up, bufs)
    return bufs.out


def gated_grad_into(gated: Gated, x, w_gate, w_up, dout, bufs: GatedBuffers):
    """gp_gated_grad into bufs.dx, dw_gate and dw_up, from dout [rows, hidden]. (Nothing of the
    forward call is needed.)"""
    if bufs.gated is not gated:
        raise ValueError("the buffers are another block's")
    if bufs.dx is None:
        raise ValueError("the buffers were made without grad")
    w, ws = gated.weight_shape, bufs.workspace
    _call(bufs.device, gated.lib.gp_gated_grad, (
        gated.ref, bufs.rows, *_matrices(bufs, (
            (x, bufs.x_shape, "x"), (w_gate, w, "w_gate"), (w_up, w, "w_up"),
            (dout, bufs.out_shape, "dout"), (bufs.dx, bufs.x_shape, "dx"),
            (bufs.dw_gate, w, "dw_gate"), (bufs.dw_up, w, "dw_up"))),
        None if ws is None else ws.data_ptr(), bufs.workspace_bytes, _stream(x)))


# ------------------------------------------------------------------ AdamW
SHARE = 256              # values of an 8-bit state that share a scale
_shape, _dtype = operator.attrgetter("shape"), operator.attrgetter("dtype")


class AdamW:
    """AdamW's states for a list of weights of one dtype, on their device: m and v of 32 bits, or of
    8 (e4m3 and e5m2 codes, with scales [blocks, 2] of each 256 values). masters: fp32 copies of
    16-bit weights, which the step is made on. grad_dtype: the gradients' (None: the weights'). A
    weight may be given once only: none of them may share memory.

    The states lie one tensor after another in m_all and v_all [blocks, 256] (and scales_all
    [blocks, 2]), each from a block of its own on; m, v and scales are views of them. They start at
    0; a checkpoint keeps the *_all tensors and the caller's step, and is copied into them: the library
    has their addresses."""

    m_all, v_all, scales_all, m, v, scales = (
        property(operator.attrgetter("_" + name)) for name in ("m_all", "v_all", "scales_all", "m", "v", "scales"))

    def __init__(self, params, masters=None, state_bits: int = 32, grad_dtype=None):
        torch = _torch()
        self.params = list(params)
        if not self.params:
            raise ValueError("no weights")
        self.masters = None if masters is None else list(masters)
        if self.masters is not None and len(self.masters) != len(self.params):
            raise ValueError("one master copy per weight")
        if state_bits not in (8, 32):
            raise ValueError("states have 8 or 32 bits")
        self.state_bits, self.dtype = state_bits, self.params[0].dtype
        self.grad_dtype = self.dtype if grad_dtype is None else grad_dtype
        self.device = self.params[0].get_device()
        if self.device < 0:
            raise ValueError("the weights must be CUDA tensors")
        self.lib = gp.load()
        dev = torch.device("cuda", self.device)
        counts = [p.numel() for p in self.params]
        first = [0]
        for n in counts:
            first.append(first[-1] + -(-n // SHARE))
        kinds = (torch.float8_e4m3fn, torch.float8_e5m2) if state_bits == 8 else (torch.float32,) * 2
        self._m_all, self._v_all = (
            torch.zeros((first[-1], SHARE * k.itemsize), dtype=torch.uint8, device=dev).view(k)
            for k in kinds)

        def views(x):
            flat = x.view(-1)
            return tuple(flat[SHARE * a:SHARE * a + n].view(p.shape)
                         for a, n, p in zip(first, counts, self.params))

        self._m, self._v = views(self.m_all), views(self.v_all)
        self._scales_all = self._scales = None
        if state_bits == 8:
            self._scales_all = torch.ones((first[-1], 2), dtype=torch.float32, device=dev)
            self._scales = tuple(self.scales_all[a:b] for a, b in zip(first, first[1:]))
        s = gp._AdamW()
        s.dtype, s.grad_dtype, s.state_bits = _dtype_code(self.dtype), _dtype_code(self.grad_dtype), state_bits
        self.struct, self.ref = s, C.byref(s)
        self.tensors = (gp._AdamWTensor * len(counts))()
        for i, t in enumerate(self.tensors):
            t.m, t.v, t.count = self.m[i].data_ptr(), self.v[i].data_ptr(), counts[i]
            t.scales = None if self.scales is None else self.scales[i].data_ptr()
        self.shapes = [p.shape for p in self.params]
        self.pointers = C.c_void_p * len(counts)
        self._weights = self.params + (self.masters or [])
        self._at = None
        self._update()

    def _update(self):
        """The weights' addresses, as they are now: a weight's storage may have been replaced, also by
        another view of the same memory or by what the allocator has put in its place."""
        torch = _torch()
        weights, n = self._weights, len(self.params)
        copies = len(weights) - n
        at = list(map(torch.Tensor.data_ptr, weights))
        if at == self._at and all(map(torch.Tensor.is_contiguous, weights)) and \
                list(map(_shape, weights)) == (self.shapes * 2 if copies else self.shapes) and \
                list(map(_dtype, weights)) == [self.dtype] * n + [torch.float32] * copies:
            return
        self._at = None
        for i, t in enumerate(self.tensors):
            p = self.params[i]
            if p.dtype is not self.dtype or p.get_device() != self.device or not p.is_contiguous() or \
                    p.shape != self.shapes[i]:
                raise ValueError(f"weight {i} must be a contiguous {self.dtype} tensor of shape "
                                 f"{tuple(self.shapes[i])} on cuda:{self.device}")
            if self.masters is not None:
                w = self.masters[i]
                if w.dtype is not torch.float32 or w.get_device() != self.device or \
                        not w.is_contiguous() or w.shape != p.shape:
                    raise ValueError(f"master copy {i} must be a contiguous float32 tensor of its "
                                     f"weight's shape on cuda:{self.device}")
                t.master = at[n + i] or None
            t.param = at[i] or None
        ends = sorted((a, a + w.numel() * w.element_size()) for a, w in zip(at, self._weights) if a)
        if any(end > begin for (_, end), (begin, _) in zip(ends, ends[1:])):
            raise ValueError("weights (and master copies) must not share memory")
        self._uncounted = any(map(torch.Tensor.is_inference, weights))
        self._at = at

    def _count(self, grads):
        """Raises the version counters of the weights that were changed: autograd refuses to use what it
        saved of them before."""
        changed = self._weights
        if any(g is None for g in grads):
            grads = list(grads) * (1 if self.masters is None else 2)
            changed = [w for w, g in zip(changed, grads) if g is not None]
        if self._uncounted:
            changed = [w for w in changed if not w.is_inference()]
        _torch().autograd.graph.increment_version(changed)

    def _gradients(self, grads):
        """Their addresses, 0 for none. (map over a method: a loop of checks would cost 17 us for 28
        tensors, whose step takes 16 on the device.)"""
        torch = _torch()
        given = [g for g in grads if g is not None]
        shapes = self.shapes
        if len(given) != len(grads):
            shapes = [s for s, g in zip(shapes, grads) if g is not None]
        of = torch.Tensor
        if list(map(_shape, given)) != shapes or not all(map(of.is_contiguous, given)) or \
                (given and (set(map(_dtype, given)) != {self.grad_dtype} or
                            set(map(of.get_device, given)) != {self.device})):
            raise ValueError(f"gradients must be contiguous {self.grad_dtype} tensors of their weights' "
                             f"shapes on cuda:{self.device}")
        at = list(map(of.data_ptr, given))
        if len(given) != len(grads):
            rest = iter(at)
            at = [0 if g is None else next(rest) for g in grads]
        return self.pointers(*at)


def _scalar(x, dtype, device, name):
    if x.numel() != 1 or x.dtype is not dtype or x.get_device() != device:
        raise ValueError(f"{name} must be a {dtype} tensor of one value on cuda:{device}")
    return x.data_ptr()


def adamw_into(opt: AdamW, grads, lr, step, betas=(0.9, 0.999), eps: float = 1e-8,
               decay: float = 0.01, factor=None, seed: int = 0):
    """gp_adamw: step number `step` (from 1) of opt's weights and states, in place. grads: a
    gradient per weight, or None for a weight that is left as it is; factor (float32, one value):
    what they are multiplied by. lr and step may be tensors of one value (float32, int64), which are
    read on the device: a captured graph is replayed with those of the time. seed: of the random
    numbers that round states of 8 bits (the same seed and steps give the same states)."""
    torch = _torch()
    dev = opt.device
    if len(grads) != len(opt.params):
        raise ValueError("one gradient (or None) per weight")
    opt._update()
    at = opt._gradients(grads)
    s = gp._AdamW.from_buffer_copy(opt.struct)
    s.beta1, s.beta2 = betas
    s.eps, s.decay, s.seed = eps, decay, int(seed) & 0xffffffffffffffff
    if isinstance(lr, torch.Tensor):
        s.lr_device = _scalar(lr, torch.float32, dev, "lr")
    else:
        s.lr = lr
    if isinstance(step, torch.Tensor):
        s.step_device = _scalar(step, torch.int64, dev, "step")
    else:
        s.step = step
    if factor is not None:
        s.factor = _scalar(factor, torch.float32, dev, "factor")
    _call(dev, opt.lib.gp_adamw, (C.byref(s), len(grads), opt.tensors, at, _stream(opt.params[0])))
    opt._count(grads)
