"""Operators of a sequence surrogate on CUDA tensors (gp_attend*, gp_logprob* of
include/baco_gp.h): attention over tuning histories packed in one batch, with its gradient,
and the log probabilities of an output row with theirs.

As in ``gp``, this module only marshals arguments. A layout of documents and an `Attention`
description are made once per batch shape, buffers once per use; the `*_into` calls are
asynchronous on the current stream, and the plain calls allocate their outputs. A
description's tensors and a call's buffers belong to one stream at a time; threads may share a
description, each with buffers of its own.
"""
from __future__ import annotations

import ctypes as C
import math
import threading
from typing import Optional, Sequence

from . import gp
from .gp import _check, _torch

MAX_REACH = 1024     # the last bucket starts at this distance at most
_INVALID = (1 << (8 * C.sizeof(C.c_size_t))) - 1


def _dtype_code(dtype):
    torch = _torch()
    code = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}.get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype}")
    return code


def _stream(x):
    """The current stream of a tensor's device. (torch.cuda.current_stream() makes an object
    for it, 2.9 us; the handle alone takes 0.1 us of a call's 6.)"""
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream(x.device).cuda_stream
    return raw(x.get_device())


def _current_device():
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getDevice", None)
    return torch.cuda.current_device() if raw is None else raw()


def _call(device, f, args):
    """f(*args) with `device` current: a launch is the current device's."""
    if _current_device() == device:
        st = f(*args)
    else:
        with _torch().cuda.device(device):
            st = f(*args)
    if st:
        _check(st)


def _workspace(nbytes, device):
    """A workspace and its size. (torch's allocator returns 512-byte aligned blocks.)"""
    if not nbytes:
        return None, 0
    torch = _torch()
    ws = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=torch.device("cuda", device))
    return ws, ws.numel()


# ------------------------------------------------------------------ layouts
class Documents:
    """The documents (tuning runs) of a packed batch.

    q_len, k_len: rows of each document (k_len None: as q_len). The query rows follow one
    another; the key rows too, unless k_begin gives each document's first key row (a cache
    with a slot per run; slots may be longer than k_len, and with gradients must not
    overlap). prefix: keys of each document that every row of it sees under a causal mask.
    q_rows, k_rows: rows of the tensors, if more than the documents take."""

    def __init__(self, q_len: Sequence[int], k_len: Optional[Sequence[int]] = None, prefix=None,
                 k_begin=None, q_rows=None, k_rows=None):
        torch = _torch()
        q_len = [int(x) for x in q_len]
        k_len = q_len if k_len is None else [int(x) for x in k_len]
        n = len(q_len)
        if len(k_len) != n or (prefix is not None and len(prefix) != n) or \
                (k_begin is not None and len(k_begin) != n):
            raise ValueError("one q_len, k_len, prefix and k_begin per document")
        if any(x < 0 for x in q_len) or any(x < 0 for x in k_len):
            raise ValueError("negative length")
        qb, at = [], 0
        for x in q_len:
            qb.append(at)
            at += x
        self.q_rows = at if q_rows is None else int(q_rows)
        if self.q_rows < at:
            raise ValueError(f"the documents have {at} query rows, q_rows is {self.q_rows}")
        self.q_full = self.q_rows == at      # every query row is some document's
        if k_begin is None:
            kb, at = [], 0
            for x in k_len:
                kb.append(at)
                at += x
        else:
            kb = [int(x) for x in k_begin]
            if any(x < 0 for x in kb):
                raise ValueError("negative k_begin")
            at = max([b + x for b, x in zip(kb, k_len)], default=0)
        self.k_rows = at if k_rows is None else int(k_rows)
        if self.k_rows < at:
            raise ValueError(f"the documents reach key row {at}, k_rows is {self.k_rows}")
        spans = sorted((b, b + x) for b, x in zip(kb, k_len) if x > 0)
        self.k_disjoint = all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
        self.k_full = self.k_disjoint and sum(k_len) == self.k_rows
        self.n, self.moving = n, False
        self.max_q, self.max_k = max(q_len, default=0), max(k_len, default=0)
        rows = [qb, [a + b for a, b in zip(qb, q_len)], kb, [a + b for a, b in zip(kb, k_len)],
                [0] * n if prefix is None else [int(x) for x in prefix]]
        # the calls get the documents with the longest first: their blocks start first, and
        # the short ones fill the device's end
        order = sorted(range(n), key=lambda d: -q_len[d] * k_len[d])
        both = torch.tensor([rows, [[r[d] for d in order] for r in rows]], dtype=torch.int32)
        both = both.reshape(2, 5, n).cuda()
        self.q_begin, self.q_end, self.k_begin, self.k_end, pre = both[0]
        self.prefix = None if prefix is None else pre
        self.sorted = both[1]
        self.device = both.get_device()

    @classmethod
    def on_device(cls, q_begin, q_end, k_begin, k_end, q_rows, k_rows, max_q, max_k, prefix=None,
                  q_full=False, k_full=False):
        """From int32 CUDA tensors that already hold the ranges (a cache whose lengths grow
        on the device, e.g. within a captured graph). max_q and max_k bound the lengths.
        Nothing is read back: disjoint key ranges are the caller's promise, and as the ranges
        may have moved since the last call, every call first clears its outputs. q_full and
        k_full promise that every query (key) row is always some document's, so that there
        is nothing to clear."""
        torch = _torch()
        self = cls.__new__(cls)
        ts = [q_begin, q_end, k_begin, k_end] + ([prefix] if prefix is not None else [])
        for t in ts:
            if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous() or \
                    t.dim() != 1 or t.shape[0] != q_begin.shape[0] or t.device != q_begin.device:
                raise ValueError("ranges must be contiguous int32 vectors of one length on one "
                                 "CUDA device")
        self.device = q_begin.get_device()
        self.q_begin, self.q_end, self.k_begin, self.k_end = ts[:4]
        self.prefix = prefix
        self.sorted = ts + [None] * (5 - len(ts))    # (in the order given)
        self.n = int(q_begin.shape[0])
        self.q_rows, self.k_rows = int(q_rows), int(k_rows)
        self.max_q, self.max_k = int(max_q), int(max_k)
        self.q_full, self.k_full = bool(q_full), bool(k_full)
        self.k_disjoint = self.moving = True
        return self


class Buckets:
    """Distance classes of a learned bias: class c of a side holds the distances from
    start[c] up to start[c + 1]; two_sided gives keys ahead of the query classes of their
    own (else they count as distance 0)."""

    def __init__(self, start: Sequence[int], two_sided: bool = False):
        self.start = [int(x) for x in start]
        self.two_sided = bool(two_sided)

    @property
    def count(self):
        return len(self.start) * (2 if self.two_sided else 1)


def log_buckets(per_side: int, max_distance: int, two_sided: bool = False) -> Buckets:
    """per_side classes a side: the first half one distance each, then steps of equal ratio
    up to max_distance; the last class takes all that is farther. The t-th class past the
    exact ones starts at the smallest a with (a / exact)^n >= (max_distance / exact)^t
    (n of them), compared in integers, or where that is no farther than the class before, at
    the next distance (classes denser than distances end past max_distance)."""
    exact = max(per_side // 2, 1)
    n = per_side - exact
    if per_side < 1 or (n > 0 and max_distance <= exact):
        raise ValueError("need per_side >= 1 and max_distance above the exact classes")
    start = list(range(exact + (1 if n > 0 else 0)))
    for t in range(1, n):
        a = start[-1] + 1
        while a ** n < exact ** (n - t) * max_distance ** t:
            a += 1
        start.append(a)
    return Buckets(start, two_sided)


# ------------------------------------------------------------------ attention
class Attention:
    """What is attended to and how, on the documents' device: documents, heads (a multiple of
    kv_heads), head size, dtype (torch.bfloat16 or torch.float16), causal or full mask (a
    prefix is the documents'), scale (1 / sqrt(dim) if None), cap of the scores by a tanh (0:
    none), and a bias by distance: slopes (float32 CUDA [heads], -slope |distance|) or Buckets
    (the table [heads, buckets.count] of dtype goes with each call)."""

    def __init__(self, docs: Documents, heads: int, kv_heads: int, dim: int, dtype,
                 causal: bool = True, scale: Optional[float] = None, cap: float = 0.0,
                 slopes=None, buckets: Optional[Buckets] = None):
        torch = _torch()
        self.docs, self.heads, self.kv_heads, self.dim = docs, int(heads), int(kv_heads), int(dim)
        self.dtype, self.buckets, self.slopes = dtype, buckets, slopes
        self.device = docs.device
        if slopes is not None and (slopes.dtype != torch.float32 or
                                   slopes.get_device() != self.device or
                                   not slopes.is_contiguous() or tuple(slopes.shape) != (heads,)):
            raise ValueError("slopes must be a contiguous float32 vector of `heads` on the "
                             "documents' device")
        s = gp._Attention()
        s.dtype, s.heads, s.kv_heads, s.dim = _dtype_code(dtype), heads, kv_heads, dim
        s.n_docs, s.q_rows, s.k_rows = docs.n, docs.q_rows, docs.k_rows
        s.max_q, s.max_k = min(docs.max_q, docs.q_rows), min(docs.max_k, docs.k_rows)
        qb, qe, kb, ke, pre = docs.sorted
        s.q_begin, s.q_end, s.k_begin, s.k_end = (t.data_ptr() for t in (qb, qe, kb, ke))
        s.prefix = pre.data_ptr() if docs.prefix is not None else None
        s.causal = 1 if causal else 0
        s.scale = 1.0 / math.sqrt(dim) if scale is None else float(scale)
        s.cap = float(cap)
        s.slopes = slopes.data_ptr() if slopes is not None else None
        if buckets is not None:
            self._start = (C.c_int32 * len(buckets.start))(*buckets.start)
            s.per_side, s.two_sided = len(buckets.start), int(buckets.two_sided)
            s.bucket_start = self._start
        self.struct = s
        self.ref = C.byref(s)
        self.lib = gp.load()
        self.workspace_bytes(False)          # raises if the description is invalid
        self.table_shape = None if buckets is None else (self.heads, buckets.count)
        self.slots = _Slots((docs.q_rows, self.heads, self.dim),
                            (docs.k_rows, self.kv_heads, self.dim), dtype, self.device)

    def workspace_bytes(self, with_grad: bool) -> int:
        lib = gp.load()
        n = lib.gp_attend_workspace_bytes(self.ref, int(with_grad))
        if n == _INVALID:   # (the size has no room for the status: a call without tensors has it)
            none = [None]
            _check(lib.gp_attend_grad(self.ref, *none * 13, 0, None) if with_grad else
                   lib.gp_attend(self.ref, *none * 8, 0, None))
        return n


class AttendBuffers:
    """Outputs and workspaces of attention calls with a description: out, lse
    [heads, q_rows], and with grad dq, dk, dv and (with buckets) dtable, and rest (what
    rounding took from out, which the gradient reads). Rows outside every document are 0
    (lse -inf); a call clears them where its documents may have others than the last call's."""

    def __init__(self, att: Attention, grad: bool = False):
        torch = _torch()
        d = att.docs
        dev = torch.device("cuda", att.device)
        f16 = dict(dtype=att.dtype, device=dev)

        def rows(full, n, heads):
            make = torch.empty if full else torch.zeros
            return make((n, heads, att.dim), **f16)

        self.out = rows(d.q_full, d.q_rows, att.heads)
        self.lse = torch.full((att.heads, d.q_rows), -math.inf, dtype=torch.float32, device=dev)
        self.workspace, self.workspace_bytes = _workspace(att.workspace_bytes(False), att.device)
        self.dq = self.dk = self.dv = self.dtable = self.rest = self.grad_workspace = None
        self.docs = self.grad_docs = d       # whose rows out and lse, and the gradients, hold
        if grad:
            if not d.k_disjoint:
                raise ValueError("gradients need documents whose key rows do not overlap")
            self.rest = rows(d.q_full, d.q_rows, att.heads)
            self.dq = rows(d.q_full, d.q_rows, att.heads)
            self.dk = rows(d.k_full, d.k_rows, att.kv_heads)
            self.dv = rows(d.k_full, d.k_rows, att.kv_heads)
            if att.buckets is not None:
                self.dtable = torch.empty((att.heads, att.buckets.count), **f16)
            self.grad_workspace, self.grad_workspace_bytes = _workspace(
                max(att.workspace_bytes(True), 1), att.device)


class _Slot:
    """One tensor argument of a description's calls: its shape, and the gp_heads struct that
    is filled for each call."""

    __slots__ = ("name", "shape", "dtype", "device", "struct", "ref")

    def __init__(self, name, shape, dtype, device):
        self.name, self.shape, self.dtype, self.device = name, shape, dtype, device
        self.struct = gp._Heads()
        self.ref = C.byref(self.struct)

    def __call__(self, x):
        if x.shape != self.shape or x.dtype is not self.dtype or x.get_device() != self.device:
            raise ValueError(f"{self.name} must be a {self.dtype} tensor of shape {self.shape} on "
                             f"cuda:{self.device}, not {x.dtype} {tuple(x.shape)} on {x.device}")
        s = self.struct
        s.row, s.head, one = x.stride()
        if one != 1:
            raise ValueError(f"{self.name}'s last axis must be contiguous")
        s.data = x.data_ptr()
        return self.ref


class _Slots(threading.local):
    """A description's slots, a set per thread: a call releases the interpreter while the
    library reads them."""

    def __init__(self, q_shape, k_shape, dtype, device):
        self.of = {n: _Slot(n, q_shape, dtype, device) for n in ("q", "out", "rest", "dout", "dq")}
        self.of.update({n: _Slot(n, k_shape, dtype, device) for n in ("k", "v", "dk", "dv")})


def _table(table, att: Attention, name="table"):
    if (table is None) != (att.buckets is None):
        raise ValueError(f"a {name} goes with a description that has buckets")
    if table is None:
        return None
    if table.shape != att.table_shape or table.dtype is not att.dtype or \
            table.get_device() != att.device or not table.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {att.dtype} tensor {att.table_shape} on "
                         f"cuda:{att.device}")
    return table.data_ptr()


def attend_into(att: Attention, q, k, v, bufs: AttendBuffers, table=None):
    """gp_attend into bufs.out and bufs.lse (asynchronous on the current stream). q
    [q_rows, heads, dim], k and v [k_rows, kv_heads, dim]; strides of rows and heads are
    free (multiples of 8)."""
    t, ws, rest = att.slots.of, bufs.workspace, bufs.rest
    args = (att.ref, t["q"](q), t["k"](k), t["v"](v), _table(table, att), t["out"](bufs.out),
            None if rest is None else t["rest"](rest), bufs.lse.data_ptr(),
            None if ws is None else ws.data_ptr(), bufs.workspace_bytes, _stream(q))
    d = att.docs
    if d.moving or bufs.docs is not d:
        if not d.q_full:
            bufs.out.zero_()
            bufs.lse.fill_(-math.inf)
        bufs.docs = d
    _call(att.device, att.lib.gp_attend, args)


def attend(att: Attention, q, k, v, table=None) -> dict:
    bufs = AttendBuffers(att)
    attend_into(att, q, k, v, bufs, table)
    return {"out": bufs.out, "lse": bufs.lse, "_buffers": bufs}


def attend_grad_into(att: Attention, q, k, v, dout, bufs: AttendBuffers, table=None):
    """gp_attend_grad into bufs.dq, dk, dv and dtable, from dout [q_rows, heads, dim] and
    the out and lse that attend_into left in bufs for the same inputs."""
    if bufs.dq is None:
        raise ValueError("the buffers were made without grad")
    if not att.docs.k_disjoint:
        raise ValueError("gradients need documents whose key rows do not overlap")
    t = att.slots.of
    args = (att.ref, t["q"](q), t["k"](k), t["v"](v), _table(table, att), t["out"](bufs.out),
            t["rest"](bufs.rest), bufs.lse.data_ptr(), t["dout"](dout), t["dq"](bufs.dq),
            t["dk"](bufs.dk), t["dv"](bufs.dv), _table(bufs.dtable, att, "dtable"),
            bufs.grad_workspace.data_ptr(), bufs.grad_workspace_bytes, _stream(q))
    d = att.docs
    if d.moving or bufs.grad_docs is not d:
        for x, full in ((bufs.dq, d.q_full), (bufs.dk, d.k_full), (bufs.dv, d.k_full)):
            if not full:
                x.zero_()
        bufs.grad_docs = d
    _call(att.device, att.lib.gp_attend_grad, args)


# ------------------------------------------------------------------ log probabilities
class LogprobBuffers:
    """Outputs and workspace, on a device (the current one if None), of logprob calls on
    [rows, width] logits: logp, entropy, lse [rows], with top the best alternatives top_logp
    and top_id [rows, top], and with grad dlogits and norm [rows, 2] (maxima and log-sums
    apart, which the gradient reads)."""

    def __init__(self, rows: int, width: int, dtype, top: int = 0, grad: bool = False,
                 device: Optional[int] = None):
        torch = _torch()
        self.rows, self.width, self.top, self.dtype = int(rows), int(width), int(top), dtype
        self.device = torch.cuda.current_device() if device is None else int(device)
        dev = torch.device("cuda", self.device)
        f32 = dict(dtype=torch.float32, device=dev)
        self.logp, self.entropy, self.lse = (torch.empty(self.rows, **f32) for _ in range(3))
        self.top_logp = torch.empty((self.rows, self.top), **f32) if top else None
        self.top_id = (torch.empty((self.rows, self.top), dtype=torch.int64, device=dev)
                       if top else None)
        self.dlogits = (torch.empty((self.rows, self.width), dtype=dtype, device=dev)
                        if grad else None)
        self.norm = torch.empty((self.rows, 2), **f32) if grad else None
        self.code = _dtype_code(dtype)
        self.shape = (self.rows, self.width)
        self.lib = gp.load()
        self.workspace, self.workspace_bytes = _workspace(
            self.lib.gp_logprob_workspace_bytes(self.rows, self.width, self.top), self.device)


def _logits(x, bufs, name="logits"):
    if x.shape != bufs.shape or x.dtype is not bufs.dtype or x.get_device() != bufs.device:
        raise ValueError(f"{name} must be a {bufs.dtype} tensor {bufs.shape} on cuda:{bufs.device}")
    row, one = x.stride()
    if one != 1 and bufs.width > 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return x.data_ptr(), row


def _row_vector(x, bufs, dtype, name):
    if x is None:
        return None
    if x.shape != (bufs.rows,) or x.dtype is not dtype or x.get_device() != bufs.device or \
            not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} vector of {bufs.rows} on "
                         f"cuda:{bufs.device}")
    return x.data_ptr()


def logprob_into(logits, targets, bufs: LogprobBuffers, scale: float = 1.0):
    """gp_logprob_norm of logits [rows, width] (the rows' stride is free): log p(targets)
    (int64 [rows]; outside 0..width-1: no target, 0), entropy and lse of
    softmax(scale * logits), and the bufs.top best entries, into bufs."""
    x, stride = _logits(logits, bufs)
    t = _row_vector(targets, bufs, _torch().int64, "targets")
    if t is None:
        raise ValueError("targets are required")
    ws, top = bufs.workspace, bufs.top
    _call(bufs.device, bufs.lib.gp_logprob_norm, (
        bufs.code, x, stride, bufs.rows, bufs.width, scale, t, top, bufs.logp.data_ptr(),
        bufs.entropy.data_ptr(), bufs.lse.data_ptr(),
        None if bufs.norm is None else bufs.norm.data_ptr(),
        bufs.top_logp.data_ptr() if top else None, bufs.top_id.data_ptr() if top else None,
        None if ws is None else ws.data_ptr(), bufs.workspace_bytes, _stream(logits)))


def logprob(logits, targets, top: int = 0, scale: float = 1.0) -> dict:
    bufs = LogprobBuffers(logits.shape[0], logits.shape[1], logits.dtype, top,
                          device=logits.get_device() if logits.is_cuda else None)
    logprob_into(logits, targets, bufs, scale)
    out = {"logp": bufs.logp, "entropy": bufs.entropy, "lse": bufs.lse}
    if top:
        out["top_logp"], out["top_id"] = bufs.top_logp, bufs.top_id
    out["_buffers"] = bufs
    return out


def logprob_grad_into(logits, targets, g_logp, g_entropy, bufs: LogprobBuffers,
                      scale: float = 1.0):
    """gp_logprob_norm_grad into bufs.dlogits, from the gradients (float32 [rows], or None) of
    logp and entropy and what logprob_into left in bufs for the same inputs."""
    torch = _torch()
    if bufs.dlogits is None:
        raise ValueError("the buffers were made without grad")
    x, stride = _logits(logits, bufs)
    dx, dstride = _logits(bufs.dlogits, bufs, "dlogits")
    _call(bufs.device, bufs.lib.gp_logprob_norm_grad, (
        bufs.code, x, stride, bufs.rows, bufs.width, scale,
        _row_vector(targets, bufs, torch.int64, "targets"), bufs.norm.data_ptr(),
        bufs.entropy.data_ptr(), _row_vector(g_logp, bufs, torch.float32, "g_logp"),
        _row_vector(g_entropy, bufs, torch.float32, "g_entropy"), dx, dstride, _stream(logits)))
