"""The Python binding of the sequence operators without a GPU: descriptions over host memory,
tensors that only have a shape and an address, and a library that records its calls."""
import ctypes as C
import types

import pytest
import torch

from paper_2212_11142_amd import gp, seq

BF = torch.bfloat16


class Tensor:
    """What the binding asks of a CUDA tensor."""
    is_cuda = True

    def __init__(self, shape, dtype=BF, at=1 << 20, device=0):
        self.shape, self.dtype, self.at, self.index = torch.Size(shape), dtype, at, device
        self.device = torch.device("cuda", device)

    def stride(self):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s)

    def dim(self):
        return len(self.shape)

    def data_ptr(self):
        return self.at

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True


class Library:
    """Takes the place of the loaded library in a description: every call returns 0."""

    def __init__(self, seen=None):
        self.calls, self.seen = [], seen

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            if self.seen:
                self.seen(name, args)
            return 0
        return call


def documents(q_rows=8, k_rows=8, docs=1, max_q=None, max_k=None, **kw):
    d = seq.Documents.__new__(seq.Documents)
    d.sorted = [torch.zeros(max(docs, 1), dtype=torch.int32) for _ in range(4)] + [None]
    d.q_begin, d.q_end, d.k_begin, d.k_end = d.sorted[:4]
    d.prefix, d.n, d.q_rows, d.k_rows = None, docs, q_rows, k_rows
    d.max_q, d.max_k = max_q or q_rows, max_k or k_rows
    d.q_full = d.k_full = d.k_disjoint = True
    d.on_dev = False
    d.device = 0
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def attention(docs=None, heads=2, kv_heads=1, dim=64, dtype=BF, **kw):
    return seq.Attention(docs or documents(), heads, kv_heads, dim, dtype, **kw)


def buffers(att, at=1 << 24, **kw):
    d, n = att.docs, att.dim
    b = types.SimpleNamespace(workspace=None, workspace_bytes=0, grad_workspace=Tensor([1 << 20], torch.uint8),
                              grad_workspace_bytes=1 << 20)
    for k, rows, heads in (("out", d.q_rows, att.heads), ("rest", d.q_rows, att.heads),
                           ("dq", d.q_rows, att.heads), ("dk", d.k_rows, att.kv_heads),
                           ("dv", d.k_rows, att.kv_heads)):
        setattr(b, k, Tensor((rows, heads, n), att.dtype, at))
    b.lse = Tensor((att.heads, d.q_rows), torch.float32, at)
    b.dtable = Tensor(att.table_shape, att.dtype, at) if att.buckets else None
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def inputs(att, at=1 << 20, **kw):
    d = att.docs
    return [Tensor((rows, heads, att.dim), att.dtype, at, **kw)
            for rows, heads in ((d.q_rows, att.heads), (d.k_rows, att.kv_heads), (d.k_rows, att.kv_heads))]


@pytest.fixture(autouse=True)
def _no_stream(monkeypatch):
    monkeypatch.setattr(seq, "_stream", lambda x: None)


def test_stand_ins_pass():
    att = attention(buckets=seq.Buckets([0, 3]))
    att.lib = Library()
    table = Tensor((2, 2))
    q, k, v = inputs(att)
    seq.attend_into(att, q, k, v, buffers(att), table=table)
    seq.attend_grad_into(att, q, k, v, q, buffers(att), table=table)
    assert att.lib.calls == ["gp_attend", "gp_attend_grad"]


def test_table_gradient_of_another_layout_refused():
    """Buffers made for fewer buckets: the table's gradient would be written past their end."""
    att = attention(buckets=seq.Buckets(list(range(64)), True))
    att.lib = Library()
    table, (q, k, v) = Tensor((2, 128)), inputs(att)
    for dtable in (Tensor((2, 2)), None, Tensor((1, 128)), Tensor((2, 128), torch.float32)):
        with pytest.raises(ValueError):
            seq.attend_grad_into(att, q, k, v, q, buffers(att, dtable=dtable), table=table)
    assert not att.lib.calls


def test_gradient_of_overlapping_keys_refused():
    """Two documents' blocks would write the same rows of dk and dv, whoever made the buffers."""
    att = attention(documents(k_disjoint=False, docs=2))
    att.lib = Library()
    q, k, v = inputs(att)
    seq.attend_into(att, q, k, v, buffers(att))
    with pytest.raises(ValueError):
        seq.attend_grad_into(att, q, k, v, q, buffers(att))
    assert att.lib.calls == ["gp_attend"]


def test_norms_are_required():
    lib = gp.load()
    def call(**kw):
        a = dict(norm=256, t=256, e=256, gl=256, ge=256, dx=256, ds=10, rows=2)
        a.update(kw)
        return lib.gp_logprob_norm_grad(2, 256, 10, a["rows"], 10, 1.0, a["t"], a["norm"], a["e"],
                                        a["gl"], a["ge"], a["dx"], a["ds"], None)
    for kw in (dict(norm=None), dict(t=None), dict(e=None), dict(dx=None), dict(ds=9), dict(rows=-1)):
        assert call(**kw) == 1, kw
    assert call(rows=0, norm=None) == 0
    assert lib.gp_logprob_norm(3, 256, 10, 2, 10, 1.0, 256, 0, 256, None, None, 256, None, None, None, 0,
                               None) == 1
