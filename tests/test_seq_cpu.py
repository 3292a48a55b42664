"""The Python binding of the sequence operators without a GPU: descriptions over host memory,
tensors that only have a shape and an address, and a library that records its calls."""
import ctypes as C
import types

import pytest
import torch

from paper_2212_11142_amd import gp, seq

BF = torch.bfloat16


class Tensor:
    """What the binding asks of a CUDA tensor (index -1: of the host's)."""
    is_cuda = property(lambda self: self.index >= 0)

    def __init__(self, shape, dtype=BF, at=1 << 20, device=0):
        self.shape, self.dtype, self.at, self.index = torch.Size(shape), dtype, at, device

    @property
    def device(self):
        return torch.device("cuda", self.index) if self.index >= 0 else torch.device("cpu")

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
    d.moving, d.device = False, 0
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def attention(docs=None, heads=2, kv_heads=1, dim=64, dtype=BF, **kw):
    return seq.Attention(docs or documents(), heads, kv_heads, dim, dtype, **kw)


def buffers(att, at=1 << 24, **kw):
    d, n = att.docs, att.dim
    b = types.SimpleNamespace(docs=d, grad_docs=d, workspace=None, workspace_bytes=0,
                              grad_workspace=Tensor([1 << 20], torch.uint8), grad_workspace_bytes=1 << 20)
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
    monkeypatch.setattr(seq, "_current_device", lambda: 0, raising=False)


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


# ------------------------------------------------------------------ limits of a launch
BIG = 1 << 30


def description(**kw):
    s = gp._Attention()
    base = dict(dtype=0, heads=4, kv_heads=2, dim=64, n_docs=1, q_rows=8, k_rows=8, max_q=8, max_k=8,
                q_begin=16, q_end=16, k_begin=16, k_end=16, causal=1, scale=0.125, cap=0.0)
    base.update(kw)
    for k, v in base.items():
        setattr(s, k, v)
    return s


def workspace(grad=0, **kw):
    return gp.load().gp_attend_workspace_bytes(C.byref(description(**kw)), grad)


REFUSED = C.c_size_t(-1).value


@pytest.mark.parametrize("docs", [1, 3, 4096, 5000, (1 << 22) - 3])
def test_ranges_of_few_rows_fit_a_launch(docs):
    """A launch has fewer than 2^32 threads, 2^24 - 1 blocks of 256: as many ranges of keys as
    that leaves, from the workspace, which holds 64 + 2 floats of each row of each range."""
    n = workspace(q_rows=docs, k_rows=BIG, max_q=1, max_k=BIG, n_docs=docs)
    rows = 2                                           # the query heads of a key head
    assert n != REFUSED
    ranges = n // (rows * 66 * 4)                      # (of all documents and key heads)
    assert ranges * 256 < 1 << 32
    assert n == 0 or ranges >= 2 * docs


def test_grids_beyond_a_launch_refused():
    assert workspace(q_rows=BIG, max_q=BIG, n_docs=1) == REFUSED             # 2^23 tiles of 4 heads
    assert workspace(q_rows=1 << 29, max_q=1 << 29, n_docs=1, heads=2) != REFUSED
    many = dict(q_rows=1 << 27, k_rows=1 << 27, max_q=1 << 27, max_k=1 << 27, heads=8, kv_heads=8)
    assert workspace(**many) != REFUSED
    assert workspace(grad=1, **many) == REFUSED                              # keys' and queries' blocks
    # many documents of which few can have rows
    assert workspace(q_rows=1 << 16, k_rows=1 << 16, max_q=100, max_k=100, n_docs=1 << 20) != REFUSED
    few = dict(q_rows=1 << 23, max_q=1, n_docs=1 << 23, heads=2)
    assert workspace(kv_heads=1, **few) != REFUSED
    assert workspace(kv_heads=2, **few) == REFUSED


# ------------------------------------------------------------------ threads
def test_threads_share_a_description():
    """A call releases the interpreter: another thread's call with the same description and
    buffers of its own must not change the arguments of this one."""
    import threading
    att = attention()
    entered, done, found = threading.Event(), threading.Event(), {}

    def seen(name, args):
        me = threading.current_thread().name
        if me == "first":
            entered.set()
            assert done.wait(20)
        found[me] = [a._obj.data for a in (args[1], args[2], args[3], args[5])]

    att.lib = Library(seen)

    def call(at):
        seq.attend_into(att, *inputs(att, at=at), buffers(att, at=2 * at))

    first = threading.Thread(target=call, args=(1 << 20,), name="first")
    first.start()
    assert entered.wait(20)
    second = threading.Thread(target=call, args=(1 << 28,), name="second")
    second.start()
    second.join(20)
    done.set()
    first.join(20)
    assert found == {"first": [1 << 20] * 3 + [1 << 21], "second": [1 << 28] * 3 + [1 << 29]}


# ------------------------------------------------------------------ devices
def test_tensors_of_another_device_refused():
    """An address of another device, or of the host, in a launch of the documents' device."""
    att = attention(buckets=seq.Buckets([0, 3]))
    att.lib = Library()
    for device in (1, -1):
        good, table = inputs(att), Tensor((2, 2))
        for n in range(3):
            x = list(good)
            x[n] = inputs(att, device=device)[n]
            with pytest.raises(ValueError):
                seq.attend_into(att, *x, buffers(att), table=table)
            with pytest.raises(ValueError):
                seq.attend_grad_into(att, *x, good[0], buffers(att), table=table)
        away = Tensor((2, 2), device=device)
        with pytest.raises(ValueError):
            seq.attend_into(att, *good, buffers(att), table=away)
        with pytest.raises(ValueError):
            seq.attend_grad_into(att, *good, inputs(att, device=device)[0], buffers(att), table=table)
        for k in ("out", "rest"):
            b = buffers(att)
            getattr(b, k).index = device
            with pytest.raises(ValueError):
                seq.attend_into(att, *good, b, table=table)
        for k in ("out", "rest", "dq", "dk", "dv", "dtable"):
            b = buffers(att)
            getattr(b, k).index = device
            with pytest.raises(ValueError):
                seq.attend_grad_into(att, *good, good[0], b, table=table)
        with pytest.raises(ValueError):
            attention(slopes=Tensor((2,), torch.float32, device=device))
    assert not att.lib.calls


def logprob_buffers(rows, width, lib, device=0):
    f = lambda *s, dtype=torch.float32: Tensor(s, dtype, device=device)
    return types.SimpleNamespace(rows=rows, width=width, top=0, dtype=torch.float32, shape=(rows, width),
                                 code=2, device=device, lib=lib, logp=f(rows), entropy=f(rows), lse=f(rows),
                                 norm=f(rows, 2), top_logp=None, top_id=None, dlogits=f(rows, width),
                                 workspace=None, workspace_bytes=0)


def test_rows_of_another_device_refused():
    lib = Library()
    b = logprob_buffers(4, 10, lib)
    x, t, g = Tensor((4, 10), torch.float32), Tensor((4,), torch.int64), Tensor((4,), torch.float32)
    seq.logprob_into(x, t, b)
    seq.logprob_grad_into(x, t, g, g, b)
    assert len(lib.calls) == 2
    for n in range(4):
        a = [Tensor((4, 10), torch.float32), Tensor((4,), torch.int64), Tensor((4,), torch.float32),
             Tensor((4,), torch.float32)]
        a[n].index = 1
        if n < 2:
            with pytest.raises(ValueError):
                seq.logprob_into(*a[:2], b)
        with pytest.raises(ValueError):
            seq.logprob_grad_into(*a, b)
    assert len(lib.calls) == 2


def test_launches_are_the_tensors_devices(monkeypatch):
    """With another device current, the call makes theirs current."""
    class Device:
        now = [0]

        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.now.append(self.index)

        def __exit__(self, *a):
            self.now.pop()

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(seq, "_current_device", lambda: Device.now[-1], raising=False)
    at = []
    lib = Library(lambda name, args: at.append(Device.now[-1]))
    for device in (0, 1):
        att = attention(documents(device=device))
        att.lib = lib
        b = buffers(att)
        for k in ("out", "rest", "dq", "dk", "dv"):
            getattr(b, k).index = device
        x = inputs(att, device=device)
        seq.attend_into(att, *x, b)
        seq.attend_grad_into(att, *x, x[0], b)
        r, t = Tensor((4, 10), torch.float32, device=device), Tensor((4,), torch.int64, device=device)
        lb = logprob_buffers(4, 10, lib, device)
        seq.logprob_into(r, t, lb)
        seq.logprob_grad_into(r, t, None, None, lb)
    assert at == [0] * 4 + [1] * 4 and Device.now == [0]


# ------------------------------------------------------------------ statuses
@pytest.mark.parametrize("kw,status", [
    (dict(heads=3, kv_heads=2), 1), (dict(dim=60), 4), (dict(dim=136), 4), (dict(dtype=torch.float32), 4),
    (dict(heads=1 << 17), 4), (dict(scale=0.0), 1), (dict(cap=-1.0), 1),
    (dict(buckets=seq.Buckets([1, 2])), 1), (dict(buckets=seq.Buckets([0, 2000])), 4),
    (dict(buckets=seq.Buckets(list(range(65)))), 4),
    (dict(docs=documents(q_rows=(1 << 30) + 1)), 1), (dict(docs=documents(k_rows=(1 << 30) + 1)), 1),
    (dict(docs=documents(q_rows=1 << 30), heads=4), 4)])
def test_descriptions_raise_the_librarys_status(kw, status):
    a = dict(heads=2, kv_heads=1, dim=64)
    a.update(kw)
    with pytest.raises(gp.GPError) as e:
        attention(**a)
    assert e.value.status == status, str(e.value)


def test_gradient_workspaces_raise_the_librarys_status():
    rows = 1 << 27
    att = attention(documents(q_rows=rows, k_rows=rows), heads=8, kv_heads=8)
    with pytest.raises(gp.GPError) as e:
        att.workspace_bytes(True)
    assert e.value.status == 4, str(e.value)


# ------------------------------------------------------------------ buckets
def test_log_buckets_known():
    b = seq.log_buckets(16, 128)
    assert b.start == [0, 1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91] and b.count == 16
    assert seq.log_buckets(16, 128, two_sided=True).count == 32
    assert seq.log_buckets(1, 5).start == [0] and seq.log_buckets(2, 2).start == [0, 1]
    assert seq.log_buckets(8, 5).start == [0, 1, 2, 3, 4, 5, 6, 7]      # denser than the distances
    for a in ((0, 5), (2, 1), (16, 8), (-3, 4)):
        with pytest.raises(ValueError):
            seq.log_buckets(*a)


@pytest.mark.parametrize("per_side,reach", [(16, 128), (32, 128), (7, 50), (64, 1024), (10, 1000), (3, 9)])
def test_log_buckets_are_logarithmic(per_side, reach):
    """Distance d past the exact ones is in the class exact + floor(n log(d / exact) /
    log(reach / exact)), the last one at most: by 60-digit logarithms, beyond doubt where those
    are not within 1e-40 of a class's edge."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    start = seq.log_buckets(per_side, reach).start
    exact = per_side // 2
    n = per_side - exact
    unit = (Decimal(reach) / exact).ln()
    for d in range(2 * reach):
        got = max(c for c in range(per_side) if start[c] <= d)
        if d < exact:
            assert got == d
            continue
        x = n * (Decimal(d) / exact).ln() / unit + Decimal(10) ** -40
        assert got == min(exact + int(x), per_side - 1), d


# ------------------------------------------------------------------ overlapping outputs
def _attend_status(out, grad=None, rows=8, heads=4, ws=None, nbytes=0, **kw):
    """Status of gp_attend (or of gp_attend_grad with `grad` in the named place) whose tensors are
    otherwise in order; 5 (no workspace) means that they all passed."""
    lib, dim = gp.load(), 64
    base = dict(q_rows=rows, max_q=rows, k_rows=1 << 20, max_k=1 << 20, heads=heads, kv_heads=2)
    base.update(kw)
    s = description(**base)
    ok, key = gp._Heads(256, heads * dim, dim), gp._Heads(256, 2 * dim, dim)
    p = lambda x: C.byref(x)
    if grad is None:
        return lib.gp_attend(p(s), p(ok), p(key), p(key), None, p(out), None, 256, ws, nbytes, None)
    t = dict(dq=ok, dk=key, dv=key)
    t[grad] = out
    return lib.gp_attend_grad(p(s), p(ok), p(key), p(key), None, p(ok), p(ok), 256, p(ok), p(t["dq"]),
                              p(t["dk"]), p(t["dv"]), None, None, 0, None)


def test_overlapping_outputs_refused():
    """Rows or heads of an output that share memory would be written by several blocks."""
    heads = lambda row, head: gp._Heads(256, row, head)
    good = [heads(256, 64), heads(64, 512), heads(64, 4096), heads(512, 128), heads(256, 64),
            heads(192, 1536 + 64), heads(128, 1024), heads(128, 64 * 17)]
    for x in good:                               # (heads interleaved with rows among them)
        assert _attend_status(x) == 5, (x.row, x.head)
    for x in (heads(0, 64), heads(256, 0), heads(256, 56), heads(56, 512), heads(64, 64), heads(128, 64),
              heads(192, 64), heads(64, 448), heads(128, 64 * 3 + 8)):
        assert _attend_status(x) == 1, (x.row, x.head)
        assert _attend_status(x, "dq") == 1
    for n in ("dk", "dv"):
        assert _attend_status(heads(128, 64), n) == 5
        assert _attend_status(heads(64, 64), n) == 1 and _attend_status(heads(0, 64), n) == 1
    # one row, or one head: its stride is not used
    assert _attend_status(heads(0, 64), rows=1) == 5
    assert _attend_status(heads(64, 0), rows=8, heads=1, kv_heads=1) == 5
