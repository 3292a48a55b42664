"""C-ABI checks of the sequence operators that need no GPU: invalid calls are refused before
any device work."""
import ctypes as C

import pytest

from paper_2212_11142_amd import gp


@pytest.fixture(scope="module")
def lib():
    return gp.load()


def _desc(**kw):
    s = gp._Attention()
    base = dict(dtype=0, heads=4, kv_heads=2, dim=64, n_docs=1, q_rows=8, k_rows=8, max_q=8, max_k=8,
                q_begin=16, q_end=16, k_begin=16, k_end=16, causal=1, scale=0.125, cap=0.0)
    base.update(kw)
    for k, v in base.items():
        setattr(s, k, v)
    return s


def _start(*v):
    return (C.c_int32 * len(v))(*v)


INVALID, UNSUPPORTED, WORKSPACE = 1, 4, 5
BAD = [(dict(dtype=2), UNSUPPORTED), (dict(heads=3), INVALID), (dict(kv_heads=0), INVALID),
       (dict(dim=60), UNSUPPORTED), (dict(dim=0), UNSUPPORTED), (dict(dim=136), UNSUPPORTED),
       (dict(n_docs=-1), INVALID), (dict(max_q=9), INVALID), (dict(q_begin=None), INVALID),
       (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID),
       (dict(cap=-1.0), INVALID), (dict(cap=float("inf")), INVALID),
       (dict(prefix=16, causal=0), INVALID), (dict(per_side=65), UNSUPPORTED),
       (dict(per_side=2), INVALID), (dict(per_side=2, bucket_start=_start(1, 2)), INVALID),
       (dict(per_side=2, bucket_start=_start(0, 0)), INVALID),
       (dict(per_side=2, bucket_start=_start(0, 1025)), UNSUPPORTED),
       (dict(per_side=1, bucket_start=_start(0), slopes=16), INVALID)]


def _call(lib, s, grad=False, table=None, ws=None, nbytes=0, tensor=None):
    h = C.byref(tensor or gp._Heads(256, 64 * 4, 64))
    if grad:
        return lib.gp_attend_grad(C.byref(s), h, h, h, table, h, h, 256, h, h, h, h, table, ws, nbytes,
                                  None)
    return lib.gp_attend(C.byref(s), h, h, h, table, h, None, 256, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", BAD)
def test_descriptions_refused(lib, kw, status):
    s = _desc(**kw)
    assert _call(lib, s) == status
    assert lib.gp_last_error()
    assert _call(lib, s, grad=True) == status
    assert lib.gp_attend_workspace_bytes(C.byref(s), 0) == C.c_size_t(-1).value
    assert lib.gp_attend_workspace_bytes(C.byref(s), 1) == C.c_size_t(-1).value


def test_tensors_refused(lib):
    s = _desc()
    for t, status in ((gp._Heads(264, 256, 64), UNSUPPORTED), (gp._Heads(256, 255, 64), UNSUPPORTED),
                      (gp._Heads(256, 256, 63), UNSUPPORTED), (gp._Heads(256, -256, 64), UNSUPPORTED),
                      (gp._Heads(256, 1 << 24, 64), UNSUPPORTED), (gp._Heads(None, 256, 64), INVALID)):
        assert _call(lib, s, tensor=t) == status
    h = C.byref(gp._Heads(256, 256, 64))
    assert lib.gp_attend(C.byref(s), None, h, h, None, h, None, 256, None, 0, None) == INVALID
    assert lib.gp_attend(C.byref(s), h, h, h, None, h, None, None, None, 0, None) == INVALID
    assert lib.gp_attend(None, h, h, h, None, h, None, 256, None, 0, None) == INVALID
    assert _call(lib, s, table=256) == INVALID          # a table without buckets
    assert _call(lib, _desc(per_side=1, bucket_start=_start(0))) == INVALID


def test_workspaces_refused(lib):
    s = _desc(q_rows=64, k_rows=1 << 20, max_q=1, max_k=1 << 16, n_docs=16)
    n = lib.gp_attend_workspace_bytes(C.byref(s), 0)
    g = lib.gp_attend_workspace_bytes(C.byref(s), 1)
    assert n > 0 and g > 0
    assert _call(lib, s, ws=None) == WORKSPACE
    assert _call(lib, s, grad=True, ws=256, nbytes=g - 1) == WORKSPACE
    assert _call(lib, s, grad=True, ws=255, nbytes=g) == WORKSPACE


def test_grids_of_loose_bounds(lib):
    """max_q and max_k may be far above the documents' lengths: the grids stay within 32 bits."""
    big = 1 << 30
    n = lib.gp_attend_workspace_bytes(C.byref(_desc(q_rows=4096, k_rows=big, max_q=1, max_k=big,
                                                    n_docs=4096)), 0)
    assert 0 < n < C.c_size_t(-1).value
    s = _desc()
    blocks = (1 << 24) + 4096 * s.kv_heads
    group = s.heads // s.kv_heads
    assert n <= blocks * min(32, group) * (128 + 2) * 4 + 4096
    s = _desc(q_rows=32, k_rows=1, max_q=32, max_k=1, n_docs=1 << 24, heads=32, kv_heads=32)
    assert _call(lib, s) == UNSUPPORTED


def test_workspace_grows_with_the_work(lib):
    f = lambda **kw: lib.gp_attend_workspace_bytes(C.byref(_desc(q_rows=1 << 16, k_rows=1 << 16,
                                                                 max_q=1 << 10, max_k=1 << 10, **kw)), 1)
    a, b = f(), f(dtype=1)
    c = f(per_side=2, bucket_start=_start(0, 3))
    d = f(per_side=2, two_sided=1, bucket_start=_start(0, 3))
    assert 0 < a < b and a < c < d and f(heads=8) > a


def test_logprob_refused(lib):
    ok = dict(dtype=2, x=256, stride=10, rows=2, width=10, scale=1.0, target=256, top=0, logp=256)

    def call(**kw):
        a = dict(ok)
        a.update(kw)
        return lib.gp_logprob(a["dtype"], a["x"], a["stride"], a["rows"], a["width"], a["scale"],
                              a["target"], a["top"], a["logp"], None, None, a.get("tl"), a.get("ti"),
                              None, 0, None)

    for kw, status in ((dict(dtype=3), INVALID), (dict(x=None), INVALID), (dict(x=258), INVALID),
                       (dict(rows=-1), INVALID), (dict(width=0), INVALID), (dict(stride=-1), INVALID),
                       (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID),
                       (dict(target=None), INVALID), (dict(top=11, tl=256, ti=256), INVALID),
                       (dict(top=129, width=200, tl=256, ti=256), UNSUPPORTED),
                       (dict(top=2), INVALID), (dict(top=-1), INVALID),
                       (dict(width=1 << 20, stride=1 << 20), WORKSPACE)):
        assert call(**kw) == status, kw
    assert call(rows=0, x=None, target=None, logp=None) == 0
    g = lambda **kw: lib.gp_logprob_grad(2, 256, 10, 2, 10, 1.0, kw.get("t", 256), kw.get("lse", 256),
                                         kw.get("e", 256), kw.get("gl", 256), kw.get("ge", 256),
                                         kw.get("dx", 256), kw.get("ds", 10), None)
    assert g(lse=None) == INVALID and g(t=None) == INVALID and g(e=None) == INVALID
    assert g(dx=None) == INVALID and g(ds=9) == INVALID
    assert lib.gp_logprob_workspace_bytes(8, 131072, 20) > 0
    assert lib.gp_logprob_workspace_bytes(8, 1024, 20) == 0
