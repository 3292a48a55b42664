"""C-ABI checks of the layers' operators that need no GPU: invalid calls are refused before any device
work, and sizes of workspaces."""
import ctypes as C

import pytest

from paper_2212_11142_amd import gp

INVALID, UNSUPPORTED, WORKSPACE = 1, 4, 5
NONE = C.c_size_t(-1).value
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return gp.load()


def make(kind, base, kw):
    s = kind()
    for k, v in {**base, **kw}.items():
        setattr(s, k, v)
    return s


# ------------------------------------------------------------------ norms
def norm(**kw):
    return make(gp._Norm, dict(dtype=0, weight_dtype=0, width=10, centre=1, eps=1e-5), kw)


def call_norm(lib, spec=None, rows=2, **kw):
    a = dict(x=256, xs=10, r=None, rs=0, w=None, b=None, out=512, os=10, sum=None, ss=0, stats=None)
    a.update(kw)
    return lib.gp_norm(None if spec is None else C.byref(spec), rows, *a.values(), None)


def call_norm_grad(lib, spec=None, rows=2, **kw):
    a = dict(h=256, hs=10, stats=256, w=None, d=256, ds=10, dsum=None, dss=0, dx=512, dxs=10, dw=None, db=None,
             ws=256, n=1 << 30)
    a.update(kw)
    return lib.gp_norm_grad(None if spec is None else C.byref(spec), rows, *a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(weight_dtype=1), UNSUPPORTED),
    (dict(dtype=2, weight_dtype=0), UNSUPPORTED), (dict(width=0), INVALID), (dict(width=(1 << 24) + 1), UNSUPPORTED),
    (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID)])
def test_norm_descriptions_refused(lib, kw, status):
    s = norm(**kw)
    assert call_norm(lib, s) == status and call_norm_grad(lib, s) == status
    assert lib.gp_last_error()
    assert lib.gp_norm_grad_workspace_bytes(C.byref(s), 2) == NONE


def test_norm_calls_refused(lib):
    s = norm()
    assert call_norm(lib, None) == INVALID and call_norm_grad(lib, None) == INVALID
    for kw in (dict(rows=-1), dict(x=None), dict(x=257), dict(out=None), dict(out=513), dict(xs=-1), dict(os=9),
               dict(w=257), dict(b=257), dict(sum=768, ss=10), dict(r=768, rs=10),
               dict(r=768, rs=10, sum=1024, ss=9), dict(r=768, rs=10, sum=512, ss=10), dict(r=769, rs=10, sum=1024, ss=10)):
        assert call_norm(lib, s, **kw) == INVALID, kw
    for kw in (dict(rows=-1), dict(h=None), dict(stats=None), dict(d=None), dict(dx=None), dict(dxs=9), dict(dx=513),
               dict(dsum=257, dss=10), dict(dsum=256, dss=-1), dict(w=257), dict(dw=257), dict(db=257)):
        assert call_norm_grad(lib, s, **kw) == INVALID, kw
    n = lib.gp_norm_grad_workspace_bytes(C.byref(s), 2)
    assert 0 < n < NONE
    for kw in (dict(ws=None), dict(ws=255), dict(n=n - 1)):
        assert call_norm_grad(lib, s, dw=1024, **kw) == WORKSPACE, kw
    assert lib.gp_norm_grad_workspace_bytes(C.byref(s), -1) == NONE
    # no rows: nothing to do
    assert call_norm(lib, s, rows=0, x=None, out=None) == 0


def test_norm_statistics_at_odd_addresses_refused(lib):
    assert call_norm(lib, norm(), stats=258) == INVALID and call_norm_grad(lib, norm(), stats=258) == INVALID


def test_norm_workspaces(lib):
    """As many sums as blocks that are resident at once, however many rows; wide rows' means beside."""
    f = lambda rows, **kw: lib.gp_norm_grad_workspace_bytes(C.byref(norm(**kw)), rows)     # noqa: E731
    assert f(0) == 0
    assert f(1 << 30, width=1024) == f(1 << 20, width=1024) <= 1024 * 2 * 1024 * 4
    assert f(10, width=1 << 24) >= 10 * 8 + 2 * (1 << 24) * 4
    assert f(1 << 20, width=40000) >= (1 << 20) * 8


# ------------------------------------------------------------------ rotary positions
def rotary(**kw):
    return make(gp._Rotary, dict(dtype=0, dim=64, rotated=32, interleaved=0, magnitude=1.0, turns=256), kw)


def heads(data=256, row=256, head=64):
    return C.byref(gp._Heads(data, row, head))


def call_rotate(lib, spec, rows=2, pos=256, n=4, x=None, out=None):
    return lib.gp_rotate(None if spec is None else C.byref(spec), rows, pos, n, x or heads(), out or heads(), 0, None)


def call_append(lib, spec, rows=2, pos=256, slots=256, n=4, kv=2, cache=9, **kw):
    a = {k: kw.get(k, heads()) for k in ("q", "out", "k", "v", "kc", "vc")}
    return lib.gp_rotate_append(None if spec is None else C.byref(spec), rows, pos, slots, n, a["q"], a["out"], kv,
                                a["k"], a["v"], cache, a["kc"], a["vc"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), INVALID), (dict(dim=60), UNSUPPORTED), (dict(dim=0), UNSUPPORTED), (dict(dim=136), UNSUPPORTED),
    (dict(rotated=0), INVALID), (dict(rotated=31), INVALID), (dict(rotated=66), INVALID), (dict(turns=None), INVALID),
    (dict(turns=260), INVALID), (dict(magnitude=NAN), INVALID), (dict(magnitude=INF), INVALID)])
def test_rotary_descriptions_refused(lib, kw, status):
    assert call_rotate(lib, rotary(**kw)) == status and call_append(lib, rotary(**kw)) == status
    assert lib.gp_last_error()


def test_rotary_calls_refused(lib):
    s = rotary()
    assert call_rotate(lib, None) == INVALID and call_append(lib, None) == INVALID
    for kw, status in ((dict(rows=-1), INVALID), (dict(rows=(1 << 30) + 1), UNSUPPORTED), (dict(pos=None), INVALID),
                       (dict(pos=258), INVALID), (dict(n=0), INVALID), (dict(n=65537), UNSUPPORTED),
                       (dict(x=heads(None)), INVALID), (dict(x=heads(264)), UNSUPPORTED),
                       (dict(x=heads(row=252)), UNSUPPORTED), (dict(x=heads(head=-8)), UNSUPPORTED),
                       (dict(x=heads(row=(1 << 23) + 8)), UNSUPPORTED), (dict(out=heads(row=56)), INVALID),
                       (dict(out=heads(head=56)), INVALID), (dict(out=heads(row=192)), INVALID),
                       (dict(out=heads(row=64, head=64)), INVALID)):
        assert call_rotate(lib, s, **kw) == status, kw
    for kw, status in ((dict(slots=None), INVALID), (dict(slots=260), INVALID), (dict(kv=0), INVALID),
                       (dict(cache=-1), INVALID), (dict(kc=heads(None)), INVALID), (dict(vc=heads(264)), UNSUPPORTED),
                       (dict(kc=heads(row=64, head=64)), INVALID), (dict(v=heads(None)), INVALID),
                       (dict(q=heads(264)), UNSUPPORTED)):
        assert call_append(lib, s, **kw) == status, kw
    # no rows: nothing to do (whatever lies in front of the cache's rows)
    assert call_rotate(lib, s, rows=0, pos=None, x=heads(None), out=heads(None)) == 0
    assert call_append(lib, s, rows=0, pos=None, slots=None) == 0


# ------------------------------------------------------------------ gated block
def gated(**kw):
    return make(gp._Gated, dict(dtype=0, width=64, hidden=72, activation=0), kw)


def matrix(data=256, row=72):
    return C.byref(gp._Matrix(data, row))


def call_gated(lib, spec, rows=2, **kw):
    return lib.gp_gated(None if spec is None else C.byref(spec), rows,
                        *[kw.get(k, matrix()) for k in ("x", "wg", "wu", "out")], None)


def call_gated_grad(lib, spec, rows=2, ws=256, n=1 << 40, **kw):
    return lib.gp_gated_grad(None if spec is None else C.byref(spec), rows, *[
        kw.get(k, matrix()) for k in ("x", "wg", "wu", "dout", "dx", "dwg", "dwu")], ws, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), UNSUPPORTED), (dict(activation=2), INVALID), (dict(width=60), UNSUPPORTED),
    (dict(hidden=0), UNSUPPORTED), (dict(hidden=76), UNSUPPORTED), (dict(width=(1 << 21) + 8), UNSUPPORTED)])
def test_gated_descriptions_refused(lib, kw, status):
    s = gated(**kw)
    assert call_gated(lib, s) == status and call_gated_grad(lib, s) == status
    assert lib.gp_gated_grad_workspace_bytes(C.byref(s), 2) == NONE


def test_gated_calls_refused(lib):
    s = gated()
    assert call_gated(lib, None) == INVALID and call_gated_grad(lib, None) == INVALID
    assert call_gated(lib, s, rows=-1) == INVALID
    for name in ("x", "wg", "wu", "out", "dout", "dx", "dwg", "dwu"):
        call = call_gated if name in ("x", "wg", "wu", "out") else call_gated_grad
        for m, status in ((None, INVALID), (matrix(None), INVALID), (matrix(264), UNSUPPORTED), (matrix(row=68), UNSUPPORTED),
                          (matrix(row=-8), UNSUPPORTED), (matrix(row=(1 << 21) + 8), UNSUPPORTED)):
            assert call(lib, s, **{name: m}) == status, (name, status)
        if name in ("out", "dx", "dwg", "dwu"):
            assert call(lib, s, **{name: matrix(row=56)}) == INVALID, name
    n = lib.gp_gated_grad_workspace_bytes(C.byref(s), 2)
    assert n >= 2 * 2 * 72 * 2
    for kw in (dict(ws=None), dict(ws=255), dict(n=n - 1)):
        assert call_gated_grad(lib, s, **kw) == WORKSPACE, kw
    assert call_gated(lib, s, rows=0, x=matrix(None), out=matrix(None)) == 0
    big = gated(width=8, hidden=1 << 21)
    assert call_gated(lib, big, rows=1 << 30, out=matrix(row=1 << 21)) == UNSUPPORTED


def test_gated_workspaces(lib):
    """dg and du, and the parts of split sums: no more parts than make the resident blocks' number."""
    for rows, width, hidden in ((1, 8, 8), (1000, 520, 1368), (16384, 1024, 4096), (1 << 20, 64, 64),
                                (64, 4096, 16384), (100000, 8, 2048)):
        n = lib.gp_gated_grad_workspace_bytes(C.byref(gated(width=width, hidden=hidden)), rows)
        own = 2 * rows * hidden * 2
        assert own <= n <= own + 1024 + 600 * 256 * 256 * 4, (rows, width, hidden)


# ------------------------------------------------------------------ AdamW
def adamw(**kw):
    return make(gp._AdamW, dict(dtype=0, grad_dtype=0, state_bits=32, beta1=0.9, beta2=0.999, lr=0.1, eps=1e-8,
                                decay=0.0, step=1), kw)


def call_adamw(lib, spec, count=1, grad=256, tensors=True, **kw):
    t = make(gp._AdamWTensor, dict(param=256, master=256, m=256, v=256, scales=None, count=0), kw)
    return lib.gp_adamw(None if spec is None else C.byref(spec), count, C.byref(t) if tensors else None,
                        (C.c_void_p * 1)(grad), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), INVALID), (dict(grad_dtype=1), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
    (dict(state_bits=16), UNSUPPORTED), (dict(beta1=1.0), INVALID), (dict(beta2=-0.1), INVALID), (dict(beta1=NAN), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=NAN), INVALID), (dict(eps=1e-60), INVALID), (dict(eps=1e60), INVALID), (dict(decay=INF), INVALID), (dict(lr=NAN), INVALID),
    (dict(step=0), INVALID), (dict(lr_device=258), INVALID), (dict(step_device=260), INVALID), (dict(factor=257), INVALID)])
def test_adamw_descriptions_refused(lib, kw, status):
    assert call_adamw(lib, adamw(**kw)) == status
    assert lib.gp_last_error()


def test_adamw_calls_refused(lib):
    s = adamw()
    assert call_adamw(lib, None) == INVALID and call_adamw(lib, s, count=-1) == INVALID
    assert call_adamw(lib, s, tensors=False) == INVALID
    for kw, status in ((dict(count=-1), INVALID), (dict(count=(1 << 40) + 1), UNSUPPORTED), (dict(param=None), INVALID),
                       (dict(m=None), INVALID), (dict(v=None), INVALID), (dict(param=257), INVALID), (dict(master=258), INVALID),
                       (dict(m=258), INVALID), (dict(scales=256), INVALID)):
        t = make(gp._AdamWTensor, dict(param=256, master=256, m=256, v=256, scales=None, count=5), kw)
        assert lib.gp_adamw(C.byref(s), 1, C.byref(t), (C.c_void_p * 1)(256), None) == status, kw
    t = make(gp._AdamWTensor, dict(param=256, master=None, m=256, v=256, count=5), {})
    assert lib.gp_adamw(C.byref(s), 1, C.byref(t), (C.c_void_p * 1)(257), None) == INVALID
    assert lib.gp_adamw(C.byref(adamw(state_bits=8)), 1, C.byref(t), (C.c_void_p * 1)(256), None) == INVALID
    full = adamw(dtype=2, grad_dtype=2)
    t.master = 256
    assert lib.gp_adamw(C.byref(full), 1, C.byref(t), (C.c_void_p * 1)(256), None) == INVALID
    # nothing to do: no tensors, empty ones, none with a gradient
    assert lib.gp_adamw(C.byref(s), 0, None, None, None) == 0
    t.count = 0
    assert lib.gp_adamw(C.byref(s), 1, C.byref(t), (C.c_void_p * 1)(256), None) == 0
    t.count = 5
    assert lib.gp_adamw(C.byref(s), 1, C.byref(t), (C.c_void_p * 1)(None), None) == 0
