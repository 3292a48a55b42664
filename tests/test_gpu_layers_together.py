"""The layers' operators together, as a surrogate uses them: a layer's gradients against float64, the
example that trains with them, and calls within captured graphs, on other streams and from threads."""
import os
import sys
import threading

import numpy as np
import pytest
import torch

from paper_2212_11142_amd import layers, seq

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ex():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import in_context_surrogate
    finally:
        sys.path.pop(0)
    return in_context_surrogate


def rand(g, *shape, dtype=BF, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


# ------------------------------------------------------------------ a layer's gradients
def plain_layer(ex, layer, x, added, sizes):
    """The example's rotary layer in float64, from its definition."""
    def norm(h, i):
        d = h - h.mean(1, keepdim=True)
        s = (d.square().mean(1, keepdim=True) + 1e-5).rsqrt()
        return d * s * layer.scale[i] + layer.shift[i]

    def rotate(y, pos):
        f = 1000.0 ** (-torch.arange(0, ex.HEAD, 2, dtype=torch.float64, device="cuda") / ex.HEAD)
        t = (pos[:, None] * f)[:, None, :]
        a, b = y[..., :ex.HEAD // 2], y[..., ex.HEAD // 2:]
        return torch.cat([a * t.cos() - b * t.sin(), a * t.sin() + b * t.cos()], -1)

    x = x + added
    y = (norm(x, 0) @ layer.qkv.weight.t()).view(-1, ex.HEADS + 2 * ex.KV_HEADS, ex.HEAD)
    pos = torch.cat([torch.arange(n + m, device="cuda", dtype=torch.float64) for n, m in sizes])
    q, k, v = y.split([ex.HEADS, ex.KV_HEADS, ex.KV_HEADS], 1)
    q, k = rotate(q, pos), rotate(k, pos)
    out, r = [], 0
    for n, m in sizes:
        rows = slice(r, r + n + m)
        r += n + m
        group = ex.HEADS // ex.KV_HEADS
        kk, vv = (z[rows].repeat_interleave(group, 1).transpose(0, 1) for z in (k, v))
        s = q[rows].transpose(0, 1) @ kk.transpose(1, 2) / ex.HEAD ** 0.5
        s = ex.CAP * torch.tanh(s / ex.CAP)
        i = torch.arange(n + m, device="cuda")
        seen = (i[None, :] <= i[:, None]) | (i[None, :] < n)
        out.append((torch.softmax(s.masked_fill(~seen, float("-inf")), -1) @ vv).transpose(0, 1))
    x = x + torch.cat(out).reshape(-1, ex.HEADS * ex.HEAD) @ layer.out.weight.t()
    z = norm(x, 1)
    g, u = z @ layer.gate.weight.t(), z @ layer.up.weight.t()
    return x, (torch.nn.functional.silu(g) * u) @ layer.down.weight.t()


def test_layer_gradients(ex):
    """fp16, half step 2^-11: a rounding is off by 2^-11 / sqrt(3) = 0.00028 of a value's size at most
    (as a root mean square over a step's places). On the longest way, from the output back to the first
    norm and its weights, lie some 25 roundings: sqrt(25) times that if they are independent, 0.0014,
    and at most 25 times, 0.007, if all add up."""
    torch.manual_seed(3)
    layer = ex.RotaryLayer(dtype=FP).cuda().half()
    with torch.no_grad():
        for p in list(layer.scale) + list(layer.shift):
            p.add_(0.2 * torch.randn_like(p))
    sizes = [(30, 20), (1, 0), (65, 64), (7, 130)]
    rows = sum(n + m for n, m in sizes)
    g = torch.Generator().manual_seed(4)
    x, added, dx, da = (rand(g, rows, ex.DIM, dtype=FP) for _ in range(4))
    docs = seq.Documents([n + m for n, m in sizes], prefix=[n for n, _ in sizes])
    att = seq.Attention(docs, ex.HEADS, ex.KV_HEADS, ex.HEAD, FP, cap=ex.CAP)
    xs = [v.clone().requires_grad_() for v in (x, added)]
    got = layer(*xs, att, layers.positions(docs))
    torch.autograd.backward(got, (dx, da))
    mine = {n: p.grad.double() for n, p in layer.named_parameters()}
    mine |= {"x": xs[0].grad.double(), "added": xs[1].grad.double()}
    ref = ex.RotaryLayer(dtype=FP).cuda().double()
    ref.load_state_dict({k: v.double() for k, v in layer.state_dict().items()})
    ys = [v.double().requires_grad_() for v in (x, added)]
    want = plain_layer(ex, ref, *ys, sizes)
    torch.autograd.backward(want, (dx.double(), da.double()))
    theirs = {n: p.grad for n, p in ref.named_parameters()} | {"x": ys[0].grad, "added": ys[1].grad}
    for a, b in zip(got, want):
        assert (a.double() - b).norm() <= 0.007 * b.norm()
    off = {n: ((mine[n] - theirs[n]).norm() / theirs[n].norm()).item() for n in theirs}
    print(off)
    assert max(off.values()) <= 0.007, off


def test_example(ex):
    lines = []
    r = ex.main(steps=60, candidates=1027, log=lines.append, order="rotary")
    print("\n".join(lines))
    assert np.isfinite(r["losses"]).all()
    assert r["ei"].isfinite().all() and (r["ei"] >= 0).all()
    # the same sums in other orders, rounded to 8 bits some dozen times on the way
    assert r["diff"] < 0.5


# ------------------------------------------------------------------ graphs, streams, threads
def operators():
    """name -> (call, its outputs, inputs that a replay changes)."""
    g = torch.Generator().manual_seed(5)
    out = {}
    for name, rows, width, dtype in (("norm", 70, 520, BF), ("norm-wide", 3, 40000, BF)):
        n = layers.Norm(width, dtype, weight=torch.float32, bias=True)
        x, r, d, s = (rand(g, rows, width, dtype=dtype) for _ in range(4))
        w, b = rand(g, width, dtype=torch.float32), rand(g, width, dtype=torch.float32)
        bufs = layers.NormBuffers(n, rows, residual=True, grad=True)

        def call(n=n, x=x, r=r, d=d, s=s, w=w, b=b, bufs=bufs):
            layers.norm_into(n, x, bufs, weight=w, bias=b, residual=r)
            layers.norm_grad_into(n, bufs.sum, d, bufs, weight=w, dsum=s)

        out[name] = (call, [bufs.out, bufs.sum, bufs.dx, bufs.dweight, bufs.dbias], [x, d])
    rot = layers.Rotary(64, BF, rotated=32)
    q, k, v = (rand(g, 9, h, 64) for h in (4, 2, 2))
    p = torch.arange(9, dtype=torch.int32).cuda()
    o, kc, vc = torch.empty_like(q), rand(g, 40, 2, 64), rand(g, 40, 2, 64)


    slots = (p.long() * 2).clone()

    def call(slots=slots):
        layers.append_into(rot, p, slots, q, k, v, o, kc, vc)

    out["append"] = (call, [o, kc, vc], [q, k, v])
    for name, rows, width, hidden in (("gated-few", 5, 264, 136), ("gated", 150, 136, 200),
                                      ("gated-large", 2050, 136, 2056)):
        t = layers.Gated(width, hidden, FP, activation="gelu")
        x, wg, wu, d = (rand(g, *s, dtype=FP, scale=0.5) for s in ((rows, width), (hidden, width), (hidden, width),
                                                                 (rows, hidden)))
        bufs = layers.GatedBuffers(t, rows, grad=True)

        def call(t=t, x=x, wg=wg, wu=wu, d=d, bufs=bufs):
            layers.gated_into(t, x, wg, wu, bufs)
            layers.gated_grad_into(t, x, wg, wu, d, bufs)

        out[name] = (call, [bufs.out, bufs.dx, bufs.dw_gate, bufs.dw_up], [x, d])
    return out


NAMES = ["norm", "norm-wide", "append", "gated-few", "gated", "gated-large"]


@pytest.fixture(scope="module")
def ops():
    return operators()


def snapshot(ts):
    return [t.clone() for t in ts]


def same(a, b):
    return all(torch.equal(x.view(torch.uint8) if x.dtype.itemsize == 1 else x, y.view(x.dtype)) for x, y in zip(a, b))


@pytest.mark.parametrize("name", NAMES)
def test_the_same_twice_and_replayed(ops, name):
    """Bit for bit: two eager calls, and replays of a captured one with other inputs, eager work and
    synchronisations between them."""
    call, outputs, inputs = ops[name]
    first = snapshot(inputs)
    call()
    want = snapshot(outputs)
    for t in outputs:
        t.fill_(float("nan")) if name != "append" else None
    call()
    assert same(outputs, want)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    others = [x * 0.5 for x in first]
    for k in range(4):
        for x, a, b in zip(inputs, first, others):
            x.copy_(b if k % 2 else a)
        call()
        want = snapshot(outputs)
        if name != "append":
            for t in outputs:
                t.fill_(float("nan"))
        if k == 2:
            torch.cuda.synchronize()
        graph.replay()
        assert same(outputs, want), (name, k)
    for x, a in zip(inputs, first):
        x.copy_(a)


@pytest.mark.parametrize("name", NAMES)
def test_another_stream(ops, name):
    call, outputs, inputs = ops[name]
    call()
    want = snapshot(outputs)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        if name != "append":
            for t in outputs:
                t.zero_()
        call()
        got = snapshot(outputs)
    s.synchronize()
    assert same(got, want)


def test_two_graphs_with_buffers_of_their_own():
    """Two captured gradients, each with its own buffers, replayed one after the other."""
    g = torch.Generator().manual_seed(6)
    t = layers.Gated(136, 200, BF)
    wg, wu = rand(g, 200, 136), rand(g, 200, 136)
    cases = []
    for rows in (33, 300):
        x, d, b = rand(g, rows, 136), rand(g, rows, 200), layers.GatedBuffers(t, rows, grad=True)
        layers.gated_grad_into(t, x, wg, wu, d, b)
        want = snapshot([b.dx, b.dw_gate, b.dw_up])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layers.gated_grad_into(t, x, wg, wu, d, b)
        cases.append((graph, b, want))
    for _ in range(3):
        for graph, b, _ in cases:
            b.dx.zero_(), b.dw_gate.zero_(), b.dw_up.zero_()
            graph.replay()
        for _, b, want in cases:
            assert same([b.dx, b.dw_gate, b.dw_up], want)


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_replayed(bits):
    """A captured step with rate and number on the device: replays are the steps that follow."""
    g = torch.Generator().manual_seed(7)
    shapes = [(300,), (70, 5), (1,)]
    w = [rand(g, *s, dtype=torch.float32) for s in shapes]
    grads = [rand(g, *s) for s in shapes]
    runs = []
    for captured in (False, True):
        m = snapshot(w)
        p = [x.to(BF) for x in m]
        opt = layers.AdamW(p, masters=m, state_bits=bits)
        lr, step = torch.zeros((), device="cuda"), torch.zeros((), dtype=torch.int64, device="cuda")
        graph = None
        if captured:
            keep = snapshot(m + p)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            step.fill_(1)
            with torch.cuda.graph(graph):
                layers.adamw_into(opt, grads, lr, step, seed=3)
            assert same(m + p, keep)                       # (captured, not run)
        for t in range(1, 5):
            rate = float(np.float32(0.01 / t))
            if captured:
                lr.fill_(rate), step.fill_(t)
                graph.replay()
            else:
                layers.adamw_into(opt, grads, rate, t, seed=3)
            if t == 2:
                torch.cuda.synchronize()
        runs.append(snapshot(m + p + [opt.m_all.view(torch.uint8), opt.v_all.view(torch.uint8)]))
    # (the corrections are computed in 64 bits on either side, by two libraries' powers: a step of fp32 apart
    # at most, 2^-23 of an update of 0.01 beside weights of some 1)
    n = len(shapes)
    for i, (a, b) in enumerate(zip(*runs)):
        if i < n:
            assert (a - b).abs().max() <= 4 * 2.0 ** -23 * 0.05 + 2.0 ** -23 * a.abs().max()
        elif i < 2 * n:
            assert (a.float() - b.float()).abs().max() <= 2.0 ** -7 * a.float().abs().max()
        else:
            assert torch.equal(a, b)


def test_threads_share_a_description():
    """Four threads, a description each, buffers and streams of their own."""
    g = torch.Generator().manual_seed(8)
    rot = layers.Rotary(64, BF)
    t = layers.Gated(72, 80, BF)
    n = layers.Norm(72, BF)
    wg, wu = rand(g, 80, 72), rand(g, 80, 72)
    work = []
    for i in range(4):
        rows = 20 + 37 * i
        x, y, p = rand(g, rows, 72), rand(g, rows, 3, 64), torch.arange(rows, dtype=torch.int32).cuda()
        want = [layers.gated(t, x, wg, wu), layers.rotate(rot, p, y), layers.norm(n, x)["out"]]
        work.append((x, y, p, want))
    torch.cuda.synchronize()
    bad = []

    def go(i):
        x, y, p, want = work[i]
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(50):
                got = [layers.gated(t, x, wg, wu), layers.rotate(rot, p, y), layers.norm(n, x)["out"]]
                s.synchronize()
                if not same(got, want):
                    bad.append(i)

    threads = [threading.Thread(target=go, args=(i,)) for i in range(4)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not bad


# ------------------------------------------------------------------ values that are not finite
def test_gated_keeps_rows_apart():
    """A row of x that is not finite reaches its own row of out and of dx alone."""
    g = torch.Generator().manual_seed(9)
    for rows, width, hidden in ((9, 72, 40), (200, 200, 264), (2100, 136, 2056)):
        t = layers.Gated(width, hidden, BF)
        x, wg, wu, d = rand(g, rows, width), rand(g, hidden, width), rand(g, hidden, width), rand(g, rows, hidden)
        b = layers.GatedBuffers(t, rows, grad=True)
        layers.gated_into(t, x, wg, wu, b)
        layers.gated_grad_into(t, x, wg, wu, d, b)
        out, dx = b.out.clone(), b.dx.clone()
        x[rows // 2, 3] = float("nan")
        x[rows - 1, width - 1] = float("inf")
        layers.gated_into(t, x, wg, wu, b)
        layers.gated_grad_into(t, x, wg, wu, d, b)
        rest = [i for i in range(rows) if i not in (rows // 2, rows - 1)]
        assert torch.equal(b.out[rest], out[rest]) and torch.equal(b.dx[rest], dx[rest])
        assert b.out[rows // 2].isnan().all() and b.dx[rows // 2].isnan().all()


def test_what_lies_behind_rows_is_not_read():
    """x, weights and dout with NaN behind their rows' ends and after the last row."""
    g = torch.Generator().manual_seed(10)
    for rows, width, hidden in ((7, 72, 40), (150, 200, 136), (2100, 136, 2056)):
        t = layers.Gated(width, hidden, FP, activation="gelu")
        plain, wide = [], []
        for n, m in ((rows, width), (hidden, width), (hidden, width), (rows, hidden)):
            big = torch.full((n + 300, m + 24), float("nan"), dtype=FP, device="cuda")
            big[:n, :m] = rand(g, n, m, dtype=FP, scale=0.3)
            wide.append(big[:n, :m])
            plain.append(wide[-1].contiguous())
        a, b = (layers.GatedBuffers(t, rows, grad=True) for _ in range(2))
        for bufs, args in ((a, plain), (b, wide)):
            layers.gated_into(t, *args[:3], bufs)
            layers.gated_grad_into(t, *args, bufs)
        assert same([a.out, a.dx, a.dw_gate, a.dw_up], [b.out, b.dx, b.dw_gate, b.dw_up])
        assert a.dx.isfinite().all() and a.dw_up.isfinite().all()


def test_outputs_stay_within_their_rows():
    """Outputs as rows of a larger matrix: what lies behind and after them is left as it was."""
    g = torch.Generator().manual_seed(11)
    for rows, width, hidden in ((5, 72, 40), (150, 200, 136), (2100, 136, 2056)):
        t = layers.Gated(width, hidden, BF)
        x, wg, wu, d = rand(g, rows, width), rand(g, hidden, width), rand(g, hidden, width), rand(g, rows, hidden)
        b = layers.GatedBuffers(t, rows, grad=True)
        layers.gated_into(t, x, wg, wu, b)
        layers.gated_grad_into(t, x, wg, wu, d, b)
        want = snapshot([b.out, b.dx, b.dw_gate, b.dw_up])
        big = []
        for name in ("out", "dx", "dw_gate", "dw_up"):
            y = getattr(b, name)
            z = torch.full((y.shape[0] + 9, y.shape[1] + 16), 7.0, dtype=BF, device="cuda")
            setattr(b, name, z[:y.shape[0], :y.shape[1]])
            big.append((z, y.shape))
        layers.gated_into(t, x, wg, wu, b)
        layers.gated_grad_into(t, x, wg, wu, d, b)
        assert same([b.out, b.dx, b.dw_gate, b.dw_up], want)
        for z, (n, m) in big:
            assert (z[n:] == 7).all() and (z[:, m:] == 7).all()
