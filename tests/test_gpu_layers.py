"""The layers' kernels against their float64 oracle: sizes, types, strides, directions, refusals.

Tolerances: half a step of the result's type, relative (bf16 2^-8, fp16 2^-11, fp32 2^-24; fp16 below
its normal numbers 2^-25 absolute), and what fp32 arithmetic may take, from the oracle's bounds.
"""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import gp_layers as ol
from paper_2212_11142_amd import gp, layers, seq

pytestmark = pytest.mark.gpu

BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32
HALF = {BF: 2.0 ** -8, FP: 2.0 ** -11, F32: 2.0 ** -24}
SMALL = {BF: 0.0, FP: 2.0 ** -25, F32: 0.0}


def rand(gen, *shape, dtype=F32, scale=1.0, at=0.0):
    return (torch.randn(shape, generator=gen) * scale + at).to(dtype).cuda()


def gen(seed=0):
    return torch.Generator().manual_seed(seed)


def host(x):
    return x.detach().double().cpu().numpy()


def near(got, want, bound, dtype, name="out"):
    got = host(got)
    tol = np.abs(want) * HALF[dtype] + SMALL[dtype] + bound * (1 + HALF[dtype])
    off = np.abs(got - want)
    bad = ~(off <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:4].tolist(),
                           got[bad][:4], want[bad][:4], tol[bad][:4])


def strided(x, by):
    """The same rows with room behind each."""
    y = torch.full((x.shape[0], x.shape[1] + by), float("nan"), dtype=x.dtype, device=x.device)
    y[:, :x.shape[1]] = x
    return y[:, :x.shape[1]]


# ------------------------------------------------------------------ norms
NORM_SIZES = [(1, 1), (3, 1), (2, 2), (5, 7), (1, 8), (3, 16), (4, 63), (1, 64), (7, 257), (3, 512), (33, 513),
              (9, 1000), (2, 1024), (3, 1025), (5, 2047), (2, 2049), (3, 3001), (2, 4096), (3, 4099),
              (2, 8191), (3, 8193), (2, 12289), (3, 16385), (2, 32769), (2, 40001), (2100, 24), (700, 300)]


def run_norm(rows, width, dtype, wdtype, bias, residual, centre, eps=1e-5, pad=0, seed=0):
    g = gen(seed + rows * 7 + width)
    x = rand(g, rows, width, dtype=dtype, scale=1.5, at=0.7)
    r = rand(g, rows, width, dtype=dtype, scale=2.0) if residual else None
    w = rand(g, width, dtype=wdtype, scale=0.3, at=1.0) if wdtype else None
    b = rand(g, width, dtype=wdtype, scale=0.5) if bias else None
    dout = rand(g, rows, width, dtype=dtype)
    dsum = rand(g, rows, width, dtype=dtype) if residual else None
    if pad:
        x, dout = strided(x, pad), strided(dout, pad + 2)
        r = None if r is None else strided(r, 2 * pad)
    n = layers.Norm(width, dtype, weight=wdtype, bias=bias, eps=eps, centre=centre)
    bufs = layers.NormBuffers(n, rows, residual=residual, grad=True)
    layers.norm_into(n, x, bufs, weight=w, bias=b, residual=r)
    h = x
    if residual:
        want = (x.float() + r.float()).to(dtype)
        assert torch.equal(bufs.sum, want)
        h = bufs.sum
    layers.norm_grad_into(n, h, dout, bufs, weight=w, dsum=dsum)
    H, W, B = host(h), None if w is None else host(w), None if b is None else host(b)
    D, S = host(dout), None if dsum is None else host(dsum)
    e = float(np.float32(eps))
    out, dx, dw, db = ol.norm_bounds(H, W, B, D, S, e, centre)
    y, m, s = ol.norm(H, W, B, e, centre)
    near(bufs.out, y, out, dtype)
    ndx, ndw, ndb = ol.norm_grad(H, D, W, S, e, centre)
    near(bufs.dx, ndx, dx, dtype, "dx")
    if w is not None:
        near(bufs.dweight, ndw, dw, wdtype, "dweight")
    if b is not None:
        near(bufs.dbias, ndb, db, wdtype, "dbias")
    return bufs


@pytest.mark.parametrize("rows,width", NORM_SIZES)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_sizes(rows, width, dtype):
    run_norm(rows, width, dtype, dtype, True, width % 2 == 0, True)


@pytest.mark.parametrize("dtype,wdtype", [(BF, None), (BF, F32), (FP, FP), (FP, F32), (F32, None)])
@pytest.mark.parametrize("bias,residual,centre", [(False, True, False), (True, False, False),
                                                  (False, False, True), (True, True, True)])
@pytest.mark.parametrize("rows,width", [(6, 40), (5, 1203), (3, 5003), (2, 33003)])
def test_norm_forms(dtype, wdtype, bias, residual, centre, rows, width):
    run_norm(rows, width, dtype, wdtype, bias and wdtype is not None, residual, centre, pad=3)


def test_norm_of_no_rows():
    """The weights' gradients of no rows are 0."""
    n = layers.Norm(70, BF, weight=F32, bias=True)
    b = layers.NormBuffers(n, 0, residual=True, grad=True)
    x = torch.empty((0, 70), dtype=BF, device="cuda")
    w = torch.ones(70, device="cuda")
    b.dweight.fill_(3), b.dbias.fill_(3)
    layers.norm_into(n, x, b, weight=w, bias=w, residual=x)
    layers.norm_grad_into(n, x, x, b, weight=w, dsum=x)
    assert not b.dweight.any() and not b.dbias.any()


def test_norm_constant_and_far_rows():
    """Rows without any variance, and rows whose mean is a thousand times their spread: deviations are
    taken before they are squared."""
    g = gen(3)
    x = torch.cat([torch.full((2, 300), 5.0), torch.zeros((2, 300)),
                   torch.randn((4, 300), generator=g) + 1000.0]).cuda()
    n = layers.Norm(300, F32)
    y = layers.norm(n, x)["out"]
    assert not y[:4].any()
    H = host(x)
    near(y[4:], ol.norm(H[4:], eps=float(np.float32(1e-5)))[0],
         ol.norm_bounds(H[4:], eps=float(np.float32(1e-5))), F32)


def test_norm_in_place_and_rows_of_nan():
    g = gen(4)
    x, r = rand(g, 9, 520, dtype=BF), rand(g, 9, 520, dtype=BF)
    x[4, 3] = float("nan")
    x[6, 5] = float("inf")
    n = layers.Norm(520, BF)
    a = layers.NormBuffers(n, 9, residual=True, grad=True)
    layers.norm_into(n, x, a, residual=r)
    b = layers.NormBuffers(n, 9, residual=True, grad=True)
    b.out, b.sum = x.clone(), r.clone()
    layers.norm_into(n, b.out, b, residual=b.sum)
    fine = [i for i in range(9) if i not in (4, 6)]
    assert torch.equal(a.out[fine], b.out[fine]) and torch.equal(a.sum[fine], b.sum[fine])
    assert a.out[fine].isfinite().all() and a.out[[4, 6]].isnan().any(1).all()
    dout = rand(g, 9, 520, dtype=BF)
    layers.norm_grad_into(n, a.sum, dout, a, dsum=dout)
    b.dx = dout.clone()
    layers.norm_grad_into(n, a.sum, b.dx, a, dsum=b.dx)
    c = layers.NormBuffers(n, 9, residual=True, grad=True)
    c.stats, c.dx = a.stats, dout.clone()
    layers.norm_grad_into(n, a.sum, c.dx, c, dsum=c.dx)
    assert torch.equal(a.dx[fine], c.dx[fine])


# ------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("dtype", [BF, FP, F32])
@pytest.mark.parametrize("dim,rotated", [(8, 2), (8, 8), (32, 32), (64, 32), (72, 36), (80, 6), (96, 96), (128, 128),
                                         (128, 126)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate(dtype, dim, rotated, interleaved):
    g = gen(dim + rotated)
    rot = layers.Rotary(dim, dtype, rotated=rotated, interleaved=interleaved, base=500.0, magnitude=1.25)
    angles = layers.frequencies(rotated, 500.0)
    for rows, heads in ((1, 1), (3, 5), (67, 2), (1030, 1)):
        x = rand(g, rows, heads + 2, dim, dtype=dtype)[:, 1:heads + 1]
        p = torch.randint(-5000, 1 << 20, (rows,), generator=g, dtype=torch.int32).cuda()
        out = torch.full((rows, heads, 2 * dim), 7.0, dtype=dtype, device="cuda")
        X = host(x)
        for inverse in (False, True):
            layers.rotate_into(rot, p, x, out[..., :dim], inverse)
            want = ol.rotate(X, host(p), angles, interleaved, 1.25, inverse)
            # (an angle of up to 2^20 radians in 64 bits: off by 2^20 2^-52, nothing beside the rest)
            near(out[..., :dim], want, ol.rotate_bound(X, angles, interleaved, 1.25), dtype)
            assert (out[..., dim:] == 7).all()
        y = x.clone()
        layers.rotate_into(rot, p, y, y, True)
        assert torch.equal(y, out[..., :dim])


def test_rotate_far_positions():
    """The whole range of positions, in fp32: angles keep their digits."""
    rot = layers.Rotary(64, F32, base=1e6)
    p = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 31 - 64, 2 ** 24 + 1], dtype=torch.int32).cuda()
    x = rand(gen(1), 4, 3, 64)
    y = layers.rotate(rot, p, x)
    a = layers.frequencies(64, 1e6)
    # the angle in long double: numpy's float64 product is itself off by 2^31 2^-53 = 2^-22
    t = np.asarray(host(p), np.longdouble)[:, None] * np.asarray(a, np.longdouble)
    t -= np.rint(t / (2 * np.longdouble(np.pi))) * 2 * np.longdouble(np.pi)
    X = host(x)
    c, s = (np.asarray(f(t), np.float64)[:, None, :] for f in (np.cos, np.sin))
    want = np.concatenate([X[..., :32] * c - X[..., 32:] * s, X[..., :32] * s + X[..., 32:] * c], -1)
    # turns per position are rounded to 2^-53 relative, their product with 2^31 again: 2^-21 2 pi turns
    # apart at the fastest pair (1 / 2 pi turns), twice; pi in 64 bits takes 2^31 2^-53 of the reference
    far = 2.0 ** 31 * 2.0 ** -52 * 3
    near(y, want, ol.rotate_bound(X, a) + far * (np.abs(X).max() * 2), F32)


def test_frequencies():
    f = layers.frequencies(8, 100.0)
    np.testing.assert_allclose(f, [1.0, 100 ** -0.25, 0.1, 100 ** -0.75])
    np.testing.assert_allclose(layers.frequencies(8, 100.0, 4.0), np.array(f) / 4)
    g = layers.frequencies(8, 100.0, 4.0, original=200.0, near=2.0, far=20.0)
    turns = 200 * np.array(f) / (2 * np.pi)
    keep = np.clip((turns - 2) / 18, 0, 1)
    assert 0 < keep[2] < 1 and keep[0] == 1
    np.testing.assert_allclose(g, np.array(f) * (keep + (1 - keep) / 4))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,heads,kv_heads,dim,rotated", [(1, 1, 1, 64, 64), (5, 4, 2, 80, 40), (70, 6, 3, 128, 128)])
def test_append(dtype, rows, heads, kv_heads, dim, rotated):
    g = gen(rows)
    n = 3 * rows + 7
    qkv = rand(g, rows, heads + 2 * kv_heads, dim, dtype=dtype)
    q, k, v = qkv.split([heads, kv_heads, kv_heads], 1)
    rot = layers.Rotary(dim, dtype, rotated=rotated)
    p = torch.randint(0, 9999, (rows,), generator=g, dtype=torch.int32).cuda()
    slots = torch.randperm(n, generator=g)[:rows]
    if rows > 3:                                       # rows that are not kept
        slots[1], slots[2] = -1, n
    kc = rand(g, kv_heads, n, dim, dtype=dtype).transpose(0, 1)     # heads far apart
    vc = rand(g, n, kv_heads, dim, dtype=dtype)
    k0, v0 = kc.clone(), vc.clone()
    out = torch.empty((rows, heads, dim), dtype=dtype, device="cuda")
    layers.append_into(rot, p, slots.cuda(), q, k, v, out, kc, vc)
    assert torch.equal(out, layers.rotate(rot, p, q))
    kept = [i for i in range(rows) if 0 <= slots[i] < n]
    k0[slots[kept].cuda()] = layers.rotate(rot, p, k)[kept]
    v0[slots[kept].cuda()] = v[kept]
    assert torch.equal(kc, k0) and torch.equal(vc, v0)
    near(out, ol.rotate(host(q), host(p), layers.frequencies(rotated)),
         ol.rotate_bound(host(q), layers.frequencies(rotated)), dtype)


def test_cache_beyond_32_bits():
    """A cache of more than 2^32 bytes: the last rows are reached, others stay."""
    heads, dim = 8, 128
    n = (1 << 32) // (heads * dim * 2) + 1000
    kc = torch.zeros((n, heads, dim), dtype=BF, device="cuda")
    vc = torch.zeros((n, heads, dim), dtype=BF, device="cuda")
    rot = layers.Rotary(dim, BF)
    x = rand(gen(2), 2, heads, dim, dtype=BF)
    p = torch.tensor([n - 1, 3], dtype=torch.int32).cuda()
    slots = torch.tensor([n - 1, 3]).cuda()
    out = torch.empty_like(x)
    layers.append_into(rot, p, slots, x, x, x, out, kc, vc)
    assert torch.equal(kc[n - 1], out[0]) and torch.equal(kc[3], out[1])
    assert torch.equal(vc[n - 1], x[0]) and torch.equal(vc[3], x[1])
    kc[n - 1] = kc[3] = vc[n - 1] = vc[3] = 0
    assert not kc.view(torch.int16).any() and not vc.view(torch.int16).any()


def test_positions():
    docs = seq.Documents([3, 0, 2, 1], [5, 4, 2, 0])
    assert layers.positions(docs).tolist() == [2, 3, 4, 0, 1, -1]
    t = lambda *x: torch.tensor(x, dtype=torch.int32).cuda()             # noqa: E731
    docs = seq.Documents.on_device(t(6, 1, 1), t(8, 1, 4), t(0, 0, 9), t(4, 0, 12), 9, 12, 5, 12)
    assert layers.positions(docs).tolist() == [0, 0, 1, 2, 0, 0, 2, 3, 0]


# ------------------------------------------------------------------ gated block
GATED_SIZES = [(1, 8, 8), (1, 64, 64), (3, 72, 40), (16, 1024, 136), (17, 200, 264), (33, 64, 72), (64, 136, 128),
               (65, 128, 192), (127, 520, 72), (129, 72, 520), (255, 264, 136), (300, 256, 1024), (1000, 64, 128),
               (2, 2056, 24), (4099, 24, 40)]


def run_gated(rows, width, hidden, dtype, kind, pad=0, grad=True, seed=0):
    g = gen(seed + rows + width + hidden)
    x = rand(g, rows, width, dtype=dtype)
    wg, wu = (rand(g, hidden, width, dtype=dtype, scale=1.5 * width ** -0.5) for _ in range(2))
    dout = rand(g, rows, hidden, dtype=dtype)
    if pad:
        x, wg, wu, dout = strided(x, pad), strided(wg, pad), strided(wu, 2 * pad), strided(dout, pad)
    t = layers.Gated(width, hidden, dtype, activation=kind)
    b = layers.GatedBuffers(t, rows, grad=grad)
    layers.gated_into(t, x, wg, wu, b)
    h = [host(v) for v in (x, wg, wu, dout)]
    out, *more = ol.gated_bounds(*h, kind, HALF[dtype])
    near(b.out, ol.gated(*h[:3], kind), out, dtype)
    if grad:
        layers.gated_grad_into(t, x, wg, wu, dout, b)
        # (fp16: dg and du below its normal numbers are off by 2^-25, absolutely)
        s = SMALL[dtype]
        sub = [s * np.abs(h[1]).sum(0) + s * np.abs(h[2]).sum(0)] + [s * np.abs(h[0]).sum(0)] * 2
        for got, want, e, z, name in zip((b.dx, b.dw_gate, b.dw_up), ol.gated_grad(*h, kind), more, sub,
                                         ("dx", "dw_gate", "dw_up")):
            near(got, want, e + z, dtype, name)
    return b


@pytest.mark.parametrize("rows,width,hidden", GATED_SIZES)
@pytest.mark.parametrize("dtype,kind", [(BF, "silu"), (FP, "gelu")])
def test_gated_sizes(rows, width, hidden, dtype, kind):
    run_gated(rows, width, hidden, dtype, kind)


@pytest.mark.parametrize("rows", list(range(2, 36, 5)) + [48, 63])
def test_gated_few_rows(rows):
    run_gated(rows, 264, 88, BF, "gelu")


@pytest.mark.parametrize("dtype,kind", [(BF, "gelu"), (FP, "silu")])
@pytest.mark.parametrize("rows,width,hidden", [(5, 104, 56), (200, 328, 264), (2048, 136, 1160)])
def test_gated_strides(rows, width, hidden, dtype, kind):
    run_gated(rows, width, hidden, dtype, kind, pad=8)


@pytest.mark.parametrize("rows,width,hidden,kind", [
    (2100, 2120, 2200, "silu"),            # larger tiles, ragged in every direction
    (8100, 1016, 1032, "gelu"),            # ... the weights' gradients in parts
    (520, 2056, 8200, "silu"),             # ... dx in parts
    (4090, 72, 1904, "gelu"),              # two steps a tile
    (3900, 328, 1000, "silu"),             # smaller tiles, as many as are resident at once
    (20000, 56, 1032, "silu"),             # a tile a step, several tiles a block
    (30000, 120, 776, "gelu"),             # ... two steps, several tiles a block
    (17000, 200, 2056, "silu"),            # ... four
    (1000, 520, 1368, "silu"),             # ... every sum in parts
    (1000, 264, 1032, "gelu"),             # two groups of wavefronts a tile: 3 and 2 steps
    (1990, 344, 968, "silu"),              # ... 3 and 3, ragged
    (300, 1080, 4104, "gelu")])            # ... 9 and 8, ragged
@pytest.mark.parametrize("dtype", [BF, FP])
def test_gated_tiles(dtype, rows, width, hidden, kind):
    """The sums' errors together, against what rounding the results alone takes: the forward pass adds
    fp32's, the gradient one more rounding of its operands, independent of the results': sqrt(2) of it, taken
    as 1.5."""
    g = gen(1)
    x = rand(g, rows, width, dtype=dtype)
    wg, wu = (rand(g, hidden, width, dtype=dtype, scale=width ** -0.5) for _ in range(2))
    dout = rand(g, rows, hidden, dtype=dtype)
    t = layers.Gated(width, hidden, dtype, activation=kind)
    b = layers.GatedBuffers(t, rows, grad=True)
    layers.gated_into(t, x, wg, wu, b)
    layers.gated_grad_into(t, x, wg, wu, dout, b)
    X, A, B, D = (v.double() for v in (x, wg, wu, dout))
    G, U = X @ A.t(), X @ B.t()
    p = torch.sigmoid(G) if kind == "silu" else torch.special.ndtr(G)
    d = p * (1 + G * (1 - p)) if kind == "silu" else p + G * torch.exp(-G * G / 2) / (2 * np.pi) ** 0.5
    dg, du = D * U * d, D * G * p
    for got, want, k in ((b.out, G * p * U, 1.0), (b.dx, dg @ A + du @ B, 1.5), (b.dw_gate, dg.t() @ X, 1.5),
                         (b.dw_up, du.t() @ X, 1.5)):
        alone = (want.to(dtype).double() - want).norm()
        assert (got.double() - want).norm() <= 1.02 * k * alone
        # each value: the operands' roundings are off by half a step of each of some hundred or thousand
        # terms, independently: 8 half steps of the largest sum are over 20 standard deviations
        assert (got.double() - want).abs().max() <= 8 * HALF[dtype] * want.abs().max()


def test_gated_of_no_rows():
    t = layers.Gated(64, 72, BF)
    b = layers.GatedBuffers(t, 0, grad=True)
    b.dw_gate.fill_(3), b.dw_up.fill_(3)
    x, d = torch.empty((0, 64), dtype=BF, device="cuda"), torch.empty((0, 72), dtype=BF, device="cuda")
    w = torch.ones((72, 64), dtype=BF, device="cuda")
    layers.gated_into(t, x, w, w, b)
    layers.gated_grad_into(t, x, w, w, d, b)
    assert not b.dw_gate.any() and not b.dw_up.any()


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_activation_values(kind):
    """One product of 1: the activation itself, over its range, to fp16's rounding; the tail of gelu too."""
    z = torch.cat([torch.linspace(-12, 12, 4801), torch.tensor([-60000.0, -200.0, -88.0, 88.0, 30000.0])])
    x = torch.zeros((len(z), 8), dtype=FP)
    x[:, 0], x[:, 1] = z.to(FP), 1.0
    w = torch.zeros((2, 8, 8), dtype=FP)
    w[0, :, 0], w[1, :, 1] = 1.0, 1.0
    x, w = x.cuda(), w.cuda()
    t = layers.Gated(8, 8, FP, activation=kind)
    b = layers.GatedBuffers(t, len(z), grad=True)
    layers.gated_into(t, x, w[0], w[1], b)
    h = host(x[:, :1])
    a, d = ol.activation(h, kind)
    rel = 2e-6 + 2 * ol.F32 * np.minimum(h * h, 1e4)
    near(b.out, np.repeat(a, 8, 1), np.repeat(np.abs(a) * rel, 8, 1), FP)
    dout = torch.zeros((len(z), 8), dtype=FP, device="cuda")
    dout[:, 0] = 1.0
    layers.gated_grad_into(t, x, w[0], w[1], dout, b)
    near(b.dx[:, :1], d, rel * (1 + np.abs(h)) * np.minimum(np.abs(d) + 1e-6, 1.2) + HALF[FP] * np.abs(d)
         + SMALL[FP], FP, "derivative")


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("rows", [1, 200])
def test_gated_values_that_are_not_finite(kind, rows):
    """act(inf) = inf, act(NaN) = NaN, and what is finite beside them stays as it is."""
    x = torch.zeros((rows, 8), dtype=BF, device="cuda")
    w = torch.zeros((2, 8, 8), dtype=BF, device="cuda")
    x[:, 0] = 1.0
    w[0, :, 0] = torch.tensor([float("inf"), float("nan"), 3e38, -3e38, 2.0, -2.0, 0.0, -0.0])
    w[1, :, 0] = 1.0
    y = layers.gated(layers.Gated(8, 8, BF, activation=kind), x, w[0], w[1])[rows - 1]
    assert y[0] == float("inf") and y[1].isnan() and y[2] == w[0, 2, 0] and y[3] == 0
    want = ol.activation(np.array([2.0, -2.0, 0.0, 0.0]), kind)[0]
    np.testing.assert_allclose(host(y[4:]), want, rtol=HALF[BF], atol=0)


# ------------------------------------------------------------------ AdamW
def weights(g, shapes, dtype, master):
    w = [rand(g, *s, scale=0.1) for s in shapes]
    p = [x.to(dtype, copy=True) for x in w]
    return p, (w if master else None)


SHAPES = [(1,), (255,), (256,), (257,), (3, 1000), (0,), (2, 5, 7), (4096,), (70001,)]


@pytest.mark.parametrize("dtype,gdtype,master", [(BF, BF, True), (BF, F32, True), (FP, FP, False), (F32, F32, False)])
@pytest.mark.parametrize("many", [False, True])
def test_adamw(dtype, gdtype, master, many):
    g = gen(5)
    shapes = SHAPES + ([(7,)] * 60 if many else [])
    p, m = weights(g, shapes, dtype, master)
    opt = layers.AdamW(p, masters=m, grad_dtype=gdtype)
    step_of = dict(lr=0.02, betas=(0.8, 0.99), eps=1e-6, decay=0.1)
    f = torch.tensor(0.5, device="cuda")
    w = [host(x) for x in (m or p)]
    M, V = ([np.zeros(x.shape) for x in w] for _ in range(2))
    for t in range(1, 4):
        grads = [rand(g, *s, dtype=gdtype, scale=0.3) for s in shapes]
        grads[4] = grads[4] if t != 2 else None              # left as it is, states and all
        before = [host(x) for x in (m or p)]
        layers.adamw_into(opt, grads, step=t, factor=f, **step_of)
        for i, x in enumerate(grads):
            if x is None:
                assert np.array_equal(host((m or p)[i]), before[i])
                continue
            G = host(x) * 0.5
            w0, m0, v0 = before[i], M[i], V[i]
            W, A, B = ol.adamw(w0, G, m0, v0, t, 0.02, 0.8, 0.99, 1e-6, 0.1)
            # fp32: betas and each product and sum, 4 roundings of m's parts, 5 of v's; the step 8 more
            em = 4 * ol.F32 * (np.abs(0.8 * m0) + np.abs(0.2 * G))
            ev = 5 * ol.F32 * (np.abs(0.99 * v0) + 0.01 * G * G)
            near(opt.m[i], A, em, F32, "m")
            near(opt.v[i], B, ev, F32, "v")
            u = 0.02 * np.abs(A / (1 - 0.8 ** t)) / (np.sqrt(B / (1 - 0.99 ** t)) + 1e-6)
            eu = u * 10 * ol.F32 + 0.02 * em / (1 - 0.8 ** t) / (np.sqrt(B / (1 - 0.99 ** t)) + 1e-6)
            near((m or p)[i], W, eu + 4 * ol.F32 * (np.abs(w0) + u), F32 if master else dtype, "w")
            if master:
                assert torch.equal(p[i], m[i].to(dtype))
            # (what the next step starts from is what is stored)
            M[i], V[i] = host(opt.m[i]), host(opt.v[i])
    assert not opt.m_all.view(-1)[1:256].any() and not opt.v_all.view(-1)[1:256].any()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_adamw_8_bits(dtype):
    """Codes and scales are those of the definition, value by value; the step takes the unrounded states."""
    g = gen(6)
    p, m = weights(g, SHAPES, dtype, dtype is BF)
    opt = layers.AdamW(p, masters=m, state_bits=8)
    seed = 0xfedcba9876543210
    b1, c1, b2, c2 = (np.float32(x) for x in (0.9, 1 - 0.9, 0.999, 1 - 0.999))
    first = np.concatenate([[0], np.cumsum([-(-x.numel() // 256) for x in p])])
    spread = [torch.exp(3 * torch.randn(s, generator=g)).cuda() for s in SHAPES]
    for t in (1, 2, 3, 70000):
        grads = [rand(g, *s, dtype=dtype) * x.to(dtype) for s, x in zip(SHAPES, spread)]
        grads[3] = torch.zeros_like(grads[3])
        old = [ol.decode(opt.m[i].view(torch.uint8).flatten().cpu().numpy(),
                         opt.v[i].view(torch.uint8).flatten().cpu().numpy(), host(opt.scales[i]))
               for i in range(len(p))]
        w0 = [host(x).ravel() for x in (m or p)]
        layers.adamw_into(opt, grads, lr=1e-2, step=t, seed=seed)
        for i, x in enumerate(grads):
            G = x.float().cpu().numpy().ravel()
            A, B = (y.astype(np.float32) for y in old[i])
            A = A * b1 + G * c1                      # fp32, each operation rounded
            B = B * b2 + G * G * c2
            cm, cv, s = ol.encode(A, B, int(first[i]), t, seed)
            assert np.array_equal(host(opt.scales[i]), s)
            assert np.array_equal(opt.m[i].view(torch.uint8).flatten().cpu().numpy(), cm), (t, i)
            assert np.array_equal(opt.v[i].view(torch.uint8).flatten().cpu().numpy(), cv), (t, i)
            W, m1, v1 = ol.adamw(w0[i], G, *old[i], t, 1e-2)
            # what m's two parts lose (4 F32 of each: they may cancel), and the step's own 10 roundings
            size = np.sqrt(v1 / (1 - 0.999 ** t)) + 1e-8
            u, em = 1e-2 / (1 - 0.9 ** t) / size, 4 * ol.F32 * (np.abs(0.9 * old[i][0]) + np.abs(0.1 * G))
            near((m or p)[i].flatten(), W, u * (em + 10 * ol.F32 * np.abs(m1)) + 4 * ol.F32 * (
                np.abs(w0[i]) + u * np.abs(m1)), F32, "w")


def test_adamw_states_that_are_not_finite():
    p = [torch.ones(600, device="cuda")]
    opt = layers.AdamW(p, state_bits=8)
    g = torch.full((600,), 0.5, device="cuda")
    g[300] = float("inf")
    layers.adamw_into(opt, [g], lr=0.1, step=1)
    s = opt.scales[0]
    assert s[1].isnan().all() and s[[0, 2]].isfinite().all()
    keep = torch.ones(600, dtype=torch.bool, device="cuda")
    keep[300] = False
    assert p[0][keep].isfinite().all() and not p[0][300].isfinite()
    layers.adamw_into(opt, [torch.ones_like(g)], lr=0.1, step=2)
    assert p[0][256:512].isnan().all() and p[0][:256].isfinite().all() and p[0][512:].isfinite().all()


def test_adamw_moved_weights():
    """A weight whose storage is replaced: the step is made on the new one."""
    a = torch.nn.Parameter(torch.ones(10, device="cuda"))
    opt = layers.AdamW([a])
    a.data = torch.full((10,), 2.0, device="cuda")
    layers.adamw_into(opt, [torch.ones(10, device="cuda")], lr=0.5, step=1, decay=0.0)
    # m / (1 - b1) = 1, v / (1 - b2) = 1, but for eps = 1e-8: a step of 0.5
    np.testing.assert_allclose(host(a), 1.5, rtol=1e-6)


def test_adamw_unaligned():
    """Weights, gradients and copies that start at any value."""
    flat = torch.zeros(1000, dtype=BF, device="cuda")
    master = torch.zeros(1000, device="cuda")
    p = [flat[1:500], flat[501:1000]]
    m = [master[3:502], master[502:1000 + 1]]
    m[1] = master[501:1000]
    m[0] = master[1:500]
    g = rand(gen(9), 1000, dtype=BF)
    opt = layers.AdamW(p, masters=m)
    layers.adamw_into(opt, [g[1:500], g[501:1000]], lr=1.0, step=1, decay=0.0)
    W, _, _ = ol.adamw(np.zeros(1000), host(g), 0.0, 0.0, 1, 1.0, decay=0.0)
    keep = np.ones(1000, bool)
    keep[[0, 500]] = False
    np.testing.assert_allclose(host(master)[keep], W[keep], rtol=2e-6)
    assert not host(master)[~keep].any() and not host(flat)[~keep].any()
