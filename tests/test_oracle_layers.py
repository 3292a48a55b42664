"""Pins of the layers' oracle: closed forms, differences, torch's own float64 layers and published
values of the generator."""
import numpy as np
import pytest
import torch

from oracle import gp_layers as ol

RNG = np.random.default_rng(0)


@pytest.mark.parametrize("centre", [True, False])
@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (True, True)])
def test_norm(centre, weight, bias):
    x, w, b = RNG.normal(size=(5, 13)) + 2, RNG.normal(size=13), RNG.normal(size=13)
    w, b = (w if weight else None), (b if bias else None)
    y, m, s = ol.norm(x, w, b, 1e-3, centre)
    t = torch.from_numpy(x).requires_grad_()
    tw = torch.from_numpy(w if weight else np.ones(13)).requires_grad_()
    tb = torch.from_numpy(b if bias else np.zeros(13)).requires_grad_()
    if centre:
        want = torch.nn.functional.layer_norm(t, (13,), tw, tb, 1e-3)
    else:
        want = t * (t.square().mean(1, keepdim=True) + 1e-3).rsqrt() * tw + tb
    np.testing.assert_allclose(y, want.detach().numpy(), rtol=1e-12, atol=1e-12)
    dout, dsum = RNG.normal(size=x.shape), RNG.normal(size=x.shape)
    want.backward(torch.from_numpy(dout))
    dx, dw, db = ol.norm_grad(x, dout, w, dsum, 1e-3, centre)
    np.testing.assert_allclose(dx, t.grad.numpy() + dsum, rtol=1e-11, atol=1e-12)
    np.testing.assert_allclose(dw, tw.grad.numpy(), rtol=1e-11, atol=1e-12)
    np.testing.assert_allclose(db, tb.grad.numpy(), rtol=1e-11, atol=1e-12)
    # and against differences
    e = 1e-6 * RNG.normal(size=x.shape)
    f = lambda z: (ol.norm(z, w, b, 1e-3, centre)[0] * dout).sum()      # noqa: E731
    np.testing.assert_allclose(f(x + e) - f(x - e), 2 * (e * (dx - dsum)).sum(), rtol=1e-5)
    for a in ol.norm_bounds(x, w, b, dout, dsum, 1e-3, centre):
        assert (a > 0).all() and a.max() < 2.0 ** -10      # (well below a step of fp16)


def test_rotate():
    x = RNG.normal(size=(4, 2, 8))
    p, a = [0, 1, -3, 100000], [0.5, 0.25, 0.1]
    for inter in (False, True):
        y = ol.rotate(x, p, a, inter)
        np.testing.assert_allclose(y[0], x[0])
        np.testing.assert_allclose(y[..., 6:], x[..., 6:])
        np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        np.testing.assert_allclose(ol.rotate(y, p, a, inter, inverse=True), x, atol=1e-11)
        # scores depend on the distance of the positions alone
        q = ol.rotate(x[:1].repeat(4, 0), [7, 8, 9, 10], a, inter)
        k = ol.rotate(x[1:2].repeat(4, 0), [2, 3, 4, 5], a, inter)
        s = (q * k).sum(-1)
        np.testing.assert_allclose(s, s[:1].repeat(4, 0))
        # the gradient is the way back
        d = RNG.normal(size=x.shape)
        np.testing.assert_allclose((ol.rotate(x, p, a, inter, 1.3) * d).sum(),
                                   (x * ol.rotate(d, p, a, inter, 1.3, inverse=True)).sum())
    z = ol.rotate(np.eye(8)[None, :2], [1], a)
    np.testing.assert_allclose(z[0, 0, [0, 3]], [np.cos(0.5), np.sin(0.5)])
    z = ol.rotate(np.eye(8)[None, :2], [1], a, True)
    np.testing.assert_allclose(z[0, 0, [0, 1]], [np.cos(0.5), np.sin(0.5)])


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gated(kind):
    z = np.linspace(-30, 30, 601)
    t = torch.from_numpy(z).requires_grad_()
    want = torch.nn.functional.silu(t) if kind == "silu" else torch.nn.functional.gelu(t)
    want.sum().backward()
    a, d = ol.activation(z, kind)
    np.testing.assert_allclose(a, want.detach().numpy(), rtol=1e-9, atol=1e-14)
    np.testing.assert_allclose(d, t.grad.numpy(), rtol=1e-9, atol=1e-12)
    x, wg, wu, dout = (RNG.normal(size=s) for s in ((5, 8), (6, 8), (6, 8), (5, 6)))
    f = lambda x, wg, wu: (ol.gated(x, wg, wu, kind) * dout).sum()      # noqa: E731
    grads = ol.gated_grad(x, wg, wu, dout, kind)
    for i, v in enumerate((x, wg, wu)):
        e = 1e-6 * RNG.normal(size=v.shape)
        args = [x, wg, wu]
        up, down = list(args), list(args)
        up[i], down[i] = v + e, v - e
        np.testing.assert_allclose(f(*up) - f(*down), 2 * (e * grads[i]).sum(), rtol=1e-5, atol=1e-12)


def test_adamw():
    w = torch.from_numpy(RNG.normal(size=9)).requires_grad_()
    opt = torch.optim.AdamW([w], lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    x, m, v = w.detach().numpy().copy(), np.zeros(9), np.zeros(9)
    for t in range(1, 6):
        g = RNG.normal(size=9)
        w.grad = torch.from_numpy(g)
        opt.step()
        x, m, v = ol.adamw(x, g, m, v, t, 0.01, 0.8, 0.95, 1e-6, 0.1)
        np.testing.assert_allclose(x, w.detach().numpy(), rtol=1e-12)


@pytest.mark.parametrize("counter,key,want", [
    ([0] * 4, [0] * 2, [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
    ([0xffffffff] * 4, [0xffffffff] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
    ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0],
     [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1])])
def test_philox(counter, key, want):
    """The published known answers of Philox4x32-10."""
    assert [int(x) for x in ol.philox4x32(counter, key)] == want


def test_state_codes():
    """The grids are torch's formats; codes keep the sign, the mean and what must not vanish."""
    codes = torch.arange(127, dtype=torch.uint8)
    np.testing.assert_array_equal(ol.M_GRID, codes.view(torch.float8_e4m3fn).double().numpy())
    np.testing.assert_array_equal(ol.V_GRID, codes[:124].view(torch.float8_e5m2).double().numpy())
    n = 200 * 256
    m = np.full(n, -0.3, np.float32)
    v = np.full(n, 1.7e-5, np.float32)
    m[::256], v[::256] = 1.0, 1e-3        # each block's scale
    v[1::256], m[1::256] = 1e-30, 1e-6
    cm, cv, s = ol.encode(m, v, 3, 11, 5)
    a, b = ol.decode(cm, cv, s)
    assert (a[::256] == 1.0).all() and (a[1::256] == 0).all() and (b[1::256] > 0).all()
    # between two codes a step apart: the mean of so many is off by step / 2 / sqrt(n) at most, 5 of these
    for x, y, bits in ((m, a, 3), (v, b, 2)):
        step = 2.0 ** (np.floor(np.log2(abs(float(x[2])))) - bits)
        keep = np.ones(n, bool)
        keep[::256] = keep[1::256] = False
        assert abs(y[keep].mean() - float(x[2])) < 5 * step / 2 / np.sqrt(keep.sum())
        assert set(np.unique(np.abs(y[keep]))) <= {step * np.floor(abs(x[2]) / step),
                                                   step * np.ceil(abs(x[2]) / step)}
    z = ol.encode(np.zeros(5), np.zeros(5), 0, 1, 0)
    assert not z[0].any() and not z[1].any() and (z[2] == 1).all()
    # the lowest scale, and values below it
    tiny = np.full(3, 2.0 ** -140)
    assert (ol.encode(tiny, tiny, 0, 1, 0)[2] == 2.0 ** -126).all()
