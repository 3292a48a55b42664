"""The gated block's gradient in fp16 where its intermediate gradients, dg and du, are beyond fp16's range or below
its normal numbers while dx and the weights' gradients are not.

Tolerances: the oracle's bounds, with one rounding of dg and du (2^-11 of a value), and for what is small beside its
neighbours 2^-32 of the largest of 64 rows x 64 hidden values; results are rounded once (2^-11, 2^-25 below the
normal numbers)."""
import numpy as np
import pytest
import torch

from oracle import gp_layers as ol
from paper_2212_11142_amd import layers

pytestmark = pytest.mark.gpu

FP, BF = torch.float16, torch.bfloat16
HALF = 2.0 ** -11


def host(x):
    return x.detach().double().cpu().numpy()


def blocks_of(n):
    return torch.arange(n) // 64


def make(rows, width, hidden, scales, mixed):
    """Inputs of the sizes 2^scales; mixed: dout differs by powers of 2^mixed from 64 rows to the next, w_up by powers
    of 2^-5 from 64 hidden values to the next."""
    g = torch.Generator().manual_seed(rows + width + hidden)
    sizes = (rows, width), (hidden, width), (hidden, width), (rows, hidden)
    x, wg, wu, dout = (torch.randn(s, generator=g) * 2.0 ** k for s, k in zip(sizes, scales))
    if mixed:
        dout *= 2.0 ** (mixed * (blocks_of(rows) * 7 % 3))[:, None]
        wu *= 2.0 ** (-5.0 * (blocks_of(hidden) * 5 % 3))[:, None]
    return [t.to(FP).cuda() for t in (x, wg, wu, dout)]


def largest(x):
    """The largest magnitude of each value's 64 x 64 block."""
    r, c = x.shape
    y = np.zeros((-(-r // 64) * 64, -(-c // 64) * 64))
    y[:r, :c] = np.abs(x)
    y = y.reshape(y.shape[0] // 64, 64, -1, 64).max((1, 3))
    return y.repeat(64, 0).repeat(64, 1)[:r, :c]


def near(got, want, bound, name):
    got = host(got)
    tol = HALF * np.abs(want) + 2.0 ** -25 + bound * (1 + HALF)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], tol[bad][:4])


# exponents of x, w_gate, w_up and dout
SCALES = {"large": (-9, -10, 12, 10),    # dg of 2^16 beside du of 2^-6
          "small": (-14, 12, 0, -14),    # dg of 2^-25, which dx comes from
          "tiny": (8, -17, -14, -20),    # dg of 2^-24 and du of 2^-27, which the weights' gradients come from
          "plain": (0, -3, -3, 0)}
MIXED = {"large": -9.0, "small": 4.0, "tiny": 9.0, "plain": -9.0}
SIZES = [(200, 72, 136), (1, 64, 64), (70, 136, 72), (300, 1080, 2056), (1000, 520, 1368), (2100, 136, 2056),
         (2100, 1048, 1032), (2500, 520, 2568)]


@pytest.mark.parametrize("rows,width,hidden", SIZES)
@pytest.mark.parametrize("scales", list(SCALES))
@pytest.mark.parametrize("mixed", [False, True])
def test_gradients(rows, width, hidden, scales, mixed):
    args = make(rows, width, hidden, SCALES[scales], MIXED[scales] if mixed else 0)
    t = layers.Gated(width, hidden, FP, activation="silu")
    b = layers.GatedBuffers(t, rows, grad=True)
    layers.gated_grad_into(t, *args, b)
    h = [host(v) for v in args]
    want = ol.gated_grad(*h, "silu")
    assert all(np.abs(w).max() < 65504 for w in want)
    _, *bounds = ol.gated_bounds(*h, "silu", HALF)
    a, d = ol.activation(h[0] @ h[1].T, "silu")
    dg, du = (2.0 ** -32 * largest(v) for v in (h[3] * (h[0] @ h[2].T) * d, h[3] * a))
    low = dg @ np.abs(h[1]) + du @ np.abs(h[2]), dg.T @ np.abs(h[0]), du.T @ np.abs(h[0])
    for got, w, e, z, name in zip((b.dx, b.dw_gate, b.dw_up), want, bounds, low, ("dx", "dw_gate", "dw_up")):
        near(got, w, e + z, name)


def test_rows_without_a_gradient_and_rows_that_are_not_finite():
    """Blocks of zeros between others; and what one row has that is not finite stays out of the others' dx."""
    args = make(330, 136, 264, SCALES["large"], 0)
    args[3][64:192] = 0
    t = layers.Gated(136, 264, FP)
    b = layers.GatedBuffers(t, 330, grad=True)
    layers.gated_grad_into(t, *args, b)
    dx = b.dx.clone()
    assert dx.isfinite().all() and not dx[64:192].any() and dx[:64].any() and dx[192:].any()
    args[3][300, 7] = float("inf")
    args[3][200] = float("nan")
    layers.gated_grad_into(t, *args, b)
    keep = [r for r in range(330) if r not in (200, 300)]
    assert torch.equal(b.dx[keep], dx[keep])
    assert b.dx[200].isnan().all() and not b.dx[300].isfinite().any()
    assert b.dw_gate.isnan().all()


def test_all_blocks_without_a_gradient():
    args = make(130, 72, 136, SCALES["plain"], 0)
    args[3].zero_()
    t = layers.Gated(72, 136, FP)
    b = layers.GatedBuffers(t, 130, grad=True)
    layers.gated_grad_into(t, *args, b)
    assert not b.dx.any() and not b.dw_gate.any() and not b.dw_up.any()
