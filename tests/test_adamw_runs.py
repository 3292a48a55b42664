"""Runs of AdamW with states of 8 bits: the rounding rule over many steps (by its definition, on the CPU),
and the kernel's steps on the GPU."""
import numpy as np
import pytest

from oracle import gp_layers as ol

SHARE = ol.SHARE
B1 = 0.9
# A value's m is 2^8 of the largest scale's 2^-9 at most, 2^17 lowest steps: 112 steps without a gradient bring
# 0.9^n of that below one step. There it goes to 0 with a chance of 0.1 or more a step: 280 steps later 200 values are
# all there but for a chance of 200 0.9^280 = 3e-11.
UNTIL = 112 + 280


def run(grads, b2, seed=5, states=True):
    """Updates (in units of the rate) of each step, and m in the end; states: of 8 bits."""
    n = len(grads[0])
    m, v = np.zeros(n), np.zeros(n)
    ups = []
    for t, g in enumerate(grads, 1):
        w, m, v = ol.adamw(np.zeros(n), g, m, v, t, 1.0, B1, b2, 1e-12, 0.0)
        ups.append(-w)
        if states:
            m, v = ol.decode(*ol.encode(m.astype(np.float32), v.astype(np.float32), 0, t, seed))
    return np.array(ups), m


@pytest.mark.parametrize("b2", [0.95, 0.999])
def test_values_whose_gradient_ends_come_to_rest(b2):
    """Among values that go on, in every block: their m becomes 0, as AdamW's does, and stays there."""
    rng = np.random.default_rng(1)
    n, stop = 4 * SHARE, 60
    dead = np.arange(n) % 8 == 0
    grads = rng.normal(size=(stop + UNTIL + 50, n))
    grads[stop:, dead] = 0
    ups, m = run(grads, b2)
    assert (m[dead] == 0).all() and (m[~dead] != 0).mean() > 0.9
    assert (ups[-50:][:, dead] == 0).all()


def test_small_values_follow():
    """Values 1 to 2^-13 of their block's largest, with a mean gradient beside the noise, travel as AdamW's do. v's
    random rounding moves it by a step of up to v / 4 with a chance of 4 (1 - b2): a variance of (1 - b2) / 4 a step, of
    1/8 in the long run, which lifts the mean of 1 / sqrt(v) by 3/8 of that, 5%; and 128 values' means are off by
    sqrt(1/8) / sqrt(128), 3%, of which 3 are allowed."""
    rng = np.random.default_rng(2)
    n = 8 * SHARE
    k = np.arange(n) % 16
    size = 2.0 ** -np.minimum(k, 13)
    grads = (rng.normal(size=(400, n)) + 0.3) * size
    got, want = (run(grads, 0.999, states=s)[0].sum(0) for s in (True, False))
    for i in range(14):
        assert abs(got[k == i].mean() / want[k == i].mean() - 1) < 0.05 + 3 * 0.031, i


def test_no_step_is_longer_than_the_largest_value_s():
    """Where a few gradients are 10^4 times the others. |m| <= c sqrt(v) for every value of AdamW, c = (1 - b1) /
    sqrt(1 - b2) / sqrt(1 - b1^2 / b2), 7.3 in the long run. An m that chance lifts to its block's lowest code,
    2^(k - 16), stands over a v of its lowest code, 2^(k' - 30), or more, k and k' the exponents of the largest: the
    ratio 2^(k - k' / 2 - 1) is c / sqrt(2) at most. Above the lowest codes one rounding makes m twice as large at most
    and v half as large: 2 sqrt(2) c."""
    rng = np.random.default_rng(3)
    n, b2 = 4 * SHARE, 0.999
    grads = rng.normal(size=(300, n)) * 2.0 ** -(np.arange(n) % 32)
    for t in range(0, 300, 37):
        grads[t, rng.integers(0, n, 3)] *= 1e4
    ups, _ = run(grads, b2)
    t = np.arange(1, 301)
    c = (1 - B1) / (1 - B1 ** t) * np.sqrt((1 - b2 ** t) / (1 - b2) / (1 - B1 ** 2 / b2))
    assert (np.abs(ups).max(1) <= 2 * np.sqrt(2) * c).all()


@pytest.mark.gpu
@pytest.mark.parametrize("b2", [0.95, 0.999])
def test_weights_whose_gradient_ends_come_to_rest(b2):
    """The same on the device: without a gradient (and without decay) weights stand still after a while."""
    import torch

    from paper_2212_11142_amd import layers
    g = torch.Generator().manual_seed(4)
    n, stop = 4 * SHARE, 60
    p = [torch.randn(n, generator=g).cuda()]
    opt = layers.AdamW(p, state_bits=8)
    live = torch.ones(n, device="cuda")
    live[::8] = 0
    for t in range(1, stop + UNTIL + 50):
        if t == stop + UNTIL:
            keep = p[0].clone()
        x = torch.randn(n, generator=g).cuda()
        layers.adamw_into(opt, [x if t <= stop else x * live], lr=1e-2, step=t, betas=(B1, b2), decay=0.0, seed=9)
    dead = live == 0
    assert torch.equal(p[0][dead], keep[dead]) and (p[0][~dead] != keep[~dead]).all()
    # (views of one byte: a code of -0 is 0 too)
    assert not (opt.m[0].view(torch.uint8)[dead] & 0x7f).any()
