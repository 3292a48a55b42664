"""Float64 definitions of the layers of a sequence surrogate (gp_norm*, gp_rotate*, gp_gated* and
gp_adamw of include/baco_gp.h), with bounds of what fp32 arithmetic and one rounding of the results may
take from them. numpy only; test infrastructure."""
import math

import numpy as np

F32 = 2.0 ** -24                       # half a step of fp32, relative
SHARE = 256


# ------------------------------------------------------------------ norms
def norm(h, weight=None, bias=None, eps=1e-5, centre=True):
    """out, mean and 1 / std of rows h."""
    h = np.asarray(h, np.float64)
    m = h.mean(1, keepdims=True) if centre else np.zeros((h.shape[0], 1))
    s = 1.0 / np.sqrt(((h - m) ** 2).mean(1, keepdims=True) + eps)
    y = (h - m) * s
    y = y if weight is None else y * weight
    return (y if bias is None else y + bias), m[:, 0], s[:, 0]


def norm_grad(h, dout, weight=None, dsum=None, eps=1e-5, centre=True):
    """dx, dweight and dbias."""
    h, dout = np.asarray(h, np.float64), np.asarray(dout, np.float64)
    _, m, s = norm(h, eps=eps, centre=centre)
    xh = (h - m[:, None]) * s[:, None]
    g = dout if weight is None else dout * weight
    e = g - xh * (g * xh).mean(1, keepdims=True)
    if centre:
        e = e - g.mean(1, keepdims=True)
    dx = e * s[:, None]
    return (dx if dsum is None else dx + dsum), (dout * xh).sum(0), dout.sum(0)


def norm_bounds(h, weight=None, bias=None, dout=None, dsum=None, eps=1e-5, centre=True, adds=64):
    """What fp32 may take from out (and from dx, dweight, dbias), before the results' rounding.
    adds: additions one after another in a row's sums at most. To first order: a sum of n terms
    in such an order is off by adds F32 times the sum of their sizes, a product or difference by F32
    of its own."""
    h = np.asarray(h, np.float64)
    _, m, s = norm(h, eps=eps, centre=centre)
    m, s = m[:, None], s[:, None]
    dev = h - m
    dm = (adds + 1) * F32 * np.abs(h).mean(1, keepdims=True) if centre else 0.0
    ddev = dm + F32 * np.abs(dev)
    var = 1.0 / s ** 2
    dvar = (2 * np.abs(dev) * ddev).mean(1, keepdims=True) + (adds + 3) * F32 * var
    rel = dvar / (2 * var) + 3 * F32                       # of s
    xh = dev * s
    dxh = s * ddev + np.abs(xh) * (rel + F32)
    w = np.ones(h.shape[1]) if weight is None else np.abs(np.asarray(weight, np.float64))
    y = np.abs(xh) * w
    out = dxh * w + 2 * F32 * y + (0 if bias is None else F32 * (y + np.abs(bias)))
    if dout is None:
        return out
    g = np.abs(np.asarray(dout, np.float64)) * w
    mean = lambda x: x.mean(1, keepdims=True)                # noqa: E731
    gx = np.asarray(dout, np.float64) * (1.0 if weight is None else weight) * xh
    c2 = np.abs(mean(gx))
    dc1 = (adds + 2) * F32 * mean(g) if centre else 0.0
    dc2 = (adds + 3) * F32 * mean(np.abs(gx)) + mean(g * dxh)
    c1 = np.abs(mean(gx / np.where(xh == 0, 1, xh))) if centre else 0.0
    e = g + c1 + np.abs(xh) * c2
    de = 4 * F32 * e + dc1 + dxh * c2 + np.abs(xh) * dc2
    dx = s * de + s * e * (rel + F32)
    if dsum is not None:
        dx = dx + F32 * (s * e + np.abs(dsum))
    rows = h.shape[0] + 48
    dw = (np.abs(dout) * dxh).sum(0) + rows * F32 * np.abs(dout * xh).sum(0)
    return out, dx, dw, rows * F32 * np.abs(dout).sum(0)


# ------------------------------------------------------------------ rotary positions
def rotate(x, positions, angles, interleaved=False, magnitude=1.0, inverse=False):
    """x [rows, heads, dim] with the first 2 len(angles) values of each head rotated."""
    x = np.asarray(x, np.float64)
    n = 2 * len(angles)
    i = np.arange(n // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n // 2)
    t = np.asarray(positions, np.float64)[:, None] * np.asarray(angles, np.float64)
    c, s = np.cos(t)[:, None, :], np.sin(t)[:, None, :]
    s = -s if inverse else s
    y = x.copy()
    y[..., a] = magnitude * (x[..., a] * c - x[..., b] * s)
    y[..., b] = magnitude * (x[..., a] * s + x[..., b] * c)
    return y


def rotate_bound(x, angles, interleaved=False, magnitude=1.0):
    """What fp32 may take: cosines and sines are off by pi 2^-24 (the rounding of an angle of up to
    one half turn) + 2 steps, 2^-23 each, of the function, each of the two products, the sum and the
    factor by F32: (3.2 + 4 + 4) F32, taken as 12."""
    x = np.abs(np.asarray(x, np.float64))
    n = 2 * len(angles)
    i = np.arange(n // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n // 2)
    y = np.zeros_like(x)
    y[..., a] = y[..., b] = 12 * F32 * abs(magnitude) * (x[..., a] + x[..., b])
    return y


# ------------------------------------------------------------------ gated block
def activation(z, kind):
    """act(z) and its derivative."""
    if kind == "silu":
        p = np.where(z >= 0, 1.0 / (1.0 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1.0 + np.exp(-np.abs(z))))
        return z * p, p + z * p * (1.0 - p)
    p = 0.5 * np.vectorize(math.erfc, otypes=[float])(-z / math.sqrt(2.0))
    return z * p, p + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)


def gated(x, w_gate, w_up, kind):
    x, w_gate, w_up = (np.asarray(v, np.float64) for v in (x, w_gate, w_up))
    return activation(x @ w_gate.T, kind)[0] * (x @ w_up.T)


def gated_grad(x, w_gate, w_up, dout, kind):
    """dx, dw_gate and dw_up."""
    x, w_gate, w_up, dout = (np.asarray(v, np.float64) for v in (x, w_gate, w_up, dout))
    a, d = activation(x @ w_gate.T, kind)
    dg, du = dout * (x @ w_up.T) * d, dout * a
    return dg @ w_gate + du @ w_up, dg.T @ x, du.T @ x


def gated_bounds(x, w_gate, w_up, dout, kind, half):
    """What fp32, and in the gradient one rounding of dg and du to a type of half step `half`, may take
    from out, dx, dw_gate and dw_up. A sum of n products is off by n F32 of their sizes; the activations
    by 2e-6 + 2 F32 z^2 of themselves (a fit to 6.6e-7, an exponential whose argument is rounded,
    a reciprocal, and products); the derivative as much of 1 + |z|."""
    x, wg, wu, dout = (np.asarray(v, np.float64) for v in (x, w_gate, w_up, dout))
    n = x.shape[1]
    g, u = x @ wg.T, x @ wu.T
    eg, eu = (n * F32 * (np.abs(x) @ np.abs(w).T) for w in (wg, wu))
    a, d = activation(g, kind)
    ea = 1.2 * eg + (2e-6 + 2 * F32 * g * g) * np.abs(a)
    ed = eg + (2e-6 + 2 * F32 * g * g) * np.minimum(1.0 + np.abs(g), 1.2 / np.maximum(F32, 2e-6))
    out = ea * np.abs(u) + np.abs(a) * eu + 2 * F32 * np.abs(a * u)
    y = np.abs(dout)
    dg, du = y * np.abs(u * d), y * np.abs(a)
    edg = y * (eu * np.abs(d) + np.abs(u) * ed) + (half + 3 * F32) * dg
    edu = y * ea + (half + 2 * F32) * du
    k, r = 2 * wg.shape[0] + 16, x.shape[0] + 16
    dx = edg @ np.abs(wg) + edu @ np.abs(wu) + k * F32 * (dg @ np.abs(wg) + du @ np.abs(wu))
    dw = [e.T @ np.abs(x) + r * F32 * (v.T @ np.abs(x)) for e, v in ((edg, dg), (edu, du))]
    return out, dx, dw[0], dw[1]


# ------------------------------------------------------------------ AdamW
def adamw(w, g, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.01):
    """w, m and v after a step."""
    w, g, m, v = (np.asarray(x, np.float64) for x in (w, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    w = w - lr * decay * w - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return w, m, v


def philox4x32(counter, key, rounds=10):
    """Philox4x32 (Salmon et al., SC 2011): counter four arrays of 32-bit values, key two numbers."""
    c = [np.asarray(x, np.uint64) for x in counter]
    k = [int(x) for x in key]
    low, half = np.uint64(0xffffffff), np.uint64(32)
    for _ in range(rounds):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> half) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> half) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return c


def state_random(first, count, step, seed):
    """The 16-bit random numbers (for m, for v) of a tensor's values whose first block is `first`."""
    e = np.uint64(first * SHARE) + np.arange(count, dtype=np.uint64)
    quad = e >> np.uint64(2)
    c = philox4x32([quad & np.uint64(0xffffffff), quad >> np.uint64(32),
                    np.full_like(quad, step & 0xffffffff), np.zeros_like(quad)],
                   [seed & 0xffffffff, seed >> 32 & 0xffffffff])
    w = np.choose((e & np.uint64(3)).astype(int), c)
    return (w & np.uint64(0xffff)).astype(int), (w >> np.uint64(16)).astype(int)


def grid(bits, bias):
    """Values of the codes 0.. of a format without sign: `bits` behind the leading one."""
    code = np.arange(128)
    e, f = code >> bits, code & ((1 << bits) - 1)
    return np.where(e > 0, (1 + f / (1 << bits)) * 2.0 ** (e - bias), f / (1 << bits) * 2.0 ** (1 - bias))


M_GRID, V_GRID = grid(3, 7)[:127], grid(2, 15)[:124]       # (above: NaN, infinity and NaN)


def _scales(x, top):
    """Scale of each block of SHARE values."""
    x = np.abs(x)
    pad = np.zeros(-len(x) % SHARE)
    big = np.concatenate([x, pad]).reshape(-1, SHARE).max(1) if len(x) else np.zeros(0)
    k = np.maximum(np.frexp(big)[1] - 1 - top, -126)
    return np.where(big > 0, 2.0 ** k, 1.0)


def encode(m, v, first, step, seed):
    """Codes and scales [blocks, 2] of fp32 states, by the definition: neighbours on the grid, the
    place between them in 65536ths; an m below an eighth of the lowest code is 0."""
    m, v = np.asarray(m, np.float64), np.asarray(v, np.float64)
    sm, sv = _scales(m, 7), _scales(v, 14)
    rm, rv = state_random(first, len(m), step, seed)
    out = []
    for x, scale, values, r, least in ((np.abs(m), sm, M_GRID, rm, M_GRID[1] / 8), (v, sv, V_GRID, rv, None)):
        x = x / np.repeat(scale, SHARE)[:len(x)]
        lo = np.searchsorted(values, x, side="right") - 1
        hi = np.minimum(lo + 1, len(values) - 1)
        place = np.where(hi > lo, (x - values[lo]) / np.where(hi > lo, values[hi] - values[lo], 1), 0.0)
        if least is not None:
            r = np.where(x < least, 0, r)
        code = np.where(place * 65536 + r >= 65536, hi, lo)
        out.append(np.where((x > 0) & (code == 0), 1, code) if least is None else code)
    cm = np.where(m < 0, out[0] | 0x80, out[0])
    return cm.astype(np.uint8), out[1].astype(np.uint8), np.stack([sm, sv], 1)


def decode(cm, cv, scales):
    cm, cv = np.asarray(cm).astype(int), np.asarray(cv).astype(int)
    sm, sv = (np.repeat(scales[:, i], SHARE)[:len(cm)] for i in range(2))
    return np.where(cm & 0x80, -1, 1) * M_GRID[cm & 0x7f] * sm, V_GRID[cv & 0x7f] * sv
