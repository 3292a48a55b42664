"""The layers of an in-context surrogate around its attention, as timed cases with their plain
forms.

A surrogate that reads a tuning run as a sequence has attention and an answer head; a step of
it, in training or when it answers, also has:

  norm          a row's residual sum and its layer norm (or root-mean-square norm)
  norm_train    the same with its gradients, those of weight and bias included
  rotate_train  rotary positions of the query and key heads of packed runs, forward and backward
  rotate        the same forward only: part of the head, frequencies scaled for long runs
  append        one new row per run: queries rotated, keys rotated into the run's cache, values
                put beside them
  gated         the gated feed-forward block's hidden values, act(x Wg') * (x Wu')
  gated_train   the same with the gradients of x and of both weights
  adamw         a step of AdamW over all weights of a model, states in 32 bits or in 8

Definitions. Norm: h = x + r, rounded to the rows' type as it is stored; with mean m (0 for the
root-mean-square form) and s = 1 / sqrt(mean((h - m)^2) + eps), out = (h - m) s w + b. Rotary:
pair i of the rotated part, (i, i + n/2) or (2i, 2i + 1), turns by pos f_i, f_i = base^(-2i/n).
Scaled by parts: n_i = original f_i / 2 pi turns over the trained length, t = (n_i - near) /
(far - near) cut to 0..1, f_i (t + (1 - t) / factor). AdamW: g times the gradients' factor,
m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2, w = w - lr decay w - lr (m / (1 - b1^t)) /
(sqrt(v / (1 - b2^t)) + eps), the step with the unrounded m and v.

States in 8 bits: 256 values share a scale, a power of two. m is e4m3 at scale 2^(k - 7), v e5m2 at
2^(k - 14), k the exponent of the largest magnitude (scales 2^-126 at least; 1 where all are 0). A
value between two codes takes the upper one if its place between them, in 65536ths, and a random
16-bit number r reach 65536 together; m below its smallest normal code goes to the nearest (upward
halfway), and a v above 0 never becomes 0. r: with e the value's number in its tensor, blocks of 256
counted through all tensors, E = 256 first + e: word E % 4 of Philox4x32-10 (Salmon et al., SC 2011)
with counter (E / 4 low, E / 4 high, t, 0) and key (seed low, seed high); low half for m, high for v.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-5
BASE, FACTOR, NEAR, FAR, ORIGINAL = 10000.0, 8.0, 1.0, 32.0, 8192
LR, BETAS, ADAM_EPS, DECAY, STEP, SEED = 1e-3, (0.9, 0.999), 1e-8, 0.01, 100, 0x5eed0123456789ab
SHARE = 256          # values of a state that share a scale


# ------------------------------------------------------------------------------ cases
def _case(name, op, **kw):
    c = {"op": op, **kw}
    if name:
        c["name"] = name
    return c


def _norm(op, name, dtype, rows, width, weight, bias, residual, centre):
    return _case(name, op, dtype=dtype, rows=rows, width=width, weight=weight, bias=bias,
                 residual=residual, centre=centre)


def _rotary(op, name, dtype, docs, rows, heads, kv_heads, dim, rotated, interleaved, scaled, lens):
    """rows: of the longest document; the others follow from it and `lens` (0: all as long)."""
    return _case(name, op, dtype=dtype, docs=docs, rows=rows, heads=heads, kv_heads=kv_heads,
                 dim=dim, rotated=rotated, interleaved=interleaved, scaled=scaled, lens=lens)


def _gated(op, name, dtype, rows, width, hidden, act):
    return _case(name, op, dtype=dtype, rows=rows, width=width, hidden=hidden, act=act)


def _adamw(name, dtype, bits, master, layers, width, hidden, bins):
    return _case(name, "adamw", dtype=dtype, bits=bits, master=master, layers=layers, width=width,
                 hidden=hidden, bins=bins)


def listed():
    return [
        # the rows of 8 proposals that a small surrogate makes at once: latency
        _norm("norm", "norm-step", "bf16", 8, 256, "bf16", True, True, True),
        # a training step's packed rows
        _norm("norm_train", "norm-train", "bf16", 16384, 1024, "bf16", True, True, True),
        # wide rows in full precision, sizes that fit no vector
        _norm("norm_train", "norm-ragged", "fp32", 1021, 10007, "fp32", False, False, False),
        # query and key heads of a training step on runs of many lengths
        _rotary("rotate_train", "rotate-packed", "bf16", 13, 1021, 16, 4, 128, 128, False, False, 3),
        # long runs, half of each head, frequencies scaled past the trained length
        _rotary("rotate", "rotate-long", "fp16", 8, 16384, 16, 4, 64, 32, True, True, 0),
        # one new row for each of 64 runs that have come to different lengths: latency
        _rotary("append", "rotate-append", "bf16", 64, 1024, 16, 4, 128, 128, False, False, 7),
        # the rows of 8 proposals: both weights are read for few products
        _gated("gated", "gated-step", "bf16", 8, 1024, 4096, "silu"),
        # a scoring batch of candidates through a small surrogate's block
        _gated("gated", "gated-candidates", "bf16", 65536, 256, 1024, "gelu"),
        # a training step in sizes that fit no tile
        _gated("gated_train", "gated-ragged", "fp16", 1021, 520, 1368, "gelu"),
        # a training step's packed rows
        _gated("gated_train", "gated-train", "bf16", 16384, 1024, 4096, "silu"),
        # all weights of a small surrogate
        _adamw("adamw-small", "bf16", 32, True, 3, 256, 1024, 128),
        # all weights of a larger one, states in 8 bits
        _adamw("adamw-large", "bf16", 8, True, 4, 1024, 4096, 512),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: sizes log-uniform over the ranges that the listed ones span."""
    op = rng.choice(("norm", "norm_train", "norm_train", "rotate", "rotate_train", "append", "gated",
                     "gated_train", "gated_train", "adamw", "adamw"))
    dtype = rng.choice(("bf16", "fp16"))
    if op.startswith("norm"):
        dtype = rng.choice(("bf16", "fp16", "fp32"))
        while True:
            rows, width = _log(rng, 1, 65536), _log(rng, 16, 32768)
            if rows * width <= 1 << 24:
                break
        weight = rng.choice((dtype, "fp32"))
        return _norm(op, None, dtype, rows, width, weight, rng.random() < 0.5, rng.random() < 0.5,
                     rng.random() < 0.7)
    if op in ("rotate", "rotate_train", "append"):
        kv_heads = rng.choice((1, 2, 3, 4, 8))
        heads = kv_heads * rng.choice((1, 2, 4))
        dim = rng.choice((32, 64, 64, 72, 80, 96, 128, 128))
        rotated = rng.choice((dim, dim, dim // 2))
        docs = _log(rng, 1, 64)
        rows = _log(rng, 1, 1024 if op == "append" else 131072 // docs)
        return _rotary(op, None, dtype, docs, rows, heads, kv_heads, dim, rotated - rotated % 2,
                       rng.random() < 0.5, rng.random() < 0.5, rng.randrange(0, 1000))
    if op.startswith("gated"):
        while True:
            rows, width, hidden = _log(rng, 1, 65536), 8 * _log(rng, 8, 512), 8 * _log(rng, 8, 1024)
            if rows * width * hidden <= 1 << 35 and rows * hidden <= 1 << 27:
                break
        return _gated(op, None, dtype, rows, width, hidden, rng.choice(("silu", "gelu")))
    dtype = rng.choice(("bf16", "fp16", "fp32"))
    width = _log(rng, 60, 1024)
    return _adamw(None, dtype, rng.choice((8, 32)), dtype != "fp32" and rng.random() < 0.7,
                  _log(rng, 1, 4), width, rng.randrange(2, 5) * width + rng.randrange(0, 7),
                  _log(rng, 8, 512))


# ------------------------------------------------------------------------------ layouts
def _lengths(c):
    rng = random.Random(c["lens"])
    return [c["rows"] if c["lens"] == 0 or d == 0 else max(1, int(c["rows"] * rng.uniform(0.05, 1.0)))
            for d in range(c["docs"])]


def _shapes(c):
    """The weights of a surrogate: an input layer, per layer the projections of attention and of
    the gated block, norms and a table of biases, and the answer head."""
    w, h = c["width"], c["hidden"]
    layer = [(2 * w, w), (w, w), (h, w), (h, w), (w, h), (w,), (w,), (8, 32)]
    return [(w, 32), (w,)] + layer * c["layers"] + [(c["bins"], w), (c["bins"],)]


def _count(shape):
    return math.prod(shape)


# ------------------------------------------------------------------------------ inputs
def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * scale).to(dtype)


def _prepare_norm(s, c, g):
    dt, wt, shape = TYPES[c["dtype"]], TYPES[c["weight"]], (c["rows"], c["width"])
    # columns with means of their own, as a residual stream has them
    s["x"] = (_randn(g, shape, torch.float32, 1.5) + _randn(g, shape[1:], torch.float32)).to(dt)
    s["residual"] = _randn(g, shape, dt, 2.0) if c["residual"] else None
    s["weight"] = (1.0 + _randn(g, shape[1:], torch.float32, 0.2)).to(wt)
    s["bias"] = _randn(g, shape[1:], wt, 0.2) if c["bias"] else None
    train = c["op"] == "norm_train"
    s["dout"] = _randn(g, shape, dt) if train else None
    s["dsum"] = _randn(g, shape, dt) if train and c["residual"] else None
    if own:
        from paper_2212_11142_amd import layers
        s["norm"] = layers.Norm(c["width"], dt, weight=wt, bias=c["bias"], eps=EPS,
                                centre=c["centre"])
        s["bufs"] = layers.NormBuffers(s["norm"], c["rows"], residual=c["residual"], grad=train)


def _prepare_rotary(s, c, g):
    dt, D, H, Hk = TYPES[c["dtype"]], c["dim"], c["heads"], c["kv_heads"]
    L = _lengths(c)
    if c["op"] == "append":
        rows = len(L)
        s["positions"] = torch.tensor([n - 1 for n in L], dtype=torch.int32, device=DEV)
        s["slots"] = torch.tensor([d * c["rows"] + n - 1 for d, n in enumerate(L)], device=DEV)
        s["k_cache"] = _randn(g, (rows * c["rows"], Hk, D), dt)
        s["v_cache"] = _randn(g, (rows * c["rows"], Hk, D), dt)
    else:
        rows = sum(L)
        s["positions"] = torch.cat([torch.arange(n, dtype=torch.int32) for n in L]).to(DEV)
        s["dout"] = _randn(g, (rows, H + Hk, D), dt) if c["op"] == "rotate_train" else None
    # the rows of one projection: query, key and value heads
    s["qkv"] = _randn(g, (rows, H + 2 * Hk, D), dt)
    if own:
        from paper_2212_11142_amd import layers
        more = dict(factor=FACTOR, original=ORIGINAL, near=NEAR, far=FAR) if c["scaled"] else {}
        s["rotary"] = layers.Rotary(D, dt, rotated=c["rotated"], base=BASE,
                                    interleaved=c["interleaved"], **more)
        s["out"] = torch.empty((rows, H if c["op"] == "append" else H + Hk, D), dtype=dt, device=DEV)
        s["dx"] = torch.empty_like(s["out"])


def _prepare_gated(s, c, g):
    dt, R, W, F = TYPES[c["dtype"]], c["rows"], c["width"], c["hidden"]
    s["x"] = _randn(g, (R, W), dt)
    s["w_gate"] = _randn(g, (F, W), dt, 1.5 / math.sqrt(W))
    s["w_up"] = _randn(g, (F, W), dt, 1.5 / math.sqrt(W))
    train = c["op"] == "gated_train"
    s["dout"] = _randn(g, (R, F), dt) if train else None
    if own:
        from paper_2212_11142_amd import layers
        s["gated"] = layers.Gated(W, F, dt, activation=c["act"])
        s["bufs"] = layers.GatedBuffers(s["gated"], R, grad=train)


def _first(c):
    """The first block of each weight's tensor, and the number of blocks, where all are kept one
    after another in rows of SHARE values."""
    first = [0]
    for shape in _shapes(c):
        first.append(first[-1] + -(-_count(shape) // SHARE))
    return first


def _flat(tensors):
    return torch.cat([_blocks(x) for x in tensors])


def _prepare_adamw(s, c, g):
    dt, shapes, first = TYPES[c["dtype"]], _shapes(c), _first(c)
    # gradients differ in size by tensor and within it; some rows get none
    size = [10.0 ** (-2 - i % 3) for i in range(len(shapes))]
    first_axis = [torch.exp(_randn(g, x[:1], torch.float32))
                  * (torch.rand(x[:1], generator=g, device=DEV) < 0.95) for x in shapes]
    spread = [a * x.reshape([-1] + [1] * (len(y) - 1)) for a, x, y in zip(size, first_axis, shapes)]
    s["grads"] = [(_randn(g, x, torch.float32) * a).to(dt) for x, a in zip(shapes, spread)]
    s["factor"] = 0.75 + 0.1 * torch.rand((), generator=g, device=DEV)
    w = _flat([_randn(g, x, torch.float32, 0.05) for x in shapes])
    m = _flat([_randn(g, x, torch.float32, 0.3) * a for x, a in zip(shapes, spread)])
    v = _flat([a ** 2 * (0.5 + torch.rand(x, generator=g, device=DEV))
               for x, a in zip(shapes, spread)])
    scales = None
    if c["bits"] == 8:
        sm, sv = _scale(m, 7), _scale(v, 14)
        m, v = (m / sm).to(torch.float8_e4m3fn), (v / sv).to(torch.float8_e5m2)
        scales = torch.cat([sm, sv], 1)
    # all weights lie in one buffer, each a view of it
    s["all"] = {"params": w.to(dt, copy=True), "masters": w if c["master"] else None, "m": m, "v": v,
                "scales": scales}
    s["step"] = STEP
    if own:
        from paper_2212_11142_amd import layers
        views = [None if x is None else
                 [x[a:b].flatten()[:_count(y)].view(y) for a, b, y in zip(first, first[1:], shapes)]
                 for x in (s["all"]["params"], s["all"]["masters"])]
        opt = layers.AdamW(views[0], masters=views[1], state_bits=c["bits"])
        for name in ("m", "v") + (("scales",) if c["bits"] == 8 else ()):
            to = getattr(opt, name + "_all")
            to.copy_(s["all"][name].view(to.shape))
            s["all"][name] = to
        s["opt"] = opt


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = {"case": c}
    if c["op"].startswith("norm"):
        _prepare_norm(s, c, g)
    elif c["op"].startswith("gated"):
        _prepare_gated(s, c, g)
    elif c["op"] == "adamw":
        _prepare_adamw(s, c, g)
    else:
        _prepare_rotary(s, c, g)
    return s


# ------------------------------------------------------------------------------ passes
def run(state):
    c = state["case"]
    if c["op"].startswith("norm"):
        return _own_norm(state, c) if own else _plain_norm(state, c)
    if c["op"].startswith("gated"):
        return _own_gated(state, c) if own else _plain_gated(state, c)
    if c["op"] == "adamw":
        return _own_adamw(state, c) if own else _plain_adamw(state, c)
    return _own_rotary(state, c) if own else _plain_rotary(state, c)


def _own_norm(s, c):
    from paper_2212_11142_amd import layers
    norm, b = s["norm"], s["bufs"]
    layers.norm_into(norm, s["x"], b, weight=s["weight"], bias=s["bias"], residual=s["residual"])
    r = {"out": b.out}
    if c["residual"]:
        r["sum"] = b.sum
    if c["op"] == "norm_train":
        layers.norm_grad_into(norm, b.sum if c["residual"] else s["x"], s["dout"], b,
                              weight=s["weight"], dsum=s["dsum"])
        r["dx"], r["dweight"] = b.dx, b.dweight
        if c["bias"]:
            r["dbias"] = b.dbias
    return r


def _own_rotary(s, c):
    from paper_2212_11142_amd import layers
    H, Hk = c["heads"], c["kv_heads"]
    q, qk, k, v = (s["qkv"][:, a:b] for a, b in ((0, H), (0, H + Hk), (H, H + Hk), (H + Hk, None)))
    if c["op"] == "append":
        layers.append_into(s["rotary"], s["positions"], s["slots"], q, k, v, s["out"], s["k_cache"],
                           s["v_cache"])
        return {"q": s["out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    layers.rotate_into(s["rotary"], s["positions"], qk, s["out"])
    r = {"out": s["out"]}
    if c["op"] == "rotate_train":
        layers.rotate_into(s["rotary"], s["positions"], s["dout"], s["dx"], inverse=True)
        r["dx"] = s["dx"]
    return r


def _own_gated(s, c):
    from paper_2212_11142_amd import layers
    b = s["bufs"]
    layers.gated_into(s["gated"], s["x"], s["w_gate"], s["w_up"], b)
    r = {"out": b.out}
    if c["op"] == "gated_train":
        layers.gated_grad_into(s["gated"], s["x"], s["w_gate"], s["w_up"], s["dout"], b)
        r["dx"], r["dw_gate"], r["dw_up"] = b.dx, b.dw_gate, b.dw_up
    return r


def _own_adamw(s, c):
    from paper_2212_11142_amd import layers
    s["step"] += 1
    layers.adamw_into(s["opt"], s["grads"], lr=LR, step=s["step"], betas=BETAS, eps=ADAM_EPS,
                      decay=DECAY, factor=s["factor"], seed=SEED)
    return {k: x for k, x in s["all"].items() if x is not None}


# ------------------------------------------------------------------------------ plain forms
def _plain_norm(s, c):
    x = s["x"].float()
    r = {}
    if c["residual"]:
        r["sum"] = (x + s["residual"].float()).to(s["x"].dtype)
        x = r["sum"].float()
    d = x - x.mean(1, keepdim=True) if c["centre"] else x
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    xh, w = d * rstd, s["weight"].float()
    out = xh * w + (s["bias"].float() if c["bias"] else 0.0)
    r["out"] = out.to(s["x"].dtype)
    if c["op"] == "norm_train":
        dy = s["dout"].float()
        g = dy * w
        e = g - xh * (g * xh).mean(1, keepdim=True)
        if c["centre"]:
            e = e - g.mean(1, keepdim=True)
        e = e * rstd
        if c["residual"]:
            e = e + s["dsum"].float()
        r["dx"] = e.to(s["x"].dtype)
        r["dweight"] = (dy * xh).sum(0).to(s["weight"].dtype)
        if c["bias"]:
            r["dbias"] = dy.sum(0).to(s["weight"].dtype)
    return r


def _frequencies(c):
    n = c["rotated"]
    f = BASE ** (-torch.arange(0, n, 2, dtype=torch.float64, device=DEV) / n)
    if c["scaled"]:
        t = ((ORIGINAL * f / (2 * math.pi) - NEAR) / (FAR - NEAR)).clamp(0.0, 1.0)
        f = f * (t + (1.0 - t) / FACTOR)
    return f


def _plain_rotate(c, x, cos, sin):
    n, y = c["rotated"], x.float()
    if c["interleaved"]:
        a, b = y[..., 0:n:2], y[..., 1:n:2]
        z = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = y[..., :n // 2], y[..., n // 2:n]
        z = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([z, y[..., n:]], -1).to(x.dtype)


def _plain_rotary(s, c):
    H, Hk = c["heads"], c["kv_heads"]
    # (far positions lose the angle's digits in 32 bits)
    angle = (s["positions"].double().unsqueeze(1) * _frequencies(c)).unsqueeze(1)
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if c["op"] == "append":
        z = _plain_rotate(c, s["qkv"][:, :H + Hk], cos, sin)
        s["k_cache"][s["slots"]] = z[:, H:]
        s["v_cache"][s["slots"]] = s["qkv"][:, H + Hk:]
        return {"q": z[:, :H].contiguous(), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    r = {"out": _plain_rotate(c, s["qkv"][:, :H + Hk], cos, sin)}
    if c["op"] == "rotate_train":
        r["dx"] = _plain_rotate(c, s["dout"], cos, -sin)
    return r


def _act(c, z):
    """The activation and its derivative."""
    if c["act"] == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return z * p, p * (1.0 + z * (1.0 - p))
    p = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z * p, p + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


def _plain_gated(s, c):
    dt = s["x"].dtype
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    a, da = _act(c, x @ wg.t())
    u = x @ wu.t()
    r = {"out": (a * u).to(dt)}
    if c["op"] == "gated_train":
        dy = s["dout"].float()
        dg, du = dy * u * da, dy * a
        r["dx"] = (dg @ wg + du @ wu).to(dt)
        r["dw_gate"], r["dw_up"] = (dg.t() @ x).to(dt), (du.t() @ x).to(dt)
    return r


def _blocks(x):
    """A tensor's values in rows of SHARE, the last one filled up with zeros."""
    x = x.flatten()
    return torch.nn.functional.pad(x, (0, -x.numel() % SHARE)).view(-1, SHARE)


def _scale(x, top):
    """2^(exponent of each row's largest magnitude - top), 2^-126 at least; 1 for rows of zeros."""
    big = x.abs().amax(1, keepdim=True)
    k = (torch.frexp(big).exponent - 1 - top).clamp_min(-126)
    return torch.where(big > 0, ((k + 127) << 23).int().view(torch.float32), torch.ones_like(big))


def _philox(quad, t):
    """Words 0..3 of Philox4x32-10 for counters (quad, t, 0): int64 tensors of 32-bit values."""
    low = 0xffffffff
    c = [quad & low, quad >> 32, torch.full_like(quad, t & low), torch.zeros_like(quad)]
    k = [SEED & low, SEED >> 32]
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57        # (64 bits of each product)
        c = [((q >> 32) & low) ^ c[1] ^ k[0], q & low, ((p >> 32) & low) ^ c[3] ^ k[1], p & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def _rounded(x, r, keep, lowest, up):
    """|x| on a grid of `keep` bits behind the leading one, 2^lowest the smallest normal number: by
    random 16-bit numbers r, and below 2^lowest by `up` in 65536ths where it is given."""
    lift = 23 - keep
    bits = (x.abs().view(torch.int32) + (r << (lift - 16))) >> lift << lift
    step = 2.0 ** (lowest - keep)
    below = torch.floor(x.abs() / step + (r if up is None else up) / 65536.0) * step
    return torch.where(x.abs() >= 2.0 ** lowest, bits.view(torch.float32), below)


def _plain_adamw(s, c):
    s["step"] += 1
    t, to = s["step"], s["all"]
    w = (to["masters"] if c["master"] else to["params"]).float()
    g = _flat(s["grads"]).float() * s["factor"]
    m, v = to["m"].float(), to["v"].float()
    if c["bits"] == 8:
        m, v = m * to["scales"][:, :1], v * to["scales"][:, 1:]
    m = m * BETAS[0] + g * (1 - BETAS[0])
    v = v * BETAS[1] + g * g * (1 - BETAS[1])
    w = w - w * (LR * DECAY) - (m / (1 - BETAS[0] ** t)) / (
        torch.sqrt(v / (1 - BETAS[1] ** t)) + ADAM_EPS) * LR
    to["params"].copy_(w)
    if c["master"]:
        to["masters"].copy_(w)
    if c["bits"] == 8:
        words = _philox(torch.arange(w.numel() // 4, device=DEV), t)
        r = torch.stack(words, 1).view(w.shape)
        sm, sv = _scale(m, 7), _scale(v, 14)
        m = _rounded(m / sm, (r & 0xffff).int(), 3, -6, 32768) * torch.sign(m)
        v = torch.where(v > 0, _rounded(v / sv, (r >> 16).int(), 2, -14, None).clamp_min(2.0 ** -16),
                        torch.zeros_like(v))
        to["scales"].copy_(torch.cat([sm, sv], 1))
    to["m"].copy_(m)
    to["v"].copy_(v)
    return {k: x for k, x in to.items() if x is not None}


# ------------------------------------------------------------------------------ work
def work(case):
    c = case
    e = SIZE[c["dtype"]]
    if c["op"].startswith("norm"):
        n, w = c["rows"] * c["width"], c["width"] * SIZE[c["weight"]] * (2 if c["bias"] else 1)
        b, f = n * e * (4 if c["residual"] else 2) + w, 8 * n
        if c["op"] == "norm_train":     # dout (and the sum's gradient) in, dx out
            b, f = b + n * e * (3 if c["residual"] else 2) + w, f + 12 * n
        return {"bytes": b, "flops": f}
    if c["op"].startswith("gated"):
        R, W, F = c["rows"], c["width"], c["hidden"]
        b, f = (R * W + 2 * F * W + R * F) * e, 4 * R * W * F
        if c["op"] == "gated_train":
            b, f = b + (R * F + R * W + 2 * F * W) * e, 3 * f
        return {"bytes": b, "flops": f}
    if c["op"] == "adamw":
        n = sum(_count(x) for x in _shapes(c))
        states = 4 + 16 / SHARE if c["bits"] == 8 else 16
        # gradient in, states in and out, the weights in and out or out beside their fp32 form
        return {"bytes": int(n * (e + states + (8 + e if c["master"] else 2 * e))), "flops": 16 * n}
    L = _lengths(c)
    rows, H, Hk, D = len(L) if c["op"] == "append" else sum(L), c["heads"], c["kv_heads"], c["dim"]
    n = rows * (H + Hk) * D
    b = 2 * e * (n + (rows * Hk * D if c["op"] == "append" else 0)) + 4 * rows
    f = 3 * rows * (H + Hk) * c["rotated"]
    return {"bytes": 2 * b, "flops": 2 * f} if c["op"] == "rotate_train" else {"bytes": b, "flops": f}


# ------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """From the definitions in 64 bits; gradients by differentiating them."""
    global own
    keep, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = keep
    c = state["case"]
    for name, f in (("norm", _exact_norm), ("gated", _exact_gated), ("adamw", _exact_adamw)):
        if c["op"].startswith(name):
            return f(state, c)
    return _exact_rotary(state, c)


def _exact_norm(s, c):
    train = c["op"] == "norm_train"
    leaf = lambda t: None if t is None else t.double().requires_grad_(train)     # noqa: E731
    w, b = leaf(s["weight"]), leaf(s["bias"])
    h = s["x"].double()
    r = {}
    if c["residual"]:
        h = (h + s["residual"].double()).to(s["x"].dtype).double()
        r["sum"] = h.clone()
    h.requires_grad_(train)
    var, mean = torch.var_mean(h, 1, correction=0, keepdim=True)
    y = ((h - mean) * (var + EPS).rsqrt() if c["centre"]
         else h * (h.square().mean(1, keepdim=True) + EPS).rsqrt()) * w
    y = y if b is None else y + b
    r["out"] = y.detach()
    if train:
        y.backward(s["dout"].double())
        r["dx"] = h.grad if s["dsum"] is None else h.grad + s["dsum"].double()
        r["dweight"] = w.grad
        if b is not None:
            r["dbias"] = b.grad
    return r


def _exact_rotary(s, c):
    n = c["rotated"]
    H, Hk = c["heads"], c["kv_heads"]
    freq = []
    for i in range(n // 2):
        f = math.exp(-2.0 * i / n * math.log(BASE))
        if c["scaled"]:
            t = min(1.0, max(0.0, (ORIGINAL * f / math.tau - NEAR) / (FAR - NEAR)))
            f = t * f + (1.0 - t) * f / FACTOR
        freq.append(f)
    at = torch.tensor([(2 * i, 2 * i + 1) if c["interleaved"] else (i, i + n // 2)
                       for i in range(n // 2)], device=DEV)
    angle = s["positions"].double()[:, None] * torch.tensor(freq, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]

    def turned(x, turn):
        x = x.double()
        z = torch.complex(x[..., at[:, 0]], x[..., at[:, 1]]) * turn
        y = x.clone()
        y[..., at[:, 0]], y[..., at[:, 1]] = z.real, z.imag
        return y

    if c["op"] == "append":
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        kc[s["slots"]] = turned(s["qkv"][:, H:H + Hk], turn)
        vc[s["slots"]] = s["qkv"][:, H + Hk:].double()
        return {"q": turned(s["qkv"][:, :H], turn), "k_cache": kc, "v_cache": vc}
    r = {"out": turned(s["qkv"][:, :H + Hk], turn)}
    if c["op"] == "rotate_train":
        r["dx"] = turned(s["dout"], turn.conj())
    return r


def _exact_gated(s, c):
    train = c["op"] == "gated_train"
    x, wg, wu = (s[k].double().requires_grad_(train) for k in ("x", "w_gate", "w_up"))
    gate = x @ wg.t()
    y = (torch.nn.functional.silu(gate) if c["act"] == "silu"
         else torch.nn.functional.gelu(gate)) * (x @ wu.t())
    r = {"out": y.detach()}
    if train:
        y.backward(s["dout"].double())
        r["dx"], r["dw_gate"], r["dw_up"] = x.grad, wg.grad, wu.grad
    return r


def _exact_adamw(s, c):
    """(The codes that random numbers choose, and their scales, have no such value.)"""
    t, of = STEP + 1, {k: None if x is None else x.double() for k, x in s["all"].items()}
    w, m, v = of["params"] if of["masters"] is None else of["masters"], of["m"], of["v"]
    if c["bits"] == 8:
        m, v = (x * of["scales"][:, i].unsqueeze(1) for i, x in enumerate((m, v)))
    g = torch.zeros_like(w)
    for a, x in zip(_first(c), s["grads"]):
        g.view(-1)[a * SHARE:a * SHARE + x.numel()] = x.reshape(-1).double() * s["factor"].double()
    m, v = torch.lerp(g, m, BETAS[0]), torch.lerp(g.square(), v, BETAS[1])
    size = torch.sqrt(v / (1 - BETAS[1] ** t)) + ADAM_EPS
    w = w * (1 - LR * DECAY) - LR * (m / (1 - BETAS[0] ** t)) / size
    r = {"params": w, "m": m, "v": v} if c["bits"] == 32 else {"params": w, "m": None, "v": None}
    if c["master"]:
        r["masters"] = w
    return r
