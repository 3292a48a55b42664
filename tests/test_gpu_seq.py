"""The sequence-surrogate operators on the GPU against their fp64 oracle.

Bounds. u is the unit roundoff of the 16-bit type (2^-8 bf16, 2^-11 fp16) and
e = 2^-19 (1 + S) bounds the relative error of a probability, S the largest absolute score:
a score carries a few fp32 roundings of its size (products of up to 128 terms, the cap, the
bias) and the exponential turns an absolute error into a relative one.
  out: its rounding, and each probability's rounding and error:  u |out| + (u + e) sum P |v|
  dv:  the same with dout in v's place
  dq, dk: the result's rounding, dS's rounding, and dS's own error, a multiple e of the
       absolute sums behind the difference dP - D (`dif`):        u |.| + u abs + (u^2 + e) dif
  dtable: no rounding of dS:                                     u |.| + e abs + (u^2 + e) dif
each with 10 % over it for the second-order terms, 1e-30 against zeros, and for fp16 results
half the spacing of its smallest numbers, 2^-25, which the relative terms do not cover."""
import math

import numpy as np
import pytest

from oracle import gp_seq as gs

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"\n[gpu] {request.node.nodeid}", flush=True)
    yield


def _torch_dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[name]


ROUND = {"bf16": 2.0 ** -7 / 2, "fp16": 2.0 ** -10 / 2}   # finfo.eps / 2


class Case:
    """Inputs rounded to the type, the description, and the oracle's answer."""

    def __init__(self, dtype, lens, heads, kv_heads, dim, causal=True, cap=0.0, bias="none",
                 prefix=None, seed=0, grad=False, size=1.0, start=(0, 1, 2, 4, 8, 20), k_begin=None,
                 k_rows=None):
        import torch
        from paper_2212_11142_amd import seq
        g = torch.Generator().manual_seed(seed)
        self.dt, self.u, self.grad = _torch_dtype(dtype), ROUND[dtype], grad
        ql, kl = [a for a, _ in lens], [b for _, b in lens]
        self.docs = seq.Documents(ql, kl, prefix=prefix, k_begin=k_begin, k_rows=k_rows)
        tq, tk = self.docs.q_rows, self.docs.k_rows

        def rnd(*shape, f=1.0):
            return (torch.randn(shape, generator=g) * f).to(self.dt).cuda()

        self.q, self.k, self.v = rnd(tq, heads, dim, f=size), rnd(tk, kv_heads, dim), rnd(tk, kv_heads, dim)
        self.dout = rnd(tq, heads, dim) if grad else None
        self.slopes = (torch.tensor([2.0 ** -(1 + h % 5) for h in range(heads)]).cuda()
                       if bias == "slope" else None)
        self.buckets = (seq.Buckets(list(start), bias == "two") if bias in ("one", "two") else None)
        self.table = rnd(heads, self.buckets.count) if self.buckets else None
        self.att = seq.Attention(self.docs, heads, kv_heads, dim, self.dt, causal=causal, cap=cap,
                                 slopes=self.slopes, buckets=self.buckets)
        self.causal, self.cap, self.lens, self.prefix = causal, cap, lens, prefix

    def oracle(self):
        f = lambda t: None if t is None else t.double().cpu().numpy()
        d = [x.cpu().tolist() for x in (self.docs.q_begin, self.docs.q_end, self.docs.k_begin,
                                        self.docs.k_end)]
        docs = [(*r, self.prefix[i] if self.prefix else 0) for i, r in enumerate(zip(*d))]
        return gs.attend(f(self.q), f(self.k), f(self.v), docs, causal=self.causal,
                         scale=1.0 / math.sqrt(self.q.shape[2]), cap=self.cap,
                         slopes=f(self.slopes), table=f(self.table),
                         start=self.buckets.start if self.buckets else None,
                         two_sided=bool(self.buckets and self.buckets.two_sided),
                         dout=f(self.dout))

    def run(self):
        import torch
        from paper_2212_11142_amd import seq
        bufs = seq.AttendBuffers(self.att, grad=self.grad)
        seq.attend_into(self.att, self.q, self.k, self.v, bufs, table=self.table)
        if self.grad:
            seq.attend_grad_into(self.att, self.q, self.k, self.v, self.dout, bufs,
                                 table=self.table)
        torch.cuda.synchronize()
        return bufs

    def check(self, bufs=None, ref=None):
        bufs = bufs or self.run()
        ref = ref or self.oracle()
        u, e = self.u, 2.0 ** -19 * (1 + ref["score"])
        grid = 2.0 ** -25 if self.u == 2.0 ** -11 else 0.0
        up = u * u if self.grad else u      # probabilities' rounding in the second product
        near(bufs.out, ref["out"], u * np.abs(ref["out"]) + (up + e) * ref["out_abs"] + grid,
             "out")
        near(bufs.lse, ref["lse"], e + 2.0 ** -22 * np.abs(np.where(np.isfinite(ref["lse"]), ref["lse"], 0)),
             "lse")
        if not self.grad:
            return
        near(bufs.dv, ref["dv"], u * np.abs(ref["dv"]) + (u + e) * ref["dv_abs"] + grid,
             "dv")
        for n in ("dq", "dk"):
            near(getattr(bufs, n), ref[n], u * np.abs(ref[n]) + (u + e) * ref[n + "_abs"]
                 + (u * u + e) * ref[n + "_dif"] + grid, n)
        if self.table is not None:
            near(bufs.dtable, ref["dtable"], u * np.abs(ref["dtable"]) + e * ref["dtable_abs"]
                 + (u * u + e) * ref["dtable_dif"] + grid, "dtable")


def near(got, want, bound, name):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape, name
    same = np.isnan(want) == np.isnan(got)
    inf = np.isinf(want)
    assert same.all() and np.array_equal(got[inf], want[inf]), name
    ok = np.isfinite(want)
    assert np.isfinite(got[ok]).all(), name
    err = np.abs(got - want)[ok]
    lim = 1.1 * np.broadcast_to(bound, want.shape)[ok] + 1e-30
    if err.size:
        worst = np.argmax(err - lim)
        assert err[worst] <= lim[worst], (name, err[worst], lim[worst])


# ------------------------------------------------------------------ attention, forward
TYPES = ("bf16", "fp16")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [8, 24, 64, 72, 128])
@pytest.mark.parametrize("lens", [[(1, 1)], [(31, 31), (33, 33)], [(65, 65), (1, 1), (130, 130)],
                                  [(129, 257)], [(200, 40), (40, 200)]])
def test_attend_sizes(dtype, dim, lens):
    Case(dtype, lens, 4, 2, dim, causal=False, seed=dim).check()
    Case(dtype, lens, 4, 2, dim, causal=True, seed=dim + 1).check()


@pytest.mark.parametrize("cap", [0.0, 2.0, 30.0])
@pytest.mark.parametrize("bias", ["none", "slope", "one", "two"])
@pytest.mark.parametrize("mask", ["full", "causal", "prefix"])
def test_attend_scores(cap, bias, mask):
    lens = [(150, 150), (70, 190), (3, 3), (260, 260)]
    Case("bf16", lens, 6, 3, 64, causal=mask != "full", cap=cap, bias=bias,
         prefix=[40, 190, 0, 131] if mask == "prefix" else None, size=3.0).check()


@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 1), (5, 5), (12, 3)])
def test_attend_head_layouts(heads, kv):
    Case("fp16", [(90, 90), (20, 75)], heads, kv, 32, bias="one").check()


def test_attend_many_documents():
    """More documents than a wavefront has lanes, some empty on either side."""
    rng = np.random.default_rng(0)
    lens = [(int(a), int(b)) for a, b in zip(rng.integers(0, 60, 150), rng.integers(0, 60, 150))]
    lens[3], lens[64], lens[70] = (0, 5), (5, 0), (0, 0)
    Case("bf16", lens, 2, 1, 64, causal=True).check()
    Case("bf16", lens, 2, 1, 64, causal=False, grad=True).check()


def test_attend_rows_that_see_nothing():
    """More queries than keys under a causal mask: the first rows stand before every key."""
    c = Case("bf16", [(300, 5), (4, 1), (150, 0)], 4, 2, 64, causal=True, grad=True)
    b = c.run()
    c.check(b)
    assert (b.out[:295] == 0).all() and b.lse[:, :295].isneginf().all() and (b.dq[:295] == 0).all()
    few = Case("bf16", [(7, 5), (4, 1), (3, 0)], 4, 2, 64, causal=True)
    few.check()


def test_attend_table_of_ruled_out_distances():
    """-inf in the table rules a distance out, all of them a row."""
    c = Case("bf16", [(80, 80), (20, 20)], 2, 1, 64, causal=True, bias="one", grad=True)
    c.table[0, 3:] = float("-inf")
    c.table[1, :] = float("-inf")
    b = c.run()
    c.check(b)
    assert (b.out[:, 1] == 0).all() and b.lse[1].isneginf().all() and (b.dq[:, 1] == 0).all()


@pytest.mark.parametrize("size", [30.0, 300.0])
def test_attend_large_scores(size):
    """Scores far beyond the exponential's range: the running maximum carries them."""
    Case("bf16", [(200, 200)], 2, 2, 64, causal=True, size=size).check()
    Case("bf16", [(200, 200)], 2, 2, 64, causal=True, size=size, cap=50.0, grad=True).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("lens", [[(200, 200)], [(6, 200)], [(1, 100), (1, 97)]])
def test_attend_anything_in_masked_places(dtype, value, lens):
    """Keys and values that a row does not see hold NaN or infinities: rows before them are
    as with finite ones, rows that see the value show it."""
    import torch
    c = Case(dtype, lens, 4, 2, 72, causal=True, k_begin=[i * 300 for i in range(len(lens))],
             k_rows=300 * len(lens))
    for i, (_, lk) in enumerate(lens):       # past the documents' ends
        c.k[i * 300 + lk:(i + 1) * 300] = value
        c.v[i * 300 + lk:(i + 1) * 300] = value
    c.check()
    lq, lk = lens[0]
    if lq > 1:
        at = lk - max(lq // 3, 2)            # a key that only the last rows see
        c.v[at, 0, 5] = value
        ref = c.oracle()
        with np.errstate(invalid="ignore"):
            ref["out_abs"][:, :2, 5] = np.where(np.isfinite(ref["out"][:, :2, 5]),
                                                ref["out_abs"][:, :2, 5], 0)
        c.check(ref=ref)
        c.k[at, 0, :] = math.nan             # scores of its own column only
        b = c.run()
        rows = torch.arange(lq, device="cuda") + (lk - lq) < at
        assert b.out[:lq][rows].isfinite().all() and b.lse[:, :lq][:, rows].isfinite().all()
        assert b.out[:lq, :2][~rows].isnan().all()


def test_attend_strides():
    """q, k, v as slices of one projection, and head-major tensors; out through strides."""
    import torch
    from paper_2212_11142_amd import seq
    H, K, D, T = 4, 2, 64, 220
    c = Case("bf16", [(T, T)], H, K, D, grad=True)
    want = c.run()
    fused = torch.zeros((T, H + 2 * K + 1, D), dtype=torch.bfloat16, device="cuda")
    fused[:, :H], fused[:, H:H + K], fused[:, H + K:H + 2 * K] = c.q, c.k, c.v
    c.q, c.k, c.v = fused[:, :H], fused[:, H:H + K], fused[:, H + K:H + 2 * K]
    got = c.run()
    for n in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(got, n), getattr(want, n)), n
    c.q, c.k, c.v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (c.q, c.k, c.v))
    assert c.q.stride(0) == D
    got = c.run()
    for n in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(got, n), getattr(want, n)), n
    bufs = seq.AttendBuffers(c.att)
    store = torch.zeros((H, T, D), dtype=torch.bfloat16, device="cuda")
    bufs.out = store.transpose(0, 1)
    seq.attend_into(c.att, c.q, c.k, c.v, bufs)
    plain = seq.attend(c.att, c.q, c.k, c.v)
    assert torch.equal(bufs.out, plain["out"])


def test_attend_shared_keys_broadcast():
    """A key head stride of 0 (heads that share one stored head)."""
    c = Case("bf16", [(100, 100)], 4, 2, 64)
    c.k, c.v = c.k[:, :1].expand(-1, 2, -1), c.v[:, :1].expand(-1, 2, -1)
    c.check()


# ------------------------------------------------------------------ larger calls
# Enough heads that the blocks of 128 queries (or keys) fill the device: the forms that small
# calls do not take.
@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("fp16", 72), ("bf16", 128)])
@pytest.mark.parametrize("cap,bias", [(0.0, "none"), (3.0, "slope"), (0.0, "one"), (20.0, "two")])
@pytest.mark.parametrize("mask", ["full", "causal", "prefix"])
def test_attend_large(dtype, dim, cap, bias, mask):
    lens = [(200, 200), (129, 257), (1, 1), (65, 40), (300, 300)]
    Case(dtype, lens, 48, 6, dim, causal=mask != "full", cap=cap, bias=bias, size=2.0,
         prefix=[90, 257, 0, 3, 131] if mask == "prefix" else None).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_attend_large_anything_in_masked_places(dtype, value):
    import torch
    c = Case(dtype, [(300, 300), (70, 150)], 96, 2, 72, causal=True, k_begin=[0, 400], k_rows=700)
    for a, b in ((300, 400), (550, 700)):
        c.k[a:b] = value
        c.v[a:b] = value
    c.check()
    c.v[180, 0, 5] = value               # a key of the first document, seen from row 180 on
    ref = c.oracle()
    with np.errstate(invalid="ignore"):
        ref["out_abs"][:, :, 5] = np.where(np.isfinite(ref["out"][:, :, 5]), ref["out_abs"][:, :, 5], 0)
    c.check(ref=ref)
    c.k[180, 0, :] = math.nan
    b = c.run()
    assert b.out[:180].isfinite().all() and b.out[180:300, :48].isnan().all()
    assert b.out[180:300, 48:].isfinite().all()


@pytest.mark.parametrize("dtype,dim", [("fp16", 64), ("bf16", 120), ("fp16", 128)])
@pytest.mark.parametrize("cap,bias", [(0.0, "none"), (3.0, "slope"), (20.0, "one"), (0.0, "two")])
@pytest.mark.parametrize("mask", ["full", "causal", "prefix"])
def test_attend_a_block_per_compute_unit(dtype, dim, cap, bias, mask):
    """Fewer blocks, whose key tiles two groups of wavefronts share; also as in training."""
    lens = [(200, 200), (129, 257), (1, 1), (65, 40), (300, 300)]
    for grad in (False, True):
        Case(dtype, lens, 20, 5, dim, causal=mask != "full", cap=cap, bias=bias, size=2.0, grad=grad,
             prefix=[90, 257, 0, 3, 131] if mask == "prefix" else None).check()


@pytest.mark.parametrize("heads", [44, 192])     # two groups of wavefronts, and one
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_attend_values_that_some_rows_see(heads, value):
    """A value and a key that no number is, in one head from one row on, in every tile's place."""
    for at in (0, 63, 64, 130, 299):
        c = Case("bf16", [(300, 300), (70, 150)], heads, 2, 64, causal=True, k_begin=[0, 400], k_rows=700)
        c.v[at, 0, 5] = value
        ref = c.oracle()
        with np.errstate(invalid="ignore"):
            ref["out_abs"][:, :, 5] = np.where(np.isfinite(ref["out"][:, :, 5]), ref["out_abs"][:, :, 5], 0)
        c.check(ref=ref)
        c.k[at, 0, :] = math.nan
        b = c.run()
        half = heads // 2
        assert b.out[:at].isfinite().all() and b.out[at:300, :half].isnan().all()
        assert b.out[at:, half:].isfinite().all() and b.out[300:].isfinite().all()


@pytest.mark.parametrize("dtype,heads,kv,dim,cap,bias,mask", [
    ("bf16", 32, 2, 64, 0.0, "slope", "causal"),     # key tiles shared by 8 blocks
    ("fp16", 32, 4, 128, 5.0, "two", "prefix"),
    ("bf16", 32, 32, 64, 0.0, "two", "full"),        # one block per key tile and head
    ("bf16", 32, 32, 128, 0.0, "none", "causal"),
    ("fp16", 32, 16, 80, 10.0, "one", "causal")])
def test_grad_large(dtype, heads, kv, dim, cap, bias, mask):
    lens = [(620, 620), (300, 90), (90, 300), (1, 1), (33, 33)]
    Case(dtype, lens, heads, kv, dim, causal=mask != "full", cap=cap, bias=bias, grad=True,
         prefix=[200, 0, 260, 0, 40] if mask == "prefix" else None).check()


@pytest.mark.parametrize("dtype,heads,kv,dim", [("bf16", 8, 1, 64), ("fp16", 16, 2, 72), ("bf16", 6, 1, 128)])
@pytest.mark.parametrize("cap,bias,mask", [(0.0, "two", "full"), (4.0, "slope", "causal"), (0.0, "one", "prefix")])
def test_grad_small_with_many_heads_per_key_head(dtype, heads, kv, dim, cap, bias, mask):
    """Small calls whose key tiles are shared, with documents shorter than the shares."""
    lens = [(260, 260), (40, 90), (1, 1), (3, 0), (97, 33)]
    Case(dtype, lens, heads, kv, dim, causal=mask != "full", cap=cap, bias=bias, grad=True,
         prefix=[31, 90, 0, 0, 12] if mask == "prefix" else None).check()


def test_grad_of_one_key_is_zero():
    """A softmax over one key does not depend on its score."""
    for heads, lens in ((2, [(1, 1), (5, 1)]), (64, [(1, 1), (300, 1), (130, 1), (260, 260)])):
        c = Case("bf16", lens, heads, heads, 64, causal=heads > 2, bias="one", grad=True)
        b = c.run()
        n = sum(a for a, k in lens if k == 1)
        assert (b.dq[:n] == 0).all()
        m = sum(k for _, k in lens if k == 1)
        assert (b.dk[:m] == 0).all() and not (b.dv[:m] == 0).all()
        c.check(b)


# ------------------------------------------------------------------ few rows, long caches
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lq", [1, 2, 5])
@pytest.mark.parametrize("bias", ["none", "slope", "one", "two"])
def test_attend_single_rows(dtype, lq, bias):
    lens = [(lq, lk) for lk in (1, 31, 32, 127, 128, 129, 1000, 2049)]
    Case(dtype, lens, 8, 2, 128, bias=bias, k_begin=[2100 * i for i in range(8)],
         k_rows=2100 * 8).check()
    Case(dtype, lens, 3, 3, 64, bias=bias, cap=20.0, size=4.0).check()


def test_attend_single_rows_agree_with_the_general_form():
    """The same rows computed by both forms (the second through documents of 33 rows)."""
    import torch
    from paper_2212_11142_amd import seq
    T, H, D = 700, 4, 64
    c = Case("bf16", [(T, T)], H, 1, D, bias="one")
    full = c.run()
    docs = seq.Documents([1], [T])
    att = seq.Attention(docs, H, 1, D, torch.bfloat16, buckets=c.buckets)
    one = seq.attend(att, c.q[-1:], c.k, c.v, table=c.table)
    torch.cuda.synchronize()
    ref = c.oracle()
    bound = c.u * np.abs(ref["out"]) + (c.u + 2.0 ** -19 * (1 + ref["score"])) * ref["out_abs"]
    near(one["out"], ref["out"][-1:], bound[-1:], "single")
    near(full.out, ref["out"], bound, "general")


def test_attend_cache_past_32_bit_offsets():
    """A cache of more than 2^32 bytes (and 2^31 elements): the last run's slot."""
    import torch
    from paper_2212_11142_amd import seq
    D, rows = 128, (1 << 24) + 4096
    c = Case("bf16", [(1, 700)], 2, 2, D)
    k = torch.zeros((rows, 2, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() > 2 ** 31
    k[-700:], v[-700:] = c.k, c.v
    docs = seq.Documents([1], [700], k_begin=[rows - 700], k_rows=rows)
    att = seq.Attention(docs, 2, 2, D, torch.bfloat16)
    got = seq.attend(att, c.q, k, v)
    want = c.run()
    torch.cuda.synchronize()
    assert torch.equal(got["out"], want.out) and torch.equal(got["lse"], want.lse)
    # and the general form
    c = Case("bf16", [(130, 130)], 2, 2, D)
    k[-130:], v[-130:] = c.k, c.v
    docs = seq.Documents([130], [130], k_begin=[rows - 130], k_rows=rows)
    got = seq.attend(seq.Attention(docs, 2, 2, D, torch.bfloat16), c.q, k, v)
    assert torch.equal(got["out"], c.run().out)


def test_large_calls_in_a_cache_past_32_bit_offsets():
    """The forms for many query rows, and the gradient, over the last rows of such a cache."""
    import types

    import torch
    from paper_2212_11142_amd import seq
    H, D, n, rows = 192, 128, 130, (1 << 24) + 4096
    c = Case("bf16", [(n, n)], H, 2, D, grad=True)
    k = torch.zeros((rows, 2, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() > 2 ** 31
    k[-n:], v[-n:] = c.k, c.v
    docs = seq.Documents([n], [n], k_begin=[rows - n], k_rows=rows)
    att = seq.Attention(docs, H, 2, D, torch.bfloat16)
    bufs = seq.AttendBuffers(att, grad=True)
    bufs.dk.fill_(7.0)
    bufs.dv.fill_(7.0)
    seq.attend_into(att, c.q, k, v, bufs)
    seq.attend_grad_into(att, c.q, k, v, c.dout, bufs)
    torch.cuda.synchronize()
    c.check(types.SimpleNamespace(out=bufs.out, lse=bufs.lse, dq=bufs.dq, dk=bufs.dk[-n:],
                                  dv=bufs.dv[-n:]))
    for d in (bufs.dk, bufs.dv):     # rows of no document keep their contents
        assert bool((d[:-n] == 7.0).all())


# ------------------------------------------------------------------ gradients
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [16, 64, 80, 128])
@pytest.mark.parametrize("lens", [[(1, 1)], [(33, 33), (2, 2)], [(128, 128), (129, 129)],
                                  [(190, 60), (60, 190)]])
def test_grad_sizes(dtype, dim, lens):
    Case(dtype, lens, 4, 2, dim, causal=False, grad=True, seed=dim).check()
    Case(dtype, lens, 4, 2, dim, causal=True, grad=True, seed=dim).check()


@pytest.mark.parametrize("cap", [0.0, 4.0])
@pytest.mark.parametrize("bias", ["slope", "one", "two"])
@pytest.mark.parametrize("mask", ["full", "causal", "prefix"])
def test_grad_scores(cap, bias, mask):
    lens = [(150, 150), (40, 130), (3, 3), (200, 200)]
    for dtype, heads, kv, dim in (("bf16", 6, 3, 64), ("fp16", 4, 1, 128)):
        Case(dtype, lens, heads, kv, dim, causal=mask != "full", cap=cap, bias=bias,
             prefix=[40, 130, 0, 131] if mask == "prefix" else None, size=2.0, grad=True).check()


@pytest.mark.parametrize("start", [(0,), (0, 1), (0, 5, 1024), tuple(range(64))])
@pytest.mark.parametrize("bias", ["one", "two"])
def test_grad_bucket_layouts(start, bias):
    """One class, classes whose reach passes the document, and 64 a side."""
    Case("bf16", [(300, 300), (50, 50)], 2, 2, 64, causal=False, bias=bias, start=start,
         grad=True).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [1e-3, 1e3])
def test_grad_scale_of_dout(dtype, size):
    """Small and large upstream gradients: fp16 keeps dS normal by its factor."""
    c = Case(dtype, [(150, 150)], 4, 2, 64, grad=True)
    c.dout = (c.dout.float() * size).to(c.dt)
    c.check()


@pytest.mark.parametrize("which", ["q", "k", "v", "table"])
def test_grad_against_differences(which):
    """A direction's central difference of sum(out * dout), out taken with what its rounding
    left (fp32 accurate). Inputs are multiples of 2^-5 and the step is 2^-5, so that the
    shifted inputs are exact; the difference's own error is a third derivative's, h^2 times
    about the value; bound 3 % of the gradient's norm times the direction's."""
    import torch
    from paper_2212_11142_amd import seq
    c = Case("fp16", [(40, 40), (25, 60)], 4, 2, 64, causal=True, cap=8.0, bias="two", grad=True,
             start=(0, 1, 3, 10))
    h = 2.0 ** -5
    for n in ("q", "k", "v", "table"):
        setattr(c, n, (torch.round(getattr(c, n).float() / h) * h).to(c.dt))

    def loss():
        b = seq.AttendBuffers(c.att, grad=True)
        seq.attend_into(c.att, c.q, c.k, c.v, b, table=c.table)
        return ((b.out.double() + b.rest.double()) * c.dout.double()).sum().item()

    b = c.run()
    grad = getattr(b, "d" + which).double()
    x = getattr(c, which)
    g = torch.Generator().manual_seed(5)
    for _ in range(4):
        d = torch.zeros(x.shape, dtype=torch.float64)
        at = torch.randperm(x.numel(), generator=g)[:32]
        d.view(-1)[at] = torch.randint(0, 2, (32,), generator=g).double() * 2 - 1
        d = d.cuda()
        vals = []
        for sign in (1, -1):
            setattr(c, which, (x.double() + sign * h * d).to(c.dt))
            assert torch.equal(getattr(c, which).double(), x.double() + sign * h * d)
            vals.append(loss())
        setattr(c, which, x)
        want = (vals[0] - vals[1]) / (2 * h)
        got = (grad * d).sum().item()
        assert abs(got - want) <= 0.03 * (grad.norm() * d.norm()).item(), (got, want)


def test_rows_outside_documents_are_left():
    """Rows that no document has: 0 in the buffers' outputs, whatever the inputs hold."""
    import torch
    from paper_2212_11142_amd import seq
    docs = seq.Documents([50, 20], [50, 20], q_rows=100, k_rows=300, k_begin=[10, 200])
    att = seq.Attention(docs, 2, 2, 64, torch.float16)
    g = torch.Generator().manual_seed(0)
    q, k, v, do = (torch.randn((n, 2, 64), generator=g).half().cuda() for n in (100, 300, 300, 100))
    bufs = seq.AttendBuffers(att, grad=True)
    for x, keep in ((q, [(0, 70)]), (do, [(0, 70)]), (k, [(10, 60), (200, 220)]),
                    (v, [(10, 60), (200, 220)])):
        m = torch.ones(x.shape[0], dtype=torch.bool, device="cuda")
        for a, b in keep:
            m[a:b] = False
        x[m] = math.nan
    seq.attend_into(att, q, k, v, bufs)
    seq.attend_grad_into(att, q, k, v, do, bufs)
    torch.cuda.synchronize()
    assert (bufs.out[70:] == 0).all() and (bufs.dq[70:] == 0).all()
    for x in (bufs.dk, bufs.dv):
        assert (x[:10] == 0).all() and (x[60:200] == 0).all() and (x[220:] == 0).all()
    for x in (bufs.out, bufs.dq, bufs.dk, bufs.dv):
        assert x.isfinite().all()


# ------------------------------------------------------------------ use
def test_repeated_calls_are_identical_on_any_stream():
    import torch
    from paper_2212_11142_amd import seq
    c = Case("bf16", [(300, 300), (129, 129)], 4, 2, 64, bias="two", cap=5.0, grad=True)
    want = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.run()
    for n in ("out", "lse", "dq", "dk", "dv", "dtable"):
        assert torch.equal(getattr(got, n), getattr(want, n)), n


def test_captured_in_a_graph():
    """Attention, its gradient, single rows with growing lengths and the output head in one
    captured graph, replayed with new inputs and other work between."""
    import torch
    from paper_2212_11142_amd import seq
    c = Case("bf16", [(200, 200), (60, 60)], 4, 2, 64, bias="one", grad=True)
    bufs = seq.AttendBuffers(c.att, grad=True)
    i32 = dict(dtype=torch.int32, device="cuda")
    kb, ke = torch.tensor([0, 1000], **i32), torch.tensor([300, 1500], **i32)
    docs = seq.Documents.on_device(torch.tensor([0, 1], **i32), torch.tensor([1, 2], **i32), kb, ke,
                                   2, 2000, 1, 1000)
    att1 = seq.Attention(docs, 4, 2, 64, torch.bfloat16)
    b1 = seq.AttendBuffers(att1)
    q1, k1, v1 = (torch.randn(s, device="cuda").bfloat16() for s in ((2, 4, 64), (2000, 2, 64), (2000, 2, 64)))
    x = torch.randn((4, 20000), device="cuda")
    t = torch.randint(0, 20000, (4,), device="cuda")
    lb = seq.LogprobBuffers(4, 20000, torch.float32, top=7, grad=True)
    one = torch.ones(4, device="cuda")

    def step(b, b1, lb):
        seq.attend_into(c.att, c.q, c.k, c.v, b, table=c.table)
        seq.attend_grad_into(c.att, c.q, c.k, c.v, c.dout, b, table=c.table)
        seq.attend_into(att1, q1, k1, v1, b1)
        seq.logprob_into(x, t, lb)
        seq.logprob_grad_into(x, t, one, None, lb)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(bufs, b1, lb)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(bufs, b1, lb)
    for n in range(4):
        c.q.normal_()
        x.normal_()
        ke += 100
        torch.cuda.synchronize()
        graph.replay()
        e, e1 = seq.AttendBuffers(c.att, grad=True), seq.AttendBuffers(att1)
        el = seq.LogprobBuffers(4, 20000, torch.float32, top=7, grad=True)
        step(e, e1, el)
        torch.cuda.synchronize()
        for a, b, names in ((bufs, e, ("out", "lse", "dq", "dk", "dv", "dtable")),
                            (b1, e1, ("out", "lse")),
                            (lb, el, ("logp", "entropy", "lse", "top_logp", "top_id", "dlogits"))):
            for k in names:
                assert torch.equal(getattr(a, k), getattr(b, k)), (n, k)


def test_python_refusals():
    import torch
    from paper_2212_11142_amd import gp, seq
    docs = seq.Documents([4], [4])
    bf = torch.bfloat16
    att = seq.Attention(docs, 2, 1, 64, bf)
    q, k = torch.zeros((4, 2, 64), dtype=bf, device="cuda"), torch.zeros((4, 1, 64), dtype=bf, device="cuda")
    b = seq.AttendBuffers(att)
    for bad in (q.half(), q.cpu(), q[:3], torch.zeros((4, 2, 128), dtype=bf, device="cuda")[:, :, ::2]):
        with pytest.raises(ValueError):
            seq.attend_into(att, bad, k, k, b)
    with pytest.raises(ValueError):
        seq.attend_into(att, q, k, k, b, table=torch.zeros((2, 4), dtype=bf, device="cuda"))
    with pytest.raises(ValueError):
        seq.attend_grad_into(att, q, k, k, q, b)
    odd = torch.zeros(4 * 2 * 64 + 8, dtype=bf, device="cuda")[1:1 + 512].view(4, 2, 64)
    with pytest.raises(gp.GPError) as e:
        seq.attend_into(att, odd, k, k, b)
    assert e.value.status == 4
    for kw in (dict(heads=3, kv_heads=2), dict(dim=60), dict(dim=136), dict(cap=-1.0),
               dict(cap=math.nan), dict(scale=0.0), dict(buckets=seq.Buckets([1, 2])),
               dict(buckets=seq.Buckets([0, 2, 2])), dict(buckets=seq.Buckets([0, 2000]))):
        a = dict(heads=2, kv_heads=1, dim=64, dtype=bf)
        a.update(kw)
        with pytest.raises(gp.GPError):
            seq.Attention(docs, **a)
    with pytest.raises(gp.GPError):
        seq.Attention(seq.Documents([4], [4], prefix=[1]), 2, 1, 64, bf, causal=False)
    with pytest.raises(ValueError):
        seq.Documents([4], [4, 5])
    with pytest.raises(ValueError):
        seq.Documents([4], [4], q_rows=3)
    with pytest.raises(ValueError):
        seq.AttendBuffers(seq.Attention(seq.Documents([1, 1], [4, 4], k_begin=[0, 2]), 2, 1, 64, bf),
                          grad=True)
    x = torch.zeros((3, 10), device="cuda")
    t = torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(gp.GPError):
        seq.logprob(x, t, top=11)
    with pytest.raises(ValueError):
        seq.logprob(x, t.int())
    with pytest.raises(gp.GPError):
        seq.logprob(x, t, scale=-1.0)
    with pytest.raises(TypeError):
        seq.logprob(x.double(), t)


# ------------------------------------------------------------------ log probabilities
def _logprob_check(x, t, top=0, scale=1.0, grad=True, seed=0, bufs=None):
    """fp32 outputs: a row's sum of n terms, at most n / 256 + 64 of them one after another,
    is off by that many times 2^-24 relative; log and entropy by as much absolute, per unit
    of the terms' size; d has a few roundings of |x - max|."""
    import torch
    from paper_2212_11142_amd import seq
    T, V = x.shape
    g = torch.Generator().manual_seed(seed)
    gl = torch.randn(T, generator=g).cuda()
    ge = torch.randn(T, generator=g).cuda()
    b = bufs or seq.LogprobBuffers(T, V, x.dtype, top=top, grad=grad)
    seq.logprob_into(x, t, b, scale=scale)
    if grad:
        seq.logprob_grad_into(x, t, gl, ge, b, scale=scale)
    torch.cuda.synchronize()
    f = lambda a: a.double().cpu().numpy()
    r = gs.logprob(f(x), t.cpu().numpy(), top=top, scale=scale, g_logp=f(gl), g_entropy=f(ge))
    e = (V / 256 + 64) * 2.0 ** -24
    fin = lambda a: np.abs(np.where(np.isfinite(a), a, 0.0))
    size = 1 + fin(r["lse"])
    near(b.lse, r["lse"], e * size, "lse")
    near(b.logp, r["logp"], e * (size + fin(r["logp"])), "logp")
    near(b.entropy, r["entropy"], e * (size + fin(r["entropy"])), "entropy")
    if top:
        assert np.array_equal(b.top_id.cpu().numpy(), r["top_id"])
        near(b.top_logp, r["top_logp"], e * (size[:, None] + fin(r["top_logp"])), "top_logp")
    if grad:
        u = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}[x.dtype]
        tiny = 2.0 ** -25 if x.dtype == torch.float16 else 0.0     # fp16's subnormal step
        w = scale * (np.abs(f(gl)) + np.abs(f(ge)) * (size + fin(r["entropy"])))[:, None]
        near(b.dlogits, r["dlogits"], u * np.abs(r["dlogits"]) + 4 * e * w * size[:, None] *
             np.minimum(1.0, np.abs(r["dlogits"]) / np.maximum(w, 1e-30) + 1e-3) + tiny + e * w * 1e-3,
             "dlogits")
    return b


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("width", [1, 2, 63, 64, 65, 511, 1024, 1025, 2049, 8193, 40001])
def test_logprob_sizes(dtype, width):
    import torch
    g = torch.Generator().manual_seed(width)
    x = (torch.randn((5, width), generator=g) * 3).to(_torch_dtype(dtype)).cuda()
    t = torch.randint(0, width, (5,), generator=g).cuda()
    _logprob_check(x, t, top=min(width, 9), scale=1.0 if width % 2 else 0.7)


@pytest.mark.parametrize("rows", [1, 3, 513, 700])
@pytest.mark.parametrize("top", [1, 32, 33, 128])
def test_logprob_alternatives(rows, top):
    """Both sides of each dispatch line (rows per device, alternatives per group)."""
    import torch
    g = torch.Generator().manual_seed(rows)
    x = torch.randn((rows, 9001), generator=g).bfloat16().cuda()    # many equal logits
    t = torch.randint(0, 9001, (rows,), generator=g).cuda()
    _logprob_check(x[:20], t[:20], top=top, grad=False)
    from paper_2212_11142_amd import seq
    b = seq.logprob(x, t, top=top)
    order = torch.sort(x.float().cpu(), dim=1, descending=True, stable=True)[1][:, :top]
    assert torch.equal(b["top_id"].cpu(), order)


@pytest.mark.parametrize("rows", [2, 600])
def test_logprob_ties_and_crowded_threads(rows):
    """Equal rows; and rows whose best entries fall on few of a block's threads, more of
    them than its candidate list holds."""
    import torch
    from paper_2212_11142_amd import seq
    V = 8192
    x = torch.zeros((rows, V), device="cuda")
    v = torch.arange(V, device="cuda")
    thread = (v // 4) % 256          # of 256 threads with vectors of 4
    x[1::2] = torch.where(thread < 127, 2.0 + (v * 7919 % V).float() / V,
                          torch.where((thread == 127) & (v < 4096), 1.0, 0.0))
    t = torch.zeros(rows, dtype=torch.int64, device="cuda")
    for top in (20, 128):
        b = seq.logprob(x, t, top=top)
        order = torch.sort(x.cpu(), dim=1, descending=True, stable=True)[1][:, :top]
        assert torch.equal(b["top_id"].cpu(), order)
    wide = torch.zeros((2, 100000), dtype=torch.float16, device="cuda")
    b = seq.logprob(wide, t[:2], top=50)
    assert torch.equal(b["top_id"].cpu(), torch.arange(50).expand(2, 50))


@pytest.mark.parametrize("width", [1, 2, 700, 4096])
def test_logprob_rows_of_one_entry(width):
    """Everything but one entry ruled out: log probability, entropy and gradient are 0."""
    import torch
    from paper_2212_11142_amd import seq
    g = torch.Generator().manual_seed(3)
    x = torch.full((300, width), -math.inf)
    t = torch.randint(0, width, (300,), generator=g)
    x[torch.arange(300), t] = torch.randn(300, generator=g) * 5
    x, t = x.cuda(), t.cuda()
    bufs = seq.LogprobBuffers(300, width, torch.float32, grad=True)
    seq.logprob_into(x, t, bufs)
    one = torch.ones(300, device="cuda")
    seq.logprob_grad_into(x, t, one, one, bufs)
    torch.cuda.synchronize()
    assert bool((bufs.logp == 0).all()) and bool((bufs.entropy == 0).all())
    assert bool((bufs.dlogits == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,width", [(3, 100003), (5, 60001), (260, 9000), (7, 3000)])
def test_logprob_alternatives_of_few_values(rows, width, dtype):
    """Rows of two, three and many equal values, in every form: the lowest indices first."""
    import torch
    from paper_2212_11142_amd import seq
    g = torch.Generator().manual_seed(5)
    x = torch.randn((rows, width), generator=g).clamp(-1, 1).round()
    x[0] = 0.0
    x[1] = (torch.rand(width, generator=g) < 1e-3).float()
    x[2, width // 2:] = 3.0
    x = x.to(_torch_dtype(dtype)).cuda()
    t = torch.zeros(rows, dtype=torch.int64, device="cuda")
    order = torch.sort(x.float().cpu(), dim=1, descending=True, stable=True)[1]
    for top in (1, 20, 32, 33, 128):
        b = seq.logprob(x, t, top=top)
        assert torch.equal(b["top_id"].cpu(), order[:, :top]), top


@pytest.mark.parametrize("width", [40, 5000, 70000])
def test_logprob_values_at_the_ends(width):
    """Ruled out entries, rows of nothing else, the type's lowest value, infinities, NaN,
    rows with fewer entries left than alternatives, targets outside the row."""
    import torch
    x = torch.randn((10, width), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    low = torch.finfo(torch.bfloat16).min
    x[0, ::2] = -math.inf
    x[1] = -math.inf
    x[2] = low
    x[3] = low
    x[3, 7] = 1.0
    x[4, 5] = math.inf
    x[5, 9] = math.nan
    x[6] = -math.inf
    x[6, [3, 30]] = torch.tensor([2.0, 1.0]).bfloat16().cuda()
    x[7] = x[7] * 1000
    t = torch.tensor([0, 1, 2, 7, 5, 0, 3, 4, -100, width], device="cuda")
    b = _logprob_check(x[[0, 1, 2, 3, 6, 7, 8, 9]], t[[0, 1, 2, 3, 6, 7, 8, 9]], top=6)
    assert b.logp[-1] == 0 and b.logp[-2] == 0
    from paper_2212_11142_amd import seq
    b = seq.logprob(x, t, top=6)
    for r in (4, 5):
        assert b["lse"][r].isnan() or b["lse"][r].isposinf()
        assert b["logp"][r].isnan() and b["entropy"][r].isnan()
    assert b["top_id"][4, 0] == 5 and 9 not in b["top_id"][5].tolist()
    assert (b["top_id"] >= -1).all() and (b["top_id"] < width).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("width", [100, 5001])
def test_logprob_strides_and_in_place(dtype, width):
    """Rows of a wider matrix from an odd offset on, and the gradient over its logits."""
    import torch
    from paper_2212_11142_amd import seq
    dt = _torch_dtype(dtype)
    big = torch.randn((6, width + 13), generator=torch.Generator().manual_seed(2)).to(dt).cuda()
    x = big[:, 5:5 + width]
    t = torch.arange(6, device="cuda")
    b = _logprob_check(x, t, top=5)
    keep = big.clone()
    same = seq.LogprobBuffers(6, width, dt, grad=True)
    same.dlogits = x
    one = torch.ones(6, device="cuda")
    ref = seq.LogprobBuffers(6, width, dt, grad=True)
    seq.logprob_into(x, t, ref)
    seq.logprob_grad_into(x, t, one, one, ref)
    seq.logprob_into(x, t, same)
    seq.logprob_grad_into(x, t, one, one, same)
    torch.cuda.synchronize()
    assert torch.equal(x, ref.dlogits)
    assert torch.equal(big[:, :5], keep[:, :5]) and torch.equal(big[:, 5 + width:], keep[:, 5 + width:])


def test_logprob_grad_parts():
    """Each upstream gradient alone, and rows without a target."""
    import torch
    from paper_2212_11142_amd import seq
    x = torch.randn((4, 300), device="cuda")
    t = torch.tensor([1, -1, 299, 300], device="cuda")
    b = seq.LogprobBuffers(4, 300, torch.float32, grad=True)
    seq.logprob_into(x, t, b)
    one = torch.ones(4, device="cuda")
    seq.logprob_grad_into(x, t, one, None, b)
    a = b.dlogits.clone()
    assert (a[1] == 0).all() and (a[3] == 0).all()
    p = torch.softmax(x.double(), 1)
    want = -p
    want[0, 1] += 1
    want[2, 299] += 1
    assert torch.allclose(a[[0, 2]].double(), want[[0, 2]], atol=1e-5)
    seq.logprob_grad_into(x, None, None, one, b)
    assert b.dlogits.isfinite().all() and not (b.dlogits[1] == 0).all()


def test_no_rows():
    import torch
    from paper_2212_11142_amd import seq
    docs = seq.Documents([], [])
    att = seq.Attention(docs, 2, 2, 64, torch.bfloat16)
    z = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    b = seq.AttendBuffers(att, grad=True)
    seq.attend_into(att, z, z, z, b)
    seq.attend_grad_into(att, z, z, z, z, b)
    # keys that no query reads: their gradients are 0
    docs = seq.Documents([0, 0], [70, 3])
    att = seq.Attention(docs, 2, 2, 64, torch.bfloat16, buckets=seq.Buckets([0, 4]))
    k = torch.ones((73, 2, 64), dtype=torch.bfloat16, device="cuda")
    tab = torch.ones((2, 2), dtype=torch.bfloat16, device="cuda")
    b = seq.AttendBuffers(att, grad=True)
    b.dk.fill_(7), b.dv.fill_(7), b.dtable.fill_(7)
    seq.attend_into(att, z, k, k, b, table=tab)
    seq.attend_grad_into(att, z, k, k, z, b, table=tab)
    torch.cuda.synchronize()
    assert (b.dk == 0).all() and (b.dv == 0).all() and (b.dtable == 0).all()
    seq.logprob(torch.zeros((0, 5), device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"))
