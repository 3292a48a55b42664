"""The sequence operators at their edges, on the GPU against the fp64 oracle: what lies outside
the documents, extremes of caps, offsets and probabilities, and calls of unusual sizes. Cases
and bounds are those of test_gpu_seq.py; what goes beyond them stands at each test."""
import math

import numpy as np
import pytest

from test_gpu_seq import TYPES, Case, _torch_dtype, near  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"\n[gpu] {request.node.nodeid}", flush=True)
    yield


# ------------------------------------------------------------------ caps without a bias
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv", [(96, 2), (24, 3), (2, 2)])   # one and two groups, few rows
@pytest.mark.parametrize("cap,bias", [(30.0, "none"), (30.0, "one"), (5.0, "slope"), (0.0, "none")])
def test_attend_whole_tiles(dtype, dim, heads, kv, cap, bias):
    """Tiles that every row sees, whose scores are not touched between the cap and the maximum."""
    for causal in (False, True):
        for grad in (False, True):
            Case(dtype, [(330, 330), (130, 400)], heads, kv, dim, causal=causal, cap=cap, bias=bias,
                 size=3.0, grad=grad).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_attend_scores_that_grow(dtype):
    """Every tile's scores are far above those before it, by more than the type's range: the
    running maximum has to follow."""
    import torch
    for heads, kv in ((96, 2), (24, 3), (2, 2)):
        for cap in (0.0, 60.0):
            c = Case(dtype, [(200, 500)], heads, kv, 64, causal=False, cap=cap)
            c.q[:] = 1.0
            c.k[:] = torch.randn((500, kv, 64), generator=torch.Generator().manual_seed(1)).cuda().to(c.dt)
            c.k[:, :, :8] += (torch.arange(500, device="cuda") // 16).to(c.dt)[:, None, None]
            c.check()


# ------------------------------------------------------------------ rows outside documents
def _gaps(x, spans, value):
    m = np.ones(x.shape[0], dtype=bool)
    for a, b in spans:
        m[a:b] = False
    y = x.clone()
    y[np.nonzero(m)[0].tolist()] = value
    return y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv,dim", [(2, 2, 64), (6, 2, 128), (64, 16, 64)])   # narrow and wide blocks
def test_grad_does_not_read_rows_outside_documents(dtype, heads, kv, dim):
    """Query and key rows that no document has hold large values, infinities and NaN: the
    gradients are bit for bit those with zeros there."""
    import torch
    from paper_2212_11142_amd import seq
    ql, kl, kb = [150, 1, 200], [150, 40, 130], [10, 300, 400]
    docs = seq.Documents(ql, kl, q_rows=400, k_rows=600, k_begin=kb)
    dt = _torch_dtype(dtype)
    att = seq.Attention(docs, heads, kv, dim, dt, buckets=seq.Buckets([0, 2, 9], True))
    g = torch.Generator().manual_seed(heads)
    q, do = (torch.randn((400, heads, dim), generator=g).to(dt).cuda() for _ in range(2))
    k, v = (torch.randn((600, kv, dim), generator=g).to(dt).cuda() for _ in range(2))
    table = torch.randn((heads, 6), generator=g).to(dt).cuda()
    keys = [(b, b + n) for b, n in zip(kb, kl)]
    want = None
    for value in (0.0, 6e4, math.inf, -math.inf, math.nan):
        x = [_gaps(t, s, value) for t, s in ((q, [(0, 351)]), (k, keys), (v, keys), (do, [(0, 351)]))]
        b = seq.AttendBuffers(att, grad=True)
        seq.attend_into(att, *x[:3], b, table=table)
        for t in (b.out, b.rest):
            t[351:] = value
        if value:
            b.lse[:, 351:] = 0.0
        seq.attend_grad_into(att, *x, b, table=table)
        torch.cuda.synchronize()
        got = [t.clone() for t in (b.dq, b.dk, b.dv, b.dtable)]
        if want is None:
            want = got
            assert all(bool((t != 0).any()) for t in want)
        for a, w, n in zip(got, want, ("dq", "dk", "dv", "dtable")):
            assert torch.equal(a, w), (n, value)


@pytest.mark.parametrize("heads,kv", [(4, 2), (64, 16)])
def test_grad_of_a_document_is_its_own(heads, kv):
    """Another document's large upstream gradients and values, and those of rows that see
    nothing, do not cost a document (fp16) its digits."""
    import torch
    c = Case("fp16", [(150, 150), (300, 5), (200, 200)], heads, kv, 64, grad=True)
    c.dout = (c.dout.float() * 2.0 ** -10).half()
    c.dout[150:445] = 6e4                     # rows 0..294 of the second document see nothing
    c.check()
    want = c.run()
    c.dout[450:] *= 2.0 ** 20                 # the third document's
    c.v[155:] *= 2.0 ** 10
    got = c.run()
    torch.cuda.synchronize()
    for n, rows in (("dq", 450), ("dk", 155), ("dv", 155)):
        assert torch.equal(getattr(got, n)[:rows], getattr(want, n)[:rows]), n


# ------------------------------------------------------------------ one class per side
@pytest.mark.parametrize("heads,kv", [(4, 2), (48, 24)])
@pytest.mark.parametrize("lens", [[(160, 193)], [(64, 65), (150, 151)], [(200, 233), (3, 36)]])
@pytest.mark.parametrize("causal", [False, True])
def test_two_sided_table_of_one_class(heads, kv, lens, causal):
    """One class per side: distance 0 belongs to the side behind, wherever the pair lies in a
    tile."""
    for grad in (False, True):
        Case("bf16", lens, heads, kv, 64, causal=causal, bias="two", start=(0,), grad=grad).check()


# ------------------------------------------------------------------ caps
@pytest.mark.parametrize("heads,kv", [(4, 2), (48, 24)])
@pytest.mark.parametrize("cap", [1e-3, 0.5, 60.0, 70.0, 1e3, 1e4, 1e6, 1e30, 3e38])
def test_caps_of_every_size(heads, kv, cap):
    """A cap far above the scores leaves them as they are, one far below leaves their signs."""
    for dtype, dim, size in (("fp16", 64, 2.0), ("bf16", 128, 30.0)):
        Case(dtype, [(140, 140), (33, 70)], heads, kv, dim, cap=cap, bias="two", size=size,
             grad=True).check()


@pytest.mark.parametrize("cap", [64.0, 65.0, 5e3])
def test_caps_about_the_scores(cap):
    """Scores on both sides of the cap."""
    for heads in (2, 96):
        c = Case("bf16", [(130, 130)], heads, 2, 64, cap=cap, grad=True)
        c.q *= cap / 8.0
        c.q[5:9] *= 2.0 ** -20
        c.check()


@pytest.mark.parametrize("cap", [1e-37, 1e-39, 1e-44])
def test_caps_near_zero(cap):
    """Scores of nothing: every visible key has the same weight, for queries of 0 too."""
    for heads in (2, 96):
        c = Case("bf16", [(130, 130)], heads, 2, 64, cap=cap)
        c.q[3:60] = 0.0
        c.check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cap", [20.0, 50.0, 64.0])
@pytest.mark.parametrize("heads,kv", [(4, 2), (96, 32)])
def test_caps_of_few_keys(dtype, cap, heads, kv):
    """Documents of up to 8 keys, where a log-sum is little more than one score: capped scores
    are off by 2^-21 of themselves, the sum and its logarithm by as much of 1 + lse."""
    c = Case(dtype, [(1, 1)] * 9 + [(2, 2), (5, 3), (8, 8), (17, 4)], heads, kv, 64, cap=cap, size=0.3,
             bias="one", grad=True)
    c.table *= 0.0
    b, ref = c.run(), c.oracle()
    lse = np.where(np.isfinite(ref["lse"]), np.abs(ref["lse"]), 0.0)
    near(b.lse, ref["lse"], 2.0 ** -21 * (1 + ref["score"]) + 2.0 ** -22 * lse, "lse")
    c.check(b, ref)


# ------------------------------------------------------------------ offsets of logits
@pytest.mark.parametrize("rows,width", [(70, 300), (5, 3000), (300, 5000), (6, 70000)])
@pytest.mark.parametrize("offset", [0.0, 2.0 ** 10, 2.0 ** 20, -2.0 ** 20])
def test_logprob_grad_of_rows_with_an_offset(rows, width, offset):
    """What a row's logits have in common cancels: the gradient has the same error with it as
    without. Logits are multiples of 2^-3 within 16 (exact with the offsets). p = e^d, d a
    few fp32 roundings of |d| < 64 and of the sum's logarithm off, e of test_gpu_seq.py and
    2^-18 together; the result is rounded."""
    import torch
    from oracle import gp_seq as gs
    from paper_2212_11142_amd import seq
    g = torch.Generator().manual_seed(width)
    x = (torch.randn((rows, width), generator=g) * 2.5).clamp(-16, 16).mul(8).round() / 8
    t = torch.randint(0, width, (rows,), generator=g)
    gl, ge = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    b = seq.LogprobBuffers(rows, width, torch.float32, grad=True)
    y, tc = (x + offset).cuda(), t.cuda()
    assert torch.equal(y.double().cpu() - offset, x.double())
    seq.logprob_into(y, tc, b)
    seq.logprob_grad_into(y, tc, gl.cuda(), ge.cuda(), b)
    torch.cuda.synchronize()
    f = lambda a: a.double().numpy()
    r = gs.logprob(f(x), t.numpy(), g_logp=f(gl), g_entropy=f(ge))
    lp = f(x) - r["lse"][:, None]
    e = (width / 256 + 64) * 2.0 ** -24 + 2.0 ** -18
    w = np.abs(f(gl))[:, None] + np.abs(f(ge))[:, None] * (1 + np.abs(lp) + r["entropy"][:, None])
    near(b.dlogits, r["dlogits"], 2.0 ** -24 * np.abs(r["dlogits"]) + 2 * e * w * np.exp(lp), "dlogits")


def test_logprob_grad_of_rows_at_the_types_ends():
    """Rows whose log-sum is beyond fp32 (the lowest value in every place, at a scale above 1)
    still have the gradient of equal entries."""
    import torch
    from paper_2212_11142_amd import seq
    for width in (40, 5000):
        x = torch.full((3, width), torch.finfo(torch.float32).min, device="cuda")
        x[1] = torch.finfo(torch.float32).max
        x[2, 1:] = -math.inf
        x[2, 0] = torch.finfo(torch.float32).max
        t = torch.tensor([1, 1, 0], device="cuda")
        b = seq.LogprobBuffers(3, width, torch.float32, grad=True)
        one = torch.ones(3, device="cuda")
        seq.logprob_into(x, t, b, scale=2.0)
        seq.logprob_grad_into(x, t, one, one, b, scale=2.0)
        want = torch.full((3, width), -2.0 / width, dtype=torch.float64)
        want[:2, 1] += 2.0
        want[2] = 0.0
        assert torch.allclose(b.dlogits.double().cpu(), want, rtol=1e-4, atol=1e-9)
        assert torch.allclose(b.logp[:2].cpu(), torch.full((2,), -math.log(width)), rtol=1e-5)


def test_logprob_grad_from_log_sums_alone():
    """gp_logprob and gp_logprob_grad, whose only memory of the forward pass is lse and
    entropy: p's relative error grows with |lse|."""
    import ctypes as C

    import torch
    from paper_2212_11142_amd import gp, seq
    lib = gp.load()
    rows, width = 9, 700
    x = torch.randn((rows, width), generator=torch.Generator().manual_seed(0)).cuda()
    t = torch.arange(rows, device="cuda")
    gl, ge = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    b = seq.LogprobBuffers(rows, width, torch.float32, grad=True)
    seq.logprob_into(x, t, b)
    seq.logprob_grad_into(x, t, gl, ge, b)
    logp, entropy, lse = (torch.empty(rows, device="cuda") for _ in range(3))
    dx = torch.empty_like(x)
    p = lambda a: C.c_void_p(a.data_ptr())
    s = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert lib.gp_logprob(2, p(x), width, rows, width, 1.0, p(t), 0, p(logp), p(entropy), p(lse), None,
                          None, None, 0, s) == 0
    assert lib.gp_logprob_grad(2, p(x), width, rows, width, 1.0, p(t), p(lse), p(entropy), p(gl),
                               p(ge), p(dx), width, s) == 0
    torch.cuda.synchronize()
    for a, w in ((logp, b.logp), (entropy, b.entropy), (lse, b.lse)):
        assert torch.equal(a, w)
    w = gl.abs()[:, None] + ge.abs()[:, None] * 16
    bound = torch.exp(x - lse[:, None]) * w * 2.0 ** -24 * 4 * (1 + lse.abs()[:, None]) + 2.0 ** -23 * dx.abs()
    assert bool(((dx - b.dlogits).abs() <= bound).all())


# ------------------------------------------------------------------ small probabilities
@pytest.mark.parametrize("heads,rows,keys", [(192, 130, 1 << 16), (24, 120, 1 << 16), (192, 130, 4096),
                                             (1, 1, 1024), (1, 5, 700)])
@pytest.mark.parametrize("grad", [False, True])
def test_small_probabilities_of_many_keys(heads, rows, keys, grad):
    """fp16: one key has nearly all of the weight and the value 0; the others, e^-18 each,
    make the output. A probability is kept to half of fp16's smallest step, 2^-25, at 2^7 times
    the row's (running) maximum, 2^14 in documents of more than 4096 keys: each is off by 2^-32
    (2^-39) of the largest beside its relative rounding u and e."""
    import torch
    from paper_2212_11142_amd import seq
    d = 64
    q = torch.zeros((rows, heads, d), dtype=torch.float16, device="cuda")
    k = torch.zeros((keys, 1, d), dtype=torch.float16, device="cuda")
    v = torch.full((keys, 1, d), 64.0, dtype=torch.float16, device="cuda")
    q[:, :, 0], k[0, 0, 0], v[0] = 8.0, 18.0, 0.0
    att = seq.Attention(seq.Documents([rows], [keys]), heads, 1, d, torch.float16, causal=False)
    b = seq.AttendBuffers(att, grad=grad)
    seq.attend_into(att, q, k, v, b)
    torch.cuda.synchronize()
    tail = (keys - 1) * math.exp(-18.0)
    want = 64.0 * tail / (1.0 + tail)
    u, e = 2.0 ** -11, 2.0 ** -19 * 19
    bound = 1.1 * ((2 * u + e) * want + 64.0 * keys * 2.0 ** (-39 if keys > 4096 else -32) + 2.0 ** -25)
    err = (b.out.double() - want).abs().max().item()
    assert err <= bound, (err, bound, want)


# ------------------------------------------------------------------ very many rows
@pytest.mark.parametrize("rows,width,grad", [((1 << 26) + 5, 3, True), ((1 << 24) + 3, 4100, False)])
def test_logprob_of_more_rows_than_a_launch_takes(rows, width, grad):
    """A launch has fewer than 2^32 threads: these rows take several. (One stored row, read
    by all.)"""
    import torch
    from paper_2212_11142_amd import seq
    x = torch.randn((1, width), generator=torch.Generator().manual_seed(0)).bfloat16().cuda()
    few = seq.LogprobBuffers(2, width, torch.bfloat16, grad=grad)
    many = seq.LogprobBuffers(rows, width, torch.bfloat16, grad=grad)
    for t in (many.logp, many.entropy, many.lse):
        t.fill_(7.0)
    for b in (few, many):
        n = b.rows
        t = torch.arange(n, device="cuda") % 2
        seq.logprob_into(x.expand(n, -1), t, b)
        if grad:
            one = torch.ones(n, device="cuda")
            seq.logprob_grad_into(x.expand(n, -1), t, one, None, b)
    names = ("logp", "entropy", "lse") + (("dlogits",) if grad else ())
    for n in names:
        a, w = getattr(many, n), getattr(few, n)
        assert bool((a[0::2] == w[0]).all()) and bool((a[1::2] == w[1]).all()), n


# ------------------------------------------------------------------ ranges that move
@pytest.mark.parametrize("heads,kv", [(4, 2), (96, 2)])
def test_rows_that_leave_the_documents_become_zero(heads, kv):
    """Ranges on the device shrink between calls: the outputs of the rows that no document has
    now are 0 (lse -inf), not the earlier call's."""
    import torch
    from paper_2212_11142_amd import seq
    i32 = dict(dtype=torch.int32, device="cuda")
    qb, qe = torch.tensor([0, 150], **i32), torch.tensor([150, 300], **i32)
    kb, ke = torch.tensor([0, 150], **i32), torch.tensor([150, 300], **i32)
    docs = seq.Documents.on_device(qb, qe, kb, ke, 300, 300, 150, 150)
    att = seq.Attention(docs, heads, kv, 64, torch.bfloat16)
    g = torch.Generator().manual_seed(0)
    q, do = (torch.randn((300, heads, 64), generator=g).bfloat16().cuda() for _ in range(2))
    k, v = (torch.randn((300, kv, 64), generator=g).bfloat16().cuda() for _ in range(2))

    def call(b):
        seq.attend_into(att, q, k, v, b)
        seq.attend_grad_into(att, q, k, v, do, b)
        torch.cuda.synchronize()

    b = seq.AttendBuffers(att, grad=True)
    call(b)
    assert bool((b.dq[100:150] != 0).any())
    qe[0], ke[0] = 100, 120
    call(b)
    fresh = seq.AttendBuffers(att, grad=True)
    call(fresh)
    for n in ("out", "dq"):
        assert bool((getattr(b, n)[100:150] == 0).all()), n
    for n in ("dk", "dv"):
        assert bool((getattr(b, n)[120:150] == 0).all()), n
    assert bool(b.lse[:, 100:150].isneginf().all())
    for n in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(b, n), getattr(fresh, n)), n


def test_ranges_that_cover_every_row():
    """The promise that documents have every query row leaves the outputs' clearing out."""
    import torch
    from paper_2212_11142_amd import seq
    i32 = dict(dtype=torch.int32, device="cuda")
    at = torch.arange(3, **i32)
    ke = torch.tensor([40, 90, 130], **i32)
    docs = seq.Documents.on_device(at, at + 1, at * 200, at * 200 + ke, 3, 600, 1, 200, q_full=True)
    att = seq.Attention(docs, 4, 2, 64, torch.bfloat16)
    q, k, v = (torch.randn(s, device="cuda").bfloat16() for s in ((3, 4, 64), (600, 2, 64), (600, 2, 64)))
    got = seq.attend(att, q, k, v)
    want = seq.attend(seq.Attention(seq.Documents([1] * 3, [40, 90, 130], k_begin=[0, 200, 400], k_rows=600),
                                    4, 2, 64, torch.bfloat16), q, k, v)
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])


# ------------------------------------------------------------------ nothing to read
@pytest.mark.parametrize("bias", [False, True])
def test_grad_of_documents_without_keys(bias):
    """Many queries over a cache in which their documents have no keys yet."""
    import torch
    from paper_2212_11142_amd import seq
    docs = seq.Documents([1000, 700], [0, 0], k_rows=640)
    buckets = seq.Buckets([0, 3]) if bias else None
    att = seq.Attention(docs, 4, 2, 64, torch.bfloat16, buckets=buckets)
    q, k = (torch.ones((n, h, 64), dtype=torch.bfloat16, device="cuda") for n, h in ((1700, 4), (640, 2)))
    table = torch.ones((4, 2), dtype=torch.bfloat16, device="cuda") if bias else None
    b = seq.AttendBuffers(att, grad=True)
    seq.attend_into(att, q, k, k, b, table=table)
    seq.attend_grad_into(att, q, k, k, q, b, table=table)
    torch.cuda.synchronize()
    for x in (b.out, b.dq, b.dk, b.dv) + ((b.dtable,) if bias else ()):
        assert bool((x == 0).all())
    assert bool(b.lse.isneginf().all())


# ------------------------------------------------------------------ alternatives beside NaN
@pytest.mark.parametrize("rows", [3, 600])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("width", [9000, 80000])
def test_ruled_out_entries_among_nan_are_alternatives(rows, dtype, width):
    """A NaN is no alternative, an entry ruled out is one (the last): where nothing else is
    left those are found, in the places behind a thread's vectors of NaN too."""
    import torch
    from paper_2212_11142_amd import seq
    x = torch.full((rows, width), math.nan)
    x[0, 2048:2056] = -math.inf
    x[1, 5000:5003] = -math.inf
    x[1, 8991] = 1.0
    x[2] = -math.inf
    x = x.to(_torch_dtype(dtype)).cuda()
    t = torch.zeros(rows, dtype=torch.int64, device="cuda")
    for top in (6, 40):
        ids = seq.logprob(x, t, top=top)["top_id"].cpu()
        none = lambda n: torch.full((n,), -1, dtype=torch.int64)
        assert torch.equal(ids[0], torch.cat([torch.arange(2048, 2056), none(40)])[:top])
        assert torch.equal(ids[1], torch.cat([torch.tensor([8991, 5000, 5001, 5002]), none(40)])[:top])
        assert torch.equal(ids[2], torch.arange(top))
        assert bool((ids[3:] == -1).all())


# ------------------------------------------------------------------ what rounding took
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv,dim", [(96, 4, 64), (40, 4, 128), (12, 4, 64)])   # one and two groups, few rows
def test_out_and_rest_are_out_before_rounding(dtype, heads, kv, dim):
    """rest is the rest of the out that was stored, where it lies halfway between two numbers
    too: their sum has the probabilities' error (two terms of u each) and rest's own rounding."""
    import torch  # noqa: F401
    c = Case(dtype, [(200, 300), (130, 130)], heads, kv, dim, grad=True, seed=heads)
    b, ref = c.run(), c.oracle()
    got = b.out.double() + b.rest.double()
    u, e = c.u, 2.0 ** -19 * (1 + ref["score"])
    grid = 2.0 ** -25 if dtype == "fp16" else 0.0
    near(got, ref["out"], u * u * np.abs(ref["out"]) + (u * u + e) * ref["out_abs"] + grid, "out + rest")


# ------------------------------------------------------------------ short documents
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 72), (48, 12, 64), (64, 64, 128)])    # narrow and wide blocks
@pytest.mark.parametrize("cap,bias", [(0.0, "none"), (30.0, "two"), (0.0, "slope")])
def test_grad_of_short_documents(dtype, heads, kv, dim, cap, bias):
    """Documents of up to 128 rows: dS enters its products in two terms, of u^2 each, so that dq
    and dk have no more than the results' own rounding, and the sums' errors."""
    lens = [(2, 2), (3, 2), (2, 128), (17, 17), (128, 128), (100, 5)]
    c = Case(dtype, lens, heads, kv, dim, causal=True, cap=cap, bias=bias, grad=True)
    b, ref = c.run(), c.oracle()
    u, e = c.u, 2.0 ** -19 * (1 + ref["score"])
    grid = 2.0 ** -25 if dtype == "fp16" else 0.0
    for n in ("dq", "dk"):
        near(getattr(b, n), ref[n], u * np.abs(ref[n]) + (u * u + e) * (ref[n + "_abs"] + ref[n + "_dif"])
             + grid, n)
    c.check(b, ref)


# ------------------------------------------------------------------ buffers of another layout
@pytest.mark.parametrize("full_first", [False, True])
def test_buffers_used_with_other_documents(full_first):
    """Buffers of one layout used with another of the same sizes: the rows of no document are 0
    there too, not the other layout's results or what the memory held."""
    import torch
    from paper_2212_11142_amd import seq
    g = torch.Generator().manual_seed(0)
    q, do = (torch.randn((300, 4, 64), generator=g).bfloat16().cuda() for _ in range(2))
    k, v = (torch.randn((300, 2, 64), generator=g).bfloat16().cuda() for _ in range(2))
    a = (seq.Documents([150, 150]) if full_first else
         seq.Documents([150, 140], q_rows=300, k_begin=[0, 160], k_rows=300))
    b = seq.Documents([90, 60], [90, 60], q_rows=300, k_begin=[20, 200], k_rows=300)
    att = [seq.Attention(d, 4, 2, 64, torch.bfloat16) for d in (a, b)]
    bufs = seq.AttendBuffers(att[0], grad=True)
    for t in (bufs.out, bufs.lse, bufs.dq, bufs.dk, bufs.dv):
        if full_first:
            t.fill_(7.0)
    big = max(x.workspace_bytes(True) for x in att)
    bufs.grad_workspace = torch.empty(big, dtype=torch.uint8, device="cuda")
    bufs.grad_workspace_bytes = big
    small = max(x.workspace_bytes(False) for x in att)
    if small:
        bufs.workspace = torch.empty(small, dtype=torch.uint8, device="cuda")
        bufs.workspace_bytes = small
    for x in (att[0], att[1], att[0], att[1]):
        seq.attend_into(x, q, k, v, bufs)
        seq.attend_grad_into(x, q, k, v, do, bufs)
        own = seq.AttendBuffers(x, grad=True)
        seq.attend_into(x, q, k, v, own)
        seq.attend_grad_into(x, q, k, v, do, own)
        torch.cuda.synchronize()
        for n in ("out", "lse", "dq", "dk", "dv"):
            assert torch.equal(getattr(bufs, n), getattr(own, n)), n
