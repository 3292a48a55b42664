"""The sequence operators' CPU oracle against closed forms and differences."""
import numpy as np
import pytest

from oracle import gp_seq as gs


def _inputs(rng, lens, H, Hk, D):
    tq, tk = sum(a for a, _, _ in lens), sum(b for _, b, _ in lens)
    docs, qb, kb = [], 0, 0
    for a, b, p in lens:
        docs.append((qb, qb + a, kb, kb + b, p))
        qb += a
        kb += b
    return (rng.normal(size=(tq, H, D)), rng.normal(size=(tk, Hk, D)),
            rng.normal(size=(tk, Hk, D)), docs)


def test_bucket_classes():
    d = np.arange(-20, 21)
    start = [0, 1, 2, 4, 9]
    one = gs.bucket_index(d, start, False)
    two = gs.bucket_index(d, start, True)
    for x, a, b in zip(d, one, two):
        back = max(-x, 0)
        assert a == max(c for c in range(5) if start[c] <= back)
        assert b == max(c for c in range(5) if start[c] <= abs(x)) + (5 if x > 0 else 0)


def test_equal_scores_average():
    rng = np.random.default_rng(0)
    q, k, v, docs = _inputs(rng, [(5, 5, 0), (3, 7, 2)], 2, 1, 4)
    r = gs.attend(np.zeros_like(q), k, v, docs, causal=True)
    for qb, qe, kb, ke, p in docs:
        for i in range(qe - qb):
            n = max(i + 1 + (ke - kb) - (qe - qb), p)
            for h in range(2):
                assert np.allclose(r["out"][qb + i, h], v[kb:kb + n, 0].mean(axis=0))
                assert np.isclose(r["lse"][h, qb + i], np.log(n))


def test_rows_that_see_nothing():
    rng = np.random.default_rng(1)
    q, k, v, docs = _inputs(rng, [(6, 2, 0)], 1, 1, 4)
    r = gs.attend(q, k, v, docs, causal=True, dout=np.ones_like(q))
    assert np.all(r["out"][:4] == 0) and np.all(np.isneginf(r["lse"][0, :4]))
    assert np.all(r["dq"][:4] == 0) and np.all(np.isfinite(r["dk"]))


@pytest.mark.parametrize("kw", [dict(causal=False), dict(causal=True, cap=1.5),
                                dict(causal=True, slopes=True), dict(causal=True, table=True),
                                dict(causal=False, table=True, cap=2.0)])
def test_gradient_against_differences(kw):
    rng = np.random.default_rng(2)
    kw = dict(kw)
    H, Hk, D = 4, 2, 3
    q, k, v, docs = _inputs(rng, [(5, 5, 0), (4, 6, 3), (3, 2, 0)], H, Hk, D)
    kw["scale"] = 0.7
    if kw.pop("slopes", False):
        kw["slopes"] = np.array([0.5, 0.25, 0.1, 0.0])
    table = None
    if kw.pop("table", False):
        table = rng.normal(size=(H, 6))
        kw.update(start=[0, 1, 3], two_sided=True)
    dout = rng.normal(size=q.shape)
    r = gs.attend(q, k, v, docs, table=table, dout=dout, **kw)

    def loss(a, b, c, t):
        return (gs.attend(a, b, c, docs, table=t, **kw)["out"] * dout).sum()

    args = [q, k, v, table]
    for n, name in enumerate(("dq", "dk", "dv", "dtable")):
        if args[n] is None:
            continue
        d = rng.normal(size=args[n].shape)
        h = 1e-6
        hi, lo = list(args), list(args)
        hi[n], lo[n] = args[n] + h * d, args[n] - h * d
        want = (loss(*hi) - loss(*lo)) / (2 * h)
        assert np.isclose((r[name] * d).sum(), want, rtol=1e-7, atol=1e-7)


def test_logprob_closed_forms_and_differences():
    rng = np.random.default_rng(3)
    x = rng.normal(size=(4, 9))
    x[1] = 0.5
    x[2, 4:] = -np.inf
    x[3] = -np.inf
    t = np.array([2, 3, 1, 0])
    r = gs.logprob(x, t, top=3, scale=1.7)
    assert np.isclose(r["entropy"][1], np.log(9)) and np.isclose(r["logp"][1], -np.log(9))
    assert list(r["top_id"][1]) == [0, 1, 2]
    assert np.isneginf(r["lse"][3]) and r["entropy"][3] == 0 and list(r["top_id"][3]) == [0, 1, 2]
    g, w = rng.normal(size=4), rng.normal(size=4)
    r = gs.logprob(x, t, scale=1.7, g_logp=g, g_entropy=w)

    def loss(y):
        s = gs.logprob(y, t, scale=1.7)
        return (g * s["logp"] + w * s["entropy"])[:3].sum()

    for i in range(3):
        for j in range(9):
            if np.isneginf(x[i, j]):
                assert r["dlogits"][i, j] == 0
                continue
            hi, lo = x.copy(), x.copy()
            hi[i, j] += 1e-6
            lo[i, j] -= 1e-6
            assert np.isclose(r["dlogits"][i, j], (loss(hi) - loss(lo)) / 2e-6, atol=1e-8)
    assert np.all(r["dlogits"][3] == 0)
