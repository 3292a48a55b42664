"""CPU fp64 definitions of the sequence-surrogate operators: attention over documents with
its gradient, and log probabilities with theirs. Loops over documents and heads; every pair
is written out.

Each function also returns error scales: the sums of absolute values that a rounded
computation's error is proportional to, from which tests derive their bounds.
"""
import numpy as np


def bucket_index(delta, start, two_sided):
    """Class of each distance delta = key - query position."""
    delta = np.asarray(delta)
    start = np.asarray(start)
    a = np.abs(delta) if two_sided else np.maximum(-delta, 0)
    c = np.searchsorted(start, a, side="right") - 1
    return np.where(delta > 0, c + len(start), c) if two_sided else c


def visible(lq, lk, causal, prefix):
    """[lq, lk] booleans."""
    pos = np.arange(lq)[:, None] + lk - lq
    key = np.arange(lk)[None, :]
    if not causal:
        return np.ones((lq, lk), bool)
    return (key <= pos) | (key < prefix)


def _scores(q, k, lq, lk, causal, prefix, scale, cap, slope, table, start, two_sided):
    z = scale * (q @ k.T)
    fac = np.ones_like(z)
    if cap > 0:
        t = np.tanh(z / cap)
        z, fac = cap * t, 1.0 - t * t
    delta = np.arange(lk)[None, :] - (np.arange(lq)[:, None] + lk - lq)
    idx = None
    s = z
    if slope is not None:
        s = s - slope * np.abs(delta)
    if table is not None:
        idx = bucket_index(delta, start, two_sided)
        s = s + table[idx]
    see = visible(lq, lk, causal, prefix)
    s = np.where(see, s, -np.inf)
    return s, fac, idx, see


def _softmax(s):
    if s.shape[1] == 0:
        return s, np.full(s.shape[0], -np.inf)
    m = s.max(axis=1, keepdims=True)
    m0 = np.where(np.isneginf(m), 0.0, m)
    with np.errstate(invalid="ignore"):
        e = np.exp(s - m0)
    l = e.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (m0 + np.log(l))[:, 0]
    return e / np.where(l == 0, 1.0, l), lse


def attend(q, k, v, docs, causal=True, scale=1.0, cap=0.0, slopes=None, table=None, start=None,
           two_sided=False, dout=None):
    """q [Tq, H, D], k and v [Tk, Hk, D] fp64; docs: (q_begin, q_end, k_begin, k_end, prefix)
    tuples. Returns out, lse and, with dout, the gradients; and the error scales. Rows of no
    document are 0 (lse -inf)."""
    H, Hk, D = q.shape[1], k.shape[1], q.shape[2]
    group = H // Hk
    r = {"out": np.zeros_like(q), "lse": np.full((H, q.shape[0]), -np.inf),
         "out_abs": np.zeros_like(q), "score": 0.0}
    if dout is not None:
        for name, x in (("dq", q), ("dk", k), ("dv", v)):
            r[name], r[name + "_abs"], r[name + "_dif"] = (np.zeros_like(x) for _ in range(3))
        if table is not None:
            r["dtable"], r["dtable_abs"], r["dtable_dif"] = (np.zeros_like(table)
                                                             for _ in range(3))
    for qb, qe, kb, ke, prefix in docs:
        lq, lk = qe - qb, ke - kb
        if lq <= 0:
            continue
        for h in range(H):
            g = h // group
            Q, K, V = q[qb:qe, h], k[kb:ke, g], v[kb:ke, g]
            s, fac, idx, see = _scores(Q, K, lq, lk, causal, prefix, scale, cap,
                                       None if slopes is None else slopes[h],
                                       None if table is None else table[h], start, two_sided)
            P, lse = _softmax(s)
            # a masked place's value takes no part, whatever it is
            Vm = np.where(np.isfinite(V), V, 0.0)
            out = P @ Vm
            for j, c in zip(*np.nonzero(~np.isfinite(V))):
                rows = see[:, j]
                out[rows, c] += V[j, c]
            r["out"][qb:qe, h] = out
            r["lse"][h, qb:qe] = lse
            r["out_abs"][qb:qe, h] = P @ np.abs(Vm)
            fin = s[np.isfinite(s)]
            size = scale * (np.abs(Q) @ np.abs(np.where(np.isfinite(K), K, 0.0)).T)
            if fin.size:
                r["score"] = max(r["score"], np.abs(fin).max(), size.max())
            if dout is None:
                continue
            dO = dout[qb:qe, h]
            dP = dO @ V.T
            Dr = (P * dP).sum(axis=1, keepdims=True)
            dS = P * (dP - Dr)
            dZ = dS * fac
            r["dq"][qb:qe, h] = scale * dZ @ K
            r["dk"][kb:ke, g] += scale * dZ.T @ Q
            r["dv"][kb:ke, g] += P.T @ dO
            # what the errors of dS are proportional to: |dS| itself (its rounding), and the
            # absolute sums behind the difference dP - D
            aP = np.abs(dO) @ np.abs(V).T
            dif = P * (aP + (P * aP).sum(axis=1, keepdims=True))
            for name, m in (("abs", np.abs(dZ)), ("dif", dif)):
                r["dq_" + name][qb:qe, h] = scale * m @ np.abs(K)
                r["dk_" + name][kb:ke, g] += scale * m.T @ np.abs(Q)
            r["dv_abs"][kb:ke, g] += P.T @ np.abs(dO)
            if table is not None:
                np.add.at(r["dtable"][h], idx, dS)
                np.add.at(r["dtable_abs"][h], idx, np.abs(dS))
                np.add.at(r["dtable_dif"][h], idx, dif)
    return r


def logprob(x, targets, top=0, scale=1.0, g_logp=None, g_entropy=None):
    """Rows of logits [T, V]: lse, logp, entropy, the best alternatives, and the gradient."""
    T, V = x.shape
    r = {"lse": np.empty(T), "logp": np.zeros(T), "entropy": np.zeros(T),
         "top_logp": np.full((T, top), np.nan), "top_id": np.full((T, top), -1, np.int64),
         "dlogits": np.zeros((T, V))}
    for t in range(T):
        row = scale * x[t]
        order = [i for i in np.argsort(-x[t], kind="stable") if not np.isnan(x[t, i])][:top]
        r["top_id"][t, :len(order)] = order
        m = np.max(row)
        has = 0 <= targets[t] < V
        if np.isneginf(m):
            r["lse"][t] = -np.inf
            r["logp"][t] = -np.inf if has else 0.0
            r["top_logp"][t, :len(order)] = -np.inf
            continue
        with np.errstate(invalid="ignore", divide="ignore"):
            e = np.exp(row - m)
            lse = m + np.log(e.sum())
            lp = row - lse
            p = np.exp(lp)
            H = -np.sum(np.where(p > 0, p * np.where(np.isneginf(lp), 0, lp), 0.0)) \
                if not np.isnan(lse) else np.nan
        r["lse"][t], r["entropy"][t] = lse, H
        if has:
            r["logp"][t] = lp[targets[t]]
        r["top_logp"][t, :len(order)] = lp[order]
        g = g_logp[t] if (g_logp is not None and has) else 0.0
        w = g_entropy[t] if g_entropy is not None else 0.0
        d = -g * p - w * np.where(p > 0, p * (np.where(p > 0, lp, 0) + H), 0.0)
        if has:
            d[targets[t]] += g
        r["dlogits"][t] = scale * d
    return r
