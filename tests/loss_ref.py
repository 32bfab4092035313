"""Plain binary64 implementations of the log probabilities, the balance loss and their
gradients (test infrastructure), each with a bound of the error that the kernels' binary32
steps may make.

With u = 2^-24, to first order.  An exponent t = (x - m) log2(e) / T has three roundings (the
difference, the constant, the product), 3 u |t|, so 2^t is off by 3 ln(2) u |t| and the
hardware's 2 u of itself: POWER(t) = u (2 + 2.1 |t|).  A sum of positive terms adds at most u of
itself an addition on the longest chain; a lane adds up to 16 vectors of 8, the lanes, wavefronts
and chunks in trees and short loops (SUM = 200 additions bounds all shapes tested here).
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8 + 2.0 ** -24}   # (bfloat16 by way of binary32)
SUM = 200
LOG2E = 1.4426950408889634


def power(t):
    return U * (2 + 2.1 * np.abs(t))


def logprob(X, tokens, K=0, temperature=1.0):
    """Row by row: dict of logp, entropy, stats, top_vals, top_idx and their bounds
    (``*_err``)."""
    N, V = X.shape
    tau = float(np.float32(temperature))
    T = 0 if tokens is None else tokens.shape[1]
    r = dict(logp=np.zeros((N, T)), entropy=np.full(N, np.nan), stats=np.full((N, 2), np.nan),
             top_vals=np.full((N, K), np.nan), top_idx=np.full((N, K), -1, np.int32))
    r.update(logp_err=np.zeros((N, T)), entropy_err=np.zeros(N), stats_err=np.zeros((N, 2)),
             top_vals_err=np.zeros((N, K)))
    for n in range(N):
        x = X[n]
        inside = [t for t in range(T) if 0 <= tokens[n, t] < V]
        m = x.max()
        if np.isnan(x).any() or not np.isfinite(m):
            r["logp"][n, inside] = np.nan
            continue
        z = (x - m) / tau
        e = np.exp(z)
        big = int(np.argmax(x))
        e[big] = 0.0
        live = e > 0
        t = np.where(live, z, 0.0) * LOG2E
        s = e.sum()
        # (the hardware's 2^t is 0 where it would be below 2^-126: such a weight is lost as a whole;
        # twice that bounds where the exponent's own error puts it there)
        gone = np.where(e < 2.0 ** -125, e, 0.0)
        ds = (e * (power(t) + SUM * U) + gone).sum()
        w = (e * -t).sum()
        dw = (e * -t * (power(t) + (SUM + 3) * U) + gone * -t).sum()
        ln_d, dln = np.log1p(s), ds / (1 + s)

        def lp(j):
            # (tokens next to the largest keep the digits of ln d)
            v = (x[j] - m) / tau - ln_d
            return v, U * abs(v) + dln if np.isfinite(v) else 0.0
        for i in inside:
            r["logp"][n, i], r["logp_err"][n, i] = lp(tokens[n, i])
        h = np.log(2.0) * w / (1 + s)
        r["entropy"][n] = ln_d + h
        r["entropy_err"][n] = U * (ln_d + h) + dln * (1 + h) + np.log(2.0) * dw / (1 + s)
        r["stats"][n], r["stats_err"][n] = (m, s), (0.0, ds + U * s)
        order = np.lexsort((np.arange(V), -x))[:K]
        r["top_idx"][n] = order
        for k, j in enumerate(order):
            r["top_vals"][n, k], r["top_vals_err"][n, k] = lp(j)
    return r


def logprob_bwd(X, tokens, dlogp, dentropy=None, temperature=1.0, dtype="f32"):
    """(dx, bound): from d ln p_t / dz_j = 1[j = t] - p_j and dH / dz_j = -p_j (ln p_j + H)."""
    N, V = X.shape
    tau = float(np.float32(temperature))
    out, err = np.zeros((N, V)), np.zeros((N, V))
    for n in range(N):
        x = X[n]
        T = 0 if tokens is None else tokens.shape[1]
        inside = [i for i in range(T) if 0 <= tokens[n, i] < V]
        g = np.array([dlogp[n, i] for i in inside])
        h = 0.0 if dentropy is None else float(dentropy[n])
        if not (g != 0).any() and h == 0:
            continue
        m = x.max()
        if np.isnan(x).any() or not np.isfinite(m) or np.isnan(g).any() or np.isnan(h):
            out[n] = np.nan
            continue
        z = (x - m) / tau
        e = np.exp(z)
        d = e.sum()
        p, ln_p = e / d, z - np.log(d)
        lnp0 = np.where(p > 0, ln_p, 0.0)
        H = -(p * lnp0).sum()
        G, A = g.sum(), np.abs(g).sum()
        dx = -p * G - h * p * (lnp0 + H)
        size = A + abs(h) * (H + np.abs(lnp0))
        t = np.where(e > 0, z, 0.0) * LOG2E
        # the weight, 1 + s as logprob_fwd sums it (``logprob``), H as given (u and of what it
        # stands in), the row's two constants and three operations; the sum of the tokens'
        # gradients
        ds = (e * (power(t) + SUM * U)).sum() / d
        bound = p * (power(t) + 8 * U + ds) * size + p * len(g) * U * A
        for i, j in enumerate(inside):
            dx[tokens[n, j]] += g[i]
        out[n] = dx / tau
        err[n] = bound / tau + HALF[dtype] * np.abs(out[n]) + 2.0 ** -125 * size / tau
        if dtype == "bf16":
            err[n] += 2.0 ** -134
    return out, err


def shares(X, score):
    """(q, 1 - sigma, bound of q's relative error, without what a slope of x adds)."""
    if score == "softmax":
        z = X - X.max(axis=1, keepdims=True)
        e, slope = np.exp(z), np.ones_like(X)
    else:
        z = np.minimum(X, 0.0)
        z = z - z.max(axis=1, keepdims=True)
        f = 1.0 / (1.0 + np.exp(-np.abs(X)))
        e, slope = np.exp(z) * f, np.where(X > 0, np.exp(-np.abs(X)) * f, f)
    q = e / e.sum(axis=1, keepdims=True)
    t = np.where(np.isfinite(z), z, 0.0) * LOG2E
    # an exponential; for the sigmoid another one, an addition and a reciprocal; the sum of at
    # most 16 a lane and 6 steps, its reciprocal, the product
    one = power(t)
    if score != "softmax":
        one = one + power(np.where(np.isfinite(X), X, 0.0) * LOG2E) + 4 * U
    err = one + (q * one).sum(axis=1, keepdims=True) + 28 * U
    return q, slope, err


def sequences(starts, N):
    if starts is None:
        return [(0, N)]
    at = np.clip(np.asarray(starts, np.int64), 0, N)
    return list(zip(at[:-1], at[1:]))


def balance(X, idx, starts=None, score="softmax", scale=1.0):
    """dict of loss, counts, probs, rows and the bounds of loss and probs."""
    N, E = X.shape
    K = idx.shape[1]
    scale = float(np.float32(scale))
    seqs = sequences(starts, N)
    S = len(seqs)
    r = dict(loss=np.zeros(S), counts=np.zeros((S, E), np.int32), probs=np.zeros((S, E)),
             rows=np.zeros(S, np.int32), loss_err=np.zeros(S), probs_err=np.zeros((S, E)))
    for i, (a, b) in enumerate(seqs):
        at = idx[a:b]
        inside = (at >= 0) & (at < E)
        took = inside.any(axis=1)
        n = int(took.sum())
        r["rows"][i] = n
        r["counts"][i] = np.bincount(at[inside], minlength=E)
        if n == 0:
            continue
        q, _, err = shares(X[a:b][took], score)
        P = q.sum(axis=0) / n
        r["probs"][i] = P
        # (up to 64 rows are added in binary32, and the sums of a wavefront's teams)
        r["probs_err"][i] = (q * err).sum(axis=0) / n + (64 + 3 + 2) * U * P
        f = scale * E / (K * n)
        r["loss"][i] = f * (r["counts"][i] * P).sum()
        r["loss_err"][i] = (abs(f) * (r["counts"][i] * r["probs_err"][i]).sum() +
                            U * abs(r["loss"][i]))
    return r


def balance_bwd(X, idx, counts, rows, dloss, starts=None, score="softmax", scale=1.0, dtype="f32"):
    """(dx, bound) for given counts and rows."""
    N, E = X.shape
    K = idx.shape[1]
    scale = float(np.float32(scale))
    out, bound = np.zeros((N, E)), np.zeros((N, E))
    for i, (a, b) in enumerate(sequences(starts, N)):
        at = idx[a:b]
        took = np.flatnonzero(((at >= 0) & (at < E)).any(axis=1)) + a
        if not len(took) or rows[i] <= 0:
            continue
        q, slope, err = shares(X[took], score)
        c = counts[i].astype(np.float64)
        n = float(rows[i])
        f = float(dloss[i]) * scale * E / (K * n * n)
        dot = (q * c).sum(axis=1, keepdims=True)
        out[took] = f * q * (c - dot) * slope
        near = np.abs(c - K * n / E)                      # what is multiplied and summed
        ddot = (q * near * (err + 28 * U)).sum(axis=1, keepdims=True)
        # the shares sum to 1 but for their errors; a slope's error, and five products
        ds = power(np.where(np.isfinite(X[took]), X[took], 0.0) * LOG2E) * (score != "softmax")
        # (and this form's own: the shares' sum is 1 to 2^-52 an expert, the counts are not centred)
        bound[took] = abs(f) * q * slope * ((err + ds + 8 * U) * np.abs(c - dot) + ddot +
                                            2 * U * near + 2.0 ** -52 * (E + 2) * c.max())
    bound += HALF[dtype] * np.abs(out) + 2.0 ** (-133 if dtype == "bf16" else -125)
    return out, bound


def check(got, want, err, what):
    """|got - want| <= err, NaN and infinities where the reference has them."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, what
    odd = ~np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what
    assert np.isfinite(got[~odd]).all(), what
    d = np.abs(got[~odd] - want[~odd])
    # (second-order terms, and a subnormal result's own step)
    lim = 1.001 * np.asarray(err)[~odd] + 2.0 ** -149
    assert (d <= lim).all(), f"{what}: {np.max(d / lim):.3g} of the bound"
