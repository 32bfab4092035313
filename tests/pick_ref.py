"""Plain binary64 implementations of sampling and routing (test infrastructure):
row by row from the formulas, sums in the host's widest floating type."""
from __future__ import annotations

import numpy as np

# Kernel results are binary64 rounded once: half a step of the output type, and
# 2^-40 for the binary64 sums (10^6 terms off by 2^-52 at most each, and less).
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
WIDE = 2.0 ** -40


def close(got, want, dtype="f32", slack=0.0):
    """|got - want| within the rounding of `dtype` (bfloat16 goes through binary32), or
    within half a step of its smallest subnormal; NaN where the reference has it.
    slack: absolute, for what cancels in `want`."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    rel = HALF[dtype] + (HALF["f32"] if dtype == "bf16" else 0.0) + WIDE
    tiny = 2.0 ** (-150 if dtype == "f32" else -134) * 1.01
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    err = np.abs(got - want)[~nan]
    lim = (rel * np.abs(want) + tiny + slack)[~nan]
    assert np.all(err <= lim), f"worst {np.max(err / lim):.3g} of the bound"


def _param(v, N):
    a = np.asarray(v, np.float32).astype(np.float64)
    return np.full(N, a) if a.ndim == 0 else a


def sample(X, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(vals, idx) of rows X (float64 values)."""
    N, V = X.shape
    T, p, q, u = (_param(v, N) for v in (temperature, top_p, min_p, u))
    k = np.full(N, top_k) if np.ndim(top_k) == 0 else np.asarray(top_k)
    vals, idx = np.full(N, np.nan), np.full(N, -1, np.int32)
    for r in range(N):
        x = X[r]
        m = x.max()
        if np.isnan(x).any() or not np.isfinite(m):
            continue
        if not T[r] > 0:
            vals[r], idx[r] = 1.0, np.argmax(x)
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            w = np.where(x == -np.inf, 0.0, np.exp((x - m) / T[r]))
        order = np.lexsort((np.arange(V), -x))
        if 0 < k[r] < V:
            order = order[:k[r]]
        if p[r] < 1:
            c = np.cumsum(w[order].astype(np.longdouble))
            order = order[:max(1, np.searchsorted(c, max(p[r], 0.0) * c[-1]) + 1)]
        if q[r] > 0:
            order = order[w[order] >= min(q[r], 1.0)]
        places = np.sort(order[w[order] > 0])
        c = np.cumsum(w[places].astype(np.longdouble))
        uu = min(max(u[r], 0.0), 1.0) if u[r] == u[r] else 0.0
        j = min(np.searchsorted(c, uu * c[-1], side="right"), len(places) - 1)
        idx[r], vals[r] = places[j], w[places[j]] / c[-1]
    return vals, idx


def _scores(x, score):
    if score == "sigmoid":
        e = np.exp(-np.abs(x))
        return np.where(x >= 0, 1.0, e) / (1.0 + e)
    e = np.exp(x - x.max())
    return e / e.sum()


def _shares(x, score):
    """Scores over their sum, without underflow."""
    if score == "sigmoid":
        z = np.minimum(x, 0.0)
        e = np.exp(z - z.max()) / (1.0 + np.exp(-np.abs(x)))
    else:
        e = np.exp(x - x.max())
    return e / e.sum()


def route(X, K, bias=None, score="softmax", groups=1, top_groups=1, group_top=1, renorm=True,
          scale=1.0):
    N, E = X.shape
    gs = E // groups
    vals, idx = np.zeros((N, K)), np.full((N, K), -1, np.int32)
    for r in range(N):
        x = X[r]
        if np.isnan(x).any() or (x == np.inf).any():
            vals[r] = np.nan
            continue
        if (x == -np.inf).all():
            continue
        s = _scores(x, score)
        may = x > -np.inf
        c = x
        if bias is not None:
            b = np.asarray(bias, np.float64)
            may = may & (b > -np.inf)
            c = s + b
        if groups > 1:
            gc = s if bias is None and group_top == 2 else c
            key = np.full(groups, -np.inf)
            for g in range(groups):
                inside = gc[g * gs:(g + 1) * gs][may[g * gs:(g + 1) * gs]]
                if len(inside):
                    key[g] = sum(sorted(inside, reverse=True)[:group_top])
            best = sorted(range(groups), key=lambda g: (-key[g], g))[:top_groups]
            may = may & np.isin(np.arange(E) // gs, best)
        pick = sorted(np.flatnonzero(may), key=lambda e: (-c[e], e))[:K]
        if not pick:
            continue
        idx[r, :len(pick)] = pick
        w = _shares(x[pick], score) if renorm else s[pick]
        vals[r, :len(pick)] = w * float(np.float32(scale))
    return vals, idx


def route_bwd(X, idx, dvals, score="softmax", renorm=True, scale=1.0):
    """From the derivatives of the weights, place by place."""
    N, E = X.shape
    scale = float(np.float32(scale))
    out = np.zeros((N, E))
    for r in range(N):
        at = [i for i in range(idx.shape[1]) if 0 <= idx[r, i] < E]
        if not at:
            continue
        j, g = idx[r, at], dvals[r, at].astype(np.float64) * scale
        s = _scores(X[r], score)
        if renorm:
            w = _shares(X[r, j], score)
            own = w * (g - (g * w).sum())
            if score == "sigmoid":
                own = own * _scores(-X[r, j], "sigmoid")
            np.add.at(out[r], j, own)
        elif score == "softmax":
            np.add.at(out[r], j, g * s[j])
            out[r] -= s * (g * s[j]).sum()
        else:
            np.add.at(out[r], j, g * s[j] * _scores(-X[r, j], "sigmoid"))
    return out
