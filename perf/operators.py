"""The picks from a softmax that a language model makes: the next token out of
the vocabulary (``softmax_sample``) and a token's experts (``route_fwd`` and its
gradient ``route_bwd``), from a single decode step to a training batch.

A case is a dict of plain values:

* ``op``: ``sample``, ``route`` or ``route_bwd``;
* ``N`` rows of ``V`` logits (vocabulary entries or experts) of ``dtype``;
* sampling: ``ld`` elements from one row to the next, ``sigma`` of the logits'
  body, and ``settings``, how the requests of the batch are set:
  ``chat`` (one temperature, top-k and top-p for all), ``plain`` (a temperature
  a row), ``nucleus`` (and a top-p), ``topk`` (a top-k a row), ``minp`` (a hot
  temperature, top-p and min-p) or ``mixed`` (every row its own kind, greedy
  ones among them);
* routing: ``K`` experts a row, ``score``, ``bias``, ``groups`` of which
  ``top_groups`` are kept by their ``group_top`` best experts, ``renorm`` and
  ``scale``.

Selections and the border of a random number are decided in 64 bits: a
vocabulary has 10^5 borders, and sums in 32 bits would move one of them past
the number in every few rows.  Outputs are new tensors of each call.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

MAX_SAMPLE = 512 * 128256     # what a drawn case may cost at most: the largest listed ones
MAX_ROUTE = 16384 * 256


def _sample(name, N, V, dtype, settings, sigma=2.0, ld=0):
    return dict(name=name, op="sample", N=N, V=V, ld=ld or V, dtype=dtype, settings=settings,
                sigma=sigma)


def _route(name, op, N, V, K, dtype, score, bias=False, groups=1, top_groups=1, group_top=1,
           renorm=True, scale=1.0):
    return dict(name=name, op=op, N=N, V=V, K=K, dtype=dtype, score=score, bias=bias,
                groups=groups, top_groups=top_groups, group_top=group_top, renorm=renorm,
                scale=scale)


def listed():
    return [
        # One sequence being decoded: a single row, where latency counts.
        _sample("sample_1x32000_bf16_chat", 1, 32000, "bf16", "chat"),
        # A batch of 33 sequences over an odd vocabulary whose rows are padded to
        # a multiple of 64 by the projection that wrote them.
        _sample("sample_33x50257_f32_minp", 33, 50257, "f32", "minp", ld=50304),
        # A decode step of a serving batch, every request with settings of its own.
        _sample("sample_64x128256_bf16_mixed", 64, 128256, "bf16", "mixed"),
        # Drawing from the whole distribution, as reinforcement learning's rollouts do.
        _sample("sample_256x128256_f32_plain", 256, 128256, "f32", "plain", sigma=3.0),
        # The largest decode batch, nucleus sampling throughout.
        _sample("sample_512x128256_bf16_nucleus", 512, 128256, "bf16", "nucleus"),
        # Many short rows: a small codebook's tokens, top-k.
        _sample("sample_4000x1000_f32_topk", 4000, 1000, "f32", "topk", sigma=1.0),
        # Routing of one decode step's 16 tokens: latency.
        _route("route_16x64_f32_softmax", "route", 16, 64, 6, "f32", "softmax", renorm=False),
        # A few experts, two of them taken, over a prefill chunk.
        _route("route_4000x8_bf16_softmax", "route", 4000, 8, 2, "bf16", "softmax"),
        # Group-limited routing of a training batch with a bias for balance.
        _route("route_16384x256_f32_sigmoid", "route", 16384, 256, 8, "f32", "sigmoid", bias=True,
               groups=8, top_groups=4, group_top=2, scale=2.5),
        # An odd batch, groups taken by their best expert.
        _route("route_10007x160_bf16_softmax", "route", 10007, 160, 6, "bf16", "softmax", groups=8,
               top_groups=3, renorm=False, scale=16.0),
        # The gradient of the training batch: every expert's logit gets one.
        _route("route_bwd_16384x256_f32_softmax", "route_bwd", 16384, 256, 8, "f32", "softmax",
               renorm=False),
        # The gradient of an odd, small batch of renormalised sigmoid weights.
        _route("route_bwd_1001x60_bf16_sigmoid", "route_bwd", 1001, 60, 4, "bf16", "sigmoid",
               scale=2.5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sample", "sample", "route", "route_bwd"])
    dtype = rng.choice(["f32", "bf16"])
    if op == "sample":
        V = _log_int(rng, 16, 262144)
        # a pass of the smallest draws still takes a few microseconds of work
        N = _log_int(rng, 1, min(4096, MAX_SAMPLE // (V * (2 if dtype == "f32" else 1))))
        ld = V if rng.random() < 0.7 else V + rng.randint(1, 64)
        return dict(op=op, N=N, V=V, ld=ld, dtype=dtype, sigma=rng.choice([1.0, 2.0, 3.0]),
                    settings=rng.choice(["chat", "plain", "nucleus", "topk", "minp", "mixed"]))
    groups = rng.choice([1, 1, 2, 4, 8])
    V = groups * _log_int(rng, 2, 512 // groups)
    top_groups = rng.randint(1, groups)
    K = rng.randint(1, min(16, top_groups * (V // groups)))
    return dict(op=op, N=_log_int(rng, 1, min(32768, MAX_ROUTE // V)), V=V, K=K, dtype=dtype,
                score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5,
                groups=groups, top_groups=top_groups, group_top=rng.choice([1, 2]),
                renorm=rng.random() < 0.5, scale=rng.choice([1.0, 2.5]))


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _uniform(g, N, lo, hi):
    return lo + (hi - lo) * torch.rand(N, device="cuda", generator=g)


def _sample_inputs(case, seed):
    """Logits with a body of about N(0, sigma^2) and a stretched upper end, as a
    language model's: a few tokens far ahead, a long tail.  One uniform number a
    row, and the settings of the requests."""
    N, V, sigma = case["N"], case["V"], case["sigma"]
    g = _gen(seed)
    buf = torch.empty((N, case["ld"]), dtype=_dtype(case), device="cuda")
    step = max(1, (1 << 26) // case["ld"])
    for a in range(0, N, step):
        r = torch.randn(min(step, N - a), case["ld"], device="cuda", generator=g)
        up = (r - 2.0).clamp_(min=0.0)
        buf[a:a + step] = (r + 0.5 * up * up) * sigma
    s = dict(x=buf[:, :V], u=torch.rand(N, device="cuda", generator=g), temperature=1.0,
             top_k=0, top_p=1.0, min_p=0.0)
    kind = case["settings"]
    if kind == "chat":
        s.update(temperature=0.8, top_k=50, top_p=0.9)
    elif kind == "plain":
        s.update(temperature=_uniform(g, N, 0.6, 1.2))
    elif kind == "nucleus":
        s.update(temperature=_uniform(g, N, 0.6, 1.2), top_p=_uniform(g, N, 0.8, 0.98))
    elif kind == "topk":
        s.update(top_k=torch.randint(1, 201, (N,), device="cuda", generator=g,
                                     dtype=torch.int32))
    elif kind == "minp":
        s.update(temperature=_uniform(g, N, 0.8, 1.5), top_p=0.95,
                 min_p=_uniform(g, N, 0.02, 0.1))
    else:  # 0 greedy, 1 plain, 2 top-k, 3 top-p, 4 min-p, 5 all of them
        c = torch.randint(0, 6, (N,), device="cuda", generator=g)
        t = _uniform(g, N, 0.6, 1.2)
        k = torch.randint(1, 201, (N,), device="cuda", generator=g)
        p = _uniform(g, N, 0.8, 0.98)
        q = _uniform(g, N, 0.02, 0.1)
        s.update(temperature=torch.where(c == 0, torch.zeros_like(t), t),
                 top_k=torch.where((c == 2) | (c == 5), k, torch.zeros_like(k)).int(),
                 top_p=torch.where((c == 3) | (c == 5), p, torch.ones_like(p)),
                 min_p=torch.where((c == 4) | (c == 5), q, torch.zeros_like(q)))
    return s


def _route_inputs(case, seed):
    """Router logits of about N(0, 1) with a common part a row; a bias of the
    size that balancing reaches.  For the gradient, each row's experts (distinct,
    as the router returns them) and the gradient of their weights."""
    N, V, K = case["N"], case["V"], case["K"]
    g = _gen(seed)
    x = torch.randn(N, V, device="cuda", generator=g)
    x += 0.5 * torch.randn(N, 1, device="cuda", generator=g)
    s = dict(x=x.to(_dtype(case)))
    if case["op"] == "route":
        s["bias"] = 0.05 * torch.randn(V, device="cuda", generator=g) if case["bias"] else None
    else:
        s["idx"] = torch.topk(x, K, dim=1).indices.int().contiguous()
        s["dvals"] = torch.randn(N, K, device="cuda", generator=g)
    return s


def prepare(case, seed):
    s = _sample_inputs(case, seed) if case["op"] == "sample" else _route_inputs(case, seed)
    s["case"] = case
    return s


# -------------------------------------------------------------- plain forms
def _column(v, x, dtype):
    """A setting as an N x 1 column."""
    t = torch.as_tensor(v, device=x.device).to(dtype)
    return t.reshape(-1, 1).expand(x.shape[0], 1)


def _sample_plain(x, u, temperature, top_k, top_p, min_p):
    V = x.shape[1]
    T = _column(temperature, x, torch.float64)
    k = _column(top_k, x, torch.int64)
    p = _column(np.float32(top_p) if isinstance(top_p, float) else top_p, x, torch.float64)
    q = _column(np.float32(min_p) if isinstance(min_p, float) else min_p, x, torch.float64)
    if isinstance(temperature, float):
        T = _column(np.float32(temperature), x, torch.float64)
    x64 = x.double()
    m = x64.amax(dim=1, keepdim=True)
    greedy = ~(T > 0)
    w = torch.exp((x64 - m) / torch.where(greedy, torch.ones_like(T), T))
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    ws = torch.gather(w, 1, order)
    rank = torch.arange(V, device=x.device).unsqueeze(0)
    keep = (rank < k) | (k <= 0)
    keep = torch.where(greedy, rank < 1, keep)
    wk = torch.where(keep, ws, torch.zeros_like(ws))
    c = torch.cumsum(wk, dim=1)
    before = torch.cat([torch.zeros_like(m), c[:, :-1]], dim=1)
    keep &= (p >= 1) | (rank == 0) | (before < p * c[:, -1:])
    keep &= ws >= q.clamp(max=1.0)
    ws = torch.where(keep, ws, torch.zeros_like(ws))
    w = torch.zeros_like(w).scatter_(1, order, ws)
    c = torch.cumsum(w, dim=1)
    total = c[:, -1:]
    idx = (c <= u.double().unsqueeze(1) * total).sum(dim=1, keepdim=True)
    last = (torch.where(w > 0, rank, torch.zeros_like(rank))).amax(dim=1, keepdim=True)
    idx = torch.minimum(idx, last)
    vals = torch.gather(w, 1, idx) / total
    return vals.squeeze(1).float(), idx.squeeze(1).int()


def _route_plain(x, bias, case):
    """The experts by scores in 64 bits (a bias brings near-ties), the weights from the
    same scores."""
    K, V, G = case["K"], case["V"], case["groups"]
    N = x.shape[0]
    x64 = x.double()
    s = torch.softmax(x64, dim=1) if case["score"] == "softmax" else torch.sigmoid(x64)
    c = x64 if bias is None else s + bias.double()
    if G > 1:
        sel = s if bias is None else c
        two = torch.sort(sel.reshape(N, G, V // G), dim=2, descending=True).values
        score = two[:, :, :case["group_top"]].sum(dim=2)
        best = torch.sort(score, dim=1, descending=True, stable=True).indices
        kept = torch.zeros_like(score, dtype=torch.bool)
        kept.scatter_(1, best[:, :case["top_groups"]], True)
        kept = kept.repeat_interleave(V // G, dim=1)
        c = torch.where(kept, c, torch.full_like(c, -math.inf))
    idx = torch.sort(c, dim=1, descending=True, stable=True).indices[:, :K]
    w = torch.gather(s, 1, idx)
    if case["renorm"]:
        w = w / w.sum(dim=1, keepdim=True)
    return (w * case["scale"]).float(), idx.int()


def _route_bwd_plain(x, idx, dvals, case):
    xf, j = x.float(), idx.long()
    g = dvals * case["scale"]
    if case["renorm"]:
        xs = torch.gather(xf, 1, j)
        if case["score"] == "softmax":
            z, slope = xs, 1.0
        else:  # log of the sigmoid, and its slope 1 - s
            z = torch.minimum(xs, torch.zeros_like(xs)) - torch.log1p(torch.exp(-xs.abs()))
            slope = 1.0 / (1.0 + torch.exp(xs))
        p = torch.exp(z - z.amax(dim=1, keepdim=True))
        p = p / p.sum(dim=1, keepdim=True)
        d = p * (g - (g * p).sum(dim=1, keepdim=True)) * slope
        return torch.zeros_like(xf).scatter_(1, j, d).to(x.dtype)
    dense = torch.zeros_like(xf).scatter_(1, j, g)
    if case["score"] == "softmax":
        s = torch.exp(xf - xf.amax(dim=1, keepdim=True))
        s = s / s.sum(dim=1, keepdim=True)
        d = s * (dense - (dense * s).sum(dim=1, keepdim=True))
    else:
        d = dense / (1.0 + torch.exp(-xf)) / (1.0 + torch.exp(xf))
    return d.to(x.dtype)


# --------------------------------------------------------------------- runs
def run(state):
    case = state["case"]
    if own:
        import paper_1805_02867_amd as osm
        if case["op"] == "sample":
            return osm.softmax_sample(state["x"], state["u"], temperature=state["temperature"],
                                      top_k=state["top_k"], top_p=state["top_p"],
                                      min_p=state["min_p"])
        if case["op"] == "route":
            return osm.route_fwd(state["x"], case["K"], bias=state["bias"], score=case["score"],
                                 groups=case["groups"], top_groups=case["top_groups"],
                                 group_top=case["group_top"], renorm=case["renorm"],
                                 scale=case["scale"])
        return osm.route_bwd(state["x"], state["idx"], state["dvals"], score=case["score"],
                             renorm=case["renorm"], scale=case["scale"])
    if case["op"] == "sample":
        return _sample_plain(state["x"], state["u"], state["temperature"], state["top_k"],
                             state["top_p"], state["min_p"])
    if case["op"] == "route":
        return _route_plain(state["x"], state["bias"], case)
    return _route_bwd_plain(state["x"], state["idx"], state["dvals"], case)


def work(case):
    """Each input read once and each output written once; an exponential and an
    add an element."""
    N, V = case["N"], case["V"]
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "sample":
        params = {"chat": 0, "plain": 4, "nucleus": 8, "topk": 4, "minp": 8, "mixed": 16}
        return {"bytes": N * (V * es + 4 + params[case["settings"]] + 8), "flops": 2 * N * V}
    K = case["K"]
    if case["op"] == "route":
        return {"bytes": N * V * es + 4 * V * case["bias"] + 8 * N * K, "flops": 2 * N * V}
    # the gradient of renormalised or sigmoid weights needs the chosen logits only
    read = V if case["score"] == "softmax" and not case["renorm"] else K
    return {"bytes": N * (read + V) * es + 8 * N * K, "flops": 2 * N * read}


# -------------------------------------------------------------------- exact
def _settings64(s, N):
    out = []
    for name in ("temperature", "top_k", "top_p", "min_p"):
        v = s[name]
        v = v.cpu().numpy() if torch.is_tensor(v) else np.full(N, v, np.float32)
        out.append(v.astype(np.float64))
    return out


def _sample_exact(case, seed):
    """Row by row from the definition, a row sorted only where a filter asks for it."""
    N, V = case["N"], case["V"]
    if N * V > 1 << 26:  # about 10 seconds
        return None
    s = _sample_inputs(case, seed)
    T, k, p, q = _settings64(s, N)
    u = s["u"].double().cpu().numpy()
    X = s["x"].float().cpu().numpy()
    vals, idx = np.empty(N), np.empty(N, np.int32)
    for r in range(N):
        x = X[r].astype(np.float64)
        m = x.max()
        if T[r] <= 0:
            vals[r], idx[r] = 1.0, int(np.argmax(x))
            continue
        w = np.exp((x - m) / T[r])
        kept = w >= min(q[r], 1.0)
        if 0 < k[r] < V or p[r] < 1:
            order = np.argsort(-x, kind="stable")
            if 0 < k[r] < V:
                order = order[:int(k[r])]
            if p[r] < 1:
                c = np.cumsum(w[order].astype(np.longdouble))
                order = order[:int(np.searchsorted(c, p[r] * c[-1])) + 1]
            chosen = np.zeros(V, bool)
            chosen[order] = True
            kept &= chosen
        places = np.flatnonzero(kept)
        c = np.cumsum(w[places].astype(np.longdouble))
        j = min(int(np.searchsorted(c, u[r] * c[-1], side="right")), len(places) - 1)
        idx[r] = places[j]
        vals[r] = float(w[places[j]] / c[-1])
    return vals, idx


def _logistic(x):
    """1 / (1 + e^-x) without overflow."""
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1.0 + e)


def _scores64(x, case):
    if case["score"] == "sigmoid":
        return _logistic(x)
    e = np.exp(x - x.max(axis=1, keepdims=True))
    return e / e.sum(axis=1, keepdims=True)


def _route_exact(case, seed):
    st = _route_inputs(case, seed)
    x = st["x"].double().cpu().numpy()
    N, V, K, G = case["N"], case["V"], case["K"], case["groups"]
    s = _scores64(x, case)
    c = x if st["bias"] is None else s + st["bias"].double().cpu().numpy()
    if G > 1:
        sel = (s if st["bias"] is None else c).reshape(N, G, V // G)
        t = min(case["group_top"], V // G)
        score = np.partition(sel, V // G - t, axis=2)[:, :, V // G - t:].sum(axis=2)
        # a group stays if fewer than top_groups come before it
        ahead = (score[:, None, :] > score[:, :, None]).sum(axis=2)
        for i in range(G):
            ahead[:, i] += (score[:, :i] == score[:, i:i + 1]).sum(axis=1)
        c = np.where(np.repeat(ahead < case["top_groups"], V // G, axis=1), c, -np.inf)
    idx = np.empty((N, K), np.int32)
    rest, rows = c.copy(), np.arange(N)
    for j in range(K):
        idx[:, j] = rest.argmax(axis=1)
        rest[rows, idx[:, j]] = -np.inf
    w = np.take_along_axis(s, idx.astype(np.int64), axis=1)
    if case["renorm"]:
        w = w / w.sum(axis=1, keepdims=True)
    return w * case["scale"], idx


def _route_bwd_exact(case, seed):
    """dx_e = sum_j dvals_j dw_j/dx_e, with the derivatives of the weights written out
    from those of the scores: ds_i/dx_e = s_i (1[i = e] - s_e) for the softmax,
    s_e (1 - s_e) 1[i = e] for the sigmoid."""
    st = _route_inputs(case, seed)
    x = st["x"].double().cpu().numpy()
    j = st["idx"].long().cpu().numpy()
    g = st["dvals"].double().cpu().numpy() * case["scale"]
    s = _scores64(x, case)
    sj = np.take_along_axis(s, j, axis=1)
    if case["renorm"]:  # w = sj / t: the gradient of sj
        t = sj.sum(axis=1, keepdims=True)
        g = g / t - (g * sj).sum(axis=1, keepdims=True) / t ** 2
    ds = np.zeros_like(x)
    np.put_along_axis(ds, j, g, axis=1)
    if case["score"] == "sigmoid":
        return ds * s * _logistic(-x)
    return s * (ds - (ds * s).sum(axis=1, keepdims=True))


def exact(case, seed):
    if case["op"] == "sample":
        return _sample_exact(case, seed)
    if case["op"] == "route":
        return _route_exact(case, seed)
    return _route_bwd_exact(case, seed)
