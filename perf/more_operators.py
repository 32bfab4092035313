"""What a language model's losses and scores read off its logits: the log
probabilities of given tokens with the entropy and the best alternatives
(``logprob_fwd``) and their gradient (``logprob_bwd``), and the loss that keeps a
router's experts in use (``balance_fwd``) and its gradient (``balance_bwd``).

A case is a dict of plain values:

* ``op``: ``logprob``, ``logprob_bwd``, ``balance`` or ``balance_bwd``;
* ``N`` rows of ``V`` logits (vocabulary entries or experts) of ``dtype``;
* log probabilities: ``ld`` elements from one row to the next, ``T`` given tokens
  and ``K`` alternatives a row, whether the ``entropy`` takes part, the
  ``temperature``, the part of the vocabulary that is ``masked`` (-inf) and the
  part of the rows that are ``ignored`` (their token is -100);
* balance: ``K`` experts a row, the ``score``, and ``segments``: how many
  sequences of different lengths the rows are packed from (0: one, without
  offsets).

Outputs are new tensors of each call.
"""
from __future__ import annotations

import math

import torch

own = False

MAX_LOGITS = 2048 * 128256 * 2    # bytes of a drawn case's logits: the largest listed ones
MAX_RANKED = 64 * 1024 * 1024     # elements of a drawn case with alternatives
MAX_ROUTER = 65536 * 256 * 4


def _logprob(name, op, N, V, dtype, T=1, K=0, entropy=False, temperature=1.0, masked=0.0,
             ignored=0.0, ld=0):
    return dict(name=name, op=op, N=N, V=V, ld=ld or V, dtype=dtype, T=T, K=K, entropy=entropy,
                temperature=temperature, masked=masked, ignored=ignored)


def _balance(name, op, N, V, K, dtype, score, segments=0, scale=1.0):
    return dict(name=name, op=op, N=N, V=V, K=K, dtype=dtype, score=score, segments=segments,
                scale=scale)


def listed():
    return [
        # One sequence being decoded, the sampled token reported with five
        # alternatives: a single row, where latency counts.
        _logprob("logprob_1x128256_bf16_top5", "logprob", 1, 128256, "bf16", K=5),
        # A serving batch under a grammar, nine tenths of an odd vocabulary masked, over
        # rows that the projection padded.
        _logprob("logprob_64x50257_f32_masked_top20", "logprob", 64, 50257, "f32", K=20,
                 entropy=True, masked=0.9, ld=50304),
        # Distillation: sixteen of a teacher's tokens a row.
        _logprob("logprob_300x32000_f32_16tokens", "logprob", 300, 32000, "f32", T=16),
        # A reinforcement learning step's forward pass over a training batch.
        _logprob("logprob_2048x128256_bf16_entropy", "logprob", 2048, 128256, "bf16",
                 entropy=True, ignored=0.1),
        # Many short rows: a small codebook's tokens.
        _logprob("logprob_16385x1000_f32", "logprob", 16385, 1000, "f32"),
        # The gradient of the training batch's cross entropy.
        _logprob("logprob_bwd_2048x128256_bf16", "logprob_bwd", 2048, 128256, "bf16",
                 ignored=0.1),
        # A policy gradient with an entropy bonus at the rollouts' temperature, odd rows.
        _logprob("logprob_bwd_1003x50257_f32_entropy", "logprob_bwd", 1003, 50257, "f32",
                 entropy=True, temperature=0.7),
        # The distillation's gradient.
        _logprob("logprob_bwd_300x32000_bf16_16tokens", "logprob_bwd", 300, 32000, "bf16", T=16),
        # The router of a small model on a few tokens: latency.
        _balance("balance_16x64_f32_softmax", "balance", 16, 64, 6, "f32", "softmax"),
        # A training batch packed from sequences of different lengths, a loss each.
        _balance("balance_65536x256_bf16_sigmoid_packed", "balance", 65536, 256, 8, "bf16",
                 "sigmoid", segments=24, scale=0.01),
        # Its gradient, from binary32 logits of a softmax router.
        _balance("balance_bwd_65536x256_f32_softmax_packed", "balance_bwd", 65536, 256, 8, "f32",
                 "softmax", segments=24, scale=0.01),
        # The gradient of an odd, small batch.
        _balance("balance_bwd_1001x60_bf16_sigmoid", "balance_bwd", 1001, 60, 4, "bf16",
                 "sigmoid", segments=3),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logprob", "logprob", "logprob_bwd", "balance", "balance_bwd"])
    dtype = rng.choice(["f32", "bf16"])
    es = 2 if dtype == "bf16" else 4
    if op.startswith("logprob"):
        V = _log_int(rng, 16, 262144)
        K = 0 if op == "logprob_bwd" else min(V, rng.choice([0, 0, 1, 5, 20, 50, 64]))
        most = min(MAX_RANKED // V if K else MAX_LOGITS // (V * es), 32768)
        return dict(op=op, N=_log_int(rng, 1, most), V=V, dtype=dtype, K=K,
                    ld=V if rng.random() < 0.7 else V + rng.randint(1, 64),
                    T=1 if rng.random() < 0.7 else rng.randint(2, 32),
                    entropy=rng.random() < 0.5, temperature=rng.choice([1.0, 1.0, 0.7, 1.3]),
                    masked=rng.choice([0.0, 0.0, 0.5, 0.9]), ignored=rng.choice([0.0, 0.1, 0.5]))
    V = _log_int(rng, 4, 512)
    N = _log_int(rng, 1, min(65536, MAX_ROUTER // (V * es)))
    return dict(op=op, N=N, V=V, K=rng.randint(1, min(8, V)), dtype=dtype,
                score=rng.choice(["softmax", "sigmoid"]),
                segments=0 if rng.random() < 0.4 else _log_int(rng, 1, min(N, 64)),
                scale=rng.choice([1.0, 0.01]))


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _steps(N, V):
    step = max(1, (1 << 26) // V)
    return [(a, min(N, a + step)) for a in range(0, N, step)]


def _logprob_inputs(case, seed):
    """Logits with a body of about N(0, 4) and a stretched upper end, as a language
    model's.  The first token of a row is drawn from its softmax, and in every second
    row raised by up to 15, as a trained model's tokens are sure of themselves; the
    others are any tokens.  For the gradient, what the forward pass gave and the gradient
    of its outputs: weights of a mean over the batch, of either sign with an entropy
    (advantages), and a small bonus."""
    N, V, T, tau = case["N"], case["V"], case["T"], case["temperature"]
    g = _gen(seed)
    buf = torch.zeros((N, case["ld"]), dtype=_dtype(case), device="cuda")
    tokens = torch.randint(0, V, (N, T), device="cuda", generator=g)
    stats = torch.empty((N, 2), device="cuda")
    entropy = torch.empty(N, device="cuda")
    for a, b in _steps(N, V):
        r = torch.randn(b - a, V, device="cuda", generator=g)
        up = (r - 2.0).clamp_(min=0.0)
        r = (r + 0.5 * up * up) * 2.0
        if case["masked"]:
            r[torch.rand(b - a, V, device="cuda", generator=g) < case["masked"]] = -math.inf
            r[:, 0] = 0.0    # (a token is left)
        noise = -torch.log(torch.empty_like(r).exponential_(generator=g))
        first = (r + noise).argmax(dim=1, keepdim=True)
        tokens[a:b, :1] = first
        sure = 15.0 * torch.rand(b - a, 1, device="cuda", generator=g)
        sure[::2] = 0.0
        r.scatter_add_(1, first, sure)
        buf[a:b, :V] = r
        if case["op"] == "logprob_bwd":
            x = buf[a:b, :V].double() / tau
            m = x.amax(dim=1, keepdim=True)
            w = torch.exp(x - m)
            d = w.sum(dim=1)
            stats[a:b, 0] = buf[a:b, :V].amax(dim=1).float()
            stats[a:b, 1] = (d - 1.0).float()
            fall = torch.where(w > 0, w * (m - x), torch.zeros_like(w)).sum(dim=1)
            entropy[a:b] = (torch.log(d) + fall / d).float()
    if case["ignored"]:
        tokens[torch.rand(N, device="cuda", generator=g) < case["ignored"]] = -100
    s = dict(x=buf[:, :V], tokens=tokens.int().contiguous())
    if case["op"] == "logprob_bwd":
        w = torch.randn(N, T, device="cuda", generator=g) if case["entropy"] else (
            -torch.rand(N, T, device="cuda", generator=g))
        s.update(stats=stats, dlogp=w / N, entropy=None, dentropy=None)
        if case["entropy"]:
            bonus = 0.01 + 0.01 * torch.rand(N, device="cuda", generator=g)
            s.update(entropy=entropy, dentropy=-bonus / N)
    return s


def _balance_inputs(case, seed):
    """Router logits of about N(0, 1) with a common part an expert, the experts as a router
    with a bias takes them; a twentieth of the rows is padding (no expert), and the rows
    behind the last sequence belong to none."""
    N, V, K, S = case["N"], case["V"], case["K"], case["segments"]
    g = _gen(seed)
    x = torch.randn(N, V, device="cuda", generator=g)
    x += 0.3 * torch.randn(V, device="cuda", generator=g)
    x = x.to(_dtype(case))
    biased = x.float() + 0.2 * torch.randn(V, device="cuda", generator=g)
    idx = torch.topk(biased, K, dim=1).indices.int()
    idx[torch.rand(N, device="cuda", generator=g) < 0.05] = -1
    starts = None
    if S:
        # lengths in proportion to the exponentials of normal numbers; a few rows are left over
        w = torch.exp(torch.randn(S + 1, device="cuda", generator=g).double())
        w[S] *= 0.1
        c = torch.cumsum(w, 0) / w.sum()
        starts = torch.zeros(S + 1, dtype=torch.int32, device="cuda")
        starts[1:] = (c[:S] * N).int()
    s = dict(x=x, idx=idx.contiguous(), starts=starts)
    if case["op"] == "balance_bwd":
        counts, rows, _, _ = _taken(s["idx"], starts, N, V)
        s.update(counts=counts, rows=rows,
                 dloss=0.5 + torch.rand(max(S, 1), device="cuda", generator=g))
    return s


def prepare(case, seed):
    make = _logprob_inputs if case["op"].startswith("logprob") else _balance_inputs
    s = make(case, seed)
    s["case"] = case
    return s


# -------------------------------------------------------------- plain forms
def _logprob_plain(x, tokens, K, entropy, tau):
    N, V = x.shape
    xf = x.float()
    m = xf.amax(dim=1, keepdim=True)
    t = xf - m if tau == 1.0 else (xf - m) / tau
    e = torch.exp(t)
    d = torch.sum(e, dim=1, keepdim=True, dtype=torch.float64)  # (log p next to 0)
    ln_d = torch.log(d)
    inside = (tokens >= 0) & (tokens < V)
    at = torch.gather(t, 1, torch.where(inside, tokens, torch.zeros_like(tokens)).long())
    logp = (at.double() - ln_d).float()
    out = dict(logp=torch.where(inside, logp, torch.zeros_like(logp)),
               stats=torch.cat([m, (d - 1.0).float()], dim=1))
    if entropy:
        fall = torch.where(e > 0, e * t, torch.zeros_like(e))
        fall = torch.sum(fall, dim=1, keepdim=True, dtype=torch.float64)
        out["entropy"] = (ln_d - fall / d).squeeze(1).float()
    if K:
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :K]
        out["top_vals"] = (torch.gather(t, 1, order).double() - ln_d).float()
        out["top_idx"] = order.int()
    return out


def _logprob_bwd_plain(x, tokens, stats, entropy, dlogp, dentropy, tau):
    N, V = x.shape
    xf = x.float()
    m, s = stats[:, :1], stats[:, 1:]
    t = xf - m if tau == 1.0 else (xf - m) / tau
    p = torch.exp(t) / (1.0 + s)
    inside = (tokens >= 0) & (tokens < V)
    g = torch.where(inside, dlogp, torch.zeros_like(dlogp))
    at = torch.where(inside, tokens, torch.zeros_like(tokens)).long()
    d = torch.zeros_like(xf).scatter_add_(1, at, g) - p * g.sum(dim=1, keepdim=True)
    if dentropy is not None:
        ln_p = t - torch.log1p(s)
        fall = torch.where(p > 0, p * (ln_p + entropy.unsqueeze(1)), torch.zeros_like(p))
        d = d - dentropy.unsqueeze(1) * fall
    return (d / tau).to(x.dtype)


def _taken(idx, starts, N, V):
    """Counts of the experts and rows of each sequence; each row's sequence and whether it
    takes part."""
    rows = torch.arange(N, device=idx.device)
    if starts is None:
        S, seg, within = 1, torch.zeros_like(rows), torch.ones_like(rows, dtype=torch.bool)
    else:
        S = starts.shape[0] - 1
        seg = torch.searchsorted(starts.long(), rows, right=True) - 1
        within = (seg >= 0) & (seg < S)
        seg = seg.clamp(0, S - 1)
    inside = (idx >= 0) & (idx < V) & within.unsqueeze(1)
    part = inside.any(dim=1)
    slot = torch.where(inside, seg.unsqueeze(1) * V + idx, torch.zeros_like(idx)).long()
    counts = torch.zeros(S * V, dtype=torch.int32, device=idx.device)
    counts.scatter_add_(0, slot.view(-1), inside.int().view(-1))
    n = torch.zeros(S, dtype=torch.int32, device=idx.device)
    n.scatter_add_(0, seg, part.int())
    return counts.view(S, V), n, seg, part


def _shares(xf, score):
    if score == "softmax":
        e = torch.exp(xf - xf.amax(dim=1, keepdim=True))
    else:
        e = 1.0 / (1.0 + torch.exp(-xf))
    return e / e.sum(dim=1, keepdim=True)


def _balance_plain(x, idx, starts, score, scale):
    N, V = x.shape
    K = idx.shape[1]
    counts, n, seg, part = _taken(idx, starts, N, V)
    q = _shares(x.float(), score)
    q = torch.where(part.unsqueeze(1), q, torch.zeros_like(q))
    member = torch.arange(counts.shape[0], device=x.device).unsqueeze(1) == seg
    total = member.double() @ q.double()
    rows = n.clamp(min=1).double().unsqueeze(1)
    probs = total / rows
    loss = scale * V / (K * rows.squeeze(1)) * (counts * probs).sum(dim=1)
    return dict(loss=loss.float(), counts=counts, probs=probs.float(), rows=n)


def _balance_bwd_plain(x, idx, starts, counts, rows, dloss, score, scale):
    N, V = x.shape
    K = idx.shape[1]
    _, _, seg, part = _taken(idx, starts, N, V)
    xf = x.float()
    q = _shares(xf, score)
    c64 = counts.double()
    c = (c64 - c64.mean(dim=1, keepdim=True)).float()[seg]  # (shares sum to 1; counts cancel)
    d = q * (c - (c * q).sum(dim=1, keepdim=True))
    if score == "sigmoid":
        d = d / (1.0 + torch.exp(xf))
    r = rows.clamp(min=1).double()
    a = (dloss.double() * scale * V / (K * r * r)).float()[seg].unsqueeze(1)
    return torch.where(part.unsqueeze(1), a * d, torch.zeros_like(d)).to(x.dtype)


# --------------------------------------------------------------------- runs
def run(state):
    case, s = state["case"], state
    op = case["op"]
    if own:
        import paper_1805_02867_amd as osm
        if op == "logprob":
            r = osm.logprob_fwd(s["x"], s["tokens"], K=case["K"], entropy=case["entropy"],
                                stats=True, temperature=case["temperature"])
            out = dict(logp=r.logp, stats=r.stats)
            if case["entropy"]:
                out["entropy"] = r.entropy
            if case["K"]:
                out.update(top_vals=r.top_vals, top_idx=r.top_idx)
            return out
        if op == "logprob_bwd":
            return osm.logprob_bwd(s["x"], s["stats"], tokens=s["tokens"], dlogp=s["dlogp"],
                                   entropy=s["entropy"], dentropy=s["dentropy"],
                                   temperature=case["temperature"])
        if op == "balance":
            r = osm.balance_fwd(s["x"], s["idx"], starts=s["starts"], score=case["score"],
                                scale=case["scale"])
            return dict(loss=r.loss, counts=r.counts, probs=r.probs, rows=r.rows)
        return osm.balance_bwd(s["x"], s["idx"], s["counts"], s["rows"], s["dloss"],
                               starts=s["starts"], score=case["score"], scale=case["scale"])
    if op == "logprob":
        return _logprob_plain(s["x"], s["tokens"], case["K"], case["entropy"],
                              case["temperature"])
    if op == "logprob_bwd":
        return _logprob_bwd_plain(s["x"], s["tokens"], s["stats"], s["entropy"], s["dlogp"],
                                  s["dentropy"], case["temperature"])
    if op == "balance":
        return _balance_plain(s["x"], s["idx"], s["starts"], case["score"], case["scale"])
    return _balance_bwd_plain(s["x"], s["idx"], s["starts"], s["counts"], s["rows"], s["dloss"],
                              case["score"], case["scale"])


def work(case):
    """Each input read once and each output written once; a subtraction, an exponential and
    an addition an element, two more operations with the entropy, three for a gradient."""
    N, V = case["N"], case["V"]
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "logprob":
        small = 4 * case["T"] + 4 * case["T"] + 8 + 4 * case["entropy"] + 8 * case["K"]
        return {"bytes": N * (V * es + small), "flops": (3 + 2 * case["entropy"]) * N * V}
    if case["op"] == "logprob_bwd":
        small = 8 * case["T"] + 8 + 8 * case["entropy"]
        return {"bytes": N * (2 * V * es + small), "flops": (3 + 3 * case["entropy"]) * N * V}
    S, K = max(case["segments"], 1), case["K"]
    if case["op"] == "balance":
        return {"bytes": N * (V * es + 4 * K) + S * (8 * V + 12), "flops": 4 * N * V}
    return {"bytes": N * (2 * V * es + 4 * K) + S * (4 * V + 12), "flops": 7 * N * V}


# -------------------------------------------------------------------- exact
def _logprob_exact(case, seed):
    """Row block by row block from p = e^z / sum e^z, the alternatives by a key of value and
    index in which no two are equal."""
    s = _logprob_inputs(case, seed)
    N, V, T, K, tau = case["N"], case["V"], case["T"], case["K"], case["temperature"]
    f64 = dict(dtype=torch.float64, device="cuda")
    logp, H, stats = torch.zeros(N, T, **f64), torch.empty(N, **f64), torch.empty(N, 2, **f64)
    top, at = torch.empty(N, K, **f64), torch.empty(N, K, dtype=torch.int32, device="cuda")
    for a, b in _steps(N, V):
        x = s["x"][a:b].double()
        big = x.max(dim=1)
        others = torch.exp((x - big.values[:, None]) / tau)
        others.scatter_(1, big.indices[:, None], 0.0)
        rest = others.sum(dim=1)
        ln_sum = big.values / tau + torch.log1p(rest)
        lnp = x / tau - ln_sum[:, None]
        tok = s["tokens"][a:b].long()
        ok = (tok >= 0) & (tok < V)
        logp[a:b] = torch.where(ok, torch.gather(lnp, 1, tok.clamp(0, V - 1)), logp[a:b])
        # (the largest one's log p from the others, so that it keeps its digits)
        hit = ok & (tok == big.indices[:, None])
        logp[a:b] = torch.where(hit, -torch.log1p(rest)[:, None], logp[a:b])
        p = torch.exp(lnp)
        H[a:b] = -(p * lnp.clamp(min=-1e4)).sum(dim=1)
        stats[a:b, 0], stats[a:b, 1] = big.values, rest
        if K:
            bits = s["x"][a:b].float().contiguous().view(torch.int32).long()
            order = torch.where(bits < 0, -1 - (bits & 0x7FFFFFFF), bits)
            order = torch.where(x == 0, torch.zeros_like(order), order)
            key = order * (1 << 31) + ((1 << 31) - 1 - torch.arange(V, device="cuda"))
            best = torch.topk(key, K, dim=1).indices
            at[a:b], top[a:b] = best.int(), torch.gather(lnp, 1, best)
    out = dict(logp=logp, stats=stats)
    if case["entropy"]:
        out["entropy"] = H
    if K:
        out.update(top_vals=top, top_idx=at)
    return out


def _logprob_bwd_exact(case, seed):
    """d ln p_t / dz_j = 1[j = t] - p_j and dH / dz_j = -p_j (ln p_j + H), from the logits."""
    s = _logprob_inputs(case, seed)
    N, V, tau = case["N"], case["V"], case["temperature"]
    out = torch.empty(N, V, dtype=torch.float64, device="cuda")
    for a, b in _steps(N, V):
        z = s["x"][a:b].double() / tau
        z = z - torch.logsumexp(z, dim=1, keepdim=True)
        p = torch.exp(z)
        tok, g = s["tokens"][a:b].long(), s["dlogp"][a:b].double()
        d = torch.zeros_like(p)
        for t in range(case["T"]):
            ok = (tok[:, t] >= 0) & (tok[:, t] < V)
            gt = torch.where(ok, g[:, t], torch.zeros_like(g[:, t]))
            d -= gt[:, None] * p
            d.scatter_add_(1, tok[:, t:t + 1].clamp(0, V - 1), gt[:, None])
        if case["entropy"]:
            zc = z.clamp(min=-1e4)
            H = -(p * zc).sum(dim=1, keepdim=True)
            d -= s["dentropy"][a:b].double()[:, None] * p * (zc + H)
        out[a:b] = d / tau
    return out


def _sequences(s, N):
    if s["starts"] is None:
        return [(0, N)]
    at = s["starts"].tolist()
    return list(zip(at[:-1], at[1:]))


def _shares64(x, score):
    if score == "softmax":
        return torch.softmax(x, dim=1)
    e = torch.sigmoid(x)
    return e / e.sum(dim=1, keepdim=True)


def _balance_exact(case, seed):
    """Sequence by sequence."""
    s = _balance_inputs(case, seed)
    N, V, K = case["N"], case["V"], case["K"]
    loss, counts, probs, rows = [], [], [], []
    for a, b in _sequences(s, N):
        idx = s["idx"][a:b].long()
        took = (idx >= 0).any(dim=1)
        n = int(took.sum())
        c = torch.bincount(idx[idx >= 0], minlength=V)
        total = _shares64(s["x"][a:b][took].double(), case["score"]).sum(dim=0)
        P = total / max(n, 1)
        loss.append(case["scale"] * (c.double() * V / (K * max(n, 1)) * P).sum())
        counts.append(c.int())
        probs.append(P)
        rows.append(n)
    return dict(loss=torch.stack(loss), counts=torch.stack(counts), probs=torch.stack(probs),
                rows=torch.tensor(rows, dtype=torch.int32))


def _balance_bwd_exact(case, seed):
    """loss = scale E / (K n^2) sum_e c_e sum_r q_re with the derivatives of the shares:
    dq_e/dx_j = q_e (1[e = j] - q_j), times 1 - sigma_j for the sigmoid."""
    s = _balance_inputs(case, seed)
    N, V, K = case["N"], case["V"], case["K"]
    out = torch.zeros(N, V, dtype=torch.float64, device="cuda")
    for i, (a, b) in enumerate(_sequences(s, N)):
        x = s["x"][a:b].double()
        q = _shares64(x, case["score"])
        n = max(int(s["rows"][i]), 1)
        c = s["counts"][i].double()
        d = q * c - q * (q * c).sum(dim=1, keepdim=True)
        if case["score"] == "sigmoid":
            d = d * torch.sigmoid(-x)
        took = (s["idx"][a:b] >= 0).any(dim=1, keepdim=True)
        factor = float(s["dloss"][i]) * case["scale"] * V / (K * n * n)
        out[a:b] = torch.where(took, factor * d, torch.zeros_like(d))
    return out


def exact(case, seed):
    return {"logprob": _logprob_exact, "logprob_bwd": _logprob_bwd_exact,
            "balance": _balance_exact, "balance_bwd": _balance_bwd_exact}[case["op"]](case, seed)
