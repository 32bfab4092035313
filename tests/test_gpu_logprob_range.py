"""logprob_fwd and logprob_bwd at the ends of their types: masks of the lowest value, rows of
the lowest and the largest one."""
import numpy as np
import pytest
import torch

import loss_ref
import paper_1805_02867_amd as osm
from test_gpu_logprob import DT, dev, host, logits, some_tokens  # noqa: F401

pytestmark = pytest.mark.gpu


def rows_of(V, dtype, dev):  # noqa: F811
    low, high = torch.finfo(DT[dtype]).min, torch.finfo(DT[dtype]).max
    x = logits(10, V, dtype, V, dev)
    few = torch.rand(V, generator=torch.Generator().manual_seed(V)) < max(0.01, 2 / V)
    x[0, ~few.to(dev)] = low
    x[1], x[1, V - 1] = low, -3.0
    x[2] = low
    x[3, : V // 2] = low
    x[4, 1:] = low
    x[5] = high
    x[6], x[6, V // 2] = low, high
    x[7], x[7, ::2] = low, 0.0
    x[8] = low / 2
    x[9], x[9, ::3] = high / 2, low
    return x


def numbers(want):
    """The reference's numbers as binary32 has them: log probabilities below its lowest value are
    -inf there (the others as they are)."""
    with np.errstate(over="ignore"):
        f = want.astype(np.float32).astype(np.float64)
    return np.where(np.isinf(f), f, want)


def check(got, want, r, each=slice(None)):
    for name in ("logp", "entropy", "stats", "top_vals"):
        t = getattr(got, name)
        if t is not None:
            loss_ref.check(host(t), numbers(want[name][each]), want[name + "_err"][each],
                           f"{r} {name}")
    if got.top_idx is not None:
        assert np.array_equal(got.top_idx.cpu().numpy(), want["top_idx"][each]), r


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 40, 1000, 3000, 9001, 40000, 66000, 300001])
def test_lowest_and_largest_values(V, dtype, dev):  # noqa: F811
    print(f"ends {dtype} {V}", flush=True)
    x, tok = rows_of(V, dtype, dev), some_tokens(10, V, 3, V, dev)
    t = tok.cpu().numpy()
    rng = torch.Generator().manual_seed(V)
    g, h = (torch.randn(n, generator=rng).to(dev) for n in ((10, 3), (10,)))
    for tau in (1.0, 0.7, 1.3):
        for K in (0, min(V, 6), min(V, 64)):
            got = osm.logprob_fwd(x, tok, K=K, entropy=True, stats=True, temperature=tau)
            check(got, loss_ref.logprob(host(x), t, K, tau), f"{tau} K={K}")
        for dh in (None, h):
            dx = osm.logprob_bwd(x, got.stats, tok, g, got.entropy if dh is not None else None, dh,
                                 temperature=tau)
            want, err = loss_ref.logprob_bwd(host(x), t, host(g), None if dh is None else host(dh),
                                             tau, dtype)
            loss_ref.check(host(dx), want, err, f"gradient {tau}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(400, 40001), (300, 1000), (2000, 24)])
def test_batches(N, V, dtype, dev):  # noqa: F811
    """Streamed rows with and without alternatives, short rows."""
    x, tok = rows_of(V, dtype, dev), some_tokens(10, V, 2, V, dev)
    each = np.arange(N) * 3 % 10
    at = torch.as_tensor(each).to(dev)
    for K in (0, 5, min(V, 32)):
        got = osm.logprob_fwd(x[at], tok[at], K=K, entropy=True, stats=True)
        check(got, loss_ref.logprob(host(x), tok.cpu().numpy(), K), f"K={K}", each)
