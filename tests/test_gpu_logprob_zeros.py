"""logprob_fwd's alternatives in streamed rows whose best elements are zeros of either sign: -0.0
and 0.0 are equal, so the lower index comes first."""
import itertools

import numpy as np
import pytest
import torch

import loss_ref
import paper_1805_02867_amd as osm
from test_gpu_logprob import DT, dev, host  # noqa: F401

pytestmark = pytest.mark.gpu

# Elements of a step of 256 lanes with 4 vectors of 8 each (of binary32 it has half as many)
STEP = 8192


def places(V):
    """The row's ends, each wavefront's first step, later steps, the last one."""
    last = (V - 1) // STEP * STEP
    return [0, 100, 600, 1100, 1700, STEP + 100, 2 * STEP + 1700, (last + V) // 2, V - 1]


def rows_of(V):
    """Rows of negative elements with a few zeros: two places with all signs but two of 0.0, one
    more at the front or the end beside five of -0.0, -0.0 in many places."""
    x = -1.0 - torch.rand(2, V, generator=torch.Generator().manual_seed(V))
    x[0] = -1.0
    rows = []

    def add(at, signs):
        r = x[len(rows) % 2].clone()
        r[torch.as_tensor(at)] = torch.as_tensor(signs)
        rows.append(r)
    for a, b in itertools.combinations(places(V), 2):
        for signs in ((-0.0, -0.0), (0.0, -0.0), (-0.0, 0.0)):
            add([a, b], list(signs))
    for end in (0, V - 1):
        for first in (0, STEP):
            add([end] + [first + i for i in (100, 200, 300, 400, 500)], [0.0] + [-0.0] * 5)
    for every in (9, 1001, 9001):
        at = torch.arange(5, V, every)
        add(at, [-0.0] * len(at))
        add(at, [0.0 if i % 3 == 2 else -0.0 for i in range(len(at))])
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V", [(400, 40001), (512, 50257), (472, 40008), (354, 131081)])
def test_zeros_of_either_sign(N, V, dtype, dev):  # noqa: F811
    """Whole rows, and (354 of 131081) in two chunks; odd lengths, so that rows begin at
    every place between two 16-byte boundaries, and whole vectors only."""
    print(f"zeros {dtype} {N} {V}", flush=True)
    x = rows_of(V).to(DT[dtype])
    want = loss_ref.logprob(x.double().numpy(), None, 32)
    each = (np.arange(N) * 7) % len(x)
    y = x.to(dev)[torch.as_tensor(each).to(dev)]
    for K in (1, 2, 5, 6, 32):
        got = osm.logprob_fwd(y, K=K, stats=True)
        idx = got.top_idx.cpu().numpy()
        bad = np.flatnonzero((idx != want["top_idx"][each, :K]).any(axis=1))
        assert len(bad) == 0, (K, len(bad), bad[:4], idx[bad[:1]],
                               want["top_idx"][each[bad[:1]], :K])
        loss_ref.check(host(got.top_vals), want["top_vals"][each, :K],
                       want["top_vals_err"][each, :K], f"top K={K}")
        loss_ref.check(host(got.stats), want["stats"][each], want["stats_err"][each], "stats")


def test_the_first_two_zeros_of_a_row(dev):  # noqa: F811
    """A row that begins 2 bytes past a boundary: -0.0 in its head, and in the first vector of
    a lane that has no other element that is not negative."""
    x = torch.full((400, 40001), -1.0, dtype=torch.bfloat16, device=dev)
    x[1, 0], x[1, 100] = -0.0, -0.0
    got = osm.logprob_fwd(x, K=2)
    assert got.top_idx[1].tolist() == [0, 100]
    assert not got.top_vals.isnan().any()
