"""balance_fwd and balance_bwd of softmax shares at logits of any magnitude: only differences of a
row's logits count, and every finite row has shares."""
import numpy as np
import pytest
import torch

import paper_1805_02867_amd as osm
from test_gpu_balance import check, dev, offsets, places  # noqa: F401
from test_gpu_logprob import DT, logits

pytestmark = pytest.mark.gpu

EXPERTS = [1, 7, 8, 24, 64, 130, 160, 256, 513, 1024]


def far_rows(E, dtype, dev):  # noqa: F811
    """Rows with a common part of any size, with equal logits, at the type's ends, with one logit
    far above or below the others."""
    low, high = torch.finfo(DT[dtype]).min, torch.finfo(DT[dtype]).max
    x = logits(64, E, "f32", E, dev)
    # (about 2^22 / log2(e) = 2.9e6 the way of taking the shares changes; with products of log2(e)
    # that are rounded first, the shares are lost from 1.5e9 on and leave the type from 2.36e38 on)
    size = [0.0, 1e3, 1e5, 2.8e6, 3e6, 1e7, 1e9, 1.6e9, 1e10, 1e20, 1e30, 2.3e38, 2.4e38, 3e38]
    for i, c in enumerate(size):
        x[2 * i] += c
        x[2 * i + 1] -= c
    x[28], x[29] = low, high
    x[30], x[30, 0] = low, high
    x[31], x[31, 0] = high, low
    x[32, E // 2], x[33, E // 2] = 3e38, -3e38
    x[34, E // 2], x[35, E // 2] = 1e10, -1e10
    x[36], x[36, E - 1] = low, 0.0
    x[37, ::2] = low
    x[38], x[39] = 1e10, -1e10
    x[39, 0] = -1e10 - 1e8
    x = x.clamp(low, high).to(DT[dtype])
    assert x.isfinite().all()
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E", EXPERTS)
def test_rows_far_from_zero(E, dtype, dev):  # noqa: F811
    print(f"far {dtype} {E}", flush=True)
    x, idx = far_rows(E, dtype, dev), places(64, E, 2, E, dev, drop=0.0)
    for starts in (None, offsets([1] * 64, dev), offsets([28, 4, 8, 24], dev)):
        r, dx = check(x, idx, starts, "softmax", dtype=dtype)
        assert r.loss.isfinite().all() and dx.isfinite().all()
        r = osm.balance_fwd(x, idx, starts, "sigmoid")
        assert r.loss.isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E", EXPERTS)
def test_equal_logits_share_equally(E, dtype, dev):  # noqa: F811
    for c in (torch.finfo(DT[dtype]).min, -1e30, -1e10, 1e10, 1e30, torch.finfo(DT[dtype]).max):
        x = torch.full((5, E), c, dtype=DT[dtype], device=dev)
        r = osm.balance_fwd(x, torch.zeros(5, 1, dtype=torch.int32, device=dev))
        # (a weight is 1; a reciprocal of 2 u, the product, sums of 5 rows, the mean)
        assert np.allclose(r.probs.cpu().numpy(), 1 / E, rtol=10 * 2.0 ** -24, atol=0), c
        assert abs(r.loss.item() - 1.0) <= 11 * 2.0 ** -24, c


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E", [8, 60, 256, 1024])
def test_other_rows_stay_as_they_are(E, dtype, dev):  # noqa: F811
    """Rows of a wavefront that has a far one beside them: the same gradient to the last bit."""
    x, idx = logits(64, E, dtype, 3, dev), places(64, E, 2, 3, dev, drop=0.0)
    y = x.clone()
    y[::5] = far_rows(E, dtype, dev)[:13] + 1e9
    r, g = osm.balance_fwd(x, idx), torch.ones(1, device=dev)
    a = osm.balance_bwd(x, idx, r.counts, r.rows, g)
    b = osm.balance_bwd(y, idx, r.counts, r.rows, g)
    rest = [i for i in range(64) if i % 5]
    assert torch.equal(a[rest], b[rest])
