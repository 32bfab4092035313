"""Sampling and routing where their short ways end: biases whose sums leave binary32,
logits that are not numbers under a gradient, rows of bfloat16 far from 0, and batches
of more than one launch."""
import numpy as np
import pytest
import torch

import paper_1805_02867_amd as osm
import pick_ref
from parity import best_us
from test_gpu_route import check_bwd, check_fwd
from test_gpu_route import logits as router
from test_gpu_sample import LOWEST, check, host, logits, uniform

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
LOW = LOWEST["f32"]


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X; none is visible")
    return torch.device("cuda:0")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E", [32, 256])
def test_groups_by_sums_that_leave_binary32(E, score, dev):
    """Two biases of the type's lowest (or largest) values: their sum is finite in binary64,
    and a group that has it comes before one that has nothing to choose."""
    x, gs = router(9, E, "f32", E, dev), E // 8
    for values in ((-INF, LOW, -INF, LOW, -INF, LOW, -INF, -INF),
                   (LOW, -3.0e38, LOW, -2.0e38, -INF, -3.2e38, LOW, LOW),
                   (-LOW, 3.0e38, -LOW, 2.0e38, INF, 3.2e38, 1.0, LOW),
                   (LOW,) * 8):
        b = torch.tensor(values, device=dev).repeat_interleave(gs)
        single = b.clone()
        single.view(8, gs)[3, 1:] = -INF      # a group of one
        for bias in (b, single):
            for top in (1, 2, 3):
                check_fwd(x, 2, bias, score=score, groups=8, top_groups=top, group_top=2)


@pytest.mark.filterwarnings("ignore:invalid value")     # of the reference, on purpose
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E,K", [(24, 4), (33, 3), (256, 8)])
def test_gradient_of_logits_that_are_not_numbers(E, K, dtype, dev):
    """A given index is taken as it is: where the weights' formula is not a number, so is its
    gradient, and no place outside of what they depend on."""
    x = router(7, E, dtype, E, dev)
    idx = torch.arange(K, dtype=torch.int32, device=dev).repeat(7, 1)
    x[0, 1] = NAN              # among the chosen
    x[1, E - 1] = NAN          # not among them
    x[2, 0] = INF
    x[3, E - 1] = INF
    x[4, 2] = -INF             # a share of 0
    x[5, 1], x[5, 2] = -INF, NAN
    g = router(7, K, "f32", 4, dev)
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            dx = check_bwd(x, idx, g, dtype, score=score, renorm=renorm)
            assert dx[0].isnan().any() and not dx[[4, 6]].isnan().any()
            none = osm.route_bwd(torch.full_like(x, -INF), idx, g, score=score, renorm=renorm)
            assert not none.any() or not renorm
            outside = torch.tensor([-1], dtype=torch.int32, device=dev).expand(7, K).contiguous()
            assert not osm.route_bwd(x, outside, g, score=score, renorm=renorm).any()
