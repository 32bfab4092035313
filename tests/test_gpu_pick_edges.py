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
