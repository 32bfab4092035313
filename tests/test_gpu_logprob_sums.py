"""The sums of long streamed rows are not one chain of additions a lane: small weights behind many
large ones are not lost one by one."""
import numpy as np
import pytest
import torch

import paper_1805_02867_amd as osm
from test_gpu_logprob import DT, dev, host  # noqa: F401

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [0, 5])
def test_small_weights_behind_large_ones(K, dtype, dev):  # noqa: F811
    """At a temperature of log2(e) weights are 2^(x - m).  A lane's first step has weights of 1, P of
    them, every later element has half a unit in the last place of P: added to the sum one by one
    they are lost, as a tie with an even number, with 1 u of the sum each.  The sum of a step's P is
    a whole multiple of that place.

    The bound counts what a row streamed by steps rounds: a weight of the hardware's exponential
    (2 u), a step's sum added to the lane's (u each; a step's own additions, of P equal powers of
    two, are exact), the largest element taken out, the wavefront's tree (6), its scale and the
    merge of up to 8 wavefronts (4 each)."""
    N, V = 400, 128256
    P = 32 if dtype == "bf16" else 16             # elements of a lane's step
    step = 64 * (4 if K else 8) * P
    steps = -(-V // step)
    small = -19.0 if dtype == "bf16" else -20.0   # P 2^-24
    assert P * 2.0 ** -24 == 2.0 ** small
    x = torch.full((N, V), small, dtype=DT[dtype], device=dev)
    x[:, :step] = 0.0
    tau = float(np.float32(np.log2(np.e)))
    got = osm.logprob_fwd(x, torch.zeros(N, dtype=torch.int32, device=dev), K=K, stats=True,
                          temperature=tau)
    d = step + (V - step) * 2.0 ** small          # 1 + s
    bound = 2 + steps + 1 + 6 + 1 + 4 * 8
    lost = (steps - 2) * P                        # of a lane's chain of single additions, at least
    assert bound < lost / 2
    off = np.abs(1.0 + host(got.stats)[:, 1] - d) / d / U
    assert off.max() <= bound, (off.max(), bound, lost)
    want = -np.log(d)
    assert np.abs(host(got.logp) - want).max() <= (bound * U + abs(want) * U) * 1.001
