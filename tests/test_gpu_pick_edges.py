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


# top-p, top-k, min-p, and all of them
FILTERS = (dict(top_p=0.9), dict(top_k=50), dict(min_p=0.02, top_p=0.98, temperature=1.3),
           dict(top_k=3000, top_p=0.95, min_p=1e-3))


@pytest.mark.parametrize("V", [128256, 32000, 9001, 5000])
def test_bfloat16_rows_with_a_constant_added(V, dev):
    """A softmax does not see it; the bins of the values do.  Chunks on both sides of where the
    bins move, of either sign, by one step and by several."""
    shift = [8, 12, 16, 20, 24, 29, 33, 200, 500, 3000, -3, -8, -13, -15, -20, -28, -33, -40, -100,
             -520, -1e4, 1e30]
    x = logits(len(shift), V, "f32", V, dev, 2.0)
    x = (x + torch.tensor(shift, device=dev).unsqueeze(1)).to(torch.bfloat16)
    u = uniform(len(shift), V, dev)
    for kw in FILTERS:
        check(x, u, dev, **kw)


@pytest.mark.parametrize("T", [1.0, 30.0, 1000.0])
def test_bfloat16_chunks_whose_bins_begin_elsewhere(T, dev):
    """Parts of a row around levels of their own: what leaves the row's bins on either side
    has weight at these temperatures, next to 0 and far below it."""
    V, part = 40000, 2500
    levels = [[40.0, 20.0, 20.0, 3.0], [700.0, 20.0, 1e-3, 300.0], [1e4, 1.0, 30.0, 600.0],
              [1e30, 1e25, 3.0, -1.0], [5.0, -5.0, -50.0, -900.0], [0.02, -0.02, -0.3, -40.0],
              [-0.05, -0.5, -40.0, -3e4], [-1e-3, -1.0, -1e3, -1e6], [-40.0, -600.0, -1e4, -1e9],
              [600.0, 40.0, -40.0, -600.0], [33.0, -33.0, 33.0, -1e-6], [2.0, 1e-4, -1e-4, -0.1]]
    g = torch.Generator().manual_seed(7)
    x = torch.randn(len(levels), V, generator=g)
    for r, at in enumerate(levels):
        order = torch.randperm(4, generator=g)
        for c in range(V // part):
            a = at[order[c % 4]]
            v = x[r, c * part:(c + 1) * part]
            v.copy_(a - abs(a) * 0.1 * v.abs())
    x = x.to(torch.bfloat16).to(dev)
    for seed, kw in enumerate(FILTERS + (dict(top_p=0.5), dict(top_k=V // 2), dict(top_p=0.999),
                                         dict(top_k=V // 3, top_p=0.8), dict(min_p=0.5))):
        check(x, uniform(len(levels), seed, dev), dev, **(dict(temperature=T) | kw))


@pytest.mark.parametrize("N", [64, 512])
def test_a_constant_costs_bfloat16_rows_little(N, dev):
    """The same batch with a constant added, by the fastest of several batches of calls."""
    V = 128256
    g = torch.Generator(device=dev).manual_seed(N)
    r = torch.randn(N, V, device=dev, generator=g)
    r = 2.0 * (r + 0.5 * (r - 2.0).clamp(min=0.0) ** 2)
    u = uniform(N, 1, dev)

    def us(shift):
        x = (r + shift).to(torch.bfloat16)
        return best_us(lambda: osm.softmax_sample(x, u, top_p=0.9), batches=5, calls=3)
    centred = us(0.0)
    for shift in (8.0, 12.0, 16.0, 20.0, -20.0, -28.0, -40.0, -100.0):
        assert us(shift) < 2.0 * centred, shift


def near_zero(N, V, g, dev):
    """Rows of which a hundredth lies within 2^-11 of 0, on both sides; and how many lie
    above 2^-11, a row."""
    x = torch.randn(N, V, device=dev, generator=g)
    few = torch.rand(N, V, device=dev, generator=g) < 0.01
    x = torch.where(few, 2.0 ** -12 * x.clamp(-1, 1), x)
    x = x.to(torch.bfloat16)
    return x, (x >= 2.0 ** -11).sum(dim=1)


@pytest.mark.parametrize("V", [128256, 9001, 6000])
def test_bfloat16_cuts_next_to_zero(V, dev):
    """Cuts among the few elements between the positive and the negative bins: by top-k, by
    top-p, by min-p and one after the other; equal elements there, and zeros of either sign."""
    N = 24
    g = torch.Generator(device=dev).manual_seed(V)
    x, above = near_zero(N, V, g, dev)
    x[1::4] = torch.where(x[1::4].abs() < 2.0 ** -11, torch.sign(x[1::4]) * 2.0 ** -13, x[1::4])
    x[2::4] = torch.where(x[2::4].abs() < 2.0 ** -11, x[2::4] * 0.0, x[2::4])
    mid = (x.abs() < 2.0 ** -11).sum(dim=1)
    k = above + 1 + torch.arange(N, device=dev) * (mid - 1) // (N - 1)  # first to last of them
    u = uniform(N, V, dev)
    u[::3] = 1 - 2.0 ** -20
    for T in (0.7, 1.5):
        w = torch.exp(x.double() / T)
        order = torch.sort(w, dim=1, descending=True).values
        c = torch.cumsum(order, dim=1)
        # between the sums before and at the k-th, so that no rounding decides
        at = (torch.gather(c, 1, k.unsqueeze(1) - 1).squeeze(1) - 0.5)
        p = (at / c[:, -1]).float()
        pk = (at / torch.gather(c, 1, (above + mid).unsqueeze(1) - 1).squeeze(1)).float()
        q = torch.exp(-x.double().amax(dim=1) / T).float()       # the weight of 0
        kt, kall = k.int().tolist(), (above + mid).int().tolist()
        for kw in (dict(top_k=kt), dict(top_p=p.tolist()), dict(min_p=q.tolist()),
                   dict(top_k=kall, top_p=pk.tolist()), dict(top_k=kt, top_p=0.999999),
                   dict(top_k=kt, top_p=0.5), dict(top_p=p.tolist(), min_p=q.tolist()),
                   dict(top_k=(k + mid).int().tolist(), min_p=q.tolist())):
            check(x, u, dev, temperature=T, **kw)


@pytest.mark.parametrize("V", [40000, 7000])
def test_bfloat16_cuts_beyond_the_bins(V, dev):
    """Cuts among elements below -32 of rows that reach above 0, at temperatures that give
    them weight."""
    N = 12
    g = torch.Generator(device=dev).manual_seed(V)
    x = 5.0 * torch.randn(N, V, device=dev, generator=g)
    x = torch.where(torch.rand(N, V, device=dev, generator=g) < 0.05, -40.0 - x.abs(), x)
    x[3::4] = x[3::4].round()
    x = x.clamp(max=31.0).to(torch.bfloat16)
    low = (x <= -32.0).sum(dim=1)
    k = (V - low + 1 + torch.arange(N, device=dev) * (low - 1) // (N - 1)).int().tolist()
    u = uniform(N, V, dev)
    u[::3] = 1 - 2.0 ** -20
    for kw in (dict(top_k=k), dict(top_p=0.99), dict(top_p=0.9999), dict(top_k=k, top_p=0.9999),
               dict(top_k=k, top_p=0.97), dict(min_p=0.15), dict(top_k=k, min_p=0.2),
               dict(top_k=k, top_p=0.5)):
        check(x, u, dev, temperature=40.0, **kw)


@pytest.mark.parametrize("N", [64, 512])
def test_cuts_next_to_zero_cost_bfloat16_rows_little(N, dev):
    V = 128256
    x = torch.randn(N, V, device=dev, generator=torch.Generator(device=dev).manual_seed(1))
    x = x.to(torch.bfloat16)
    above = (x >= 2.0 ** -11).sum(dim=1)
    u = uniform(N, 1, dev)

    def us(k):
        k = k.int()
        return best_us(lambda: osm.softmax_sample(x, u, top_k=k), batches=5, calls=3)
    assert us(above + 5) < 3.0 * us(above // 2)


def test_routing_twice_the_rows_takes_longer(dev):
    """4096 x 160 has the lanes of the larger batch (0.76 of its time; with half the experts a
    lane 0.91)."""
    def us(N):
        x, b = router(N, 160, "f32", N, dev), 0.05 * router(1, 160, "f32", 1, dev).view(-1)
        kw = dict(score="sigmoid", groups=8, top_groups=3, group_top=2)
        vals, idx = osm.route_fwd(x, 6, b, **kw)
        return best_us(lambda: osm.route_fwd(x, 6, b, vals=vals, idx=idx, **kw))
    assert us(4096) < 0.84 * us(8192)


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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_flat_and_cold_short_rows_cost_little(dtype, dev):
    """Rows whose cut lies among more elements than a list holds, or below the histogram,
    against ordinary ones; and their tokens."""
    N, V = 4000, 1000
    x, u = logits(N, V, dtype, 3, dev, 1.0), uniform(N, 3, dev)
    flat = torch.ones_like(x)

    def us(x, **kw):
        return best_us(lambda: osm.softmax_sample(x, u, **kw), batches=5, calls=3)
    ordinary = us(x, top_p=0.9)
    for y, kw in ((x, dict(top_p=0.9, temperature=30.0)), (x, dict(top_k=700, temperature=30.0)),
                  (flat, dict(top_p=0.9)), (x, dict(top_k=50, temperature=0.05))):
        check(y[:64], u[:64], dev, **kw)
        assert us(y, **kw) < 3.0 * ordinary, kw


@pytest.mark.parametrize("N,V", [(1000, 7000), (2000, 8000)])
def test_bfloat16_rows_of_a_workgroup_take_no_longer_than_binary32(N, V, dev):
    """Of as many elements a lane, in half the bytes."""
    x, u = logits(N, V, "f32", 3, dev), uniform(N, 3, dev)

    def us(x, kw):
        return best_us(lambda: osm.softmax_sample(x, u, **kw), batches=5, calls=3)
    for kw in (dict(), dict(top_p=0.9), dict(top_k=50), dict(temperature=0.0)):
        assert us(x.to(torch.bfloat16), kw) < 1.25 * us(x, kw), kw


def test_one_more_row_does_not_cost_a_launch(dev):
    """256 and 300 binary32 rows of a vocabulary, with a filter."""
    V = 128256
    x = torch.randn(300, V, device=dev, generator=torch.Generator(device=dev).manual_seed(1)) * 2
    u = uniform(300, 1, dev)

    def us(N):
        return best_us(lambda: osm.softmax_sample(x[:N], u[:N], top_p=0.9), batches=5, calls=3)
    assert us(300) < 1.4 * us(256)


@pytest.mark.parametrize("dtype,N,V", [("f32", 2100, 20000), ("bf16", 2100, 20000),
                                       ("f32", 1100, 50257), ("bf16", 1037, 50257),
                                       ("f32", 4200, 12000), ("f32", 1400, 20000)])
def test_batches_of_more_than_one_launch(dtype, N, V, dev):
    """4096 chunks a launch, in the same scratch: rows on both sides of each launch's border and
    the last ones, and the whole batch the same with a workspace and once more."""
    g = torch.Generator(device=dev).manual_seed(N)
    r = torch.randn(N, V, device=dev, generator=g)
    x = (2.0 * r).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    u = torch.rand(N, device=dev, generator=g)
    rows = sorted({r for S in (2, 3, 4, 5, 7, 8) for b in range(4096 // S, N + 1, 4096 // S)
                   for r in range(b - 3, b + 3) if 0 <= r < N} | set(range(4)) |
                  set(range(N - 4, N)))
    at = torch.tensor(rows, device=dev)
    ws = torch.full((osm.sample_workspace(N, V, x.dtype),), 255, dtype=torch.uint8, device=dev)
    # a launch is full with a filter or without
    assert 0 < ws.numel() and abs(ws.numel() - osm.sample_workspace(2 * N, V, x.dtype)) < 1 << 16
    for kw in (dict(), dict(top_p=0.9), dict(top_k=300, top_p=0.95, min_p=1e-3)):
        vals, idx = osm.softmax_sample(x, u, **kw)
        rv, ri = pick_ref.sample(host(x[at]), host(u[at]), **kw)
        assert np.array_equal(idx[at].cpu().numpy(), ri)
        pick_ref.close(host(vals[at]), rv)
        for w in (ws, None):
            v, i = osm.softmax_sample(x, u, workspace=w, **kw)
            assert torch.equal(i, idx) and torch.equal(v, vals)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_streamed_rows(dtype, dev):
    """Rows of more than 64 chunks."""
    V = 2200003
    assert osm.sample_workspace(3, V, torch.float32 if dtype == "f32" else torch.bfloat16) == 0
    x, u = logits(3, V, dtype, 4, dev), uniform(3, 4, dev)
    x[1, : V // 2] = -INF
    x[2, 77] = NAN
    for kw in (dict(), dict(top_p=0.9), dict(top_k=300), dict(min_p=0.01), dict(temperature=0.0),
               dict(top_k=100000, top_p=0.99)):
        check(x, u, dev, **kw)
