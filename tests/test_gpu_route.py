"""route_fwd and route_bwd against plain binary64 implementations: experts equal,
weights and gradients within the rounding of their type."""
import itertools

import numpy as np
import pytest
import torch

import paper_1805_02867_amd as osm
import pick_ref

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X; none is visible")
    return torch.device("cuda:0")


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def logits(N, E, dtype, seed, dev, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    return (sigma * torch.randn(N, E, generator=g)).to(TYPES[dtype]).to(dev)


def check_fwd(x, K, bias=None, **kw):
    vals, idx = osm.route_fwd(x, K, bias=bias, **kw)
    torch.cuda.synchronize()
    rv, ri = pick_ref.route(host(x), K, host(bias), **kw)
    got = idx.cpu().numpy()
    assert np.array_equal(got, ri), [(r, got[r], ri[r])
                                     for r in np.flatnonzero((got != ri).any(1))[:3]]
    pick_ref.close(host(vals), rv)
    return vals, idx


def check_bwd(x, idx, g, dtype, **kw):
    dx = osm.route_bwd(x, idx, g, **kw)
    torch.cuda.synchronize()
    want = pick_ref.route_bwd(host(x), idx.cpu().numpy(), host(g), **kw)
    # what cancels (g_i - sum g p) is a binary64 difference of the g
    slack = 2.0 ** -44 * abs(kw.get("scale", 1.0)) * float(g.abs().max()) if g.numel() else 0.0
    pick_ref.close(host(dx), want, dtype, slack)
    return dx


# (E, K, groups, top_groups)
SHAPES = [(1, 1, 1, 1), (2, 1, 1, 1), (8, 2, 1, 1), (8, 8, 1, 1), (16, 4, 4, 2), (33, 5, 1, 1),
          (60, 4, 1, 1), (64, 6, 8, 3), (64, 64, 1, 1), (100, 10, 5, 2), (128, 1, 1, 1),
          (160, 6, 8, 3), (256, 8, 8, 4), (257, 8, 1, 1), (384, 12, 1, 1), (512, 16, 64, 7),
          (1024, 64, 1, 1), (1024, 8, 16, 4), (990, 33, 30, 9)]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,K,groups,top_groups", SHAPES)
def test_shapes(E, K, groups, top_groups, dtype, score, dev):
    for N in (1, 37):
        x = logits(N, E, dtype, E + N, dev)
        b = 0.1 * logits(1, E, "f32", E, dev).view(-1)
        g = logits(N, K, "f32", 7, dev)
        for renorm, bias, top in itertools.product((True, False), (None, b), (1, 2)):
            kw = dict(score=score, renorm=renorm, scale=2.5)
            vals, idx = check_fwd(x, K, bias, groups=groups, top_groups=top_groups,
                                  group_top=top, **kw)
            if top == 1:
                check_bwd(x, idx, g, dtype, **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [2, 63, 64, 65, 1000, 5001])
def test_batches(N, dtype, dev):
    x = logits(N, 64, dtype, N, dev)
    vals, idx = check_fwd(x, 6)
    g = logits(N, 6, "f32", 1, dev)
    for score, renorm in itertools.product(("softmax", "sigmoid"), (True, False)):
        check_bwd(x, idx, g, dtype, score=score, renorm=renorm)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", TYPES)
def test_ties_and_far_logits(dtype, score, dev):
    """Equal experts and groups go to the lower index; weights of logits far below (or
    above) do not vanish together when they are renormalised."""
    g = torch.Generator().manual_seed(5)
    few = torch.randint(0, 3, (50, 96), generator=g).to(TYPES[dtype]).to(dev)
    zero = torch.where(torch.rand(50, 96, generator=g) < 0.5, 0.0, -0.0).to(TYPES[dtype]).to(dev)
    for x in (few, zero):
        for kw in (dict(), dict(groups=8, top_groups=3), dict(groups=8, top_groups=3, group_top=2)):
            check_fwd(x, 9, score=score, **kw)
            check_fwd(x, 9, torch.zeros(96, device=dev), score=score, **kw)
    for shift in (-3e4, -900.0, -120.0, 90.0, 1e4):
        x = (logits(20, 40, dtype, 6, dev, 3.0) + shift).to(TYPES[dtype])
        vals, idx = check_fwd(x, 5, score=score)
        assert (vals > 0).any(dim=1).all()
        gr = logits(20, 5, "f32", 2, dev)
        check_bwd(x, idx, gr, dtype, score=score)
        check_fwd(x, 5, score=score, renorm=False)
        check_bwd(x, idx, gr, dtype, score=score, renorm=False)


def test_a_bias_decides_between_close_scores(dev):
    """Sums s + bias that binary32 cannot tell apart."""
    x = torch.zeros(4, 32, device=dev)
    x[:, 5] = 2.0 ** -20
    x[:, 9] = 2.0 ** -21
    b = torch.full((32,), 0.75, device=dev)
    for score in ("softmax", "sigmoid"):
        _, idx = check_fwd(x, 3, b, score=score)
        assert idx[0].tolist() == [5, 9, 0]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,K,groups", [(8, 3, 2), (40, 6, 4), (256, 8, 8), (1000, 20, 10)])
def test_near_ties_everywhere(E, K, groups, score, dev):
    """Scores that differ by less than a binary32 sum with the bias can show: at every
    place, at the last one, and between the groups at the line; beside ordinary rows."""
    g = torch.Generator().manual_seed(E)
    n = 48
    x = torch.randn(n, E, generator=g)
    x[::3] = 0.5 + 2.0 ** -22 * torch.randint(0, 9, (n // 3, E), generator=g)
    x[1::3] = x[1::3].round()
    x = x.to(dev)
    for b in (torch.full((E,), 3.0), torch.zeros(E), 0.1 * torch.randn(E, generator=g),
              1e6 * torch.randint(-1, 2, (E,), generator=g)):
        b = b.to(dev)
        for top in (1, 2):
            check_fwd(x, K, b, score=score, groups=groups, top_groups=groups - 1, group_top=top)
    check_fwd(x, K, score=score, groups=groups, top_groups=groups - 1, group_top=2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,groups", [(24, 1), (24, 4), (200, 8), (600, 1)])
def test_masks(E, groups, dtype, score, dev):
    x = logits(9, E, dtype, E, dev)
    x[0] = -INF
    x[1] = -INF
    x[1, E - 1] = 0.5
    x[2, 1:] = -INF
    x[3, ::2] = -INF
    x[4, E // 2] = NAN
    x[5, 0] = INF
    x[6, :E // 2] = -INF
    x[7] = torch.finfo(x.dtype).min
    b = 0.1 * logits(1, E, "f32", 3, dev).view(-1)
    b[3] = -INF
    b[4] = NAN
    b[7] = INF
    K = 5
    g = logits(9, K, "f32", 4, dev)
    for bias, renorm in itertools.product((None, b), (True, False)):
        kw = dict(score=score, renorm=renorm)
        vals, idx = check_fwd(x, K, bias, groups=groups, top_groups=groups, group_top=2, **kw)
        assert (idx[[0, 4, 5]] == -1).all()
        assert (vals[0] == 0).all() and vals[[4, 5]].isnan().all()
        dx = check_bwd(x, idx, g, dtype, **kw)
        assert (dx[[0, 4, 5]] == 0).all()


def test_gradient_indices_outside_and_twice(dev):
    x = logits(6, 30, "f32", 1, dev)
    idx = torch.tensor([[0, 3, 29], [-1, 30, 4], [-1, -1, -1], [5, 5, 2], [7, 7, 7],
                        [2 ** 31 - 1, -2 ** 31, 1]], dtype=torch.int32, device=dev)
    g = logits(6, 3, "f32", 2, dev)
    for score, renorm in itertools.product(("softmax", "sigmoid"), (True, False)):
        dx = check_bwd(x, idx, g, "f32", score=score, renorm=renorm)
        assert (dx[2] == 0).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(score, renorm, dev):
    """The weights of the kernel itself at x +- h: the difference of two binary32 weights
    (each off by 2^-25 or less of a value under 2.5) over 2h, and h^2 / 6 of a third
    derivative under 10 * 2.5."""
    x = logits(3, 16, "f32", 8, dev)
    g = logits(3, 4, "f32", 9, dev)
    kw = dict(score=score, renorm=renorm, scale=2.5)
    _, idx = osm.route_fwd(x, 4, **kw)
    dx = osm.route_bwd(x, idx, g, **kw).double()
    h = 2.0 ** -7
    bound = (4 * 2 * 2.0 ** -24 * 2.5 / (2 * h) + h * h / 6 * 25 * 4) * g.abs().max().item()
    for e in range(16):
        d = torch.zeros_like(x)
        d[:, e] = h
        vh, ih = osm.route_fwd(x + d, 4, **kw)
        vl, il = osm.route_fwd(x - d, 4, **kw)
        ok = ((ih == idx) & (il == idx)).all(dim=1)
        diff = ((vh.double() - vl.double()) * g.double()).sum(dim=1) / (2 * h)
        assert ((diff - dx[:, e]).abs()[ok] <= bound).all()


def test_outputs_in_place_and_unaligned(dev):
    N, E, K = 13, 37, 5
    for dtype in TYPES:
        buf = torch.full((N * E + 3,), NAN, dtype=TYPES[dtype], device=dev)
        x = buf[3:].view(N, E)
        x.copy_(logits(N, E, dtype, 3, dev))
        vals = torch.full((N * K + 2,), -7.0, device=dev)
        idx = torch.full((N * K + 2,), -7, dtype=torch.int32, device=dev)
        osm.route_fwd(x, K, vals=vals[1:-1], idx=idx[1:-1])
        rv, ri = pick_ref.route(host(x), K)
        assert np.array_equal(idx[1:-1].view(N, K).cpu().numpy(), ri)
        assert (vals[[0, -1]] == -7).all() and (idx[[0, -1]] == -7).all()
        out = torch.full((N * E + 4,), -7.0, dtype=TYPES[dtype], device=dev)
        g = logits(N, K, "f32", 4, dev)
        osm.route_bwd(x, idx[1:-1].view(N, K), g, dx=out[1:-3].view(N, E))
        pick_ref.close(host(out[1:-3].view(N, E)), pick_ref.route_bwd(host(x), ri, host(g)), dtype,
                       2.0 ** -40)
        assert (out[[0, -1, -2, -3]] == -7).all()
    v, i = osm.route_fwd(x[:0], K)
    assert v.shape == (0, K) and osm.route_bwd(x[:0], i, v).shape == (0, E)


def test_refusals(dev):
    x = logits(4, 32, "f32", 1, dev)
    v, i = osm.route_fwd(x, 4)
    for f in (lambda: osm.route_fwd(x.half(), 4), lambda: osm.route_fwd(x.t(), 4),
              lambda: osm.route_fwd(x, 4, bias=x[0, :31]),
              lambda: osm.route_fwd(x, 4, bias=x[0].double()),
              lambda: osm.route_fwd(x, 4, score="tanh"),
              lambda: osm.route_fwd(x, 4, vals=v[:, :3]),
              lambda: osm.route_bwd(x, i.long(), v), lambda: osm.route_bwd(x, i, v.double()),
              lambda: osm.route_bwd(x, i, v[:, :3]), lambda: osm.route_bwd(x, i, v, dx=v)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: osm.route_fwd(x, 0), lambda: osm.route_fwd(x, 33),
              lambda: osm.route_fwd(x, 4, groups=5), lambda: osm.route_bwd(x, i, v, dx=x)):
        with pytest.raises(osm.OsmError):
            f()


def test_captured_replays(dev):
    x = logits(300, 96, "bf16", 1, dev)
    g = logits(300, 4, "f32", 2, dev)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        vals, idx = osm.route_fwd(x, 4, groups=8, top_groups=2, group_top=2)
        dx = osm.route_bwd(x, idx, g)
    rv, ri = osm.route_fwd(x, 4, groups=8, top_groups=2, group_top=2)
    rd = osm.route_bwd(x, ri, g)
    for rep in range(3):
        for t in (vals, idx, dx):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(vals, rv) and torch.equal(idx, ri) and torch.equal(dx, rd)
        check_fwd(x, 4)


@pytest.mark.parametrize("E", [1024, 1021])
def test_offsets_past_32_bits(E, dev):
    """A batch of more than 2^31 logits: its last rows."""
    N, K, last = (1 << 31) // E + 100, 4, 64
    x = torch.zeros(N, E, dtype=torch.bfloat16, device=dev)
    x[-last:] = logits(last, E, "bf16", 1, dev)
    g = torch.zeros(N, K, device=dev)
    g[-last:] = logits(last, K, "f32", 2, dev)
    vals, idx = osm.route_fwd(x, K)
    dx = osm.route_bwd(x, idx, g)
    rv, ri = pick_ref.route(host(x[-last:]), K)
    assert np.array_equal(idx[-last:].cpu().numpy(), ri)
    pick_ref.close(host(vals[-last:]), rv)
    want = pick_ref.route_bwd(host(x[-last:]), ri, host(g[-last:]))
    pick_ref.close(host(dx[-last:]), want, "bf16", 2.0 ** -44 * float(g.abs().max()))
    assert (idx[:-last] == torch.arange(K, device=dev, dtype=torch.int32)).all()
    assert not dx[:-last].any()
