"""softmax_sample against a plain binary64 implementation: tokens equal, their
probabilities within the rounding of binary32."""
import numpy as np
import pytest
import torch

import paper_1805_02867_amd as osm
import pick_ref

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LOWEST = {t: float(torch.finfo(d).min) for t, d in TYPES.items()}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X; none is visible")
    return torch.device("cuda:0")


def host(t):
    return t.detach().double().cpu().numpy()


def logits(N, V, dtype, seed, dev, sigma=2.0):
    g = torch.Generator().manual_seed(seed)
    r = torch.randn(N, V, generator=g)
    up = (r - 2.0).clamp(min=0.0)
    return ((r + 0.5 * up * up) * sigma).to(TYPES[dtype]).to(dev)


def uniform(N, seed, dev):
    return torch.rand(N, generator=torch.Generator().manual_seed(seed)).to(dev)


def on_device(kw, dev):
    out = {}
    for n, v in kw.items():
        if np.ndim(v):
            v = torch.tensor(v, dtype=torch.int32 if n == "top_k" else torch.float32).to(dev)
        out[n] = v
    return out


def check(x, u, dev, **kw):
    """One call against the reference; the settings are numbers or lists of N."""
    vals, idx = osm.softmax_sample(x, u, **on_device(kw, dev))
    torch.cuda.synchronize()
    rv, ri = pick_ref.sample(host(x if x.dim() == 2 else x.unsqueeze(0)), host(u), **kw)
    got = idx.cpu().numpy()
    assert np.array_equal(got, ri), [(r, got[r], ri[r]) for r in np.flatnonzero(got != ri)[:5]]
    pick_ref.close(host(vals), rv)
    return vals, idx


SETTINGS = {
    "plain": {}, "hot": dict(temperature=1.7), "cold": dict(temperature=0.05),
    "greedy": dict(temperature=0.0), "k1": dict(top_k=1), "k7": dict(top_k=7),
    "k300": dict(top_k=300), "p": dict(top_p=0.9), "small_p": dict(top_p=0.01),
    "large_p": dict(top_p=0.9999), "q": dict(min_p=0.05), "q1": dict(min_p=1.0),
    "kp": dict(temperature=0.8, top_k=50, top_p=0.9),
    "pq": dict(temperature=1.3, top_p=0.95, min_p=0.03),
    "kpq": dict(top_k=900, top_p=0.7, min_p=0.001),
}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 2, 3, 63, 64, 65, 257, 1000, 2049, 4099, 8193, 16411, 50257])
def test_settings(V, dtype, dev):
    N = 7
    x = logits(N, V, dtype, V, dev)
    for i, kw in enumerate(SETTINGS.values()):
        check(x, uniform(N, 31 * V + i, dev), dev, **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,V", [(1, 128256), (3, 131073), (70, 32000), (600, 1000),
                                 (2, 1000003), (2, 1200007)])
def test_a_setting_a_row(N, V, dtype, dev):
    rng = np.random.default_rng(V + N)
    x = logits(N, V, dtype, N, dev)
    kind = rng.integers(0, 6, N)
    kw = dict(temperature=np.where(kind == 0, 0.0, rng.uniform(0.5, 1.5, N)).tolist(),
              top_k=np.where(kind % 3 == 2, rng.integers(1, 2000, N), 0).tolist(),
              top_p=np.where(kind >= 3, rng.uniform(0.3, 0.999, N), 1.0).tolist(),
              min_p=np.where(kind >= 4, rng.uniform(0.0, 0.1, N), 0.0).tolist())
    check(x, uniform(N, 5, dev), dev, **kw)
    check(x, uniform(N, 6, dev), dev, top_p=0.95)
    check(x, uniform(N, 7, dev), dev)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [8, 1000, 20000])
def test_ties(V, dtype, dev):
    """Cuts inside runs of equal logits: the lower indices stay.  Equal weights make the
    part of a top-p fall exactly on an element."""
    n = 64
    u = torch.linspace(0, 1 - 2.0 ** -24, n).to(dev)
    same = torch.full((n, V), 1.25, dtype=TYPES[dtype], device=dev)
    g = torch.Generator().manual_seed(V)
    few = torch.randint(0, 4, (n, V), generator=g).to(TYPES[dtype]).to(dev)
    zeros = torch.where(torch.rand(n, V, generator=g) < 0.5, 0.0, -0.0).to(TYPES[dtype]).to(dev)
    for x in (same, few, zeros):
        check(x, u, dev)
        check(x, u, dev, top_k=V // 2 + 1)
        check(x, u, dev, top_k=3, top_p=0.5)
        check(x, u, dev, top_p=0.5)
        check(x, u, dev, top_p=0.3, top_k=V - 1)
        check(x, u, dev, min_p=1.0)
        check(x, u, dev, temperature=0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [5, 300, 9000, 40000])
def test_masks(V, dtype, dev):
    """Masks of -inf and of the type's lowest value; rows with one element left, with
    none, and with what a row must not hold."""
    x = logits(12, V, dtype, V, dev)
    g = torch.Generator().manual_seed(V)
    masked = (torch.rand(12, V, generator=g) < 0.9).to(dev)
    masked[:, V // 2] = False
    x[:4] = x[:4].masked_fill(masked[:4], -INF)
    x[4:6] = x[4:6].masked_fill(masked[4:6], LOWEST[dtype])
    x[6] = -INF
    x[7] = -INF
    x[7, V - 1] = -3.0
    x[8] = LOWEST[dtype]
    x[9, V // 3] = NAN
    x[10, V - 1] = INF
    x[11] = LOWEST[dtype]
    x[11, 0] = -INF
    u = uniform(12, 9, dev)
    for kw in SETTINGS.values():
        vals, idx = check(x, u, dev, **kw)
        assert idx[[6, 9, 10]].tolist() == [-1, -1, -1] and vals[[6, 9, 10]].isnan().all()
        assert idx[7].item() == V - 1 and vals[7].item() == 1.0


@pytest.mark.parametrize("dtype", TYPES)
def test_ends_of_the_settings(dtype, dev):
    N, V = 9, 700
    x = logits(N, V, dtype, 1, dev)
    x[0, :300] = -INF
    u = [0.0, 2.0 ** -24, 0.5, 1 - 2.0 ** -24, 1.0, 7.0, -3.0, NAN, 0.25]
    ut = torch.tensor(u, device=dev)
    for kw in (dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF),
               dict(temperature=1e-30), dict(temperature=1e-42), dict(temperature=1e30),
               dict(top_k=-5), dict(top_k=V), dict(top_k=V + 9), dict(top_k=V - 1),
               dict(top_k=2 ** 31 - 1), dict(top_p=0.0), dict(top_p=-1.0), dict(top_p=2.0),
               dict(top_p=NAN), dict(top_p=1e-30), dict(top_p=1 - 2.0 ** -24),
               dict(min_p=-1.0), dict(min_p=NAN), dict(min_p=2.0), dict(min_p=1e-30),
               dict(top_k=5, top_p=1e-9, min_p=1.0)):
        check(x, ut, dev, **kw)
        check(x[1:2], ut[4:5], dev, **{n: [v] for n, v in kw.items()})


@pytest.mark.parametrize("dtype", TYPES)
def test_far_values(dtype, dev):
    """Magnitudes from the smallest to the largest of the type, and rows shifted far."""
    g = torch.Generator().manual_seed(2)
    e = torch.rand(6, 5000, generator=g) * 76 - 38
    x = (torch.sign(torch.randn(6, 5000, generator=g)) * 10.0 ** e).to(TYPES[dtype])
    x[4:] = x[4:] * 1e-38
    x = x.to(dev)
    shifted = logits(6, 5000, dtype, 3, dev) + torch.tensor([1e3, -1e3, 1e4, -1e4, 88.0, -88.0],
                                                            device=dev).unsqueeze(1)
    for t in (x, shifted.to(TYPES[dtype])):
        for kw in (dict(), dict(top_k=1700), dict(top_p=0.8), dict(temperature=1e30, top_p=0.8),
                   dict(temperature=1e38, top_k=2500, top_p=0.5)):
            check(t, uniform(6, 4, dev), dev, **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [9001, 40000, 300000])
def test_values_of_every_kind(V, dtype, dev):
    """What a histogram over the values themselves could get wrong: elements next to 0 (and a
    cut among them), beyond its ends, rows far from 0 whose parts lie in different octaves,
    rows all negative, and equal elements cut in the middle, in any part of the row."""
    g = torch.Generator().manual_seed(V)
    r = torch.randn(16, V, generator=g)
    x = r.clone()
    x[0] = 2.0 ** -13 * r[0]                           # all next to 0
    x[1] = torch.where(r[1] > 1.0, r[1], 2.0 ** -14 * r[1])
    x[2] = 0.0
    x[3] = r[3].clamp(max=0.0)                         # half of them 0, at the top
    x[4] = 1000.0 + 20.0 * r[4]
    x[4, : V // 2] = x[4, : V // 2].clamp(max=1010.0)  # 2^10 is reached in one half only
    x[5] = -700.0 + r[5]
    x[6] = -30.0 - 25.0 * r[6].abs()                   # beyond the negative end
    x[7] = 31.0 + 2.0 * r[7]                           # both sides of 2^5
    x[8] = (2.0 * r[8]).round()                        # a dozen values
    x[9] = r[9] * 2.0 ** -10
    x[10] = 3e38 * r[10].clamp(-1, 1)
    x[11] = r[11] * 1e-40
    x[12] = torch.where(r[12] > 2.5, 5.0, -40.0)
    x[13] = torch.where(r[13] > 0.0, -2.0 ** -20, 2.0 ** -20)
    x[14] = 100.0 * r[14]
    x[15, : V - 3] = -INF
    x = x.to(TYPES[dtype]).to(dev)
    u = uniform(16, V, dev)
    u[3], u[8] = 0.0, 1.0
    for kw in (dict(), dict(top_p=0.5), dict(top_p=0.9999), dict(top_k=V // 3), dict(top_k=17),
               dict(top_k=V - 2, top_p=0.7), dict(min_p=0.7), dict(top_p=0.9, min_p=1e-6),
               dict(temperature=0.02, top_p=0.9), dict(temperature=40.0, top_p=0.8, min_p=0.3),
               dict(temperature=40.0, top_k=V // 2), dict(temperature=INF, top_p=0.25),
               dict(temperature=1e-35, top_p=0.5, top_k=V // 2)):
        check(x, u, dev, **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V,ld,first", [(1000, 1003, 1), (50257, 50304, 0), (4097, 5000, 3),
                                        (1, 64, 5), (33, 33, 1)])
def test_rows_apart_and_unaligned(V, ld, first, dtype, dev):
    N = 11
    buf = torch.full((N * ld + first,), NAN, dtype=TYPES[dtype], device=dev)
    x = buf[first:].view(N, ld)[:, :V]
    x.copy_(logits(N, V, dtype, V, dev))
    for kw in (dict(), dict(top_k=40, top_p=0.9), dict(top_p=0.97, temperature=1.5)):
        check(x, uniform(N, V, dev), dev, **kw)
    check(x[::2], uniform(6, V, dev), dev, top_p=0.9)     # every other row
    check(x[3], uniform(1, V, dev), dev, top_k=9)         # one row, 1-D
    assert buf.view(-1)[:first].isnan().all()


def test_outputs_are_written_in_place_and_nothing_else(dev):
    x, u = logits(5, 300, "f32", 1, dev), uniform(5, 1, dev)
    vals = torch.full((9,), -7.0, device=dev)
    idx = torch.full((9,), -7, dtype=torch.int32, device=dev)
    v, i = osm.softmax_sample(x, u, vals=vals[2:7], idx=idx[2:7])
    assert v.data_ptr() == vals[2:7].data_ptr() and i.data_ptr() == idx[2:7].data_ptr()
    rv, ri = pick_ref.sample(host(x), host(u))
    assert np.array_equal(idx[2:7].cpu().numpy(), ri)
    assert (vals[[0, 1, 7, 8]] == -7).all() and (idx[[0, 1, 7, 8]] == -7).all()
    v, i = osm.softmax_sample(x[:0], u[:0])
    assert v.shape == (0,) and i.shape == (0,)


def test_refusals(dev):
    x, u = logits(4, 64, "f32", 1, dev), uniform(4, 1, dev)
    bad = [dict(u=u[:3]), dict(u=u.double()), dict(u=u.cpu()), dict(x=x.half()),
           dict(x=x.t()), dict(x=x[:, ::2]), dict(x=x[0].expand(4, 64)), dict(x=x.view(2, 2, 64)),
           dict(temperature=u[:2]), dict(temperature=u.double()),
           dict(top_k=torch.ones(4, device=dev)), dict(top_p=u.cpu()),
           dict(min_p=u.new_zeros(8)[::2]), dict(vals=u.double()), dict(idx=u)]
    for b in bad:
        kw = dict(x=x, u=u) | b
        with pytest.raises(ValueError):
            osm.softmax_sample(kw.pop("x"), kw.pop("u"), **kw)
    with pytest.raises(osm.OsmError):
        osm.softmax_sample(x, u, vals=u)                  # overlaps an input


@pytest.mark.parametrize("N,V", [(3, 128256), (40, 5000)])
def test_streams_and_captured_replays(N, V, dev):
    """Two streams at once, and captured calls replayed with eager calls between."""
    kw = dict(temperature=0.9, top_k=400, top_p=0.9)
    xs = [logits(N, V, "bf16", s, dev) for s in range(2)]
    us = [uniform(N, s, dev) for s in range(2)]
    want = [pick_ref.sample(host(x), host(u), **kw) for x, u in zip(xs, us)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for s, x, u in zip(streams, xs, us):                  # warm
        with torch.cuda.stream(s):
            osm.softmax_sample(x, u, **kw)
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for s, x, u in zip(streams, xs, us):
            with torch.cuda.stream(s):
                got.append(osm.softmax_sample(x, u, **kw))
    torch.cuda.synchronize()
    for n, (v, i) in enumerate(got):
        assert np.array_equal(i.cpu().numpy(), want[n % 2][1])
    graphs, outs = [], []
    for s, x, u in zip(streams, xs, us):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(osm.softmax_sample(x, u, **kw))
        graphs.append(g)
    for rep in range(4):
        for v, i in outs:
            i.fill_(-5)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):                 # both graphs at once
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for (v, i), (rv, ri) in zip(outs, want):
            assert np.array_equal(i.cpu().numpy(), ri), f"replay {rep}"
            pick_ref.close(host(v), rv)
        check(xs[0], us[0], dev, **kw)                    # eager between replays


@pytest.mark.parametrize("N,V", [(3, 128256), (70, 32000)])
def test_workspaces(N, V, dev):
    """Two calls at once in workspaces of their own, of any contents; a small one is refused."""
    kw = dict(top_p=0.9, temperature=1.1)
    n = osm.sample_workspace(N, V, torch.bfloat16)
    assert n > 0
    ws = [torch.full((n,), 255, dtype=torch.uint8, device=dev) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    xs = [logits(N, V, "bf16", s, dev) for s in range(2)]
    us = [uniform(N, s, dev) for s in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, w, x, u in zip(streams, ws, xs, us):
            with torch.cuda.stream(s):
                got.append(osm.softmax_sample(x, u, workspace=w, **kw))
    torch.cuda.synchronize()
    for j in range(2):
        want = pick_ref.sample(host(xs[j]), host(us[j]), **kw)
        for v, i in got[j::2]:
            assert np.array_equal(i.cpu().numpy(), want[1])
            pick_ref.close(host(v), want[0])
    for bad in (ws[0][:n - 1], ws[0][:0], ws[0][1:]):
        with pytest.raises(osm.OsmError):
            osm.softmax_sample(xs[0], us[0], workspace=bad, **kw)


def test_same_bits_every_time(dev):
    x, u = logits(20, 60000, "f32", 8, dev), uniform(20, 8, dev)
    for kw in (dict(), dict(top_p=0.9), dict(top_k=3000, top_p=0.9, min_p=1e-4)):
        first = osm.softmax_sample(x, u, **kw)
        for _ in range(5):
            again = osm.softmax_sample(x, u, **kw)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_a_captured_call_on_another_stream_brings_its_workspace(dev):
    """Else the graph's memory for it could be given to the current stream's next call."""
    x, u = logits(3, 128256, "bf16", 1, dev), uniform(3, 1, dev)
    n = osm.sample_workspace(3, 128256, torch.bfloat16)
    ws = torch.empty(n, dtype=torch.uint8, device=dev)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        main = torch.cuda.current_stream()
        with pytest.raises(ValueError):
            osm.softmax_sample(x, u, top_p=0.9, stream=other)
        other.wait_stream(main)
        vals, idx = osm.softmax_sample(x, u, top_p=0.9, stream=other, workspace=ws)
        main.wait_stream(other)
    rv, ri = pick_ref.sample(host(x), host(u), top_p=0.9)
    for _ in range(3):
        idx.fill_(-5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(idx.cpu().numpy(), ri)
        pick_ref.close(host(vals), rv)


@pytest.mark.parametrize("dtype,V", [("bf16", 700), ("f32", 700), ("bf16", 6000), ("f32", 40000),
                                     ("bf16", 40000)])
def test_offsets_past_32_bits(dtype, V, dev):
    """Rows 1.5 * 2^30 elements apart: the last one begins past 2^31."""
    ld = 3 << 29
    buf = torch.empty(2 * ld + V, dtype=TYPES[dtype], device=dev)
    x = buf.as_strided((3, V), (ld, 1))
    x.copy_(logits(3, V, dtype, 2, dev))
    for kw in (dict(), dict(top_k=50, top_p=0.9)):
        check(x, uniform(3, 3, dev), dev, **kw)


@pytest.mark.parametrize("dtype", TYPES)
def test_masked_chunks_and_a_workspace_of_any_contents(dtype, dev):
    """Chunks that are masked as a whole write no sums: what the workspace held is not read."""
    N, V = 4, 128256
    x, u = logits(N, V, dtype, 5, dev), uniform(N, 5, dev)
    x[0, 5000:] = -INF
    x[1, :100000] = -INF
    x[2, 40000:90000] = LOWEST[dtype]
    x[3] = -INF
    for kw in (dict(), dict(top_k=60), dict(top_k=60000), dict(top_k=30, top_p=0.9),
               dict(top_p=0.99, min_p=1e-3), dict(temperature=0.0)):
        want = pick_ref.sample(host(x), host(u), **kw)
        for fill in (255, 1, 0):
            ws = torch.full((osm.sample_workspace(N, V, x.dtype),), fill, dtype=torch.uint8,
                            device=dev)
            vals, idx = osm.softmax_sample(x, u, workspace=ws, **kw)
            assert np.array_equal(idx.cpu().numpy(), want[1]), (kw, fill)
            pick_ref.close(host(vals), want[0])
