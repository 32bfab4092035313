"""balance_fwd and balance_bwd against the plain binary64 implementation (loss_ref.py): numbers of
experts around every team's width, sequences of every kind of length, padding, repeated and
missing indices, rows that are no numbers, streams, graphs and threads.  And the losses of a
mixture-of-experts language model's training step together."""
import threading

import numpy as np
import pytest
import torch

import loss_ref
import paper_1805_02867_amd as osm
from test_gpu_logprob import DT, host, logits, some_tokens

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X; none is visible")
    return torch.device("cuda:0")


def places(N, E, K, seed, dev, drop=0.1):
    """Indices as a router gives them, some of them missing, some rows without any; a few twice."""
    g = torch.Generator().manual_seed(seed)
    i = torch.randint(0, E, (N, K), generator=g)
    i[torch.rand(N, K, generator=g) < drop] = -1
    i[torch.rand(N, generator=g) < drop] = -1
    i[torch.rand(N, K, generator=g) < 0.02] = E
    return i.int().to(dev)


def offsets(lengths, dev, first=0):
    return torch.tensor(np.cumsum([first] + list(lengths)), dtype=torch.int32, device=dev)


def check(x, idx, starts=None, score="softmax", scale=1.0, dtype="f32", seed=0, what=""):
    r = osm.balance_fwd(x, idx, starts, score, scale)
    at = None if starts is None else starts.cpu().numpy()
    i = idx.cpu().numpy().reshape(x.shape[0], -1)
    want = loss_ref.balance(host(x), i, at, score, scale)
    what = f"{what} {tuple(x.shape)} {score}"
    assert np.array_equal(r.counts.cpu().numpy(), want["counts"]), what
    assert np.array_equal(r.rows.cpu().numpy(), want["rows"]), what
    loss_ref.check(host(r.probs), want["probs"], want["probs_err"], what + " probs")
    loss_ref.check(host(r.loss), want["loss"], want["loss_err"], what + " loss")
    g = torch.randn(r.loss.shape, generator=torch.Generator().manual_seed(seed)).to(x.device)
    dx = osm.balance_bwd(x, idx, r.counts, r.rows, g, starts, score, scale)
    d, err = loss_ref.balance_bwd(host(x), i, want["counts"], want["rows"], host(g), at, score,
                                  scale, dtype)
    loss_ref.check(host(dx), d, err, what + " gradient")
    return r, dx


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E", [1, 2, 7, 8, 9, 32, 60, 64, 65, 128, 130, 160, 256, 384, 511, 512,
                               513, 1000, 1024])
def test_experts(E, dtype, dev):
    print(f"experts {dtype} {E}", flush=True)
    for N, K, lengths in ((1, 1, None), (37, 3, None), (500, 5, [100, 0, 1, 250, 100]),
                          (700, 64, [650])):
        x, idx = logits(N, E, dtype, E, dev), places(N, E, K, N, dev)
        starts = None if lengths is None else offsets(lengths, dev)
        for score in ("softmax", "sigmoid"):
            check(x, idx, starts, score, 0.01, dtype, E)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unaligned_batches(dtype, dev):
    for E in (64, 160, 1024):
        x, idx = logits(90, E, dtype, E, dev, offset=1), places(90, E, 4, 1, dev)
        check(x, idx, dtype=dtype)
        assert x.data_ptr() % 16 != 0


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_sequences(score, dev):
    """Of one token, of none (at the front, in between, at the end), longer than a workgroup's span
    and than many; rows in front of the first and behind the last; more sequences than rows."""
    g = torch.Generator().manual_seed(2)
    for N, E, lengths, first in (
            (40000, 64, [1, 0, 0, 20000, 7, 0, 19992, 0], 0), (40000, 64, [39999], 1),
            (30000, 16, [10000, 0, 15000], 3000), (5000, 256, [1] * 5000, 0),
            (20000, 60, torch.randint(0, 300, (130,), generator=g).tolist(), 5),
            (12000, 256, torch.randint(0, 70, (300,), generator=g).tolist(), 9),
            (9000, 8, [0] * 300 + [9000] + [0] * 300, 0), (100, 8, [0] * 70, 50),
            (66000, 32, [32768, 1, 32767, 64, 64], 300), (100, 24, [100], 0)):
        print(N, E, len(lengths), flush=True)
        assert first + sum(lengths) <= N
        x, idx = logits(N, E, "f32", E, dev, sigma=1.0), places(N, E, 2, 3, dev)
        _, dx = check(x, idx, offsets(lengths, dev, first), score)
        assert not dx[:first].any() and not dx[first + sum(lengths):].any()


@pytest.mark.parametrize("E", [8, 64, 65, 128, 130, 256, 300, 512, 513, 1024])
def test_sequences_of_many_spans(E, dev):
    """All rows as one sequence, one that begins late, two; the same every time, also with scratch
    memory that held something else."""
    N = 9000 if E <= 64 else 5000
    x, idx = logits(N, E, "bf16", E, dev), places(N, E, 3, 4, dev)
    for lengths, first in ((None, 0), ([N - 8], 8), ([N - 100], 0), ([N // 2, N // 3], N // 6)):
        starts = None if lengths is None else offsets(lengths, dev, first)
        r, _ = check(x, idx, starts, "sigmoid", dtype="bf16", what=str(lengths))
        n = osm.balance_workspace(N, E, 1 if lengths is None else len(lengths))
        for fill in (0, 255):
            ws = torch.full((n,), fill, dtype=torch.uint8, device=dev)
            again = osm.balance_fwd(x, idx, starts, "sigmoid", workspace=ws)
            assert all(torch.equal(a, b) for a, b in zip(r, again))


def test_every_place_of_a_border(dev):
    """Two sequences whose border moves over the rows of several spans."""
    N, E = 3000, 8
    x, idx = logits(N, E, "f32", 1, dev), places(N, E, 2, 1, dev)
    q, _, err = loss_ref.shares(host(x), "softmax")
    i = idx.cpu().numpy()
    took = ((i >= 0) & (i < E)).any(axis=1)
    before = np.concatenate([np.zeros((1, E)), np.cumsum(q * took[:, None], axis=0)])
    n = np.concatenate([[0], np.cumsum(took)])
    for at in list(range(0, 300)) + list(range(300, N + 1, 37)) + [N - 1, N]:
        r = osm.balance_fwd(x, idx, offsets([at, N - at], dev))
        assert r.rows.tolist() == [n[at], n[N] - n[at]], at
        P = np.stack([before[at] / max(n[at], 1), (before[N] - before[at]) / max(n[N] - n[at], 1)])
        # (every share's error is below that of the largest; the differences of the sums 2^-40)
        assert (np.abs(host(r.probs) - P) <= (err.max() + 2.0 ** -24) * P + 2.0 ** -40).all(), at


def test_offsets_outside_the_batch(dev):
    x, idx = logits(50, 12, "f32", 1, dev), places(50, 12, 2, 1, dev)
    starts = torch.tensor([-5, 10, 10, 50, 99, 1 << 30], dtype=torch.int32, device=dev)
    check(x, idx, starts)


def test_no_rows(dev):
    for S in (None, 3):
        starts = None if S is None else torch.zeros(S + 1, dtype=torch.int32, device=dev)
        x, idx = torch.zeros(0, 12, device=dev), torch.zeros(0, 2, dtype=torch.int32, device=dev)
        r = osm.balance_fwd(x, idx, starts, loss=torch.full((S or 1,), 7.0, device=dev))
        assert not r.loss.any() and not r.counts.any() and not r.probs.any() and not r.rows.any()
        assert osm.balance_bwd(x, idx, r.counts, r.rows, r.loss, starts).shape == (0, 12)
    x = logits(9, 12, "f32", 1, dev)
    none = torch.full((9, 2), -1, dtype=torch.int32, device=dev)
    r, dx = check(x, none)
    assert not dx.any() and not r.loss.any()


@pytest.mark.filterwarnings("ignore:invalid value")     # of the reference, on purpose
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_are_no_numbers(dtype, dev):
    """They spoil their sequence, and no other; rows that take no part may hold anything."""
    x, idx = logits(40, 24, dtype, 1, dev), places(40, 24, 2, 1, dev, drop=0.0)
    x[3, 5], x[25, 0] = NAN, INF
    x[12] = -INF
    x[13] = NAN
    x[31, 4] = -INF
    idx[12:14] = -1
    starts = offsets([10, 10, 10, 10], dev)
    r = osm.balance_fwd(x, idx, starts)
    assert r.loss.isnan().tolist() == [True, False, True, False]
    check(x, idx, starts, "sigmoid", dtype=dtype)
    dx = osm.balance_bwd(x, idx, r.counts, r.rows, torch.ones(4, device=dev), starts)
    assert dx[3].isnan().all() and dx[25].isnan().all() and not dx[12:14].any()
    keep = [i for i in range(40) if i not in (3, 25)]
    assert not dx[keep].isnan().any()
    clean = x.clone()
    clean[3], clean[25] = 0.0, 0.0
    check(clean, idx, starts, dtype=dtype)
    # all sigmoids next to 0, and next to 1
    for c in (-200.0, 200.0):
        y = logits(9, 24, dtype, 2, dev) + c
        check(y, places(9, 24, 2, 1, dev), None, "sigmoid", dtype=dtype)


def test_balanced_counts_keep_their_digits(dev):
    """Counts of 10^8 that differ by a few: what cancels is not in the sum."""
    N, E = 64, 16
    x, idx = logits(N, E, "f32", 1, dev, sigma=0.5), places(N, E, 2, 1, dev, drop=0.0)
    g = torch.Generator().manual_seed(1)
    counts = (10 ** 8 + torch.randint(-3, 4, (1, E), generator=g)).int()
    rows = torch.tensor([int(counts.long().sum()) // 2], dtype=torch.int32)
    dloss = torch.tensor([1e9])
    dx = osm.balance_bwd(x, idx, counts.to(dev), rows.to(dev), dloss.to(dev))
    d, err = loss_ref.balance_bwd(host(x), idx.cpu().numpy(), counts.numpy(), rows.numpy(),
                                  dloss.numpy())
    loss_ref.check(host(dx), d, err, "counts")
    assert np.abs(d).max() > 0


def test_counts_of_all_ranks(dev):
    """Two halves of a batch with counts and rows summed over them: the gradient of the whole."""
    x, idx = logits(200, 32, "f32", 1, dev), places(200, 32, 4, 1, dev)
    g = torch.ones(1, device=dev)
    whole = osm.balance_fwd(x, idx)
    want = osm.balance_bwd(x, idx, whole.counts, whole.rows, g)
    parts = [osm.balance_fwd(x[a:a + 100], idx[a:a + 100]) for a in (0, 100)]
    counts = parts[0].counts + parts[1].counts
    rows = parts[0].rows + parts[1].rows
    assert torch.equal(counts, whole.counts) and torch.equal(rows, whole.rows)
    for a in (0, 100):
        dx = osm.balance_bwd(x[a:a + 100], idx[a:a + 100], counts, rows, g)
        assert torch.equal(dx, want[a:a + 100])


def test_gradient_against_differences(dev):
    """Of the kernels' own forward pass: losses of order 1, 2^-22 each, over a step of 1/4; h^2 / 6
    times third derivatives below 1/2."""
    x, idx = logits(12, 6, "f32", 1, dev, sigma=1.0), places(12, 6, 2, 1, dev)
    starts, w = offsets([5, 7], dev), torch.tensor([1.0, -2.0], device=dev)
    for score in ("softmax", "sigmoid"):
        r = osm.balance_fwd(x, idx, starts, score)
        dx = osm.balance_bwd(x, idx, r.counts, r.rows, w, starts, score)
        for n in range(12):
            for j in range(6):
                lo, hi = x.clone(), x.clone()
                lo[n, j] -= 0.125
                hi[n, j] += 0.125
                d = osm.balance_fwd(hi, idx, starts, score).loss.double()
                d = ((d - osm.balance_fwd(lo, idx, starts, score).loss.double()) * w).sum()
                diff = float(d) / float(hi[n, j] - lo[n, j])
                assert abs(diff - float(dx[n, j])) < 3 * (0.125 ** 2 / 12 + 2.0 ** -18)


def test_refused(dev):
    x, idx = logits(8, 12, "f32", 1, dev), places(8, 12, 2, 1, dev)
    starts = offsets([4, 4], dev)
    r = osm.balance_fwd(x, idx, starts)
    g = torch.ones(2, device=dev)
    for call in (lambda: osm.balance_fwd(x, idx.long()), lambda: osm.balance_fwd(x, idx[:7]),
                 lambda: osm.balance_fwd(x.t(), idx),
                 lambda: osm.balance_fwd(x, idx, starts.long()),
                 lambda: osm.balance_fwd(x, idx, starts[:1]),
                 lambda: osm.balance_fwd(x, idx, score="tanh"),
                 lambda: osm.balance_fwd(x, idx, score=1 << 32),
                 lambda: osm.balance_fwd(x, idx, loss=torch.empty(2, device=dev)),
                 lambda: osm.balance_bwd(x, idx, r.counts, r.rows, g),
                 lambda: osm.balance_bwd(x, idx, r.counts, r.rows, g.half(), starts),
                 lambda: osm.balance_bwd(x, idx, r.counts, r.rows, g, starts, dx=x.half())):
        with pytest.raises(ValueError):
            call()
    wide = torch.zeros(2, 1025, device=dev)
    for call in (lambda: osm.balance_fwd(wide, idx[:2]), lambda: osm.balance_fwd(x, idx, score=7),
                 lambda: osm.balance_bwd(x, idx, r.counts, r.rows, g, starts, dx=x)):
        with pytest.raises(osm.OsmError) as e:
            call()
        assert e.value.status == osm.EINVAL
    x, idx, starts = logits(9000, 12, "f32", 1, dev), places(9000, 12, 2, 1, dev), None
    r = osm.balance_fwd(x, idx)
    n = osm.balance_workspace(9000, 12)
    assert n > 0
    ws = torch.full((n,), 255, dtype=torch.uint8, device=dev)
    assert torch.equal(osm.balance_fwd(x, idx, starts, workspace=ws).loss, r.loss)
    with pytest.raises(osm.OsmError) as e:
        osm.balance_fwd(x, idx, starts, workspace=ws[:n - 1])
    assert e.value.status == osm.ESCRATCH


def test_threads_graphs_and_streams(dev):
    """Threads on one stream and on their own; two graphs with memory of their own at once."""
    data, want = [], []
    for i, (N, E, S) in enumerate([(30000, 64, 3), (50, 8, 1), (9000, 256, 40), (20000, 160, 1)]):
        x, idx = logits(N, E, "bf16", i, dev), places(N, E, 4, i, dev)
        starts = offsets([N // S] * S, dev)
        data.append((x, idx, starts))
        want.append(osm.balance_fwd(x, idx, starts))
    torch.cuda.synchronize()
    shared, bad = torch.cuda.Stream(), []

    def work(i, stream):
        with torch.cuda.stream(stream):
            for _ in range(10):
                got = osm.balance_fwd(*data[i])
        stream.synchronize()
        bad.extend(i for a, b in zip(got, want[i]) if not torch.equal(a, b))
    for streams in ([shared] * 4, [torch.cuda.Stream() for _ in range(4)]):
        threads = [threading.Thread(target=work, args=(i, s)) for i, s in enumerate(streams)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not bad
        for s in set(streams):
            osm.stream_release(s)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for graph, s, d in zip(graphs, streams, (data[0], data[2])):
        with torch.cuda.graph(graph, stream=s):
            r = osm.balance_fwd(*d)
            dx = osm.balance_bwd(d[0], d[1], r.counts, r.rows, r.loss, d[2])
        outs.append(tuple(r) + (dx,))
    for rep in range(4):
        for i, (x, idx, starts) in enumerate((data[0], data[2])):
            x.copy_(logits(*x.shape, "bf16", 20 + 2 * rep + i, dev))
            idx.copy_(places(*idx.shape[:1], x.shape[1], 4, rep, dev))
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for (x, idx, starts), out in zip((data[0], data[2]), outs):
            r = osm.balance_fwd(x, idx, starts)
            dx = osm.balance_bwd(x, idx, r.counts, r.rows, r.loss, starts)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, tuple(r) + (dx,))), f"replay {rep}"


def test_training_step(dev):
    """A mixture-of-experts language model's losses: route the tokens, balance them by sequence,
    project to the vocabulary, cross entropy with an entropy bonus; the gradients down to both
    matrices against autograd in binary64, eagerly and replayed from a graph."""
    N, H, E, V, K = 45, 64, 24, 5003, 4
    g = torch.Generator().manual_seed(3)
    h = torch.randn(N, H, generator=g).to(torch.bfloat16).to(dev)
    wr = (torch.randn(E, H, generator=g) / 8).to(torch.bfloat16).to(dev)
    wv = (torch.randn(V, H, generator=g) / 4).to(torch.bfloat16).to(dev)
    tokens = some_tokens(N, V, 1, 1, dev)
    starts = offsets([20, 5, 17], dev)
    weight = -torch.ones(N, 1, device=dev) / N
    bonus = torch.full((N,), -0.01 / N, device=dev)
    each = torch.full((3,), 1.0 / 3, device=dev)

    def step():
        router = osm.proj(h, wr)
        _, idx = osm.route_fwd(router, K)
        bal = osm.balance_fwd(router, idx, starts, scale=0.1)
        drouter = osm.balance_bwd(router, idx, bal.counts, bal.rows, each, starts, scale=0.1)
        x = osm.proj(h, wv)
        r = osm.logprob_fwd(x, tokens, entropy=True, stats=True)
        dx = osm.logprob_bwd(x, r.stats, tokens, weight, r.entropy, bonus)
        return router, idx, bal.loss, drouter, x, r.logp, r.entropy, dx

    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        out = step()
    for rep in range(3):
        h.copy_(torch.randn(N, H, generator=g).to(torch.bfloat16))
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager)), f"replay {rep}"
        router, idx, loss, drouter, x, logp, entropy, dx = eager
        xr = router.double().cpu().requires_grad_()
        xv = x.double().cpu().requires_grad_()
        q = torch.softmax(xr, 1)
        i, total = idx.long().cpu(), 0.0
        for a, b in ((0, 20), (20, 25), (25, 42)):
            f = torch.bincount(i[a:b].reshape(-1), minlength=E).double() * E / (K * (b - a))
            total = total + 0.1 * (f * q[a:b].mean(0)).sum() / 3
        lp = torch.log_softmax(xv, 1)
        t = tokens.long().cpu()
        ok = (t >= 0) & (t < V)
        lt = torch.where(ok, torch.gather(lp, 1, t.clamp(0, V - 1)), torch.zeros(N, 1).double())
        H64 = -(lp.exp() * lp).sum(1)
        total = total + (lt * weight.double().cpu()).sum() + (H64 * bonus.double().cpu()).sum()
        total.backward()
        mine = float(loss.double().sum() / 3 + (logp.double() * weight.double()).sum() +
                     (entropy.double() * bonus.double()).sum())
        assert abs(mine - total.item()) < 1e-5 * abs(total.item())     # 160 roundings of 2^-24
        for d, want, ref in ((drouter, xr.grad, h), (dx, xv.grad, h)):
            # an element's error is below 300 roundings of its row's largest, or of g
            lim = 300 * 2.0 ** -24 * want.abs().max()
            assert (d.double().cpu() - want).abs().max() <= lim
            dw = d.double().t().contiguous() @ ref.double()
            w64 = want.t().contiguous() @ ref.double().cpu()
            assert (dw.cpu() - w64).abs().max() <= lim * N * ref.double().abs().max().item()
