"""logprob_fwd and logprob_bwd against the plain binary64 implementation (loss_ref.py): every
kernel shape and its borders, types, strides, masks, ties, ignored and repeated tokens, rows that
are no numbers, streams, graphs and threads."""
import threading

import numpy as np
import pytest
import torch

import loss_ref
import paper_1805_02867_amd as osm

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X; none is visible")
    return torch.device("cuda:0")


def host(t):
    return t.detach().double().cpu().numpy()


def logits(N, V, dtype, seed, dev, ld=0, offset=0, sigma=2.0):
    """N x V logits in rows of ld elements, the first at an offset from an aligned place."""
    ld = ld or V
    g = torch.Generator().manual_seed(seed)
    buf = torch.randn(N * ld + offset, generator=g) * sigma
    return buf.to(DT[dtype]).to(dev)[offset:].view(N, ld)[:, :V]


def some_tokens(N, V, T, seed, dev):
    """Tokens of all kinds: among them ignored ones, repeated ones, the first and the last."""
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, V, (N, T), generator=g)
    t[torch.rand(N, T, generator=g) < 0.15] = -100
    t[:, 0] = torch.tensor([0, V - 1, V, -1])[torch.arange(N) % 4]
    if T > 2:
        t[:, 2] = t[:, 1]
    return t.int().to(dev)


def check_fwd(x, tokens, K=0, temperature=1.0, what="", **kw):
    """All outputs of a call, and the same from calls that ask for one thing only."""
    got = osm.logprob_fwd(x, tokens, K=K, entropy=True, stats=True, temperature=temperature, **kw)
    t = None if tokens is None else tokens.cpu().numpy().reshape(x.shape[0], -1)
    want = loss_ref.logprob(host(x), t, K, temperature)
    what = f"{what} {tuple(x.shape)} K={K}"
    if tokens is not None:
        loss_ref.check(host(got.logp).reshape(want["logp"].shape), want["logp"], want["logp_err"],
                       what + " logp")
    loss_ref.check(host(got.entropy), want["entropy"], want["entropy_err"], what + " entropy")
    loss_ref.check(host(got.stats), want["stats"], want["stats_err"], what + " stats")
    if K:
        assert np.array_equal(got.top_idx.cpu().numpy(), want["top_idx"]), what
        loss_ref.check(host(got.top_vals), want["top_vals"], want["top_vals_err"], what + " top")
    return got


def check_bwd(x, tokens, dlogp, dentropy=None, temperature=1.0, dtype="f32", dx=None, what=""):
    r = osm.logprob_fwd(x, entropy=True, stats=True, temperature=temperature)
    got = osm.logprob_bwd(x, r.stats, tokens, dlogp, r.entropy if dentropy is not None else None,
                          dentropy, temperature=temperature, dx=dx)
    N = x.shape[0]
    t = None if tokens is None else tokens.cpu().numpy().reshape(N, -1)
    g = None if dlogp is None else host(dlogp).reshape(N, -1)
    want, err = loss_ref.logprob_bwd(host(x), t, g,
                                     None if dentropy is None else host(dentropy), temperature,
                                     dtype)
    loss_ref.check(host(got), want, err, f"{what} {tuple(x.shape)}")
    return got


# lengths around a vector, a wavefront's, a workgroup's and a chunk's share
LENGTHS = [1, 2, 3, 5, 8, 9, 31, 64, 255, 257, 1000, 1023, 2049, 4096, 4097, 8191, 8200, 16385,
           32768, 32771, 65537, 70001, 131075]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", LENGTHS)
def test_rows(V, dtype, dev):
    N = 5
    print(f"rows {dtype} {V}", flush=True)
    for ld, offset, T, K, tau in ((V, 0, 1, 0, 1.0), (V + 3, 1, 3, min(V, 5), 0.7),
                                  (V + 8, 2, 64, min(V, 64), 1.3)):
        x = logits(N, V, dtype, V + T, dev, ld, offset)
        check_fwd(x, some_tokens(N, V, T, V, dev), K, tau, f"{dtype} ld {ld} offset {offset}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(1, 128256), (1, 1000003), (2, 300007), (700, 1500), (1500, 4000),
                                 (3000, 300), (600, 9000), (260, 33000), (1030, 20)])
def test_batches(N, V, dtype, dev):
    """Batches that take the other plans: one long row, many short ones, more than the chip."""
    print(f"batch {dtype} {N} {V}", flush=True)
    x = logits(N, V, dtype, N, dev)
    tok = some_tokens(N, V, 2, V, dev)
    for K in (0, min(V, 20)):
        got = osm.logprob_fwd(x, tok, K=K, entropy=True, stats=True)
        rows = sorted(set(range(min(N, 6))) | {N // 2, N - 1})
        at = torch.tensor(rows, device=dev)
        want = loss_ref.logprob(host(x[at]), tok[at].cpu().numpy(), K)
        for name in ("logp", "entropy", "stats") + (("top_vals",) if K else ()):
            loss_ref.check(host(getattr(got, name)[at]), want[name], want[name + "_err"], name)
        if K:
            assert np.array_equal(got.top_idx[at].cpu().numpy(), want["top_idx"])
        again = osm.logprob_fwd(x, tok, K=K, entropy=True, stats=True)
        assert all(torch.equal(a, b) for a, b in zip(got, again) if a is not None)


@pytest.mark.filterwarnings("ignore:invalid value")     # of the reference, on purpose
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,nv,offset", [(16, 2049, 0), (16, 3001, 1), (16, 20011, 0),
                                         (16, 33000, 3), (400, 2500, 0), (300, 8200, 1)])
def test_long_rows_of_every_kind(N, nv, offset, dtype, dev):
    """Rows that do not fit into registers, whole and in chunks, by nv 16-byte vectors: masked ones,
    ties, sure tokens, logits far from 0, rows that are no numbers; and their gradients."""
    V = nv * (4 if dtype == "f32" else 8) - 2
    print(f"long rows {dtype} {N} {V}", flush=True)
    x = logits(16, V, "f32", V, dev)
    at = torch.randint(0, V, (16,), generator=torch.Generator().manual_seed(nv)).to(dev)
    x[0] = -INF
    x[1] = -INF
    x[1, at[1]] = -3.0
    x[2, : at[2]] = -INF
    x[3, torch.arange(V, device=dev) % 97 != 5] = -INF
    x[4] = torch.finfo(DT[dtype]).min / 4
    x[4, at[4]] = 0.0
    x[5, at[5]] = NAN
    x[6, at[6]] = INF
    x[7] = 1.5
    x[8, ::3] = 9.0
    for r, up in ((9, 20.0), (10, 45.0)):
        x[r, at[r]] = x[r].max() + up
    x[11] += 1e4
    x[12] = x[12] * 1e5 - 1e7
    x[13, V - 1] = 12.0
    x[14, 0] = 12.0
    tok = some_tokens(16, V, 3, V, dev)
    tok[:, 1] = at.int()
    ld = V + (3 if offset else 2)
    rows = torch.arange(N, device=dev) % 16
    each = rows.cpu().numpy()
    buf = torch.zeros(N * ld + offset, dtype=DT[dtype], device=dev)
    y = buf[offset:].view(N, ld)[:, :V]
    y.copy_(x[rows])
    got = osm.logprob_fwd(y, tok[rows], entropy=True, stats=True, temperature=0.8)
    first = y[:16].contiguous()
    want = loss_ref.logprob(host(first), tok.cpu().numpy(), 0, 0.8)
    for name in ("logp", "entropy", "stats"):
        loss_ref.check(host(getattr(got, name)), want[name][each], want[name + "_err"][each], name)
    only = osm.logprob_fwd(y, tok[rows], temperature=0.8)
    loss_ref.check(host(only.logp), want["logp"][each], want["logp_err"][each], "logp alone")
    g = torch.Generator().manual_seed(nv)
    dlogp, dent = torch.randn(16, 3, generator=g).to(dev), torch.randn(16, generator=g).to(dev)
    dx = osm.logprob_bwd(y, got.stats, tok[rows], dlogp[rows], got.entropy, dent[rows],
                         temperature=0.8)
    d, err = loss_ref.logprob_bwd(host(first), tok.cpu().numpy(), host(dlogp), host(dent), 0.8,
                                  dtype)
    loss_ref.check(host(dx), d[each], err[each], "gradient")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,nv", [(12, 1900), (12, 2100), (12, 8190), (12, 8300), (300, 2500)])
def test_alternatives_of_long_rows(N, nv, dtype, dev):
    """With alternatives rows are held: by four wavefronts, by eight, in chunks."""
    V = nv * (4 if dtype == "f32" else 8) - 1
    print(f"alternatives {dtype} {N} {V}", flush=True)
    x = logits(N, V, dtype, V, dev)
    x[1, : V // 2] = -INF
    x[2] = 1.5
    x[3] = -INF
    x[3, V - 1] = 2.0
    x[4, ::5] = 9.0
    for K in (5, 40):
        check_fwd(x, some_tokens(N, V, 3, V, dev), K, what=dtype)


@pytest.mark.filterwarnings("ignore:invalid value")     # of the reference, on purpose
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 15, 16, 17, 33, 64, 67, 100, 127, 130, 255, 256, 263,
                               500, 520, 777, 1000, 1024, 1030, 2047, 2055, 2060])
def test_short_rows_of_every_kind(V, dtype, dev):
    """Batches of several rows a wavefront, the last of them not full: masked rows, ties, sure
    tokens, logits far from 0, rows that are no numbers, beside each other; up to 64 tokens."""
    print(f"short rows {dtype} {V}", flush=True)
    M, N = 18, 269
    x = logits(M, V, "f32", V, dev)
    g = torch.Generator().manual_seed(V)
    at = torch.randint(0, V, (M,), generator=g).to(dev)
    x[0] = -INF
    x[1] = -INF
    x[1, at[1]] = -3.0
    x[2, : at[2]] = -INF
    x[3] = torch.finfo(DT[dtype]).min / 4
    x[4] = torch.finfo(DT[dtype]).min / 4
    x[4, at[4]] = 0.0
    x[5, at[5]] = NAN
    x[6, at[6]] = INF
    x[7] = 1.5
    x[8, ::3] = 9.0
    for r, up in ((9, 20.0), (10, 45.0), (11, 70.0)):
        x[r, at[r]] = x[r].max() + up
    x[12] += 1e4
    x[13] = x[13] * 1e5 - 1e7
    x[14, V - 1] = 12.0
    x[15, 0] = 12.0
    x[16] = -x[16].abs() - 50.0
    rows = torch.arange(N, device=dev) % M
    each = rows.cpu().numpy()
    for ld, offset, T, tau in ((V, 0, 3, 1.0), (V + 3, 1, 64, 0.8)):
        buf = torch.zeros(N * ld + offset, dtype=DT[dtype], device=dev)
        y = buf[offset:].view(N, ld)[:, :V]
        y.copy_(x[rows])
        tok = some_tokens(M, V, T, V, dev)
        tok[:, 1] = at.int()
        want = loss_ref.logprob(host(y[:M].contiguous()), tok.cpu().numpy(), 0, tau)
        got = osm.logprob_fwd(y, tok[rows], entropy=True, stats=True, temperature=tau)
        for name in ("logp", "entropy", "stats"):
            loss_ref.check(host(getattr(got, name)), want[name][each], want[name + "_err"][each],
                           name)
        only = osm.logprob_fwd(y, tok[rows], stats=True, temperature=tau)
        loss_ref.check(host(only.logp), want["logp"][each], want["logp_err"][each], "logp alone")
        assert torch.equal(only.stats.nan_to_num(7.0), got.stats.nan_to_num(7.0))


@pytest.mark.filterwarnings("ignore:invalid value")     # of the reference, on purpose
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,nv,offset", [(400, 4200, 1), (256, 8300, 0), (270, 16500, 3)])
def test_alternatives_of_large_batches(N, nv, offset, dtype, dev):
    """Streamed rows and chunks with up to 32 alternatives: rows that rise and fall, of few values,
    masked ones with the rest at the front, at the end and anywhere, no numbers."""
    V = nv * (4 if dtype == "f32" else 8) - 3
    print(f"alternatives {dtype} {N} {V}", flush=True)
    x = logits(16, V, "f32", V, dev)
    at = torch.randint(0, V, (16,), generator=torch.Generator().manual_seed(nv)).to(dev)
    x[0] = -INF
    x[1] = -INF
    x[1, at[1]] = -3.0
    x[2, 20:] = -INF
    x[3, :-20] = -INF
    x[4, torch.arange(V, device=dev) % 997 != 5] = -INF
    x[5] = x[5].sort().values
    x[6] = x[6].sort(descending=True).values
    x[7] = x[7].round()
    x[8] = -1.25
    x[9, V // 2:] = 9.0
    x[10] = torch.arange(V, device=dev) // 5000
    x[11, at[11]] = NAN
    x[12] = x[12] - 50.0
    x[13, -1], x[13, 0], x[13, 1] = 20.0, 20.0, 21.0
    x[14] = x[14].sort().values.view(-1, 1)[:, 0].round()
    rows = torch.arange(N, device=dev) % 16
    each = rows.cpu().numpy()
    ld = V + (3 if offset else 0)
    buf = torch.zeros(N * ld + offset, dtype=DT[dtype], device=dev)
    y = buf[offset:].view(N, ld)[:, :V]
    y.copy_(x[rows])
    tok = some_tokens(16, V, 2, V, dev)
    for K in (1, 6, 32):
        got = osm.logprob_fwd(y, tok[rows], K=K, entropy=True, stats=True)
        want = loss_ref.logprob(host(y[:16].contiguous()), tok.cpu().numpy(), K)
        assert np.array_equal(got.top_idx.cpu().numpy(), want["top_idx"][each]), K
        for name in ("logp", "entropy", "stats", "top_vals"):
            loss_ref.check(host(getattr(got, name)), want[name][each], want[name + "_err"][each],
                           f"{name} K={K}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [7, 1000, 40000, 300001])
def test_masked_rows(V, dtype, dev):
    """-inf almost everywhere, everywhere but in one place, everywhere; fewer elements left than
    alternatives; the type's lowest value."""
    low = torch.finfo(DT[dtype]).min
    x = logits(7, V, dtype, V, dev)
    g = torch.Generator().manual_seed(V)
    few = (torch.rand(V, generator=g) < max(0.01, 2 / V)).to(dev)
    x[0, ~few] = -INF
    x[1] = -INF
    x[1, V - 1] = -3.0
    x[2] = -INF
    x[3, : V // 2] = -INF
    x[4, 1:] = low / 4
    x[5] = low / 4
    x[6, :] = -INF
    x[6, V // 2] = 5.0
    for K in (0, 1, min(V, 6), min(V, 64)):
        check_fwd(x, some_tokens(7, V, 3, V, dev), K, what=dtype)
    tok = some_tokens(7, V, 3, V, dev)
    check_bwd(x, tok, torch.randn(7, 3, device=dev), torch.randn(7, device=dev), dtype=dtype)
    check_bwd(x, tok, torch.randn(7, 3, device=dev), dtype=dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [5, 1200, 50001])
def test_rows_that_are_no_numbers(V, dtype, dev):
    x = logits(6, V, dtype, V, dev)
    for r, (j, v) in enumerate([(0, NAN), (V - 1, NAN), (V // 2, INF), (0, INF)]):
        x[r, j] = v
    x[4, 0], x[4, 1] = NAN, INF
    tok = some_tokens(6, V, 2, V, dev)
    got = check_fwd(x, tok, min(V, 5), what=dtype)
    assert (got.top_idx[:5] == -1).all() and (got.top_idx[5] >= 0).all()
    # a gradient that is not 0 is not a number there; where none comes in it is 0
    g = torch.ones(6, 2, device=dev)
    check_bwd(x, tok, g, dtype=dtype)
    dx = check_bwd(x, tok, torch.zeros_like(g), torch.zeros(6, device=dev), dtype=dtype)
    assert not dx.any()
    ignored = torch.full_like(tok, -100)
    assert not check_bwd(x, ignored, g, dtype=dtype).any()
    g[5, 0] = NAN
    tok[5] = 1
    assert check_bwd(x, tok, g, dtype=dtype)[5].isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 3000, 66000])
def test_ties(V, dtype, dev):
    """Equal elements everywhere, at the top, at the line; -0.0 and 0.0; by index."""
    x = logits(5, V, dtype, V, dev)
    x[0] = 1.5
    x[1, ::3] = 9.0
    x[2] = (x[2] * 2).round() / 2
    x[3] = 0.0
    x[3, ::2] = -0.0
    x[4, V // 2:] = x[4].max()
    for K in (1, 5, min(V, 64)):
        check_fwd(x, some_tokens(5, V, 3, V, dev), K, what=dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [90, 700, 2500, 4877, 9001, 20005, 70001])
def test_negative_zeros_beside_the_largest(V, dtype, dev):
    """-0.0 at the row's ends, which is not above what the same lanes have of its vectors."""
    for N, ld in ((48, V + 5), (300, V)):
        x = logits(N, V, dtype, V, dev, ld, 1).round()
        x[:, :9], x[:, -9:] = -0.0, -0.0
        g = torch.Generator().manual_seed(V)
        step = torch.tensor([0, 512, 1024, 2048, 4096])[torch.randint(0, 5, (N,), generator=g)]
        at = (step + torch.randint(9, 120, (N,), generator=g)) % (V - 18) + 9
        x[torch.arange(N), at] = 11.0
        got = osm.logprob_fwd(x, entropy=True, stats=True)
        assert (got.stats[:, 0] == 11.0).all()
        only = osm.logprob_fwd(x, stats=True)
        assert torch.equal(only.stats, got.stats)
        want = loss_ref.logprob(host(x[:48].contiguous()), None)
        for name in ("entropy", "stats"):
            loss_ref.check(host(getattr(got, name)[:48]), want[name], want[name + "_err"], name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [10, 700, 33333, 140000])
def test_sure_rows_keep_their_digits(V, dtype, dev):
    """A token with almost all the weight: its log p, and 1 - p in its gradient, are numbers of
    1e-3 to 1e-30 with the type's precision."""
    x = logits(8, V, dtype, V, dev, sigma=1.0).float()
    at = torch.tensor([0, 1, V - 1, V // 2, V // 3, 7, 8, 9], device=dev) % V
    up = torch.tensor([5.0, 10.0, 16.0, 20.0, 30.0, 40.0, 60.0, 70.0], device=dev)
    x.scatter_(1, at.unsqueeze(1), (x.amax(dim=1) + up).unsqueeze(1))
    x = x.to(DT[dtype])
    tok = at.int().unsqueeze(1).contiguous()
    got = check_fwd(x, tok, 2, what=dtype)
    assert (got.logp < 0).all()
    dx = check_bwd(x, tok, torch.ones(8, 1, device=dev), dtype=dtype)
    assert (torch.gather(dx, 1, at.unsqueeze(1)) > 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_far_from_zero(dtype, dev):
    """A constant added; magnitudes at which steps of the type are large; the largest numbers."""
    x = logits(6, 9001, dtype, 3, dev)
    for r, c in enumerate((1e2, -1e3, 1e4, 1e6)):
        x[r] += c
    x[4] = x[4] * 1e5
    x[5] = x[5].sign() * 1e37
    tok = some_tokens(6, 9001, 2, 1, dev)
    for tau in (1.0, 0.5, 30.0):
        check_fwd(x, tok, 4, tau, what=dtype)
        check_bwd(x, tok, torch.randn(6, 2, device=dev), torch.randn(6, device=dev), tau, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", LENGTHS)
def test_gradients(V, dtype, dev):
    print(f"gradients {dtype} {V}", flush=True)
    N = 5
    g = torch.Generator().manual_seed(V)
    for ld, ldd, off, T, tau in ((V, V, 0, 1, 1.0), (V + 3, V, 1, 3, 0.7),
                                 (V + 8, V + 5, 2, 64, 1.0)):
        x = logits(N, V, dtype, V + T, dev, ld, off)
        tok = some_tokens(N, V, T, V, dev)
        dlogp = torch.randn(N, T, generator=g).to(dev)
        dent = torch.randn(N, generator=g).to(dev)
        buf = torch.full((N * ldd + 3,), 7.0, dtype=DT[dtype], device=dev)
        rows = buf[3:].view(N, ldd)
        what = f"{dtype} ld {ld} {ldd}"
        dx = check_bwd(x, tok, dlogp, None, tau, dtype, what=what)
        assert torch.equal(check_bwd(x, tok, dlogp, None, tau, dtype, rows[:, :V], what), dx)
        assert (rows[:, V:] == 7.0).all() and (buf[:3] == 7.0).all()
        check_bwd(x, tok, dlogp, dent, tau, dtype, what=what)
        check_bwd(x, None, None, dent, tau, dtype, what=what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(1, 128256), (3000, 300), (1030, 20), (300, 5000), (5000, 1)])
def test_gradients_of_batches(N, V, dtype, dev):
    x = logits(N, V, dtype, N, dev)
    tok = some_tokens(N, V, 2, V, dev)
    dlogp = torch.randn(N, 2, device=dev)
    r = osm.logprob_fwd(x, stats=True)
    dx = osm.logprob_bwd(x, r.stats, tok, dlogp)
    rows = sorted(set(range(min(N, 6))) | {N // 2, N - 1})
    at = torch.tensor(rows, device=dev)
    want, err = loss_ref.logprob_bwd(host(x[at]), tok[at].cpu().numpy(), host(dlogp[at]),
                                     dtype=dtype)
    loss_ref.check(host(dx[at]), want, err, f"{N} {V}")
    assert torch.equal(dx, osm.logprob_bwd(x, r.stats, tok, dlogp))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 7, 16, 33, 255, 256, 257, 264, 511, 512, 520])
def test_gradients_of_short_rows(V, dtype, dev):
    """Several rows a wavefront, with up to sixteen tokens and more, rows without any, without
    gradients and with no numbers beside others; a batch that does not fill the last wavefront."""
    for N, T in ((1, 1), (37, 16), (37, 17), (18, 64), (70, 3)):
        x = logits(N, V, dtype, V + T, dev, V + 3, 1)
        tok = some_tokens(N, V, T, V, dev)
        dlogp, dent = torch.randn(N, T, device=dev), torch.randn(N, device=dev)
        if N > 9:
            tok[2] = -100
            dlogp[3], dent[3] = 0.0, 0.0
            x[4] = -INF
            x[5, V // 2] = NAN
            x[6], dlogp[6], dent[6] = NAN, 0.0, 0.0
            x[7, : V - 1] = -INF
            x[8, V // 2] += 30.0
            dlogp[9, 0] = NAN
            tok[9, 0] = 0
        for h in (dent, None):
            check_bwd(x, tok, dlogp, h, 0.9, dtype, what=f"{T} tokens")


def test_gradient_against_differences(dev):
    """Of the kernels' own forward pass: a step of 1/8 in binary32, differences of sums of 12
    outputs of order 10 (2^-20 each), and h^2 / 6 times third derivatives below 2."""
    x = logits(3, 11, "f32", 1, dev, sigma=1.0)
    tok = some_tokens(3, 11, 4, 2, dev)
    g, h = torch.randn(3, 4, device=dev), torch.randn(3, device=dev)
    r = osm.logprob_fwd(x, tok, entropy=True, stats=True)
    dx = osm.logprob_bwd(x, r.stats, tok, g, r.entropy, h)

    def value(x):
        r = osm.logprob_fwd(x, tok, entropy=True)
        return float((r.logp.double() * g.double()).sum() + (r.entropy.double() * h.double()).sum())
    size = float(g.abs().sum() + h.abs().sum())
    for n in range(3):
        for j in range(11):
            lo, hi = x.clone(), x.clone()
            lo[n, j] -= 0.125
            hi[n, j] += 0.125
            step = float(hi[n, j] - lo[n, j])
            diff = (value(hi) - value(lo)) / step
            assert abs(diff - float(dx[n, j])) < size * (0.125 ** 2 / 3 + 2.0 ** -16)


def test_what_is_asked_for(dev):
    """Outputs do not depend on which others are asked for; given tensors are written; shapes."""
    for V in (100, 50000):
        x, tok = logits(4, V, "f32", 1, dev), some_tokens(4, V, 1, 1, dev)
        full = check_fwd(x, tok, 5)
        assert full.logp.shape == (4, 1) and full.top_idx.shape == (4, 5)
        flat = osm.logprob_fwd(x, tok.view(4))
        assert flat.logp.shape == (4,) and flat.entropy is None and flat.top_idx is None
        assert torch.equal(flat.logp, full.logp.view(4))
        assert torch.equal(osm.logprob_fwd(x, entropy=True).entropy, full.entropy)
        assert torch.equal(osm.logprob_fwd(x, stats=True).stats, full.stats)
        top = osm.logprob_fwd(x, K=5)
        assert top.logp is None and torch.equal(top.top_idx, full.top_idx)
        e, s = torch.empty(4, device=dev), torch.empty(4, 2, device=dev)
        r = osm.logprob_fwd(x, tok, entropy=e, stats=s, logp=torch.empty(4, 1, device=dev))
        assert r.entropy is e and torch.equal(e, full.entropy) and torch.equal(s, full.stats)
        one = osm.logprob_fwd(x[0], tok.view(4)[:1], K=2)
        assert torch.equal(one.logp, full.logp[0]) and one.top_idx.shape == (1, 2)


def test_empty_and_refused(dev):
    x = logits(4, 50, "f32", 1, dev)
    tok = some_tokens(4, 50, 2, 1, dev)
    r = osm.logprob_fwd(x[:0], tok[:0], K=3, entropy=True, stats=True)
    assert r.logp.shape == (0, 2) and r.top_idx.shape == (0, 3)
    assert osm.logprob_bwd(x[:0], r.stats, tok[:0], r.logp).shape == (0, 50)
    stats, g = torch.zeros(4, 2, device=dev), torch.zeros(4, 2, device=dev)
    for call in (lambda: osm.logprob_fwd(x, tok.long()), lambda: osm.logprob_fwd(x, tok[:3]),
                 lambda: osm.logprob_fwd(x.half(), tok), lambda: osm.logprob_fwd(x.t(), tok),
                 lambda: osm.logprob_fwd(x, tok.cpu()), lambda: osm.logprob_fwd(x, logp=g),
                 lambda: osm.logprob_fwd(x, top_vals=g),
                 lambda: osm.logprob_fwd(x, tok, logp=g.half()),
                 lambda: osm.logprob_fwd(x, tok, stats=torch.zeros(4, device=dev)),
                 lambda: osm.logprob_bwd(x, stats, tok), lambda: osm.logprob_bwd(x, g[:2], tok, g),
                 lambda: osm.logprob_bwd(x, stats, tok, g, dentropy=g[:, 0].contiguous()),
                 lambda: osm.logprob_bwd(x, stats, tok, g, dx=x.to(torch.bfloat16)),
                 lambda: osm.logprob_bwd(x, stats, tok, g, dx=torch.empty(4, 49, device=dev))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: osm.logprob_fwd(x), lambda: osm.logprob_fwd(x, tok, K=51),
                 lambda: osm.logprob_fwd(x, tok, temperature=0.0),
                 lambda: osm.logprob_fwd(x, torch.zeros(4, 65, dtype=torch.int32, device=dev)),
                 lambda: osm.logprob_bwd(x, stats),
                 lambda: osm.logprob_bwd(x, stats, tok, g, dx=x)):
        with pytest.raises(osm.OsmError) as e:
            call()
        assert e.value.status == osm.EINVAL


def test_workspaces(dev):
    """A workspace of any contents, one that is too small, and one shared by calls in turn."""
    x, tok = logits(3, 200000, "f32", 1, dev), some_tokens(3, 200000, 2, 1, dev)
    want = osm.logprob_fwd(x, tok, K=7, entropy=True)
    n = osm.logprob_workspace(3, 200000, 7)
    assert n > 0
    ws = torch.full((n,), 255, dtype=torch.uint8, device=dev)
    for _ in range(3):
        got = osm.logprob_fwd(x, tok, K=7, entropy=True, workspace=ws)
        assert all(torch.equal(a, b) for a, b in zip(got, want) if a is not None)
    with pytest.raises(osm.OsmError) as e:
        osm.logprob_fwd(x, tok, K=7, workspace=ws[:n - 1])
    assert e.value.status == osm.ESCRATCH


@pytest.mark.parametrize("V", [3000, 150000])
def test_graphs_share_nothing(V, dev):
    """Two graphs of the same shapes, captured without a call before, replayed on two streams at
    once with other inputs, with eager calls between."""
    xs = [logits(4, V, "bf16", s, dev) for s in range(2)]
    toks = [some_tokens(4, V, 2, s, dev) for s in range(2)]
    g = torch.randn(4, 2, device=dev)
    outs, graphs, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for s, x, t in zip(streams, xs, toks):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            r = osm.logprob_fwd(x, t, K=9, entropy=True, stats=True)
            dx = osm.logprob_bwd(x, r.stats, t, g)
        outs.append(tuple(r) + (dx,))
        graphs.append(graph)
    for rep in range(4):
        for i, x in enumerate(xs):
            x.copy_(logits(4, V, "bf16", 10 * rep + i, dev))
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for x, t, out in zip(xs, toks, outs):
            r = osm.logprob_fwd(x, t, K=9, entropy=True, stats=True)
            want = tuple(r) + (osm.logprob_bwd(x, r.stats, t, g),)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want)), f"replay {rep}"


def test_a_captured_call_on_another_stream_brings_its_workspace(dev):
    x = logits(4, 150000, "f32", 1, dev)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ValueError):
            osm.logprob_fwd(x, K=3, stream=other)
        out = osm.logprob_fwd(x, K=3)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.top_idx, osm.logprob_fwd(x, K=3).top_idx)


def test_threads_and_streams(dev):
    """Calls from several threads, on one stream and on their own."""
    shapes = [(3, 200000, 5), (40, 70000, 0), (1, 128256, 20), (500, 900, 3)]
    want, data = [], []
    for i, (N, V, K) in enumerate(shapes):
        x, t = logits(N, V, "f32", i, dev), some_tokens(N, V, 2, i, dev)
        data.append((x, t, K))
        want.append(osm.logprob_fwd(x, t, K=K, entropy=True, stats=True))
    torch.cuda.synchronize()
    shared, bad = torch.cuda.Stream(), []

    def work(i, stream):
        x, t, K = data[i]
        with torch.cuda.stream(stream):
            for _ in range(10):
                got = osm.logprob_fwd(x, t, K=K, entropy=True, stats=True)
        stream.synchronize()
        bad.extend(i for a, b in zip(got, want[i]) if a is not None and not torch.equal(a, b))
    for streams in ([shared] * 4, [torch.cuda.Stream() for _ in range(4)]):
        threads = [threading.Thread(target=work, args=(i, s)) for i, s in enumerate(streams)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert not bad
        for s in set(streams):
            osm.stream_release(s)


def test_offsets_past_32_bits(dev):
    """The last rows of a batch of more than 2^32 bytes, and elements past 2^31."""
    N, V = 70, 33000000
    x = torch.zeros(N, V, dtype=torch.bfloat16, device=dev)
    g = torch.Generator(device=dev).manual_seed(1)
    x[N - 1] = torch.randn(V, device=dev, generator=g).to(torch.bfloat16)
    x[N - 1, V - 2] = 12.0
    tok = torch.full((N,), V - 2, dtype=torch.int32, device=dev)
    r = osm.logprob_fwd(x, tok, K=2, entropy=True, stats=True)
    last = x[N - 1].double()
    lse = torch.logsumexp(last, 0)
    assert r.top_idx[N - 1].tolist()[0] == V - 2 and r.top_idx[0].tolist() == [0, 1]
    # flat rows of V, a sum of V terms; 500 additions a lane, chunk and merge at most
    assert abs(float(r.logp[N - 1]) - float(12.0 - lse)) < 700 * 2.0 ** -24 + 20 * 2.0 ** -24
    assert abs(float(r.entropy[0]) - np.log(V)) < 700 * 2.0 ** -24 + 20 * 2.0 ** -24
    dx = osm.logprob_bwd(x, r.stats, tok, torch.ones(N, device=dev))
    p = torch.exp(last - lse)
    p[V - 2] -= 1.0
    d = (dx[N - 1].double() + p).abs()
    assert bool((d <= (2.0 ** -8 + 2.0 ** -12) * p.abs()).all())


def test_more_rows_than_a_launch_has_threads_for(dev):
    """2^26 rows and a few: 2^32 threads and more."""
    N = (1 << 26) + 5
    x = torch.zeros(N, 2, device=dev)
    at = [0, 1, (1 << 22) - 1, 1 << 22, (1 << 26) - 1, 1 << 26, N - 1]
    for i, r in enumerate(at):
        x[r, 1] = i + 1.0
    tok = torch.ones(N, dtype=torch.int32, device=dev)
    got = osm.logprob_fwd(x, tok, K=1, stats=True)
    only = osm.logprob_fwd(x, tok)
    rows = torch.tensor(at, device=dev)
    want = loss_ref.logprob(host(x[rows]), tok[rows].cpu().numpy().reshape(-1, 1), 1)
    for r in (got, only):
        loss_ref.check(host(r.logp[rows])[:, None], want["logp"], want["logp_err"], "logp")
        assert int((r.logp == r.logp[2]).sum()) == N - len(at)
    assert got.top_idx[rows].tolist() == [[1]] * len(at)
    assert int(got.top_idx.sum()) == len(at)
    dx = osm.logprob_bwd(x, got.stats, tok, torch.ones(N, device=dev))
    d, err = loss_ref.logprob_bwd(host(x[rows]), np.ones((len(at), 1), int),
                                  np.ones((len(at), 1)))
    loss_ref.check(host(dx[rows]), d, err, "gradient")
