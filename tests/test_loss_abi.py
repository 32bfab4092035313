"""logprob_fwd, logprob_bwd, balance_fwd and balance_bwd: arguments they refuse, on the host and
before anything is launched (fake, never dereferenced pointers), and the plain
implementations that the GPU tests compare with, by hand and against differences."""
import ctypes
import re

import numpy as np
import pytest
import torch

import loss_ref
import paper_1805_02867_amd as osm
from test_abi import HEADER

X, T_, L, H, S_, V_, I_, D, W = (0x10000000 * i for i in range(1, 10))
INF, NAN = float("inf"), float("nan")


def _params(tokens=T_, logp=L, entropy=H, stats=S_, top=V_, idx=I_, T=2, K=3, temperature=1.0):
    return osm.Logprob(tokens, logp, entropy, stats, top, idx, T, K, temperature)


def _fwd(x=X, ld=10, p=None, N=4, V=10, dtype=0, **kw):
    p = _params(**kw) if p is None else p
    return osm.lib().logprob_fwd(x, ld, ctypes.byref(p), N, V, dtype, None)


@pytest.mark.parametrize("bad", [
    dict(N=-1), dict(N=1 << 31), dict(V=0, ld=1), dict(V=1 << 31, ld=1 << 31), dict(ld=9),
    dict(ld=1 << 31), dict(dtype=2), dict(dtype=-1), dict(x=0), dict(tokens=0), dict(logp=0),
    dict(top=0), dict(idx=0), dict(T=-1), dict(T=65), dict(K=-1), dict(K=11),
    dict(K=65, V=100, ld=100),
    dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=INF), dict(temperature=NAN),
    dict(temperature=1e-45),
    dict(x=X + 2), dict(tokens=T_ + 1), dict(logp=L + 2), dict(entropy=H + 3), dict(stats=S_ + 1),
    dict(top=V_ + 2), dict(idx=I_ + 2), dict(T=0, K=0, entropy=0, stats=0),
    dict(logp=X + 8), dict(logp=T_ + 4), dict(entropy=L + 4), dict(stats=H + 12), dict(top=S_ + 28),
    dict(idx=V_ + 44), dict(logp=X + 4 * 45, ld=20, T=1),            # between two rows of x
])
def test_logprob_fwd_refuses(bad):
    assert _fwd(**bad) == osm.EINVAL


def test_logprob_fwd_refuses_no_params_and_bad_workspaces():
    f = osm.lib().logprob_fwd_ws
    p = _params()
    assert osm.lib().logprob_fwd(X, 10, None, 4, 10, 0, None) == osm.EINVAL
    for ws in (W + 16, X, L - 256, V_):
        assert f(X, 10, ctypes.byref(p), 4, 10, 0, ws, 1 << 12, None) == osm.EINVAL


def _bwd(x=X, ld=10, tokens=T_, stats=S_, entropy=H, dlogp=L, dentropy=V_, dx=D, ldd=10, N=4, V=10,
         T=2, dtype=0, temperature=1.0):
    return osm.lib().logprob_bwd(x, ld, tokens, stats, entropy, dlogp, dentropy, dx, ldd, N, V, T,
                                 dtype, temperature, None)


@pytest.mark.parametrize("bad", [
    dict(N=-1), dict(N=1 << 31), dict(V=0), dict(ld=9), dict(ldd=9), dict(ldd=1 << 31),
    dict(ld=1 << 31), dict(dtype=2), dict(x=0), dict(stats=0), dict(dx=0), dict(tokens=0),
    dict(dlogp=0), dict(entropy=0), dict(T=0, dentropy=0), dict(T=-1), dict(T=65),
    dict(temperature=0.0), dict(temperature=NAN), dict(temperature=-2.0), dict(temperature=1e-45),
    dict(x=X + 2), dict(dx=D + 2), dict(tokens=T_ + 2), dict(stats=S_ + 2), dict(entropy=H + 2),
    dict(dlogp=L + 2), dict(dentropy=V_ + 2), dict(dx=X), dict(dx=X + 4 * 45, ld=20),
    dict(dx=T_), dict(dx=S_ - 4), dict(dx=H), dict(dx=L), dict(dx=V_),
])
def test_logprob_bwd_refuses(bad):
    assert _bwd(**bad) == osm.EINVAL


def _bal(x=X, idx=I_, starts=T_, loss=L, counts=H, probs=V_, rows=S_, N=4, E=10, K=2, S=3, dtype=0,
         score=0, scale=1.0):
    return osm.lib().balance_fwd(x, idx, starts, loss, counts, probs, rows, N, E, K, S, dtype,
                                 score, scale, None)


def _bal_bwd(x=X, idx=I_, starts=T_, counts=H, rows=S_, dloss=L, dx=D, N=4, E=10, K=2, S=3, dtype=0,
             score=0, scale=1.0):
    return osm.lib().balance_bwd(x, idx, starts, counts, rows, dloss, dx, N, E, K, S, dtype, score,
                                 scale, None)


SIZES = [dict(N=-1), dict(N=1 << 31), dict(N=1 << 30, K=2), dict(E=0), dict(E=1025), dict(K=0),
         dict(K=65), dict(S=0), dict(S=-1), dict(S=1 << 31), dict(S=(1 << 31) // 10 + 1),
         dict(starts=0), dict(dtype=2), dict(score=2), dict(score=-1), dict(x=0), dict(idx=0),
         dict(x=X + 2), dict(idx=I_ + 2), dict(starts=T_ + 1)]


@pytest.mark.parametrize("bad", SIZES + [
    dict(loss=0), dict(counts=0), dict(probs=0), dict(rows=0), dict(loss=L + 2),
    dict(counts=H + 1), dict(probs=V_ + 2), dict(rows=S_ + 3), dict(loss=X + 8), dict(counts=I_),
    dict(probs=T_ + 12), dict(rows=L + 8), dict(probs=H + 116), dict(N=0, loss=0),
])
def test_balance_fwd_refuses(bad):
    assert _bal(**bad) == osm.EINVAL


@pytest.mark.parametrize("bad", SIZES + [
    dict(counts=0), dict(rows=0), dict(dloss=0), dict(dx=0), dict(counts=H + 2), dict(rows=S_ + 2),
    dict(dloss=L + 2), dict(dx=D + 2), dict(dx=X), dict(dx=I_), dict(dx=T_), dict(dx=H),
    dict(dx=S_), dict(dx=L),
])
def test_balance_bwd_refuses(bad):
    assert _bal_bwd(**bad) == osm.EINVAL


def test_balance_refuses_bad_workspaces():
    for ws in (W + 128, X, H):
        assert osm.lib().balance_fwd_ws(X, I_, T_, L, H, V_, S_, 4, 10, 2, 3, 0, 0, 1.0, ws,
                                        1 << 20, None) == osm.EINVAL


def test_empty_batches_are_noops():
    assert _fwd(N=0, x=0, tokens=0, logp=0, entropy=0, stats=0, top=0, idx=0) == osm.OK
    assert _bwd(N=0, x=0, tokens=0, stats=0, entropy=0, dlogp=0, dentropy=0, dx=0) == osm.OK
    assert _bal_bwd(N=0, x=0, idx=0, counts=0, rows=0, dloss=0, dx=0) == osm.OK
    assert _fwd(N=0, temperature=0.0) == osm.EINVAL


def test_workspace_sizes():
    n = ctypes.c_size_t()
    size = osm.lib().osm_logprob_workspace
    assert size(4, 0, 0, 0, ctypes.byref(n)) == osm.EINVAL
    assert size(4, 10, 11, 0, ctypes.byref(n)) == osm.EINVAL
    assert size(4, 100, 65, 0, ctypes.byref(n)) == osm.EINVAL
    assert size(4, 100, -1, 0, ctypes.byref(n)) == osm.EINVAL
    assert size(4, 10, 0, 3, ctypes.byref(n)) == osm.EINVAL
    assert size(4, 10, 0, 0, None) == osm.EINVAL
    assert osm.logprob_workspace(0, 128256) == 0 and osm.logprob_workspace(4000, 1000, 5) == 0
    # at most 2^16 chunks a launch: 16 bytes and the keys each; 4 a row
    assert osm.logprob_workspace(5000, 128256) == 0
    for N in (1, 64, 5000, 1 << 20):
        for K in (0, 64) if N < 100 else (64,):
            assert 0 < osm.logprob_workspace(N, 128256, K) <= (1 << 16) * (16 + 8 * K + 4) + 256
    size = osm.lib().osm_balance_workspace
    assert size(4, 0, 1, ctypes.byref(n)) == osm.EINVAL
    assert size(4, 1025, 1, ctypes.byref(n)) == osm.EINVAL
    assert size(4, 10, 0, ctypes.byref(n)) == osm.EINVAL
    assert size(-1, 10, 1, ctypes.byref(n)) == osm.EINVAL
    assert size(4, 10, 1, None) == osm.EINVAL
    assert osm.balance_workspace(0, 8) == 0
    # at most 64 rows a team, 32 teams a workgroup: of each two slots of E + 1 words of 8 bytes
    spans = (1 << 24) // (64 * 32)
    most = spans * (2 * 257 * 8 + 64) + 512
    assert 0 < osm.balance_workspace(1 << 24, 256, 9) <= most


def test_constants_match_the_header():
    text = open(HEADER).read()
    assert re.search(rf"#define OSM_LOGPROB_TMAX {osm.LOGPROB_TMAX}\b", text)


def test_binding_refuses_what_is_not_there():
    x, t = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: osm.logprob_fwd(x, t), lambda: osm.balance_fwd(x, t),
                 lambda: osm.logprob_bwd(x, x, t, x),
                 lambda: osm.balance_bwd(x, t, t, t, t),
                 lambda: osm.logprob_workspace(4, 10, 1 << 32)):
        with pytest.raises(ValueError):
            call()


def test_reference_by_hand():
    x = np.log(np.array([[1.0, 4.0, 2.0, 1.0], [1.0, 1.0, 1.0, 1.0]]))
    r = loss_ref.logprob(x, np.array([[1, 3, -1], [2, 4, 0]]), K=2)
    assert np.allclose(r["logp"], [[np.log(0.5), np.log(0.125), 0.0],
                                   [np.log(0.25), 0.0, np.log(0.25)]])
    assert np.allclose(r["entropy"], [np.log(2) * (0.5 + 0.5 + 2 * 3 / 8), np.log(4)])
    assert np.allclose(r["stats"], [[np.log(4), 1.0], [0.0, 3.0]])
    assert r["top_idx"].tolist() == [[1, 2], [0, 1]]
    half = loss_ref.logprob(2 * x, np.array([[1], [0]]), temperature=2.0)
    assert np.allclose(half["logp"][:, 0], [np.log(0.5), np.log(0.25)])
    # two rows of a softmax over two experts, one index each; a row without one
    x = np.log(np.array([[1.0, 3.0], [1.0, 1.0], [9.0, 1.0]]))
    r = loss_ref.balance(x, np.array([[1], [1], [-1]]))
    assert r["rows"].tolist() == [2] and r["counts"].tolist() == [[0, 2]]
    assert np.allclose(r["probs"], [[0.375, 0.625]]) and np.allclose(r["loss"], [1.25])
    r = loss_ref.balance(x, np.array([[1], [1], [0]]), starts=[0, 2, 2, 3])
    assert r["rows"].tolist() == [2, 0, 1] and np.allclose(r["loss"], [1.25, 0.0, 1.8])


def test_reference_gradients_against_differences():
    rng = np.random.default_rng(5)
    x = rng.normal(size=(2, 7))
    tok = np.array([[2, 5, 2, 9], [0, -1, 6, 1]])
    g, h = rng.normal(size=(2, 4)), rng.normal(size=2)

    def value(x, T):
        r = loss_ref.logprob(x, tok, temperature=T)
        return (r["logp"] * g).sum() + (r["entropy"] * h).sum()

    for T in (1.0, 0.5):
        d, _ = loss_ref.logprob_bwd(x, tok, g, h, temperature=T)
        for n in range(2):
            for j in range(7):
                lo, hi = x.copy(), x.copy()
                lo[n, j] -= 1e-5
                hi[n, j] += 1e-5
                # central difference: h^2 / 6 times a third derivative of order 10 / T^3
                assert abs((value(hi, T) - value(lo, T)) / 2e-5 - d[n, j]) < 2e-8
    x = rng.normal(size=(9, 5))
    idx = rng.integers(-1, 6, size=(9, 2))
    starts, w = [1, 4, 4, 8], rng.normal(size=3)
    for score in ("softmax", "sigmoid"):
        kw = dict(starts=starts, score=score, scale=0.5)
        r = loss_ref.balance(x, idx, **kw)
        d, _ = loss_ref.balance_bwd(x, idx, r["counts"], r["rows"], w, **kw)
        for n in range(9):
            for j in range(5):
                lo, hi = x.copy(), x.copy()
                lo[n, j] -= 1e-5
                hi[n, j] += 1e-5
                diff = ((loss_ref.balance(hi, idx, **kw)["loss"] -
                         loss_ref.balance(lo, idx, **kw)["loss"]) * w).sum() / 2e-5
                assert abs(diff - d[n, j]) < 2e-8
