"""softmax_sample, route_fwd and route_bwd: arguments they refuse, on the host and
before anything is launched (fake, never dereferenced pointers), and the
plain implementations that the GPU tests compare with, on cases worked by hand."""
import ctypes
import re

import numpy as np
import pytest
import torch

import paper_1805_02867_amd as osm
import pick_ref
from test_abi import HEADER

X, U, V_, I_, B_, D_ = (0x10000000 * i for i in range(1, 7))


def _sample(x=X, ld=10, u=U, params=None, vals=V_, idx=I_, N=4, V=10, dtype=0):
    p = None if params is None else ctypes.byref(params)
    return osm.lib().softmax_sample(x, ld, u, p, vals, idx, N, V, dtype, None)


@pytest.mark.parametrize("bad", [
    dict(N=-1), dict(N=1 << 31), dict(V=0, ld=1), dict(V=1 << 31, ld=1 << 31), dict(ld=9),
    dict(ld=1 << 31), dict(dtype=2), dict(x=0), dict(u=0), dict(vals=0), dict(idx=0),
    dict(x=X + 2), dict(u=U + 1), dict(vals=V_ + 2), dict(idx=I_ + 3),
    dict(vals=X + 100), dict(idx=V_ + 8), dict(vals=U), dict(idx=U + 12),
    dict(vals=X + 4 * 45, ld=20),                       # between two rows of x
    dict(params=osm.SampleParams(B_ + 1, None, None, None, 1, 0, 1, 0)),
    dict(params=osm.SampleParams(None, V_, None, None, 1, 0, 1, 0)),   # overlaps vals
    dict(params=osm.SampleParams(None, None, None, I_ + 4, 1, 0, 1, 0)),
])
def test_sample_refuses(bad):
    assert _sample(**bad) == osm.EINVAL


@pytest.mark.parametrize("ws,n", [(D_ + 16, 1 << 24), (X, 1 << 24), (V_ - 256, 1 << 20)])
def test_sample_refuses_a_bad_workspace(ws, n):
    assert osm.lib().softmax_sample_ws(X, 10, U, None, V_, I_, 4, 10, 0, ws, n, None) == osm.EINVAL


def test_workspace_sizes():
    n = ctypes.c_size_t()
    size = osm.lib().osm_sample_workspace
    assert size(4, 0, 0, ctypes.byref(n)) == osm.EINVAL
    assert size(4, 10, 7, ctypes.byref(n)) == osm.EINVAL
    assert size(-1, 10, 0, ctypes.byref(n)) == osm.EINVAL
    assert size(4, 10, 0, None) == osm.EINVAL
    assert osm.sample_workspace(0, 128256) >= 0 and osm.sample_workspace(1000, 1000) == 0
    for V, rows in ((32000, (1, 64)), (128256, (1, 64, 4000)), (1000000, (1, 4000))):
        for N in rows:
            # a launch's rows at a time, at most 4096 chunks: of each 1024 bins of 8 + 4 bytes
            # and six words of 8 (its sum and maximum, and two classes of bfloat16 values);
            # rounded up to 256; and 4 bytes for each row, of which there are no more than chunks
            most = 4096 * (12 * 1024 + 6 * 8) + 256 + 4 * 4096
            assert 0 < osm.sample_workspace(N, V) <= most


def test_empty_batches_are_noops():
    assert _sample(N=0, x=0, u=0, vals=0, idx=0) == osm.OK
    assert _fwd(N=0, x=0, vals=0, idx=0) == osm.OK
    assert _bwd(N=0, x=0, idx=0, dvals=0, dx=0) == osm.OK


def _route(score=0, groups=1, top_groups=1, group_top=1, renorm=1, scale=1.0):
    return osm.Route(score, groups, top_groups, group_top, renorm, scale)


def _fwd(x=X, bias=None, vals=V_, idx=I_, N=4, E=12, K=2, dtype=0, r=_route()):
    return osm.lib().route_fwd(x, bias, vals, idx, N, E, K, dtype,
                               None if r is None else ctypes.byref(r), None)


def _bwd(x=X, idx=I_, dvals=V_, dx=D_, N=4, E=12, K=2, dtype=0, r=_route()):
    return osm.lib().route_bwd(x, idx, dvals, dx, N, E, K, dtype,
                               None if r is None else ctypes.byref(r), None)


SIZES = [dict(N=-1), dict(N=1 << 31), dict(E=0), dict(E=1025), dict(K=0), dict(K=65, E=100),
         dict(dtype=2), dict(r=None), dict(r=_route(score=2)), dict(r=_route(score=-1)),
         dict(x=0), dict(idx=0), dict(x=X + 1), dict(idx=I_ + 2)]


@pytest.mark.parametrize("bad", SIZES + [
    dict(K=13), dict(vals=0), dict(vals=V_ + 1), dict(bias=B_ + 2), dict(bias=V_),
    dict(vals=X + 8), dict(idx=V_ + 4), dict(r=_route(groups=0)),
    dict(r=_route(groups=5)), dict(E=130, r=_route(groups=65)),
    dict(r=_route(groups=4, top_groups=0)), dict(r=_route(groups=4, top_groups=5)),
    dict(r=_route(groups=4, group_top=0)), dict(r=_route(groups=4, group_top=3)),
    dict(K=4, r=_route(groups=4)),                      # three experts to choose from
])
def test_route_fwd_refuses(bad):
    assert _fwd(**bad) == osm.EINVAL


@pytest.mark.parametrize("bad", SIZES + [
    dict(dvals=0), dict(dx=0), dict(dvals=V_ + 2), dict(dx=D_ + 2), dict(dx=X), dict(dx=I_ + 8),
    dict(dx=V_),
])
def test_route_bwd_refuses(bad):
    assert _bwd(**bad) == osm.EINVAL


def test_constants_match_the_header():
    text = open(HEADER).read()
    assert re.search(rf"#define OSM_ROUTE_EMAX {osm.ROUTE_EMAX}\b", text)
    assert re.search(rf"#define OSM_ROUTE_GMAX {osm.ROUTE_GMAX}\b", text)
    for name, val in (("SOFTMAX", 0), ("SIGMOID", 1)):
        assert re.search(rf"OSM_SCORE_{name} = {val}\b", text)
        assert osm.SCORES[name.lower()] == val


def test_binding_refuses_cpu_tensors_and_bad_scores():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        osm.softmax_sample(x, torch.zeros(2))
    with pytest.raises(ValueError):
        osm.route_fwd(x, 2)
    with pytest.raises(ValueError):
        osm.route_bwd(x, torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 2))
    with pytest.raises(ValueError):
        osm._score("tanh")


def test_reference_sampling_by_hand():
    x = np.log(np.array([[1.0, 4.0, 2.0, 4.0, 1.0]]))   # order 1, 3, 2, 0, 4; sum 12

    def at(u, **kw):
        v, i = pick_ref.sample(x, [u], **kw)
        return int(i[0]), round(float(v[0]) * 1000)
    assert at(0.0) == (0, 83) and at(0.09) == (1, 333) and at(0.95) == (4, 83)
    assert at(1.0) == (4, 83)
    assert at(0.0, top_k=1) == (1, 1000) and at(0.6, top_k=2) == (3, 500)
    assert at(0.99, top_k=4) == (3, 364)                # 0, 1, 2, 3 of weights 1 4 2 4
    assert at(0.0, top_p=0.5) == (1, 500)               # 4 / 12 is short, 8 / 12 is not
    assert at(0.99, top_p=0.7) == (3, 400) and at(0.5, top_p=0.7) == (2, 200)
    assert at(0.99, min_p=0.49) == (3, 400) and at(0.3, min_p=0.51) == (1, 500)
    assert at(0.9, temperature=0.0) == (1, 1000)
    assert at(0.9, top_p=0.0) == (1, 1000)


def test_reference_gradient_against_differences():
    rng = np.random.default_rng(3)
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            x = rng.normal(size=(1, 9))
            kw = dict(score=score, renorm=renorm, scale=2.5)
            _, idx = pick_ref.route(x, 4, **kw)
            g = rng.normal(size=(1, 4))
            d = pick_ref.route_bwd(x, idx, g, **kw)
            for e in range(9):
                h = 1e-5
                lo, hi = x.copy(), x.copy()
                lo[0, e] -= h
                hi[0, e] += h
                vl, il = pick_ref.route(lo, 4, **kw)
                vh, ih = pick_ref.route(hi, 4, **kw)
                assert np.array_equal(il, idx) and np.array_equal(ih, idx)
                # central difference: h^2 / 6 times a third derivative of order 10
                assert abs(((vh - vl) * g).sum() / (2 * h) - d[0, e]) < 1e-8
