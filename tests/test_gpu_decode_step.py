"""Routing and sampling as a mixture-of-experts model runs them: a router's projection,
the experts of every token and their weighted sum, the vocabulary's projection,
one token sampled of each row.  And the training step of the router."""
import numpy as np
import pytest
import torch

import paper_1805_02867_amd as osm
import pick_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X; none is visible")
    return torch.device("cuda:0")


def host(t):
    return t.detach().double().cpu().numpy()


class Model:
    """A layer of E experts (a matrix each) between a router and a vocabulary."""

    def __init__(self, H, E, V, dev):
        g = torch.Generator().manual_seed(1)

        def w(*shape):
            return (torch.randn(*shape, generator=g) / H ** 0.5).to(torch.bfloat16).to(dev)
        self.router, self.head = w(E, H), 4 * w(V, H)
        self.experts = w(E, H, H).float()
        self.bias = 0.05 * torch.randn(E, generator=g).to(dev)

    def step(self, h, u, K, seen=None):
        scores = osm.proj(h, self.router)
        vals, idx = osm.route_fwd(scores, K, bias=self.bias, score="sigmoid", groups=4,
                                  top_groups=2, group_top=2, scale=2.5)
        y = h.float()
        for i in range(K):
            m = self.experts[idx[:, i].long()]                   # N x H x H
            y = y + vals[:, i:i + 1] * torch.bmm(m, h.float().unsqueeze(2)).squeeze(2)
        logits = osm.proj(y.to(torch.bfloat16), self.head)
        out = osm.softmax_sample(logits, u, temperature=0.8, top_k=40, top_p=0.95)
        if seen is not None:
            seen.update(scores=scores, vals=vals, idx=idx, logits=logits)
        return out


@pytest.mark.parametrize("N", [1, 17])
def test_decode_steps(N, dev):
    H, E, V, K = 64, 16, 5003, 3
    model = Model(H, E, V, dev)
    g = torch.Generator().manual_seed(N)
    h = torch.randn(N, H, generator=g).to(torch.bfloat16).to(dev)
    u = torch.rand(N, generator=g).to(dev)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        model.step(h, u, K)
    torch.cuda.synchronize()
    graph, out = torch.cuda.CUDAGraph(), None
    with torch.cuda.graph(graph, stream=s):
        out = model.step(h, u, K)
    for rep in range(4):
        h.copy_(torch.randn(N, H, generator=g).to(torch.bfloat16))
        u.copy_(torch.rand(N, generator=g))
        seen = {}
        vals, idx = model.step(h, u, K, seen)
        torch.cuda.synchronize()
        rv, ri = pick_ref.route(host(seen["scores"]), K, host(model.bias), score="sigmoid",
                                groups=4, top_groups=2, group_top=2, scale=2.5)
        assert np.array_equal(seen["idx"].cpu().numpy(), ri)
        pick_ref.close(host(seen["vals"]), rv)
        rv, ri = pick_ref.sample(host(seen["logits"]), host(u), temperature=0.8, top_k=40,
                                 top_p=0.95)
        assert np.array_equal(idx.cpu().numpy(), ri)
        pick_ref.close(host(vals), rv)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], vals) and torch.equal(out[1], idx), f"replay {rep}"


def test_router_training_step(dev):
    """The gradient of a loss over the weighted experts, down to the router's matrix."""
    N, H, E, K = 45, 64, 24, 4
    g = torch.Generator().manual_seed(3)
    h = torch.randn(N, H, generator=g).to(torch.bfloat16).to(dev)
    w = (torch.randn(E, H, generator=g) / 8).to(torch.bfloat16).to(dev)
    value = torch.randn(E, generator=g).to(dev)                  # what an expert adds to the loss
    for score, renorm in (("softmax", True), ("softmax", False), ("sigmoid", True)):
        kw = dict(score=score, renorm=renorm)
        logits = osm.proj(h, w)
        vals, idx = osm.route_fwd(logits, K, **kw)
        dlogits = osm.route_bwd(logits, idx, value[idx.long()].contiguous(), **kw)
        dw = dlogits.double().t().contiguous() @ h.double()
        x = logits.double().requires_grad_()
        s = torch.softmax(x, 1) if score == "softmax" else torch.sigmoid(x)
        p = torch.gather(s, 1, idx.long())
        if renorm:
            p = p / p.sum(1, keepdim=True)
        (p * value.double()[idx.long()]).sum().backward()
        want = x.grad.t().contiguous() @ h.double()
        # binary32 roundings of dlogits, |.| under |value| <= 4, summed over N rows of |h| <= 5
        assert (dw - want).abs().max().item() <= N * 5 * 4 * 2.0 ** -24
