"""The library's first call of a process made while a stream is captured: the graph is right,
and so are the calls after it, which need the library's own memory."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import sys
import torch
sys.path.insert(0, {root!r})
import paper_1805_02867_amd as osm
g = torch.Generator().manual_seed(1)
dev = torch.device("cuda:0")
x = torch.randn(3, 128256, generator=g).to(torch.bfloat16).to(dev)
u = torch.rand(3, generator=g).to(dev)
r = torch.randn(300, 64, generator=g).to(dev)
call = {{"softmax_sample": lambda: osm.softmax_sample(x, u, top_p=0.9),
        "route_fwd": lambda: osm.route_fwd(r, 4),
        "softmax_topk_noalloc": lambda: osm.softmax_topk_noalloc(x, 5)}}[{name!r}]
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    out = call()
got = []
for _ in range(3):
    for t in out:
        t.zero_()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    got.append([t.clone() for t in out])
osm.softmax_fwd(torch.randn(2, 300000, device=dev))      # split rows: the library's scratch
want = call()
osm.softmax_topk(x.float(), 5)
osm.softmax_sample(x, u, top_k=9)
torch.cuda.synchronize()
assert all(torch.equal(a, b) for o in got for a, b in zip(o, want))
print("same")
"""


@pytest.mark.parametrize("name", ["softmax_sample", "route_fwd", "softmax_topk_noalloc"])
def test_first_call_under_capture(name):
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X; none is visible")
    r = subprocess.run([sys.executable, "-c", PROGRAM.format(root=ROOT, name=name)], timeout=100,
                       capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.split() == ["same"], r.stdout + r.stderr
