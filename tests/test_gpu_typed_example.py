"""The example network runs the 8-bit operators and the aggregation together.

Against the same network in float64 without 8 bits: e4m3 holds a normal value with a
relative error of 2.6% rms, so a product of two such matrices is off by 3.7% of its
2-norm. Four products (three layers and the scores) follow one another, each error
added to a stream that holds the earlier ones: sqrt(4) * 3.7% = 7.4%; twice that."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from conftest import ROOT  # noqa: E402

sys.path.insert(0, os.path.join(ROOT, "examples"))

import paper_2308_11825_amd as agcn  # noqa: E402
import typed_residual_gcn as example  # noqa: E402


@pytest.mark.parametrize("nodes,f,types,classes", [(3000, 128, 4, 40), (1111, 100, 3, 7), (2500, 256, 1, 16)])
def test_example_against_float64(nodes, f, types, classes):
    csr, rest, x = example.make(nodes, f=f, types=types, classes=classes, seed=f)
    plan = agcn.Plan(*csr, n_cols=nodes)
    net = example.TypedResidualGCN(plan, *rest)
    x0 = x.clone()
    got = net.forward(x)
    rows = torch.repeat_interleave(torch.arange(nodes, device=x.device), torch.diff(csr[0]).long())
    A = torch.zeros((nodes, nodes), dtype=torch.float64, device=x.device)
    A.index_put_((rows, csr[1].long()), csr[2].double(), accumulate=True)
    want = example.reference(A, *rest, x)
    off = float((got.double() - want).norm() / want.norm())
    print(f"[example] {nodes} nodes: {off:.4f} off", flush=True)
    assert off < 0.148
    assert torch.equal(x, x0)                       # the features are not written to
    assert torch.equal(net.forward(x), got)       # the same bits again
    plan.destroy()


def test_example_in_a_graph():
    csr, rest, x = example.make(2000, seed=9)
    net = example.TypedResidualGCN(agcn.Plan(*csr, n_cols=2000), *rest)
    want = net.forward(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        net.forward(x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = net.forward(x)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert torch.equal(net.forward(x), want)
