"""Inference of a deep typed graph network, its dense half in 8 bits.

Nodes of several types, ordered by type, keep a residual stream h. Per layer:

    z = relu(A (rms_norm(h) W[type]))        h <- h + z

The norm adds the layer before's z to h, normalises and writes 8 bits in one pass
(``rms_norm``); the transformation takes a weight per node type
(``grouped_linear``, float32 out); the aggregation is the plan's (``Plan.spmm``
with its ReLU). A last norm and one product for all types give class scores.

    python examples/typed_residual_gcn.py [nodes]
"""
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2308_11825_amd as agcn

EPS = 1e-6


class TypedResidualGCN:
    """Weights quantised once; forward(features) -> class scores, (nodes, classes)."""

    def __init__(self, plan, offsets, norms, weights, last_norm, head):
        """offsets: int32, node types + 1; norms: (f,) per layer; weights: (types, f, f)
        per layer; head: (f, classes). All float32 on the plan's GPU."""
        self.plan, self.offsets, self.norms, self.last_norm = plan, offsets, norms, last_norm
        self.weights = [agcn.quantize_weight(w) for w in weights]
        self.head = agcn.quantize_weight(head)

    def forward(self, x):
        h, z = x, None
        for norm, (wq, ws) in zip(self.norms, self.weights):
            q, s, h = self._norm(h, z, norm)
            t = agcn.grouped_linear(q, s, wq, ws, self.offsets)
            z = self.plan.spmm(t, act="relu")
        q, s, h = self._norm(h, z, self.last_norm)
        return agcn.quantized_linear(q, s, *self.head)

    @staticmethod
    def _norm(h, z, weight):
        if z is None:
            return (*agcn.rms_norm(h, weight, eps=EPS), h)
        return agcn.rms_norm(z, weight, residual=h, eps=EPS)


def reference(A, offsets, norms, weights, last_norm, head, x):
    """The same network without 8 bits, in float64 (A: sparse or dense matrix)."""
    def norm(h, g):
        return h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * g.double()

    h, ends = x.double(), offsets.tolist()
    for g, w in zip(norms, weights):
        y = norm(h, g)
        t = torch.cat([y[a:b] @ w[i].double() for i, (a, b) in enumerate(zip(ends, ends[1:]))])
        h = h + (A @ t).clamp(min=0)
    return norm(h, last_norm) @ head.double()


def make(nodes, f=128, types=4, layers=3, classes=40, degree=12, device="cuda:0", seed=0):
    """A random graph and random weights: (A as (rowptr, colidx, vals), the other
    arguments of the network, features)."""
    gen = torch.Generator(device=device).manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=device)

    colidx = torch.randint(0, nodes, (nodes * degree,), generator=gen, device=device).int()
    rowptr = (torch.arange(nodes + 1, device=device) * degree).int()
    vals = torch.full((nodes * degree,), 1.0 / degree ** 0.5, device=device)
    cuts = torch.rand(types - 1, generator=gen, device=device).sort().values * nodes
    offsets = torch.cat([cuts.new_zeros(1), cuts.floor(), cuts.new_full((1,), nodes)]).int()
    norms = [1 + 0.1 * randn(f) for _ in range(layers)]
    weights = [randn(types, f, f) / f ** 0.5 for _ in range(layers)]
    return (rowptr, colidx, vals), (offsets, norms, weights, 1 + 0.1 * randn(f),
                                    randn(f, classes) / f ** 0.5), randn(nodes, f)


def main(nodes=170_000):
    csr, rest, x = make(nodes)
    net = TypedResidualGCN(agcn.Plan(*csr, n_cols=nodes), *rest)
    scores = net.forward(x)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(10):
        scores = net.forward(x)
    torch.cuda.synchronize()
    print(f"{nodes} nodes, {len(net.weights)} layers: {(time.perf_counter() - began) * 100:.3f} ms "
          f"a forward pass, scores {tuple(scores.shape)}", flush=True)


if __name__ == "__main__":
    main(*(int(a) for a in sys.argv[1:]))
