"""Memory of calls on a stream of the caller's choice: results are allocated on that stream, and what
the call reads is not handed out again before its work is done."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from routed_helpers import randn  # noqa: E402

DEV = "cuda:0"
N, F = 4096, 512  # matrices of 8 MB: blocks of their own


def plan():
    i = torch.arange(N + 1, device=DEV).int()
    return agcn.Plan(i, i[:N].clone(), torch.ones(N, device=DEV))


def calls():
    p, W, g = plan(), randn((F, F), torch.float32, 2), torch.ones(F, device=DEV)
    _, place = agcn.sort_groups(torch.zeros((N, 1), dtype=torch.int32, device=DEV), 1)
    return {"spmm": lambda X, s: p.spmm(X, stream=s), "gcn_layer": lambda X, s: p.gcn_layer(X, W, stream=s),
            "linear": lambda X, s: agcn.linear(X, W, stream=s), "layer_norm": lambda X, s: agcn.layer_norm(X, g, stream=s),
            "dispatch": lambda X, s: agcn.dispatch(X, place, stream=s)}


@pytest.mark.parametrize("name", ["spmm", "gcn_layer", "linear", "layer_norm", "dispatch"])
def test_results_are_allocated_on_the_stream(name):
    call, X, side = calls()[name], randn((N, F), torch.float32, 1), torch.cuda.Stream()
    want = call(X, None)
    t = torch.empty((N, F), device=DEV)
    free = t.data_ptr()
    torch.cuda.synchronize()
    del t  # free again for work of the current stream, which nothing orders with the other's
    out = call(X, side)
    assert out.data_ptr() != free
    side.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("name", ["spmm", "gcn_layer", "linear", "layer_norm", "dispatch"])
def test_inputs_are_kept_until_the_stream_has_read_them(name):
    call, X, side = calls()[name], randn((N, F), torch.float32, 1), torch.cuda.Stream()
    want = call(X, None)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)  # the call's work comes after this
    out = call(X, side)
    held = X.data_ptr()
    del X
    other = torch.full((N, F), float("nan"), device=DEV)
    assert other.data_ptr() != held
    side.synchronize()
    assert torch.equal(out, want)
