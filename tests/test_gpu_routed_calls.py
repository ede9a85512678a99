"""Calls of the routed layer's operators that are refused or fail, and how they say so."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from routed_helpers import randn  # noqa: E402

DEV = "cuda:0"


class Elsewhere:
    """A stream of a device that the tensors are not on."""
    device = torch.device("cuda", 1)
    cuda_stream = 0


def test_a_stream_of_another_device_is_refused_by_every_function():
    n, f = 6, 32
    x, g, W = randn((n, f), torch.float32, 1), randn((f,), torch.float32, 2), randn((f, 8), torch.float32, 3)
    s = Elsewhere()
    Q, S = agcn.quantize(x)
    WQ, WS = agcn.quantize_weight(W)
    rowptr, colidx, vals = torch.arange(n + 1, device=DEV).int(), torch.arange(n, device=DEV).int(), g[:n].clone()
    plan = agcn.Plan(rowptr, colidx, vals)
    offsets = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    for call in (lambda: agcn.quantize_weight_int(W, stream=s), lambda: agcn.quantize_weight(W, stream=s),
                 lambda: agcn.quantize(x, stream=s), lambda: agcn.quantize(x, out=(Q, S), stream=s),
                 lambda: agcn.rms_norm(x, g, stream=s), lambda: agcn.quantized_linear(Q, S, WQ, WS, stream=s),
                 lambda: agcn.grouped_linear(Q, S, WQ[None], WS[None], offsets, stream=s),
                 lambda: agcn.linear(x, W, stream=s), lambda: agcn.Plan(rowptr, colidx, vals, stream=s),
                 lambda: plan.spmm(x, stream=s), lambda: plan.gcn_layer(x, W, stream=s)):
        with pytest.raises(ValueError, match="stream must be one of cuda:0"):
            call()


def test_memory_that_runs_out_is_torchs_error():
    """The same exception from all functions, whichever of them allocates."""
    x = randn((1000, 1024), torch.float32, 1)
    _, place = agcn.sort_groups(torch.zeros((1000, 256), dtype=torch.int32, device=DEV), 1)
    W = torch.zeros((1, 1024), device=DEV).expand(1024, 1024).contiguous()
    torch.cuda.empty_cache()
    total = torch.cuda.get_device_properties(0).total_memory
    try:
        # What is held now and 256 MB more: the allocator itself refuses the gigabyte of results.
        torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + 2 ** 28) / total)
        with pytest.raises(torch.OutOfMemoryError):
            x.new_empty((256000, 1024))
        with pytest.raises(torch.OutOfMemoryError) as e:
            agcn.dispatch(x, place)
        assert isinstance(e.value, RuntimeError) and "memory" in str(e.value)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert agcn.dispatch(x, place).shape == (256000, 1024) and agcn.quantize_weight_int(W)[0].shape == (1024, 1024)


def test_expanded_gradients_are_refused_with_the_way_out():
    """The gradient of a sum has strides of 0: what to do about it is said."""
    n, k, f = 6, 2, 16
    x, g, w = randn((n, f), torch.float32, 1), randn((f,), torch.float32, 2), randn((n, k), torch.float32, 3)
    _, stats = agcn.layer_norm(x, g, stats=True)
    _, place = agcn.sort_groups(torch.zeros((n, k), dtype=torch.int32, device=DEV), 1)
    R = agcn.dispatch(x, place)
    for grad in (torch.ones((), device=DEV).expand(n, f), torch.ones(f, device=DEV).expand(n, f),
                 torch.ones((n, 1), device=DEV).expand(n, f), randn((f, n), torch.float32, 4).t()):
        for call in (lambda grad: agcn.layer_norm_backward(grad, x, stats, g), lambda grad: agcn.layer_norm(grad, g),
                     lambda grad: agcn.combine_backward(grad, R, place, w), lambda grad: agcn.quantize_int(grad)):
            with pytest.raises(ValueError, match=r"contiguous\(\)"):
                call(grad)
            call(grad.contiguous())
    with pytest.raises(ValueError, match=r"contiguous\(\)"):
        agcn.combine(R, place, torch.ones(k, device=DEV).expand(n, k))


def test_linear_refuses_an_out_that_is_not_on_its_device():
    """(Its address would be written to by the kernel.)"""
    x, W = randn((6, 8), torch.float32, 1), randn((8, 4), torch.float32, 2)
    with pytest.raises(ValueError, match="device"):
        agcn.linear(x, W, out=torch.zeros((6, 4)))
