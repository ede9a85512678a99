"""Views whose memory is not their values: torch conjugates complex tensors, and negates the
imaginary parts of such, by a bit on the view. Functions that read the memory itself refuse them."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from routed_helpers import dispatch, randn  # noqa: E402

DEV = "cuda:0"


def negated(t):
    """t's values behind the bit."""
    v = torch._neg_view(-t)
    assert v.is_neg() and torch.equal(v, t)
    return v


def refused(call, *args):
    """Each of the tensors among args in turn as such a view; with all of them plain the call works."""
    call(*args)
    for i, a in enumerate(args):
        if a is not None:
            with pytest.raises(TypeError, match="resolve_neg"):
                call(*args[:i], negated(a), *args[i + 1:])


@pytest.mark.parametrize("dtype", [torch.complex64, torch.complex128])
def test_dispatch_of_complex_rows(dtype):
    x = torch.complex(randn((20, 6), torch.float32, 1), randn((20, 6), torch.float32, 2)).to(dtype)
    _, place = agcn.sort_groups(torch.arange(40, device=DEV).view(20, 2) % 3, 3)
    assert torch.equal(agcn.dispatch(x, place), dispatch(x, place))
    with pytest.raises(TypeError, match="resolve_conj"):
        agcn.dispatch(x.conj(), place)
    with pytest.raises(TypeError, match="resolve_conj"):
        agcn.dispatch(x, place, out=torch.zeros((40, 6), dtype=dtype, device=DEV).conj())
    resolved = x.conj().resolve_conj()
    assert torch.equal(agcn.dispatch(resolved, place), dispatch(resolved, place))


def test_an_imaginary_part():
    """One column of a conjugate's imaginary part has the strides that the functions take."""
    x = torch.complex(randn((12, 1), torch.float32, 1), randn((12, 1), torch.float32, 2))
    part = x.conj().imag
    assert part.is_neg()
    _, place = agcn.sort_groups(torch.zeros((12, 1), dtype=torch.int32, device=DEV), 1)
    for call in (lambda: agcn.dispatch(part, place), lambda: agcn.combine(part, place), lambda: agcn.quantize_int(part),
                 lambda: agcn.quantize_weight_int(part), lambda: agcn.layer_norm(part, torch.ones(1, device=DEV)),
                 lambda: agcn.quantize(part), lambda: agcn.linear(part, part[:1])):
        with pytest.raises(TypeError, match="resolve_neg"):
            call()


def test_routed_operators():
    n, k, f = 10, 2, 32
    x, r, g, b = (randn(s, torch.float32, i) for i, s in enumerate(((n, f), (n, f), (f,), (f,))))
    refused(lambda x, g, b, r: agcn.layer_norm(x, g, b, residual=r), x, g, b, r)
    refused(lambda h, y: agcn.layer_norm(x, g, b, residual=r, hidden=h, out=y), x.clone(), x.clone())
    _, stats = agcn.layer_norm(x, g, b, stats=True)
    refused(lambda dy, h, s, g, dh: agcn.layer_norm_backward(dy, h, s, g, grad_hidden=dh), r, x, stats, g, r)
    refused(lambda o: agcn.layer_norm_backward(r, x, stats, g, out=o), x.clone())
    ids = torch.arange(n * k, device=DEV).view(n, k) % 3
    refused(lambda i: agcn.sort_groups(i, 3), ids)
    offsets, place = agcn.sort_groups(ids, 3)
    refused(lambda o, p: agcn.sort_groups(ids, 3, out=(o, p)), offsets.clone(), place.clone())
    refused(agcn.dispatch, x, place)
    R, w = agcn.dispatch(x, place), randn((n, k), torch.float32, 7)
    refused(lambda o: agcn.dispatch(x, place, out=o), R.clone())
    refused(agcn.combine, R, place, w)
    refused(lambda o: agcn.combine(R, place, w, out=o), x.clone())
    refused(agcn.combine_backward, x, R, place, w)
    refused(lambda o: agcn.combine_backward(x, R, place, w, out=o), R.clone())
    refused(agcn.quantize_int, x)
    Q, S = agcn.quantize_int(x)
    refused(lambda q, s: agcn.quantize_int(x, out=(q, s)), Q.contiguous().clone(), S.clone())
    refused(agcn.quantize_weight_int, randn((f, 5), torch.float32, 8))
    WQ, WS = (torch.stack([v] * 3).contiguous() for v in agcn.quantize_weight_int(randn((f, 5), torch.float32, 8)))
    refused(agcn.int_linear, Q[:n].contiguous(), S, WQ[0], WS[0])
    refused(lambda y: agcn.int_linear(Q, S, WQ[0], WS[0], out=y), torch.zeros((n, 5), device=DEV))
    offsets = torch.tensor([0, 2, 2, 9], dtype=torch.int32, device=DEV)
    refused(agcn.grouped_int_linear, Q.contiguous(), S, WQ, WS, offsets)


def test_8_bit_operators_and_the_aggregation():
    n, f = 10, 32
    x, r, g = (randn(s, torch.float32, i) for i, s in enumerate(((n, f), (n, f), (f,))))
    refused(agcn.quantize, x)
    refused(agcn.quantize_weight, x)
    refused(lambda x, g, r, h: agcn.rms_norm(x, g, residual=r, hidden=h), x, g, r, x.clone())
    Q, S = agcn.quantize(x)
    WQ, WS = agcn.quantize_weight(randn((3, f, 5), torch.float32, 8))
    refused(lambda y: agcn.quantized_linear(Q, S, WQ[0], WS[0], out=y), torch.zeros((n, 5), device=DEV))
    offsets = torch.tensor([0, 2, 2, 9], dtype=torch.int32, device=DEV)
    refused(lambda o: agcn.grouped_linear(Q, S, WQ, WS, o), offsets)
    W = randn((f, 5), torch.float32, 9)
    refused(lambda x, w, o: agcn.linear(x, w, out=o), x, W, torch.zeros((n, 5), device=DEV))
    rowptr, colidx, vals = (torch.arange(n + 1, device=DEV).int(), torch.arange(n, device=DEV).int(),
                            randn((n,), torch.float32, 10))
    refused(lambda *a: agcn.Plan(*a), rowptr, colidx, vals)
    plan = agcn.Plan(rowptr, colidx, vals)
    refused(lambda x, o: plan.spmm(x, out=o), x, torch.zeros((n, f), device=DEV))
    refused(lambda x, w, o: plan.gcn_layer(x, w, out=o), x, W, torch.zeros((n, 5), device=DEV))
