"""A routed layer as it is used: norm, groups, products per group and the sum of the slots, for
inference with both 8-bit forms and for a training step, against the same in 64 bits."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from quant_helpers import values, weight_values  # noqa: E402
from routed_helpers import gen, randn, rows_of  # noqa: E402

DEV = "cuda:0"


def make(n, f, e, k, dtype, seed=0):
    x = randn((n, f), torch.float32, 1, seed).to(dtype)
    g, b = 1 + 0.2 * randn((1, f), torch.float32, 2)[0], 0.1 * randn((1, f), torch.float32, 3)[0]
    W = torch.randn((e, f, f), generator=gen(e, f), device=DEV) / f ** 0.5
    ids = torch.rand((n, e), generator=gen(n, e, seed), device=DEV).topk(k, dim=1).indices
    ids[n // 2] = -1  # a row that no group takes
    w = torch.softmax(randn((n, k), torch.float32, 4, seed), 1)
    return x, g, b, W, ids, w


def serve(x, g, b, ids, w, e, WQ, WS, integers):
    """One layer with 8-bit weights: the rows are cut to 8 bits once and laid out k times."""
    offsets, place = agcn.sort_groups(ids, e)
    if integers:
        Q, S = agcn.quantize_int(agcn.layer_norm(x, g, b))
        rows, scales = agcn.dispatch(Q, place), agcn.dispatch(S[:, None], place)[:, 0]
        y = agcn.grouped_int_linear(rows, scales, WQ, WS, offsets, dtype=x.dtype, act="relu")
    else:
        Q, S = agcn.rms_norm(x, g)
        rows, scales = agcn.dispatch(Q, place), agcn.dispatch(S, place)
        y = agcn.grouped_linear(rows, scales, WQ, WS, offsets, dtype=x.dtype, act="relu")
    return agcn.combine(y, place, w), rows, scales, offsets, place


@pytest.mark.parametrize("integers", [False, True])
@pytest.mark.parametrize("n,f,e,k", [(1, 256, 8, 2), (37, 200, 5, 3), (3000, 384, 16, 4)])
def test_inference(n, f, e, k, integers):
    """Against the same products of the values that the 8 bits stand for: what differs is
    the rounding of the slots' results and of their sum to bfloat16, half a step (2^-8) each,
    fp32 sums and the 8-bit matrix instruction (1.5e-5)."""
    x, g, b, W, ids, w = make(n, f, e, k, torch.bfloat16)
    WQ, WS = (agcn.quantize_weight_int if integers else agcn.quantize_weight)(W)
    out, rows, scales, offsets, place = serve(x, g, b, ids, w, e, WQ, WS, integers)
    if integers:
        A, V = rows.double() * scales.double()[:, None], WQ.double() * WS.double()[..., None]
    else:
        A, V = values(rows, scales), torch.stack([weight_values(q, s) for q, s in zip(WQ, WS)])
    y = torch.zeros((n * k, f), dtype=torch.float64, device=DEV)
    for i in range(e):
        a, z = int(offsets[i]), int(offsets[i + 1])
        if integers:  # their sums exactly: one of 0 is 0
            y[a:z] = ((rows[a:z].double() @ WQ[i].double().t()) * scales[a:z, None].double() * WS[i].double()).clamp(min=0)
        else:
            y[a:z] = (A[a:z] @ V[i].t()).clamp(min=0)
    at, kept = rows_of(place)
    parts = (w.double() * kept)[..., None] * y[at]
    size = parts.abs().sum(1)
    # the instruction's cut-off is relative to the products' sizes, not to their sum
    cut = 7 * 2.0 ** -13 * ((w.double() * kept)[..., None] * (A.abs().amax(1, keepdim=True) * V.abs().amax() * f / 8)[at]).sum(1)
    off = 2.01 * 2.0 ** -8 * size + (0 if integers else cut)
    assert bool(((out.double() - parts.sum(1)).abs() <= off).all())
    assert not out[n // 2].any()


def test_inference_in_a_graph():
    """Captured once, replayed with new rows and ids, eager calls in between."""
    n, f, e, k = 200, 256, 12, 3
    x, g, b, W, ids, w = make(n, f, e, k, torch.bfloat16)
    weights = [(agcn.quantize_weight(W), False), (agcn.quantize_weight_int(W), True)]
    serve(x, g, b, ids, w, e, *weights[0][0], False)
    graphs = []
    for (WQ, WS), integers in weights:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = serve(x, g, b, ids, w, e, WQ, WS, integers)[0]
        graphs.append((graph, out, WQ, WS, integers))
    for i in range(3):
        nx, _, _, _, nids, nw = make(n, f, e, k, torch.bfloat16, seed=i + 1)
        x.copy_(nx), ids.copy_(nids), w.copy_(nw)
        for graph, out, *_ in graphs:
            out.zero_()
            graph.replay()
        for graph, out, WQ, WS, integers in graphs:
            assert torch.equal(out, serve(x, g, b, ids, w, e, WQ, WS, integers)[0])


@pytest.mark.parametrize("n,f,e,k", [(5, 40, 4, 2), (900, 128, 6, 3)])
def test_training_step(n, f, e, k):
    """h = x + r, y = combine(dispatch(norm(h)) W), loss = sum(y a + h c): the gradients of x, the
    norm's parameters, the groups' weights and the slots' weights against those of the same in
    64 bits. Products in torch, float32: each is off by f u of the sum of its terms' sizes at
    most, typically by sqrt(f) u; norms of the differences stay below 50 u of the norms."""
    x, g, b, W, ids, w = make(n, f, e, k, torch.float32)
    r, a, c = (randn((n, f), torch.float32, s) for s in (7, 8, 9))
    y, h, stats = agcn.layer_norm(x, g, b, residual=r, stats=True)
    offsets, place = agcn.sort_groups(ids, e)
    rows = agcn.dispatch(y, place)
    ends = offsets.tolist()
    z = torch.zeros((n * k, f), device=DEV)
    for i in range(e):
        z[ends[i]:ends[i + 1]] = agcn.linear(rows[ends[i]:ends[i + 1]], W[i])
    out = agcn.combine(z, place, w)
    dz, dw = agcn.combine_backward(a, z, place, w)
    drows, dW = torch.zeros_like(rows), torch.zeros_like(W)
    for i in range(e):
        at = slice(ends[i], ends[i + 1])
        drows[at] = agcn.linear(dz[at], W[i].t().contiguous())
        dW[i] = rows[at].t() @ dz[at]
    dy = agcn.combine(drows, place)
    dx, dg, db = agcn.layer_norm_backward(dy, h, stats, g, grad_hidden=c)

    p = [v.double().requires_grad_() for v in (x, g, b, W, w)]
    H = p[0] + r.double()
    mean = H.mean(1, keepdim=True)
    Y = (H - mean) / torch.sqrt(((H - mean) ** 2).mean(1, keepdim=True) + 1e-5) * p[1] + p[2]
    parts = [p[4][:, s, None] * (Y[:, None] @ p[3][ids[:, s].clamp(min=0)])[:, 0] * (ids[:, s, None] >= 0)
             for s in range(k)]
    want = sum(parts)
    grads = torch.autograd.grad((want * a.double()).sum() + (H * c.double()).sum(), p)
    for got, ref in zip((out, dx, dg, db, dW, dw), (want, *grads)):
        assert (got.double() - ref).norm() <= 50 * 2.0 ** -24 * ref.norm()


def test_on_another_stream():
    """Every call with a stream of its own, its inputs made there: nothing of it runs before
    them, and results are those of the current stream."""
    n, f, e, k = 400, 512, 9, 2
    x, g, b, W, ids, w = make(n, f, e, k, torch.bfloat16)
    want, *_ = serve(x, g, b, ids, w, e, *agcn.quantize_weight_int(W), True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        x2 = x + 0
    WQ, WS = agcn.quantize_weight_int(W, stream=s)
    y = agcn.layer_norm(x2, g, b, stream=s)
    Q, S = agcn.quantize_int(y, stream=s)
    offsets, place = agcn.sort_groups(ids, e, stream=s)
    rows, scales = agcn.dispatch(Q, place, stream=s), agcn.dispatch(S[:, None], place, stream=s)[:, 0]
    z = agcn.grouped_int_linear(rows, scales, WQ, WS, offsets, dtype=x.dtype, act="relu", stream=s)
    out = agcn.combine(z, place, w, stream=s)
    dz, dw = agcn.combine_backward(x2, z, place, w, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    again = agcn.combine_backward(x, z, place, w)
    assert torch.equal(dz, again[0]) and torch.equal(dw, again[1])


def test_sorts_in_graphs():
    """Two captured sorts of many slots, with workspaces, replayed in turn with other ids."""
    cases = [(20000, 4, 50), (3000, 2, 3000), (300, 3, 12)]
    ids = [torch.randint(-1, e + 1, (n, k), generator=gen(n, e), device=DEV).int() for n, k, e in cases]
    graphs = []
    for x, (n, k, e) in zip(ids, cases):
        agcn.sort_groups(x, e)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = agcn.sort_groups(x, e)
        graphs.append((graph, out))
    for i in range(4):
        for x, (n, k, e) in zip(ids, cases):
            x.copy_(torch.randint(-1, e + 1, (n, k), generator=gen(n, e, i), device=DEV))
        for graph, _ in graphs:
            graph.replay()
        for (_, out), x, (n, k, e) in zip(graphs, ids, cases):
            want = agcn.sort_groups(x, e)
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_a_stream_of_another_device_is_refused():
    class Elsewhere:
        device = torch.device("cuda", torch.cuda.device_count())

    x, ids = torch.randn(5, 64, device=DEV), torch.zeros((5, 1), dtype=torch.int64, device=DEV)
    for call in (lambda s: agcn.layer_norm(x, x[0], stream=s), lambda s: agcn.sort_groups(ids, 3, stream=s),
                 lambda s: agcn.quantize_int(x, stream=s)):
        with pytest.raises(ValueError, match="stream"):
            call(Elsewhere())


def test_two_streams_at_once():
    """The same calls on two streams at a time, each with workspaces of its own."""
    n, f = 3000, 512
    x = [randn((n, f), torch.bfloat16, s) for s in (1, 2)]
    ids = [torch.randint(0, 40, (n, 6), generator=gen(s), device=DEV).int() for s in (1, 2)]
    g = torch.ones(f, device=DEV)

    def step(i, stream=None):
        y, stats = agcn.layer_norm(x[i], g, stats=True, stream=stream)
        grads = agcn.layer_norm_backward(y, x[i], stats, g, stream=stream)
        offsets, place = agcn.sort_groups(ids[i], 40, stream=stream)
        rows = agcn.dispatch(y, place, stream=stream)
        return (y, stats, *grads, offsets, place, rows, agcn.combine(rows, place, stream=stream))

    want = [step(0), step(1)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[step(i, s) for i, s in enumerate(streams)] for _ in range(5)]
    torch.cuda.synchronize()
    for pair in got:
        for a, b in zip(pair, want):
            assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_python_refuses_what_does_not_fit():
    """Types, shapes, strides and devices, before anything runs; the C call's refusals as its error."""
    x, g, s = torch.zeros((6, 8), device=DEV), torch.ones(8, device=DEV), torch.zeros((6, 2), device=DEV)
    ids = torch.zeros((6, 2), dtype=torch.int32, device=DEV)
    off, place = agcn.sort_groups(ids, 3)
    R, w = torch.zeros((12, 8), device=DEV), torch.ones((6, 2), device=DEV)
    Q, S = agcn.quantize_int(x)
    WQ, WS = agcn.quantize_weight_int(torch.ones((8, 5), device=DEV))
    WQ3, WS3 = agcn.quantize_weight_int(torch.ones((2, 8, 5), device=DEV))
    offs = torch.zeros(3, dtype=torch.int32, device=DEV)
    wrong_type = [
        lambda: agcn.layer_norm(x.double(), g), lambda: agcn.layer_norm(x, g.half()), lambda: agcn.layer_norm(x, g.cpu()),
        lambda: agcn.layer_norm(x, g, g.bfloat16()), lambda: agcn.layer_norm(x, g, residual=x.half()),
        lambda: agcn.layer_norm(x, g, out=x.half()), lambda: agcn.layer_norm(x, None),
        lambda: agcn.layer_norm_backward(x, x.half(), s, g), lambda: agcn.layer_norm_backward(x, x, s.double(), g),
        lambda: agcn.sort_groups(ids.short(), 3), lambda: agcn.sort_groups(ids, 3, out=off),
        lambda: agcn.sort_groups(ids, "3"), lambda: agcn.dispatch(x, place.long()), lambda: agcn.combine(R, place.long()),
        lambda: agcn.combine(R.int(), place), lambda: agcn.combine(R, place, w.half()),
        lambda: agcn.combine_backward(x.half(), R, place, w), lambda: agcn.combine_backward(x, R, place, None),
        lambda: agcn.quantize_int(x.int()), lambda: agcn.int_linear(Q.float(), S, WQ, WS),
        lambda: agcn.int_linear(Q, S.double(), WQ, WS), lambda: agcn.int_linear(Q, S, WQ, WS, dtype=torch.int32),
        lambda: agcn.int_linear(Q, S, WQ, WS, dtype="float32"), lambda: agcn.int_linear(Q, S, WQ, WS.cpu()),
        lambda: agcn.int_linear(Q, S, WQ, WS, dtype=torch.float16, out=torch.zeros((6, 5), device=DEV)),
        lambda: agcn.grouped_int_linear(Q, S, WQ3, WS3, offs.long())]
    for call in wrong_type:
        with pytest.raises(TypeError):
            call()
    wrong_value = [
        lambda: agcn.layer_norm(x[0], g), lambda: agcn.layer_norm(x, g[:7]), lambda: agcn.layer_norm(x, g, g[:7]),
        lambda: agcn.layer_norm(x, g, hidden=x), lambda: agcn.layer_norm(x.t(), torch.ones(6, device=DEV)),
        lambda: agcn.layer_norm(x, torch.ones(16, device=DEV)[::2]), lambda: agcn.layer_norm(x, g, residual=x[:5]),
        lambda: agcn.layer_norm(x[:, :0], g[:0], stats=True), lambda: agcn.layer_norm_backward(x, x[:5], s, g),
        lambda: agcn.layer_norm_backward(x, x, s[:, :1], g), lambda: agcn.sort_groups(ids[0], 3),
        lambda: agcn.sort_groups(ids, -1), lambda: agcn.sort_groups(ids, 3, out=(off[:3], place)),
        lambda: agcn.dispatch(x, place[:5]), lambda: agcn.dispatch(x, place[0]), lambda: agcn.dispatch(x, place, out=x),
        lambda: agcn.combine(R[:11], place), lambda: agcn.combine(R, place, w[:, :1]),
        lambda: agcn.combine_backward(x[:5], R, place, w), lambda: agcn.int_linear(Q, S[:5], WQ, WS),
        lambda: agcn.int_linear(Q[:, :7], S, WQ, WS), lambda: agcn.int_linear(Q, S, WQ, WS, act="gelu"),
        lambda: agcn.int_linear(Q, S, WQ3, WS3), lambda: agcn.grouped_int_linear(Q, S, WQ, WS, offs),
        lambda: agcn.grouped_int_linear(Q, S, WQ3, WS3, offs[:2])]
    for call in wrong_value:
        with pytest.raises(ValueError):
            call()
    for call, status in ((lambda: agcn.layer_norm(x, g, eps=0.0), agcn.AGCN_ERR_INVALID_ARGUMENT),
                         (lambda: agcn.layer_norm(x, g, out=x), agcn.AGCN_ERR_INVALID_ARGUMENT),
                         (lambda: agcn.sort_groups(ids, 65537), agcn.AGCN_ERR_UNSUPPORTED),
                         (lambda: agcn.combine(R[:, :0].expand(12, 0), place, out=torch.zeros((6, 0), device=DEV)), None)):
        if status is None:
            call()
            continue
        with pytest.raises(agcn.AgcnError) as e:
            call()
        assert e.value.status == status and agcn.agcn_last_error() in str(e.value)
