"""Layer norm and its gradients against the formulas in 64 bits.

u = 2^-24. A lane adds V NV <= 40 values of a row one after the other (1024 threads f / 1024
of a long one), and at most 16 more steps join the lanes: D = max(40, f / 1024) + 16
additions deep. A difference to the pivot, and then to the mean, is off by u of itself, the
mean by D u times the mean size of the differences, which the row's 1 / sqrt(var + eps) brings to
1 at most; that factor is off by D / 2 + 8 u of itself. So the normalised value is off by
(D / 2 + 10) u |xh| + (D + 2) u, and y by that times |g|, u of both terms of its sum and its
own rounding. Gradients are bounded term by term in the same way in the tests."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from routed_helpers import TYPES, U, half_step, norm, norm_grad, padded, randn, tiniest  # noqa: E402

DEV = "cuda:0"
EPS = 1e-5


def depth(f):
    return max(40, -(-f // 1024)) + 16


def check_norm(y, stats, h, g, b, dtype, eps=EPS):
    """h: the rows as 32 bits hold them, in float64."""
    f = h.shape[1]
    g, b = g.double(), torch.zeros_like(g.double()) if b is None else b.double()
    want, xh, mean, rs = norm(h, g, b, eps)
    D = depth(f)
    off = U * (((D / 2 + 10) * xh.abs() + D + 2) * g.abs() + (xh * g).abs() + want.abs())
    off = off + half_step(dtype) * (want.abs() + off) + tiniest(dtype)
    assert bool(((y.double() - want).abs() <= off).all()), ((y.double() - want).abs() / off).max()
    if stats is not None:
        size = (h - mean).abs().mean(1, keepdim=True)
        assert bool(((stats[:, :1].double() - mean).abs() <= U * (2 * mean.abs() + D * size)).all())
        assert bool(((stats[:, 1:].double() - rs).abs() <= U * (D / 2 + 8) * rs).all())


def check_grad(got, dy, h, stats, g, dh, dtype, p_dtype):
    dx, dg, db = got
    n, f = h.shape
    want, want_g, want_b = norm_grad(dy, h, stats, g)
    rs = stats[:, 1:].double()
    xh = ((h.double() - stats[:, :1].double()) * rs)
    d = (dy.double() * g.double()).abs()
    D = depth(f)
    m1, m2 = d.mean(1, keepdim=True), (d * xh.abs()).mean(1, keepdim=True)
    off = rs * U * (6 * d + (D + 6) * m1 + (D + 12) * xh.abs() * m2)
    if dh is not None:
        want = want + dh.double()
    off = off + U * want.abs()
    off = off + half_step(dtype) * (want.abs() + off) + tiniest(dtype)
    assert bool(((dx.double() - want).abs() <= off).all()), ((dx.double() - want).abs() / off).max()
    # Rows: a lane's own one after the other (256 workgroups or more; of long rows every 25th or more),
    # 16 rows of a workgroup, the workgroups' sums 32 apart and then 32.
    R = n // (25 if f > 8192 else 256) + 96
    for a, w, size in ((dg, want_g, (dy.double() * xh).abs().sum(0)), (db, want_b, dy.double().abs().sum(0))):
        off = U * (R + 4) * size
        off = off + half_step(p_dtype) * (w.abs() + off) + tiniest(p_dtype)
        assert a.dtype == p_dtype
        assert bool(((a.double() - w).abs() <= off).all()), ((a.double() - w).abs() / off).max()


def inputs(n, f, dtype, p_dtype, *seed):
    x = randn((n, f), torch.float32, 1, *seed) * torch.exp(randn((n, 1), torch.float32, 2, *seed))
    x = x + 2 * randn((n, 1), torch.float32, 3, *seed)
    return (x.to(dtype), randn((n, f), dtype, 4, *seed), (1 + 0.3 * randn((1, f), torch.float32, 5, *seed)[0]).to(p_dtype),
            randn((1, f), torch.float32, 6, *seed)[0].to(p_dtype))


# Every shape of lanes and pieces, both sides of each border, and rows past the registers.
WIDTHS = [1, 2, 3, 4, 7, 8, 9, 15, 16, 63, 64, 65, 127, 128, 129, 192, 193, 255, 256, 257, 300, 384, 385,
          512, 513, 601, 768, 769, 1000, 1024, 1025, 1536, 1537, 2048, 2049, 2432, 2561, 3000, 3080, 4096, 4097, 5120, 6145, 8191, 8192,
          8193, 10112, 12289, 16384, 16385, 20480, 24577, 32768, 32769, 40001]


@pytest.mark.parametrize("dtype,p_dtype", [("float32", "float32"), ("bfloat16", "float32"), ("bfloat16", "bfloat16"),
                                           ("float16", "float32"), ("float16", "float16")])
@pytest.mark.parametrize("f", WIDTHS)
def test_every_width(f, dtype, p_dtype):
    dtype, p_dtype = TYPES[dtype], TYPES[p_dtype]
    for n in (1, 19):
        x, r, g, b = inputs(n, f, dtype, p_dtype)
        y, h, stats = agcn.layer_norm(x, g, b, residual=r, stats=True)
        full = (x.float() + r.float()).double()
        assert torch.equal(h, full.to(dtype))
        check_norm(y, stats, full, g, b, dtype)
        dy, dh = randn((n, f), dtype, 7), randn((n, f), dtype, 8)
        check_grad(agcn.layer_norm_backward(dy, h, stats, g, grad_hidden=dh), dy, h, stats, g, dh, dtype, p_dtype)


@pytest.mark.parametrize("n,f,dtype", [(5000, 128, "float32"), (40000, 41, "bfloat16"), (3000, 601, "float16"),
                                       (1500, 4096, "bfloat16"), (2500, 1024, "float32"), (100, 20000, "bfloat16"),
                                       (300, 33001, "float16"), (200, 17001, "float32")])
def test_many_rows_without_residual_or_bias(n, f, dtype):
    dtype = TYPES[dtype]
    x, _, g, _ = inputs(n, f, dtype, torch.float32)
    x[n // 2] = 0
    y, stats = agcn.layer_norm(x, g, stats=True)
    assert torch.equal(y, agcn.layer_norm(x, g))
    check_norm(y, stats, x.double(), g, None, dtype)
    dy = randn((n, f), dtype, 9)
    got = agcn.layer_norm_backward(dy, x, stats, g)
    check_grad(got, dy, x, stats, g, None, dtype, torch.float32)
    again = agcn.layer_norm_backward(dy, x, stats, g)
    assert all(torch.equal(a, b) for a, b in zip(got, again))  # sums in a fixed order
    dx, dg, db = agcn.layer_norm_backward(dy, x, stats, g, bias=False)
    assert db is None and torch.equal(dx, got[0]) and torch.equal(dg, got[1])


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("f", [5, 200, 601, 3001])
def test_strides_alignment_and_given_outputs(f, dtype):
    dtype, n = TYPES[dtype], 30
    x, r, g, b = inputs(n, f, dtype, torch.float32)
    want, hidden, stats = agcn.layer_norm(x, g, b, residual=r, stats=True)
    xs, rs, out, hs = padded(x, 3, 1), padded(r, 5), padded(torch.zeros_like(x), 2, 1), padded(torch.zeros_like(x), 1)
    around = out._base.clone() if out._base is not None else None
    y, h, s = agcn.layer_norm(xs, g, b, residual=rs, stats=True, hidden=hs, out=out)
    assert y is out and h is hs and torch.equal(y, want) and torch.equal(h, hidden) and torch.equal(s, stats)
    if around is not None:
        full = out._base.clone()
        full[1:].view(n, f + 2)[:, :f] = 0
        around[1:].view(n, f + 2)[:, :f] = 0
        assert torch.equal(torch.nan_to_num(full, nan=7.0), torch.nan_to_num(around, nan=7.0))
    # h in place of x, and of the residual
    x2 = padded(x, 3, 1)
    y, h = agcn.layer_norm(x2, g, b, residual=r, hidden=x2)
    assert h is x2 and torch.equal(y, want) and torch.equal(x2, hidden)
    r2 = r.clone()
    y, h = agcn.layer_norm(x, g, b, residual=r2, hidden=r2)
    assert torch.equal(y, want) and torch.equal(r2, hidden)
    dy, dh = randn((n, f), dtype, 7), randn((n, f), dtype, 8)
    want = agcn.layer_norm_backward(dy, hidden, stats, g, grad_hidden=dh)
    st = padded(stats, 1, 1)
    got = agcn.layer_norm_backward(padded(dy, 1, 1), padded(hidden, 2), st, g, grad_hidden=padded(dh, 3), out=out)
    assert got[0] is out and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("f", [40, 600, 5000, 20000])
def test_rows_of_one_value_far_from_zero_and_past_the_range(f):
    """Rows of one value give b, whatever their size; large means cost no bits of the
    differences; squares past fp32's range are summed scaled."""
    g, b = randn((1, f), torch.float32, 1)[0], randn((1, f), torch.float32, 2)[0]
    x = randn((9, f), torch.float32, 3)
    x[0], x[1], x[2], x[3] = 0, 1000.1, -3.0e38, 1e-30
    x[4] = 1000 + torch.round(x[4] * 64) / 64  # exactly held
    x[5] *= 1e20
    x[6] *= 2.0 ** 124 / x[6].abs().max()
    x[7] *= 1e-4
    x[8] = torch.where(torch.arange(f, device=DEV) % 2 == 0, 3.0e38, -3.0e38)
    y, stats = agcn.layer_norm(x, g, b, stats=True)
    assert all(torch.equal(y[i], b) for i in range(4))
    check_norm(y[4:], stats[4:], x[4:].double(), g, b, torch.float32)
    assert bool(torch.isfinite(stats).all())
    dy = randn((9, f), torch.float32, 4)
    dx, dg, db = agcn.layer_norm_backward(dy, x, stats, g)
    assert bool(torch.isfinite(dx).all()) and bool(torch.isfinite(db).all())
    check_grad((dx[4:], *agcn.layer_norm_backward(dy[4:], x[4:].contiguous(), stats[4:].contiguous(), g)[1:]), dy[4:],
               x[4:], stats[4:], g, None, torch.float32, torch.float32)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_not_finite_rows_stay_by_themselves(dtype):
    dtype = TYPES[dtype]
    for f in (20, 200, 3000, 20001):
        x, _, g, b = inputs(6, f, dtype, torch.float32)
        clean, stats = agcn.layer_norm(x, g, b, stats=True)
        x[1, f // 2], x[3, f - 1], x[4, 0] = float("nan"), float("inf"), float("-inf")
        y, s = agcn.layer_norm(x, g, b, stats=True)
        for i in (1, 3, 4):
            assert bool(torch.isnan(y[i]).all()) and bool(torch.isnan(s[i, 1]))
        for i in (0, 2, 5):
            assert torch.equal(y[i], clean[i]) and torch.equal(s[i], stats[i])
        dx, _, db = agcn.layer_norm_backward(torch.ones_like(x), x, s, g)
        assert bool(torch.isnan(dx[1]).all()) and bool(torch.isfinite(dx[0]).all()) and bool(torch.isfinite(db).all())


@pytest.mark.parametrize("eps", [1e-12, 1.0, 2.9e38])
def test_eps(eps):
    for f in (30, 2500):
        x, _, g, b = inputs(8, f, torch.float32, torch.float32)
        x[2] = 1e19 * x[2]
        y, stats = agcn.layer_norm(x, g, b, eps=eps, stats=True)
        check_norm(y, stats, x.double(), g, b, torch.float32, torch.tensor(eps, dtype=torch.float32).double().item())


def test_empty():
    for n, f in ((0, 8), (0, 0), (5, 0)):
        x, g = torch.zeros((n, f), device=DEV), torch.ones(f, device=DEV)
        assert agcn.layer_norm(x, g, g, residual=x)[0].shape == (n, f)
        dx, dg, db = agcn.layer_norm_backward(x, x, torch.zeros((n, 2), device=DEV), g)
        assert dx.shape == (n, f) and not dg.any() and not db.any() and dg.shape == (f,)


@pytest.mark.parametrize("f", [6, 130])
def test_gradients_against_differences(f):
    """The kernels' gradients against central differences of the formula in 64 bits, of step t:
    they are off by t^2 / 6 of its third derivative, which the smooth rows here keep below 50."""
    n, t = 7, 1e-5
    x, _, g, b = inputs(n, f, torch.float32, torch.float32, 5)
    x = x / x.std(1, keepdim=True)
    _, stats = agcn.layer_norm(x, g, b, stats=True)
    dy, dh = randn((n, f), torch.float32, 1), randn((n, f), torch.float32, 2)
    dx, dg, db = (v.double() for v in agcn.layer_norm_backward(dy, x, stats, g, grad_hidden=dh))

    def loss(x, g, b):
        return (norm(x, g, b, EPS)[0] * dy.double()).sum() + (x * dh.double()).sum()

    p = [v.double() for v in (x, g, b)]
    for i, grad in enumerate((dx, dg, db)):
        to = randn(tuple(p[i].shape), torch.float32, 30 + i).double()
        up, down = list(p), list(p)
        up[i], down[i] = p[i] + t * to, p[i] - t * to
        want = (loss(*up) - loss(*down)) / (2 * t)
        size = (grad.abs() * to.abs()).sum() + (dh.double().abs() * to.abs()).sum() if i == 0 else \
            (dy.double().abs() * 4).sum()
        assert abs((grad * to).sum() - want) <= 200 * U * size + 50 * n * f * t * t, i


def test_on_another_stream_and_in_a_graph():
    """A backward pass captured and replayed, with other eager calls between the replays."""
    n, f = 700, 300
    x, r, g, b = inputs(n, f, torch.bfloat16, torch.float32)
    dy = randn((n, f), torch.bfloat16, 7)

    def step():
        y, h, stats = agcn.layer_norm(x, g, b, residual=r, stats=True)
        return (y, h, stats, *agcn.layer_norm_backward(dy, h, stats, g, grad_hidden=y))

    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y, h, stats = agcn.layer_norm(x, g, b, residual=r, stats=True, stream=s)
    got = (y, h, stats, *agcn.layer_norm_backward(dy, h, stats, g, grad_hidden=y, stream=s))
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for i in range(4):
        x.copy_(randn((n, f), torch.bfloat16, 40 + i))
        want = step()
        for graph, out in graphs:
            for v in out:
                v.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, c) for a, c in zip(out, want)), i
