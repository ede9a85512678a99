"""Products of 8-bit integers: quantising is exact as defined; a product's sum is exact, so it
is off by its conversion to 32 bits, two products and the rounding to the type (u = 2^-24)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from routed_helpers import TYPES, U, gen, half_step, padded, randn, tiniest  # noqa: E402

DEV = "cuda:0"


def quantized(x):
    """(q, s) of the rows of x as defined: 127 / a and its product with x rounded to 32 bits,
    each from a 64-bit value that holds it exactly enough (a quotient of 24-bit numbers in 53
    bits rounds to 24 as the exact one does; a product is exact)."""
    top = x.double().abs().amax(1, keepdim=True) if x.shape[1] else x.new_zeros((x.shape[0], 1)).double()
    up = torch.where(top < 2.0 ** -100, 2.0 ** 100, 1.0).double()
    factor = (127 / torch.where(top > 0, top * up, 1.0)).float().double()
    q = torch.round((x.double() * up * factor).float().double())
    return q, (top / 127).float()[:, 0]


def ints(shape, *seed, low=-127):
    return torch.randint(low, 128, shape, generator=gen(*shape, *seed), device=DEV).to(torch.int8)


def check(y, q, s, wq, ws, act=None):
    want = (q.double() @ wq.double().t()) * s.double()[:, None] * ws.double()
    if act == "relu":
        want = want.clamp(min=0)
    off = 3.01 * U * want.abs() + tiniest(torch.float32)
    off = off + half_step(y.dtype) * (want.abs() + off) + tiniest(y.dtype)
    off = torch.where(want == 0, 0.0, off)
    close = (y.double() - want).abs() <= off
    # Rounding to nearest makes an infinity of what lies half a step or more above the type's
    # largest value, most = (2 - eps) 2^e: of most + eps / 2 2^e on (65520 for float16). Which
    # side of it a value within its 32-bit error of it comes to is open.
    info = torch.finfo(y.dtype)
    border = info.max * (1 + info.eps / 2 / (2 - info.eps))
    same = y.double() == torch.copysign(torch.full_like(want, float("inf")), want)
    below, above = want.abs() < border * (1 - 4 * U), want.abs() > border * (1 + 4 * U)
    right = torch.where(below, close, torch.where(above, same, close | same))
    assert bool(right.all()), (y.double() - want)[~right].abs().max()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("f", [1, 3, 4, 7, 8, 9, 64, 128, 129, 250, 256, 385, 512, 601, 1000, 1536, 2048, 4096, 4097,
                               8192, 8193, 16385, 40001])
def test_rows(f, dtype):
    x = randn((21, f), TYPES[dtype]) * torch.exp(2 * randn((21, 1), torch.float32, 2)).to(TYPES[dtype])
    x[4] = 0
    Q, S = agcn.quantize_int(x)
    q, s = quantized(x)
    assert Q.dtype == torch.int8 and Q.shape == (21, f) and S.shape == (21,)
    assert torch.equal(Q.double(), q) and torch.equal(S, s) and S[4] == 0 and not Q[4].any()
    raw = torch.full((21, f + 9), 77, dtype=torch.int8, device=DEV)
    more = torch.full((23,), 77.0, device=DEV)
    got = agcn.quantize_int(padded(x, 3, 1), out=(raw[:, 5:5 + f], more[1:22]))
    assert torch.equal(got[0], Q) and torch.equal(got[1], S) and more[0] == 77 and more[22] == 77
    assert raw[:, :5].eq(77).all() and raw[:, 5 + f:].eq(77).all()


def test_rows_of_every_size_and_not_finite():
    x = randn((16, 300), torch.float32)
    for i, e in enumerate((-149, -140, -127, -126, -120, -101, -100, -99, 0, 100, 126)):
        x[i] = torch.clamp(x[i] / x[i].abs().max(), -1, 1) * 2.0 ** e
    Q, S = agcn.quantize_int(x)
    q, s = quantized(x)
    assert torch.equal(Q.double(), q) and torch.equal(S, s)
    for f in (5, 300, 3000, 40000):
        x = randn((5, f), torch.float32)
        clean = agcn.quantize_int(x)
        x[1, f - 1], x[2, 0], x[3, f // 2] = float("inf"), float("nan"), float("-inf")
        Q, S = agcn.quantize_int(x)
        assert bool(torch.isnan(S[1:4]).all()) and not Q[1:4].any()
        assert torch.equal(Q[::4], clean[0][::4]) and torch.equal(S[::4], clean[1][::4])


def test_halves_go_to_even():
    x = torch.arange(-254, 255, device=DEV).float()[None] / 2
    Q, _ = agcn.quantize_int(x)
    assert torch.equal(Q.float(), torch.round(x))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("lead,fin,fout", [((), 1, 1), ((), 128, 128), ((), 602, 41), ((), 130, 300), ((3,), 65, 129),
                                           ((1,), 16, 8), ((5,), 256, 100), ((), 5000, 64)])
def test_weights(lead, fin, fout, dtype):
    W = randn((*lead, fin, fout), TYPES[dtype])
    WQ, WS = agcn.quantize_weight_int(W)
    assert WQ.shape == (*lead, fout, fin) and WS.shape == (*lead, fout)
    for w, q, s in zip(W.reshape(-1, fin, fout), WQ.reshape(-1, fout, fin), WS.reshape(-1, fout)):
        want = quantized(w.t())
        assert torch.equal(q.double(), want[0]) and torch.equal(s, want[1])
    wide = torch.full((*lead, fin, fout + 3), float("nan"), dtype=TYPES[dtype], device=DEV)
    wide[..., 1:1 + fout] = W
    got = agcn.quantize_weight_int(wide[..., 1:1 + fout])
    assert torch.equal(got[0], WQ) and torch.equal(got[1], WS)


def test_weights_not_finite():
    W = randn((40, 70), torch.float32)
    W[3, 5], W[39, 66] = float("nan"), float("inf")
    WQ, WS = agcn.quantize_weight_int(W)
    bad = torch.isnan(WS)
    assert bad.nonzero().flatten().tolist() == [5, 66] and not WQ[bad].any()


SHAPES = [(1, 1, 1), (1, 4096, 4096), (2, 127, 33), (5, 128, 16), (16, 1000, 100), (17, 256, 300), (33, 2048, 128),
          (48, 8192, 256), (64, 640, 64), (100, 602, 41), (130, 4096, 512), (300, 128, 128), (256, 2048, 2048),
          (1000, 96, 1000), (1024, 2048, 1024), (700, 4096, 700), (3000, 602, 256), (5000, 128, 41), (9000, 256, 16),
          (2048, 1024, 2048), (4100, 640, 4100), (70000, 128, 40), (66000, 1536, 300), (40000, 528, 512)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,fin,fout", SHAPES)
def test_products(n, fin, fout, dtype):
    """Every kernel and tile size; rows that start on 16 bytes and rows that do not."""
    s, ws = randn((1, n), torch.float32, 1)[0].abs(), randn((1, fout), torch.float32, 2)[0].abs()
    q = torch.zeros((n, -(-fin // 16) * 16), dtype=torch.int8, device=DEV)[:, :fin]
    wq = torch.zeros((fout, -(-fin // 16) * 16), dtype=torch.int8, device=DEV)[:, :fin]
    q.copy_(ints((n, fin), 3, low=-128)), wq.copy_(ints((fout, fin), 4, low=-128))
    for act in (None, "relu"):
        y = agcn.int_linear(q, s, wq, ws, dtype=TYPES[dtype], act=act)
        check(y, q, s, wq, ws, act)
        if n * fin * fout < 2 ** 33:
            odd = [padded(v, 1, 1) for v in (q, wq)]
            assert torch.equal(agcn.int_linear(odd[0], s, odd[1], ws, dtype=TYPES[dtype], act=act), y)


@pytest.mark.parametrize("fin", [1, 15, 16, 17, 31, 64, 100, 127, 128, 129, 255, 257, 383, 385, 520, 700, 1100])
def test_ends_of_rows(fin):
    """Bytes behind a row's last value, in the same 16 and in the next row, do not count."""
    for n, fout in ((3, 40), (70, 64), (513, 513), (3000, 520)):
        q = torch.full((n, -(-fin // 16) * 16), 99, dtype=torch.int8, device=DEV)[:, :fin]
        wq = torch.full((fout, -(-fin // 16) * 16), 99, dtype=torch.int8, device=DEV)[:, :fin]
        q.copy_(ints((n, fin), 1)), wq.copy_(ints((fout, fin), 2))
        s, ws = torch.rand(n, device=DEV), torch.rand(fout, device=DEV)
        check(agcn.int_linear(q, s, wq, ws), q, s, wq, ws)


def test_the_largest_sums():
    """fin = 2^17 - 1 values of -128: 2^31 - 2^14, the last sum that 32 bits hold."""
    fin = 2 ** 17 - 1
    for n, fout in ((1, 3), (70, 70), (600, 520)):
        q = torch.full((n, fin), -128, dtype=torch.int8, device=DEV)
        w = torch.full((fout, fin), -128, dtype=torch.int8, device=DEV)
        y = agcn.int_linear(q, torch.ones(n, device=DEV), w, torch.ones(fout, device=DEV))
        assert bool((y == float(2 ** 31 - 2 ** 14)).all())
        y = agcn.int_linear(q, torch.ones(n, device=DEV), -1 - w, torch.ones(fout, device=DEV))
        assert bool((y.double() == -float(fin) * 128 * 127).all() | ((y.double() / (-float(fin) * 128 * 127) - 1).abs() <= U).all())


def offsets_of(sizes, n, first=0):
    at = [first]
    for s in sizes:
        at.append(at[-1] + s)
    assert at[-1] <= n
    return torch.tensor(at, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,fin,fout,sizes,first", [
    (1, 128, 64, [1], 0), (10, 100, 33, [0, 3, 0, 5], 1), (64, 2048, 256, [2] * 16 + [0] * 16, 0),
    (500, 602, 41, [100, 0, 7, 300, 1], 50), (900, 256, 128, [300, 1, 299, 0, 255], 0), (3000, 512, 512, [1200, 700, 900], 100),
    (6000, 128, 128, [100] * 50, 7), (2000, 1024, 300, [13] * 150, 0), (20000, 2048, 512, [9000, 0, 10900], 0),
    (40, 64, 64, [], 0), (30, 64, 64, [0, 0, 0], 0)])
def test_groups(n, fin, fout, sizes, first, dtype):
    e = len(sizes)
    off = offsets_of(sizes, n, first)
    q, wq = ints((n, fin), 1), ints((e, fout, fin), 2)
    s, ws = torch.rand(n, device=DEV), torch.rand((e, fout), device=DEV)
    s[:first] = float("nan")  # rows of no group are 0 whatever they hold
    s[int(off[-1]):] = float("nan")
    pad = torch.zeros((e, fout, -(-fin // 16) * 16), dtype=torch.int8, device=DEV)[..., :fin]
    pad.copy_(wq)
    for w in (wq, pad):
        y = agcn.grouped_int_linear(q, s, w, ws, off, dtype=TYPES[dtype])
        for i in range(e):
            a, b = int(off[i]), int(off[i + 1])
            if b > a:
                check(y[a:b], q[a:b], s[a:b], wq[i], ws[i])
        assert not y[:first].any() and not y[int(off[-1]):].any()


@pytest.mark.parametrize("n,groups,fin,fout", [(20, 64, 130, 300), (60, 40, 500, 70), (60, 40, 512, 1030), (700, 30, 96, 257),
                                               (700, 30, 1000, 515), (700, 30, 1040, 64), (9, 3, 4099, 41), (33, 1, 2050, 4100),
                                               (2000, 33, 640, 128), (40, 1, 300, 50)])
def test_few_rows_of_a_group(n, groups, fin, fout):
    """Short and long rows, on 16 bytes and not: the same sums; some groups have no rows, one most."""
    ids = torch.randint(0, groups, (n // 2,), generator=gen(n, groups), device=DEV) // 2
    sizes = torch.bincount(ids, minlength=groups)
    sizes[groups // 2] += n - n // 2 - 2
    off = offsets_of(sizes.tolist(), n, 1)
    q, wq = ints((n, fin), 1), ints((groups, fout, fin), 2)
    s, ws = torch.rand(n, device=DEV), torch.rand((groups, fout), device=DEV)
    to = -(-fin // 16) * 16
    rows, weights = (torch.full((*v.shape[:-1], to), 99, dtype=torch.int8, device=DEV)[..., :fin] for v in (q, wq))
    rows.copy_(q), weights.copy_(wq)
    y = agcn.grouped_int_linear(rows, s, weights, ws, off)
    for i in range(groups):
        a, b = int(off[i]), int(off[i + 1])
        if b > a:
            check(y[a:b], q[a:b], s[a:b], wq[i], ws[i])
    assert not y[0].any() and not y[int(off[-1]):].any()
    odd = padded(wq.view(-1, fin), 1, 1).unflatten(0, (groups, fout))
    assert torch.equal(agcn.grouped_int_linear(padded(q, 1, 1), s, odd, ws, off), y)
    for bad in (off.flip(0).contiguous(), off * 1000 - 700, off - 5):
        raw = torch.full((n + 2, fout), 7.0, device=DEV)
        agcn.grouped_int_linear(rows, s, weights, ws, bad, out=raw[1:-1])
        agcn.grouped_int_linear(q, s, wq, ws, bad, out=raw[1:-1])
        assert raw[0].eq(7).all() and raw[-1].eq(7).all()


def test_offsets_that_break_the_rules_stay_inside():
    n, fin, fout = 300, 128, 64
    q, wq, s, ws = ints((n, fin), 1), ints((3, fout, fin), 2), torch.rand(n, device=DEV), torch.rand((3, fout), device=DEV)
    for bad in ([0, 200, 100, 300], [-5, 100, 400, 2 ** 31 - 1], [300, 200, 100, 0]):
        raw = torch.full((n + 2, fout), 7.0, device=DEV)
        agcn.grouped_int_linear(q, s, wq, ws, torch.tensor(bad, dtype=torch.int32, device=DEV), out=raw[1:-1])
        assert raw[0].eq(7).all() and raw[-1].eq(7).all()


def test_scales_zero_and_not_a_number():
    for n, fin, fout in ((3, 40, 20), (300, 256, 256), (3000, 602, 300)):
        q, wq = ints((n, fin), 1), ints((fout, fin), 2)
        s, ws = torch.rand(n, device=DEV), torch.rand(fout, device=DEV)
        clean = agcn.int_linear(q, s, wq, ws)
        s[1], s[2], ws[fout - 1] = 0, float("nan"), float("nan")
        y = agcn.int_linear(q, s, wq, ws)
        assert not y[1, :-1].any() and bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[:, -1]).all())
        assert torch.equal(y[3:, :-1], clean[3:, :-1])


def test_empty():
    z = torch.zeros((4, 0), dtype=torch.int8, device=DEV)
    Q, S = agcn.quantize_int(torch.zeros((4, 0), device=DEV))
    assert Q.shape == (4, 0) and not S.any()
    WQ, WS = agcn.quantize_weight_int(torch.zeros((0, 6), device=DEV))
    assert WQ.shape == (6, 0) and not WS.any()
    y = agcn.int_linear(Q, S, WQ, WS, out=torch.full((4, 6), 7.0, device=DEV))
    assert not y.any()
    assert agcn.int_linear(z[:0], S[:0], WQ, WS).shape == (0, 6)
    assert agcn.int_linear(Q, S, WQ[:0], WS[:0]).shape == (4, 0)
