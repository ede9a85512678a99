"""Products of matrices in 8 bits against 64 bits.

Bounds per element, with S = |A| |W|^T in 64 bits:

* float32: products of e4m3 values are exact; a block of 128 k is four steps of
  the bf16 matrix instruction, which cuts off what falls below the last bit of what
  it adds (32 products and the accumulator: at most 33 * 2^-23 of the block's S per
  step), then one rounding per block: (4 * 33 + blocks) * 2^-23 * S.
* 16-bit types: the 8-bit instruction keeps 13 bits or more below the largest
  product it adds at a time (7.7e-5 S the worst measured on random bit patterns): 2^-12 S,
  and half a unit of the type's last place, 2^-8 (bfloat16) or 2^-11 (float16) of the
  result."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from quant_helpers import TYPES, values, weight_values  # noqa: E402

DEV = "cuda:0"


def _gen(*seed):
    s = 0
    for x in seed:
        s = s * 1000003 + int(x)
    return torch.Generator(device=DEV).manual_seed(s % (1 << 40))


def _rows(n, f, seed=0):
    g = _gen(n, f, seed)
    x = torch.randn((n, f), generator=g, device=DEV)
    return agcn.quantize(x * torch.exp(torch.randn((n, 1), generator=g, device=DEV)))


def _weight(fin, fout, lead=(), seed=0):
    g = _gen(fin, fout, seed)
    w = torch.randn((*lead, fin, fout), generator=g, device=DEV)
    return agcn.quantize_weight(w * torch.exp(torch.randn((*lead, fin, 1), generator=g, device=DEV)))


def _layout(q, kind):
    """q as its quantiser lays it out, with packed rows, or off any alignment."""
    if kind == "packed":
        return q.contiguous()
    if kind == "odd":
        *lead, n, f = q.shape
        raw = torch.full((*lead, n, f + 5), 0x7f, dtype=torch.uint8, device=DEV)  # NaN around it
        raw[..., 3:f + 3] = q.contiguous().view(torch.uint8)
        return raw.view(torch.float8_e4m3fn)[..., 3:f + 3]
    if kind == "padded":  # rows on 16 bytes, NaN in the padding
        *lead, n, f = q.shape
        raw = torch.full((*lead, n, (f + 15) // 16 * 16 + 16), 0x7f, dtype=torch.uint8, device=DEV)
        raw[..., :f] = q.contiguous().view(torch.uint8)
        return raw.view(torch.float8_e4m3fn)[..., :f]
    return q


def _bound(Y, S, dtype, fin):
    if dtype == "float32":
        return (4 * 33 + (fin + 127) // 128) * 2.0 ** -23 * S + 1e-37
    half = 2.0 ** -8 if dtype == "bfloat16" else 2.0 ** -11
    tiny = 1e-37 if dtype == "bfloat16" else 2.0 ** -25  # float16's subnormals
    return 2.0 ** -12 * S * (1 + half) + half * Y.abs() + tiny


def _check(got, A, W, dtype, act, fin):
    Y, S = A @ W.t(), A.abs() @ W.abs().t()
    if act == "relu":
        Y = Y.clamp(min=0)
    err = (got.double() - Y).abs() - _bound(Y, S, dtype, fin)
    assert got.dtype == TYPES[dtype] and got.shape == Y.shape
    assert float(err.max() if err.numel() else 0.0) <= 0.0, float(err.max())  # NaN fails too


_SIZES = [
    (1, 1, 1), (1, 128, 16), (1, 4096, 300), (2, 41, 3), (3, 129, 41), (15, 600, 130), (16, 128, 128),
    (17, 1000, 64), (33, 256, 17), (48, 2048, 160), (63, 15, 65), (64, 8192, 32), (65, 128, 127),
    (100, 500, 500), (128, 384, 256), (129, 130, 129), (200, 4096, 48), (255, 640, 256),
    (257, 513, 300), (300, 3000, 1000), (513, 1024, 1030), (1000, 128, 16), (1025, 70, 8),
    (2000, 602, 41), (4097, 128, 64), (5000, 256, 257), (10000, 100, 100), (300, 16, 5000),
    (2049, 1100, 2050), (70000, 64, 40), (4500, 257, 4400)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,fin,fout", _SIZES)
def test_linear(n, fin, fout, dtype):
    Q, S = _rows(n, fin)
    WQ, WS = _weight(fin, fout)
    A, W = values(Q, S), weight_values(WQ, WS)
    for kind, act in (("own", None), ("padded", "relu"), ("packed", None), ("odd", "relu")):
        print(f"[linear] {n} x {fin} -> {fout} {dtype} {kind}", flush=True)
        got = agcn.quantized_linear(_layout(Q, kind), S, _layout(WQ, kind), WS, dtype=TYPES[dtype],
                                    act=act)
        _check(got, A, W, dtype, act, fin)


def test_default_type_and_out():
    Q, S = _rows(40, 200)
    WQ, WS = _weight(200, 50)
    Y = agcn.quantized_linear(Q, S, WQ, WS)
    assert Y.dtype == torch.float32
    raw = torch.full((40, 61), 7.0, device=DEV)
    out = raw[:, 3:53]
    assert agcn.quantized_linear(Q, S, WQ, WS, out=out) is out
    assert torch.equal(out, Y) and raw[:, :3].eq(7).all() and raw[:, 53:].eq(7).all()
    half = torch.empty((40, 50), dtype=torch.float16, device=DEV)
    agcn.quantized_linear(Q, S, WQ, WS, out=half)
    assert torch.equal(half, agcn.quantized_linear(Q, S, WQ, WS, dtype=torch.float16))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,fin,fout", [(3, 300, 70), (130, 300, 150), (700, 512, 600), (5000, 200, 300)])
def test_not_finite(n, fin, fout, dtype):
    """NaN in a row of A, in a row of W or as a scale reaches the outputs it belongs to
    and no others; ReLU keeps it."""
    Q, S = _rows(n, fin)
    WQ, WS = _weight(fin, fout)
    A, W = values(Q, S), weight_values(WQ, WS)
    Q.view(torch.uint8)[n - 2, 5] = 0x7f
    WQ.view(torch.uint8)[fout - 1, fin - 1] = 0xff
    S.view(torch.uint8)[0, 1] = 255
    got = agcn.quantized_linear(Q, S, WQ, WS, dtype=TYPES[dtype], act="relu")
    nan = torch.zeros((n, fout), dtype=torch.bool, device=DEV)
    nan[n - 2], nan[0], nan[:, fout - 1] = True, True, True
    assert torch.equal(torch.isnan(got), nan)
    rest = torch.arange(1, n, device=DEV)[torch.arange(1, n, device=DEV) != n - 2]
    _check(got[rest][:, :fout - 1], A[rest], W[:fout - 1], dtype, "relu", fin)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,fout", [(20, 40), (300, 300)])
def test_scales_of_any_size(n, fout, dtype):
    """Scales whose product is in range although neither is near 1, and blocks whose
    values vanish beside the others'."""
    fin = 384
    Q, S = _rows(n, fin)
    WQ, WS = _weight(fin, fout)
    S.view(torch.uint8)[:, 0] = 5
    WS.view(torch.uint8)[:, 0] = 245
    S.view(torch.uint8)[:, 1] = 240
    WS.view(torch.uint8)[:, 1] = 2
    got = agcn.quantized_linear(Q, S, WQ, WS, dtype=TYPES[dtype])
    _check(got, values(Q, S), weight_values(WQ, WS), dtype, None, fin)


def test_no_columns_gives_zero():
    Q, S = _rows(20, 0)
    WQ, WS = _weight(0, 30)
    assert agcn.quantized_linear(Q, S, WQ, WS).eq(0).all()
    off = torch.tensor([0, 20], dtype=torch.int32, device=DEV)
    assert agcn.grouped_linear(Q, S, WQ[None], WS[None], off, dtype=torch.float16).eq(0).all()
    Q, S = _rows(0, 30)
    WQ, WS = _weight(30, 10)
    assert agcn.quantized_linear(Q, S, WQ, WS).shape == (0, 10)
    Q, S = _rows(5, 30)
    WQ, WS = _weight(30, 0)
    assert agcn.quantized_linear(Q, S, WQ, WS).shape == (5, 0)


# --- grouped ------------------------------------------------------------------------------


def _check_grouped(n, fin, fout, offsets, dtype, act=None, kind="own", seed=0):
    groups = len(offsets) - 1
    Q, S = _rows(n, fin, seed)
    WQ, WS = _weight(fin, fout, (groups,), seed)
    off = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    print(f"[grouped] {n} x {fin} -> {fout} groups {groups} {dtype} {kind}", flush=True)
    got = agcn.grouped_linear(_layout(Q, kind), S, _layout(WQ, kind), WS, off, dtype=TYPES[dtype],
                              act=act)
    assert got[:offsets[0]].eq(0).all() and got[offsets[-1]:].eq(0).all()
    for e in range(groups):
        a, b = offsets[e], offsets[e + 1]
        if b > a:
            _check(got[a:b], values(Q[a:b], S[a:b]), weight_values(WQ[e], WS[e]), dtype, act, fin)


def _offsets(n, groups, empty, seed, first=0, spare=0):
    g = torch.Generator().manual_seed(seed)
    share = torch.rand(groups, generator=g) ** 2 + 0.05
    share[torch.randperm(groups, generator=g)[:empty]] = 0
    rows = n - first - spare
    sizes = torch.bincount(torch.multinomial(share, rows, replacement=True, generator=g),
                           minlength=groups) if rows else torch.zeros(groups, dtype=torch.int64)
    return [first] + (first + sizes.cumsum(0)).tolist()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,fin,fout,groups,empty,first,spare", [
    (1, 128, 32, 4, 3, 0, 0), (7, 41, 9, 3, 1, 0, 2), (64, 2048, 100, 32, 4, 0, 5),
    (64, 256, 64, 64, 0, 0, 0), (300, 602, 41, 7, 1, 3, 0), (500, 128, 128, 1, 0, 0, 0),
    (1000, 300, 257, 5, 2, 17, 30), (1500, 640, 300, 200, 50, 0, 0), (4000, 130, 200, 3, 0, 0, 0),
    (6000, 512, 513, 20, 3, 100, 100), (20000, 128, 64, 6, 0, 0, 7), (9000, 1024, 1100, 4, 1, 0, 0)])
def test_grouped(n, fin, fout, groups, empty, first, spare, dtype):
    off = _offsets(n, groups, empty, n + groups, first, spare)
    for kind, act in (("own", None), ("odd", "relu"), ("padded", None)):
        _check_grouped(n, fin, fout, off, dtype, act, kind)


def test_groups_that_end_inside_and_at_tiles():
    for dtype in ("float32", "bfloat16"):
        _check_grouped(600, 200, 130, [0, 1, 1, 16, 32, 33, 64, 128, 129, 256, 257, 512, 600], dtype)
        _check_grouped(600, 200, 130, [0, 0, 600, 600, 600], dtype)
        _check_grouped(40, 200, 130, [40, 40, 40], dtype)
        _check_grouped(40, 200, 130, [0, 0, 0], dtype)
        _check_grouped(40, 200, 130, [0], dtype)


def test_equal_to_the_single_product_where_there_is_one_group():
    for n, fin, fout in [(30, 500, 70), (3000, 500, 300)]:
        Q, S = _rows(n, fin)
        WQ, WS = _weight(fin, fout)
        off = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        for dtype in sorted(TYPES):
            A, W = values(Q, S), weight_values(WQ, WS)
            got = agcn.grouped_linear(Q, S, WQ[None], WS[None], off, dtype=TYPES[dtype])
            _check(got, A, W, dtype, None, fin)


def test_one_weight_shared_by_all_groups():
    """A group stride of 0."""
    Q, S = _rows(100, 300)
    WQ, WS = _weight(300, 40)
    off = torch.tensor([0, 30, 31, 100], dtype=torch.int32, device=DEV)
    got = agcn.grouped_linear(Q, S, WQ.expand(3, -1, -1), WS.expand(3, -1, -1), off)
    _check(got, values(Q, S), weight_values(WQ, WS), "float32", None, 300)


@pytest.mark.parametrize("offsets", [[5, 3, 60, 20], [-7, 10, 10, 500], [200, 300, 400, 500],
                                     [-2 ** 31, 2 ** 31 - 1, -5, 40]])
@pytest.mark.parametrize("n,fout", [(50, 40), (700, 300)])
def test_offsets_out_of_range_stay_inside_the_output(offsets, n, fout):
    """Clamped to the rows: nothing outside Y is written."""
    Q, S = _rows(n, 256)
    WQ, WS = _weight(256, fout, (3,))
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV).to(torch.int32)
    for dtype in sorted(TYPES):
        raw = torch.full((n + 20, fout + 6), 7.0, device=DEV, dtype=TYPES[dtype])
        agcn.grouped_linear(Q, S, WQ, WS, off, out=raw[10:n + 10, 3:fout + 3])
        raw[10:n + 10, 3:fout + 3] = 7.0
        assert raw.eq(7.0).all()


def test_spans_past_4_gib():
    """Row offsets past 32 bits in A, in the groups' weights and in Y."""
    n, fin, fout = 70_000, 130, 24
    Q, S = _rows(n, fin)
    raw = torch.empty((n, 65_000), dtype=torch.uint8, device=DEV)
    far = raw.view(torch.float8_e4m3fn)[:, 64:64 + fin]
    far.copy_(Q)
    WQ, WS = _weight(fin, fout, (2,))
    Y = torch.empty((n, 20_000), device=DEV)[:, 8:8 + fout]
    off = torch.tensor([0, 69_000, n], dtype=torch.int32, device=DEV)
    agcn.grouped_linear(far, S, WQ, WS, off, out=Y)
    _check(Y[69_000:], values(Q[69_000:], S[69_000:]), weight_values(WQ[1], WS[1]), "float32", None,
           fin)
    agcn.quantized_linear(far, S, WQ[0], WS[0], out=Y)
    _check(Y[-500:], values(Q[-500:], S[-500:]), weight_values(WQ[0], WS[0]), "float32", None, fin)
    big = raw.view(-1)[:2 * 2_200_000_000].view(2, -1)[:, :fout * 144].view(2, fout, 144)
    big = big.view(torch.float8_e4m3fn)[..., :fin]
    big.copy_(WQ)
    agcn.grouped_linear(Q, S, big, WS, off, out=Y)
    _check(Y[69_000:], values(Q[69_000:], S[69_000:]), weight_values(WQ[1], WS[1]), "float32", None,
           fin)


def test_same_bits_every_time_on_any_stream_and_in_a_graph():
    Q, S = _rows(777, 1500)
    WQ, WS = _weight(1500, 300, (3,))
    off = torch.tensor([0, 100, 101, 700], dtype=torch.int32, device=DEV)
    one = [agcn.grouped_linear(Q, S, WQ, WS, off, dtype=t) for t in TYPES.values()]
    two = [agcn.quantized_linear(Q, S, WQ[1], WS[1], dtype=t) for t in TYPES.values()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t, a, b in zip(TYPES.values(), one, two):
        x = agcn.grouped_linear(Q, S, WQ, WS, off, dtype=t, stream=side)
        y = agcn.quantized_linear(Q, S, WQ[1], WS[1], dtype=t, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(x, a) and torch.equal(y, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = agcn.grouped_linear(Q, S, WQ, WS, off, dtype=torch.bfloat16)
        cap2 = agcn.quantized_linear(Q, S, WQ[1], WS[1])
    for ends in ([0, 0, 400, 777], [50, 60, 70, 80], [0, 777, 777, 777]):
        off.copy_(torch.tensor(ends, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(cap, agcn.grouped_linear(Q, S, WQ, WS, off, dtype=torch.bfloat16))
        assert torch.equal(cap2, agcn.quantized_linear(Q, S, WQ[1], WS[1]))


def test_refusals():
    Q, S = _rows(20, 200)
    WQ, WS = _weight(200, 130)
    W3, S3 = WQ.expand(2, -1, -1), WS.expand(2, -1, -1)
    off = torch.tensor([0, 5, 20], dtype=torch.int32, device=DEV)
    out = torch.empty((20, 130), device=DEV)
    for call in (lambda: agcn.quantized_linear(Q, S, WQ[:, :128], WS), lambda: agcn.quantized_linear(S, Q, WQ, WS),
                 lambda: agcn.quantized_linear(Q.float(), S, WQ, WS),
                 lambda: agcn.quantized_linear(Q, S[:, :1], WQ, WS),
                 lambda: agcn.quantized_linear(Q, S, WQ, WS[:1]),
                 lambda: agcn.quantized_linear(Q, S, W3, S3),
                 lambda: agcn.quantized_linear(Q, S, WQ, WS, dtype=torch.float64),
                 lambda: agcn.quantized_linear(Q, S, WQ, WS, act="gelu"),
                 lambda: agcn.quantized_linear(Q, S, WQ, WS, out=out[:, :100]),
                 lambda: agcn.quantized_linear(Q, S, WQ, WS, out=out, dtype=torch.float16),
                 lambda: agcn.quantized_linear(Q, S, WQ, WS, out=out.double()),
                 lambda: agcn.quantized_linear(Q, S, WQ, WS, out=out.cpu()),
                 lambda: agcn.quantized_linear(Q, S.cpu(), WQ, WS),
                 lambda: agcn.grouped_linear(Q, S, WQ, WS, off),
                 lambda: agcn.grouped_linear(Q, S, W3, S3, off[:2]),
                 lambda: agcn.grouped_linear(Q, S, W3, S3, off.long()),
                 lambda: agcn.grouped_linear(Q, S, W3, S3, off.cpu()),
                 lambda: agcn.grouped_linear(Q, S, W3, S3[:1], off)):
        with pytest.raises((TypeError, ValueError)):
            call()


# --- each way through the sizes -----------------------------------------------------------


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("n,fin,fout", [
    (8200, 1100, 1100), (4200, 1030, 2100), (8192, 1280, 1024), (6000, 1160, 1500),  # 256 x 256 tiles:
    # whole and partial last blocks of k after odd and even numbers, partial row and column tiles
    (10000, 200, 1000), (3900, 130, 700), (1500, 200, 1000), (40000, 200, 30),   # smaller tiles
    (1000, 300, 1000), (1100, 4100, 1200), (500, 1000, 1000), (130, 2000, 900),    # k split over waves
    (20, 10000, 700)])
def test_every_tile_shape(n, fin, fout, dtype):
    Q, S = _rows(n, fin, seed=3)
    WQ, WS = _weight(fin, fout, seed=3)
    A, W = values(Q, S), weight_values(WQ, WS)
    for kind, act in (("padded", "relu"), ("own", None), ("odd", None)):
        print(f"[linear] {n} x {fin} -> {fout} {dtype} {kind}", flush=True)
        raw = torch.full((n + 2, fout + 3), 7.0, dtype=TYPES[dtype], device=DEV)
        got = agcn.quantized_linear(_layout(Q, kind), S, _layout(WQ, kind), WS, act=act,
                                    out=raw[1:n + 1, 2:fout + 2])
        _check(got, A, W, dtype, act, fin)
        raw[1:n + 1, 2:fout + 2] = 7.0
        assert raw.eq(7.0).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,fin,fout", [
    (4090, 1700, 4000), (8300, 1550, 2050), (8192, 1664, 2048), (200_000, 600, 250),  # 256 x 256
    (40_000, 100, 300), (40_000, 16, 100), (40_000, 256, 128), (40_000, 270, 200),  # 128 x 128
    (900, 3000, 1000), (4000, 250, 250)])  # few: k split over waves, a short k not
def test_large_tiles(n, fin, fout, dtype):
    """Whole and partial last blocks of k after odd and even numbers of blocks, one block
    alone, partial row and column tiles."""
    Q, S = _rows(n, fin, seed=5)
    WQ, WS = _weight(fin, fout, seed=5)
    A, W = values(Q, S), weight_values(WQ, WS)
    for act in (None, "relu"):
        print(f"[linear] {n} x {fin} -> {fout} {dtype} {act}", flush=True)
        raw = torch.full((n + 2, fout + 3), 7.0, dtype=TYPES[dtype], device=DEV)
        got = agcn.quantized_linear(_layout(Q, "padded"), S, _layout(WQ, "padded"), WS, act=act,
                                    out=raw[1:n + 1, 2:fout + 2])
        _check(got, A, W, dtype, act, fin)
        raw[1:n + 1, 2:fout + 2] = 7.0
        assert raw.eq(7.0).all()


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_large_tiles_of_groups(dtype):
    off = [0, 0, 4000, 4000, 4003, 7900, 7900, 11_990]
    _check_grouped(12_000, 1600, 1600, off, dtype, kind="padded", act="relu")
    _check_grouped(12_000, 1540, 1601, off, dtype, kind="padded")
    _check_grouped(12_000, 90, 700, off, dtype, kind="padded")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_groups_of_very_different_sizes(dtype):
    """All rows in one of many groups, where the average group has few; many groups of
    one row among large ones; large groups beside empty ones."""
    for n, fin, fout, groups in [(300, 256, 100, 100), (900, 640, 130, 40), (5000, 128, 70, 600)]:
        for at in (0, groups // 2, groups - 1):
            off = [0] * (at + 1) + [n] * (groups - at)
            _check_grouped(n, fin, fout, off, dtype, kind="own")
            _check_grouped(n, fin, fout, off, dtype, kind="odd", act="relu")
    sizes = [1] * 70 + [700] + [0] * 5 + [65, 64, 63, 16, 17, 15, 32, 33] + [1] * 50
    off = [3]
    for size in sizes:
        off.append(off[-1] + size)
    _check_grouped(off[-1] + 9, 300, 100, off, dtype)
    off = [0, 0, 4000, 4000, 4003, 7900, 7900, 12000]
    _check_grouped(12000, 1100, 1100, off, dtype, kind="padded")
    _check_grouped(12000, 1100, 1100, off, dtype, kind="odd", act="relu")


def test_more_groups_than_a_grid_has_rows():
    groups, fin, fout = 66_000, 32, 8
    Q, S = _rows(groups, fin)
    WQ, WS = _weight(fin, fout, (groups,))
    off = torch.arange(groups + 1, dtype=torch.int32, device=DEV)
    got = agcn.grouped_linear(Q, S, WQ, WS, off)
    A, W = values(Q, S), weight_values(WQ, WS)
    Y, T = (W @ A[:, :, None])[..., 0], (W.abs() @ A.abs()[:, :, None])[..., 0]
    assert bool(((got.double() - Y).abs() <= _bound(Y, T, "float32", fin)).all())


def test_every_scale_code():
    """Codes 0 to 255 of A with 254 - code of W: the product of the scales is 1, and NaN
    with 255. Values that bf16 holds (down to 2^-133) come out exactly scaled."""
    code = torch.arange(256, device=DEV)
    Q = torch.full((256, 128), 1.5, device=DEV).to(torch.float8_e4m3fn)
    S = code.to(torch.uint8)[:, None].contiguous().view(torch.float8_e8m0fnu)
    WQ = torch.zeros((256 * 128, 128), device=DEV)
    WQ[::128, 7] = 1
    WQ = WQ.to(torch.float8_e4m3fn)
    WS = (254 - code).clamp(min=0).to(torch.uint8)[:, None].contiguous().view(torch.float8_e8m0fnu)
    for dtype in ("float32", "bfloat16"):
        Y = agcn.quantized_linear(Q, S, WQ, WS, dtype=TYPES[dtype])[:, ::128]
        d = Y.diagonal()
        assert d[:255].float().eq(1.5).all() and torch.isnan(d[255])
        assert torch.isnan(Y[255]).all()


def test_rows_of_zeros_beside_others():
    """Blocks of zeros have the least scale."""
    x = torch.randn((300, 256), generator=_gen(5), device=DEV)
    x[::7] = 0
    x[3, 128:] = 0
    Q, S = agcn.quantize(x)
    WQ, WS = _weight(256, 90)
    for dtype in sorted(TYPES):
        got = agcn.quantized_linear(Q, S, WQ, WS, dtype=TYPES[dtype])
        assert got[::7].eq(0).all()
        _check(got, values(Q, S), weight_values(WQ, WS), dtype, None, 256)
