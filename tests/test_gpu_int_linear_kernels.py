"""Integer products at sizes that reach each of the kernels' shapes for rows on 16 bytes, named beside
the size, on both sides of their partial tiles, with even and odd numbers of blocks of k and an end of k
inside one. The sums are exact, so the results are those of every other kernel bit by bit; rows
that start anywhere go through others."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from routed_helpers import TYPES, gen, padded  # noqa: E402
from test_gpu_int_linear import check, ints, offsets_of  # noqa: E402

DEV = "cuda:0"


def aligned(q):
    """q with rows on 16 bytes and other values behind them."""
    fin = q.shape[-1]
    to = torch.full((*q.shape[:-1], -(-fin // 16) * 16), 99, dtype=torch.int8, device=DEV)[..., :fin]
    return to.copy_(q)


def rand(n, *seed):
    return torch.rand(n, generator=gen(n, *seed), device=DEV) + 0.5


@pytest.mark.parametrize("n,fin,fout", [
    (16300, 1536, 1000),  # 256 x 256, 12 blocks
    (16300, 1664, 1000),  # 13
    (16384, 1700, 1024),  # 14, the last one 36 wide, whole tiles
    (16129, 1580, 769),   # 13, the last one 44 wide; one row and one column in the last tiles
    (99000, 520, 500),    # 256 x 256, narrow outputs: 5, the last one 8 wide
    (98700, 640, 512),    # 5
    (100, 1000, 2000),    # k_qlinear_stream, 32 x 32, blocks dealt to four waves
    (100, 2100, 2000),
    (1100, 4096, 1100),   # k_qlinear_stream, 64 x 64, two workgroups a compute unit
    (1100, 4200, 1050),
    (40000, 600, 16),     # 128 x 32
    (33000, 128, 31),
    (1100, 600, 1100),    # 64 x 64
    (70001, 300, 50)])    # 128 x 64
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_products(n, fin, fout, dtype):
    q, wq, s, ws = ints((n, fin), 1, low=-128), ints((fout, fin), 2, low=-128), rand(n, 3), rand(fout, 4)
    a, w = aligned(q), aligned(wq)
    odd = padded(q, 1, 1), padded(wq, 1, 1)
    for act in (None, "relu"):
        y = agcn.int_linear(a, s, w, ws, dtype=TYPES[dtype], act=act)
        check(y, q, s, wq, ws, act)
        assert torch.equal(agcn.int_linear(odd[0], s, odd[1], ws, dtype=TYPES[dtype], act=act), y)


@pytest.mark.parametrize("n,fin,fout,sizes,first", [
    (40000, 1536, 512, [13000, 0, 25000], 100),  # 256 x 256, 12 blocks
    (40000, 1700, 500, [256, 12544, 27000], 0),  # 14, the last one 36 wide
    (36000, 1580, 700, [1, 17000, 18999], 0),    # 13, the last one 44 wide
    (1000, 2048, 128, [600, 399], 1),            # k_qlinear_stream, 32 x 32, few outputs
    (1000, 2500, 100, [31, 0, 960], 3),
    (1660, 4200, 141, [400, 0, 900, 1, 300], 0),  # 128 x 128, a long k
    (40000, 600, 16, [15000, 1, 24000], 5),      # 128 x 32
    (40000, 600, 60, [15000, 127, 24000], 5)])   # 128 x 64
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_groups(n, fin, fout, sizes, first, dtype):
    e, off = len(sizes), offsets_of(sizes, n, first)
    q, wq, s, ws = ints((n, fin), 1, low=-128), ints((e, fout, fin), 2, low=-128), rand(n, 3), rand(e * fout, 4).view(e, fout)
    a, w = aligned(q), aligned(wq)
    odd = padded(q, 1, 1), padded(wq.view(-1, fin), 1, 1).unflatten(0, (e, fout))
    for act in (None, "relu"):
        y = agcn.grouped_int_linear(a, s, w, ws, off, dtype=TYPES[dtype], act=act)
        for i in range(e):
            f, t = int(off[i]), int(off[i + 1])
            if t > f:
                check(y[f:t], q[f:t], s[f:t], wq[i], ws[i], act)
        assert not y[:first].any() and not y[int(off[-1]):].any()
        assert torch.equal(agcn.grouped_int_linear(odd[0], s, odd[1], ws, off, dtype=TYPES[dtype], act=act), y)


@pytest.mark.parametrize("fin", [1536, 1664])
def test_the_least_sums_in_the_largest_tiles(fin):
    """Sums of products of one sign, as far from 0 as that many values allow: exact in 32 bits."""
    n, fout = 16300, 1000
    q = torch.full((n, fin), -128, dtype=torch.int8, device=DEV)
    w = torch.full((fout, fin), 127, dtype=torch.int8, device=DEV)
    y = agcn.int_linear(q, torch.ones(n, device=DEV), w, torch.ones(fout, device=DEV))
    assert bool((y == -128.0 * 127 * fin).all())


def test_rows_far_apart():
    """Strides that a tile's 32-bit offsets cannot hold, both sides; as the rows close together."""
    for n, fin, fout in ((20, 300, 40), (3, 1100, 20), (40, 129, 17)):
        q, wq, s, ws = ints((n, fin), 1, low=-128), ints((fout, fin), 2, low=-128), rand(n, 3), rand(fout, 4)
        far = torch.zeros((max(n, fout), 9_000_000), dtype=torch.int8, device=DEV)
        a, w = far[:n, :fin].copy_(q), far[:fout, 5_000_000:5_000_000 + fin].copy_(wq)
        for dtype in TYPES.values():
            y = agcn.int_linear(a, s, w, ws, dtype=dtype)
            check(y, q, s, wq, ws)
            assert torch.equal(agcn.int_linear(aligned(q), s, aligned(wq), ws, dtype=dtype), y)
