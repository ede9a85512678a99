"""How many bits the sums of the 8-bit products keep, where sums cancel.

float32 and float16 outputs: products of e4m3 values are exact in bfloat16's matrix
instruction, and a block of 128 k is four of its steps, each of which cuts off what
falls below the last bit of what it adds (32 products and the accumulator, at most
33 * 2^-23 of the step's sum of magnitudes), then one rounding per block. So a result is
within (4 * 33 + blocks) * 2^-23 * S of the exact sum, S = |A| |W|^T, and float16 rounds
that once, by 2^-11 of it or 2^-25."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from quant_helpers import TYPES, values, weight_values  # noqa: E402

DEV = "cuda:0"


def _cancelling(n, fin, fout, groups=None):
    """Of every eight columns two cancel and six are 2^-14 of them: sums that keep 13
    bits below the largest of eight products lose all but the two."""
    g = torch.Generator(device=DEV).manual_seed(n + fin + fout)
    a = 1 + torch.rand((n, fin), generator=g, device=DEV)
    w = 1 + torch.rand((groups or 1, fin, fout), generator=g, device=DEV)
    k = torch.arange(fin, device=DEV)
    pairs = fin // 8 * 8
    first, second = (k % 8 == 0) & (k < pairs), (k % 8 == 1) & (k < pairs)
    a[:, first] *= 64
    a[:, second] = -a[:, first]
    w[:, first] *= 64
    w[:, second] = w[:, first]
    a[:, ~(first | second)] /= 2
    w[:, ~(first | second)] /= 2
    return agcn.quantize(a), agcn.quantize_weight(w if groups else w[0])


def _check(got, A, W, fin, dtype):
    Y, S = A @ W.t(), A.abs() @ W.abs().t()
    off = (4 * 33 + (fin + 127) // 128) * 2.0 ** -23 * S
    if dtype == "float16":
        off = off + 2.0 ** -11 * (Y.abs() + off) + 2.0 ** -25
    err = (got.double() - Y).abs() - off
    assert float(err.max()) <= 0.0, float(err.max())


def _odd(q):
    *lead, n, f = q.shape
    raw = torch.zeros((*lead, n, f + 5), dtype=torch.uint8, device=DEV)
    raw[..., 3:f + 3] = q.contiguous().view(torch.uint8)
    return raw.view(torch.float8_e4m3fn)[..., 3:f + 3]


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("n,fin,fout", [
    (1, 1024, 64), (16, 128, 32), (40, 2048, 200), (200, 2048, 300), (300, 257, 100), (2000, 602, 41),
    (700, 4200, 800), (40_000, 256, 128), (40_000, 130, 300), (50_000, 128, 24), (8192, 1664, 2048)])
def test_sums_that_cancel(n, fin, fout, dtype):
    (Q, S), (WQ, WS) = _cancelling(n, fin, fout)
    A, W = values(Q, S), weight_values(WQ, WS)
    for layout in ((lambda q: q), _odd):
        print(f"[sums] {n} x {fin} -> {fout} {dtype}", flush=True)
        _check(agcn.quantized_linear(layout(Q), S, layout(WQ), WS, dtype=TYPES[dtype]), A, W, fin, dtype)


@pytest.mark.parametrize("dtype", ["float32", "float16"])
@pytest.mark.parametrize("n,fin,fout,groups", [(40, 512, 64, 8), (300, 640, 130, 7), (9000, 384, 300, 4)])
def test_grouped_sums_that_cancel(n, fin, fout, groups, dtype):
    (Q, S), (WQ, WS) = _cancelling(n, fin, fout, groups)
    ends = [n * i // groups for i in range(groups + 1)]
    off = torch.tensor(ends, dtype=torch.int32, device=DEV)
    for layout in ((lambda q: q), _odd):
        print(f"[sums] {n} x {fin} -> {fout} groups {groups} {dtype}", flush=True)
        got = agcn.grouped_linear(layout(Q), S, layout(WQ), WS, off, dtype=TYPES[dtype])
        for e, (a, b) in enumerate(zip(ends, ends[1:])):
            _check(got[a:b], values(Q[a:b], S[a:b]), weight_values(WQ[e], WS[e]), fin, dtype)
