"""Grouped products over more groups than are looked through one after another: every
row against its own group's weight in 64 bits, with the bounds of
test_gpu_quantized_linear.py for float32."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from quant_helpers import values, weight_values  # noqa: E402

DEV = "cuda:0"


def _offsets(n, groups, kind):
    g = torch.Generator().manual_seed(n + groups)
    if kind == "spread":
        off = torch.randint(0, n + 1, (groups + 1,), generator=g).sort().values
    elif kind == "even":
        off = torch.arange(groups + 1) * n // groups
    else:  # all rows in one group, which starts past the first rows
        off = torch.full((groups + 1,), n // 10)
        off[groups // 3:] = n
    return off.to(torch.int32).to(DEV)


@pytest.mark.parametrize("n,fin,fout,groups", [
    (19_000, 200, 70, 126), (19_000, 200, 70, 127), (19_000, 200, 200, 300), (70_000, 64, 130, 1000),
    (3000, 32, 8, 40_000), (5000, 32, 8, 70_000), (200_000, 32, 8, 70_000), (1, 32, 8, 70_000)])
@pytest.mark.parametrize("kind", ["spread", "even", "one"])
def test_many_groups(n, fin, fout, groups, kind):
    g = torch.Generator(device=DEV).manual_seed(n + groups)
    Q, S = agcn.quantize(torch.randn((n, fin), generator=g, device=DEV))
    WQ, WS = agcn.quantize_weight(torch.randn((groups, fin, fout), generator=g, device=DEV))
    off = _offsets(n, groups, kind)
    print(f"[groups] {n} x {fin} -> {fout} over {groups} {kind}", flush=True)
    out = torch.full((n + 2, fout), 7.0, device=DEV)
    got = agcn.grouped_linear(Q, S, WQ, WS, off, out=out[1:n + 1])
    rows = torch.arange(n, device=DEV)
    group = torch.searchsorted(off[1:].long(), rows, right=True).clamp(max=groups - 1)
    used = (rows >= off[0]) & (rows < off[-1])
    A = values(Q, S)
    for at in range(0, n, 4000):
        part = slice(at, at + 4000)
        W = weight_values(WQ[group[part]], WS[group[part]])
        Y = (W * A[part, None]).sum(-1) * used[part, None]
        T = (W.abs() * A[part, None].abs()).sum(-1)
        bound = (4 * 33 + (fin + 127) // 128) * 2.0 ** -23 * T + 1e-37
        assert bool(((got[part].double() - Y).abs() <= bound).all())
    assert got[~used].eq(0).all() and out[0].eq(7).all() and out[n + 1].eq(7).all()
