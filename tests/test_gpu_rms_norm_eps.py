"""rms_norm with an eps near float32's largest value: the mean of the squares plus eps may
overflow although either is in range, and rows whose squares overflow still add eps.
Bounds as in test_gpu_quantize.py: the norm's relative error is at most
(f / 8 + 16) * 2^-24, and a quantised value then is a neighbour."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from quant_helpers import power, row_blocks, scales, step  # noqa: E402

DEV = "cuda:0"


@pytest.mark.parametrize("f", [4, 300, 3000, 9000, 40000])
@pytest.mark.parametrize("eps", [1e-6, 1e30, 1e38, 3e38])
def test_large_eps(f, eps):
    gen = torch.Generator(device=DEV).manual_seed(f)
    X = 1 + torch.rand((6, f), generator=gen, device=DEV)
    X *= torch.tensor([1.0, 1e15, 1e18, 1e19, 2e19, 1e20], device=DEV)[:, None]
    g = torch.rand(f, generator=gen, device=DEV) + 0.5
    Q, S = agcn.rms_norm(X, g, eps=eps)
    h, eps = X.double(), float(torch.tensor(eps, dtype=torch.float32))
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * g.double()
    rel = (f / 8 + 16) * 2.0 ** -24
    v = (row_blocks(y) * power(-scales(S).long())[..., None]).reshape(6, -1)[:, :f]
    q = Q.double()
    off = (q - v).abs() - 0.5 * torch.maximum(step(q), step(v)) - rel * v.abs()
    assert float(off.max()) <= 1e-12, float(off.max())
    assert bool((row_blocks(v).abs().amax(-1) > 200).all())  # each block's scale is the least
