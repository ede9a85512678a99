"""More rows than one launch of the quantiser takes: every launch's first and last rows."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402
from quant_helpers import quantize_rows, scales  # noqa: E402

DEV = "cuda:0"


@pytest.mark.parametrize("f", [2, 300])
def test_more_blocks_than_a_launch(f):
    """2^28 blocks are 2^32 threads, which no launch can have."""
    blocks = (f + 127) // 128
    n = (2 ** 28 + 5000) // blocks
    X = torch.empty((n, f), dtype=torch.float16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(f)
    X.normal_(generator=g)
    Q, S = agcn.quantize(X)
    piece = (2 ** 31 - 1) // 256 * 16 // blocks
    assert piece < n
    for at in [0, *range(piece, n, piece), n]:
        rows = slice(max(0, at - 500), min(n, at + 500))
        q, e = quantize_rows(X[rows].double())
        assert torch.equal(scales(S[rows]), e.to(torch.int32)) and torch.equal(Q[rows].double(), q)
