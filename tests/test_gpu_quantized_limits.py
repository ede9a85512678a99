"""Sizes that the library counts in 32 bits are refused by the Python functions, not cut
to their lower half."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2308_11825_amd as agcn  # noqa: E402

DEV = "cuda:0"
WIDE = 2 ** 32 + 8


def test_rows_of_over_2_31_columns():
    X = torch.empty((1, WIDE), dtype=torch.float16, device=DEV)
    for call in (lambda: agcn.quantize(X), lambda: agcn.rms_norm(X, X[0])):
        with pytest.raises(ValueError):
            call()
    Q = X.view(torch.uint8)[:, :WIDE].view(torch.float8_e4m3fn)
    S = torch.empty((1, (WIDE + 127) // 128), dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu)
    with pytest.raises(ValueError):
        agcn.quantized_linear(Q, S, Q, S)


def test_weights_of_over_2_31_rows_columns_or_groups():
    W = torch.empty((WIDE,), dtype=torch.float16, device=DEV)
    for shape in ((WIDE, 1), (1, WIDE), (WIDE, 1, 1), (1, WIDE, 1), (1, 1, WIDE)):
        with pytest.raises(ValueError):
            agcn.quantize_weight(W.view(shape))
