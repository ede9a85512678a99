"""Sizes past the 8-bit operators' limits are refused by the C ABI on the host, before any
HIP call. No GPU needed."""
import pytest

pytest.importorskip("torch")

import paper_2308_11825_amd as agcn


@pytest.mark.parametrize("groups", [2 ** 24 + 1, 2 ** 31 - 65536, 2 ** 31 - 1])
def test_quantize_weight_groups(groups):
    """Groups are counted in steps of 65535 in 32 bits."""
    lib = agcn.load_library()
    status = lib.agcn_quantize_weight(groups, 1, 1, agcn.AGCN_FLOAT, 0x10000000000, 1, 1, 0x20000000000, 1,
                                      1, 0x30000000000, 1, 1, None)
    assert status == agcn.AGCN_ERR_UNSUPPORTED, agcn.agcn_last_error()
