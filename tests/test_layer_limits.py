"""Sizes at the ends of 32 bits that include/pf_layer.h refuses on the host, before any work (no GPU needed)."""
import pytest

from test_layer_host import BF16, F32, SHAPE, UNSUPPORTED, _matmul, _quant, layer  # noqa: F401  (fixture)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("K", [2**31 - 127, 2**31 - 16, 2**31 - 15, 2**31 - 1])
def test_columns_that_32_bits_do_not_count(layer, K, dt):  # noqa: F811
    """Blocks of 128 columns, and rows of whole 16 bytes, would end behind the largest 32-bit number."""
    for b_rows in (1, 128):
        for M in (1, 40):
            assert _matmul(layer, M=M, K=K, lda=2**31, ldb=2**31, b_rows=b_rows, dt=dt) == UNSUPPORTED
            assert layer.pf_matmul_fp8_workspace_bytes(M, 8, K, b_rows) == 0
    assert _quant(layer, K=K, ldx=2**31, ldq=2**31, ldqt=16, dt=dt) == UNSUPPORTED


def test_the_deepest_product_is_known(layer):  # noqa: F811
    """The largest K passes the checks of sizes (a row shorter than K is what is wrong here)."""
    assert _matmul(layer, K=2**31 - 128, lda=2**31, ldb=64) == SHAPE
