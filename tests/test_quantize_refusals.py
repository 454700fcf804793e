"""Rows to 8 bits of more elements than the kernels can count are refused before any launch (no GPU needed)."""
import pytest

from paper_2412_06354_b200 import gnn
from test_dense_refusals import P, UNSUPPORTED


@pytest.mark.parametrize("K", [2 ** 31 - 256, 2 ** 31 - 1])
@pytest.mark.parametrize("dtype", [gnn.F32, gnn.BF16])
def test_longest_rows(K, dtype):
    lib = gnn.load()
    for N in (0, 1):
        assert lib.gnn_quantize_rows(P, N, K, dtype, P, P, None) == UNSUPPORTED
    assert b"2^31" in lib.gnn_last_error_string()


@pytest.mark.parametrize("N", [1, 100])
def test_product_of_too_many_columns_or_rows(N):
    """Blocks of columns are counted in an int."""
    call = lambda n, M: gnn.load().gnn_linear_i8(P, P, P, P, n, 16, M, gnn.F32, None, 0, P, P, 1 << 40, None)
    assert call(N, 2 ** 31 - 256) == call(N, 2 ** 31 - 1) == UNSUPPORTED
    assert call(2 ** 31 - 129, 8) == UNSUPPORTED
