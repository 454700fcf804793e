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
