"""How the rows of dW are cut, seen in the workspace that the call asks for (no GPU needed)."""
import pytest

from paper_2412_06354_b200 import gnn


def parts(N, K, M):
    """Parts of an fp32 gradient: K and M on 16 bytes, so that the workspace holds the weights' terms and two partials a part."""
    ws = gnn.load().gnn_linear_segments_workspace
    none = 256 + -(-6 * K * M // 256) * 256
    return (ws(N, 1, K, M, gnn.F32, 1) - none) // (2 * K * M * 4)


@pytest.mark.parametrize("N", [2049, 4096, 16384, 40000, 100000, 1000000, 20000000])
@pytest.mark.parametrize("K,M", [(8, 8), (64, 64), (128, 256), (1024, 1024), (2048, 2048)])
def test_fp32_parts_are_short_enough_for_their_sums(N, K, M):
    assert parts(N, K, M) * 2048 >= N
