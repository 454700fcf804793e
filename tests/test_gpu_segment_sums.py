"""fp32 gradients of the weights over many rows whose terms have one sign, where the tensor cores' cut-off sums drift furthest.

Tolerance: 1e-5 of the terms' sum, as in test_gpu_segments.py.  A sum over 2048 rows is 128 steps, each of which cuts off up to 2^-24 of the
result on average (the accumulator's last bit is 2^-23 to 2^-24 of it while it grows): 7.6e-6, and the rounding of a few partials behind it."""
import pytest

from test_segment_parts import parts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gnn():
    from paper_2412_06354_b200 import gnn as g
    g.load()
    return g


@pytest.mark.parametrize("N,K,M", [(16384, 2048, 2048), (100000, 1024, 1024), (1000000, 64, 64)])
def test_longest_parts(gnn, N, K, M):
    """Every 16 rows end in what the accumulator has no bits for: fifteen rows of 1 + 2^-7 (squared: one unit of 2^-14) and one of 1, by 1 to 1.75."""
    import torch
    assert -(-N // parts(N, K, M)) > 1024  # the parts are long ones
    a = torch.full((N, 1), 1 + 2.0 ** -7)
    a[::16] = 1.0
    ptr, W = torch.tensor([0, N]).cuda(), torch.zeros(1, K, M, device="cuda")
    X = a.expand(N, K).contiguous().cuda()
    for scale in (1.0, 1.25, 1.5, 1.75):
        _, dW = gnn.linear_segments_backward(X, ptr, W, (a * scale).expand(N, M).contiguous().cuda(), want_dX=False)
        ref = float((a.double() * a.double() * scale).sum())
        assert float((dW.double() - ref).abs().max()) <= 1e-5 * ref, scale
