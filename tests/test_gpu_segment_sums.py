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


@pytest.mark.parametrize("size", [1e-30, 1e-34, 1e-36, 1e-38, 1e-40])
def test_smallest_values(gnn, size):
    """fp32 values of which the second and third bf16 term have few bits or none: within 2^-134 of each value, beside the sums' 1e-5."""
    import torch
    g = torch.Generator().manual_seed(1)
    X, W, dY = torch.randn(300, 72, generator=g) * size, torch.randn(2, 72, 40, generator=g), torch.randn(300, 40, generator=g) * size
    ptr = torch.tensor([0, 130, 300])
    Xd, Wd, pd = X.cuda(), W.cuda(), ptr.cuda()
    Y = gnn.linear_segments(Xd, pd, Wd).double().cpu()
    dX, _ = gnn.linear_segments_backward(None, pd, Wd, dY.cuda(), want_dW=False)
    Z = torch.randn(300, 40, generator=g)
    _, dW = gnn.linear_segments_backward(Xd, pd, Wd, Z.cuda(), want_dX=False)
    for s in range(2):
        r = slice(int(ptr[s]), int(ptr[s + 1]))
        for got, a, b in ((Y[r], X[r], W[s]), (dX[r].double().cpu(), dY[r], W[s].t()), (dW[s].double().cpu(), X[r].t(), Z[r])):
            a, b = a.double(), b.double()
            # and products of either factor's terms under the smallest fp32 number, 2^-149 of each at most
            room = 1e-5 * (a.abs() @ b.abs()) + 2.0 ** -134 * b.abs().sum(0) + a.shape[1] * 6 * 2.0 ** -149
            assert bool(((got - a @ b).abs() <= room).all()), float(((got - a @ b).abs() / room).max())
