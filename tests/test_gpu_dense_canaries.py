"""Guard bands around the outputs and workspaces of the typed, 8-bit and last-layer calls (see test_gpu_canaries.py): sizes that
end inside tiles, boxes, chunks and parts, rows of no segment, descending segment bounds."""
import pytest

from test_gpu_canaries import guarded  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def randn(*shape, dtype="f32"):
    import torch
    return torch.randn(*shape, device="cuda").to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,lead,tail,K,M", [([1], 0, 0, 1, 1), ([3, 0, 130], 5, 9, 33, 47), ([1000, 1, 255], 0, 1, 128, 64), ([20000, 7, 0, 30001], 3, 700, 100, 72),
                                                 ([25000, 129, 16000], 0, 0, 520, 264), ([64] * 50, 0, 0, 16, 24)])
def test_segments(guarded, dtype, sizes, lead, tail, K, M):  # noqa: F811
    import torch
    gnn, gt = guarded
    N, G = lead + sum(sizes) + tail, len(sizes)
    ptr = torch.cumsum(torch.tensor([lead] + sizes), 0).cuda()
    X, W, b, dY = randn(N, K, dtype=dtype), randn(G, K, M, dtype=dtype), randn(G, M), randn(N, M, dtype=dtype)
    gnn.linear_segments(X, ptr, W, bias=b, relu=True)
    gt.check("Y")
    gnn.linear_segments_backward(X, ptr, W, dY)
    gt.check("dX, dW")
    gnn.linear_segments_backward(X, ptr, W, dY, want_dX=False, return_ws=True)
    gt.check("dW")
    # bounds that descend or leave the rows: any result, nothing outside the arguments
    for bad in (ptr.flip(0).contiguous(), ptr - 50, ptr + N, torch.randint(-N, 2 * N, (G + 1,), device="cuda")):
        gnn.linear_segments(X, bad, W, bias=b)
        gnn.linear_segments_backward(X, bad, W, dY)
        gt.check("descending bounds")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,K,M", [(1, 1, 1), (8, 17, 5), (9, 40, 33), (130, 100, 47), (5000, 256, 72), (40000, 64, 264), (40001, 1040, 250)])
def test_8_bits(guarded, dtype, n, K, M):  # noqa: F811
    gnn, gt = guarded
    q, s = gnn.quantize_rows(randn(n, K, dtype=dtype))
    w, sw = gnn.quantize_rows(randn(M, K))
    gt.check("rows to 8 bits")
    x, sx, wq, sw2 = (t.clone() for t in (q, s, w, sw))
    import torch
    gnn.linear_i8(x, sx, wq, sw2, bias=randn(M), relu=True, dtype={"f32": torch.float32, "bf16": torch.bfloat16}[dtype], return_ws=True)
    gt.check("Y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C,top", [(1, 1, 1), (7, 33, 5), (5000, 47, 5), (4099, 64, 32), (300, 129, 3), (50, 1025, 32), (3, 40001, 7), (1, 1000003, 32), (700, 5000, 0)])
def test_log_probs(guarded, dtype, n, C, top):  # noqa: F811
    import torch
    gnn, gt = guarded
    Z = randn(n, C, dtype=dtype)
    y = torch.randint(-2, C + 2, (n,), device="cuda", dtype=torch.int32)
    logp, H, lse, _, _ = gnn.log_probs(Z, y, top=top)
    gt.check("forward")
    d = torch.ones(n, device="cuda")
    gnn.log_probs_backward(Z, y, lse.clone(), dlogp=d, entropy=H.clone(), dentropy=d)
    gt.check("gradient")
    Z[:] = float("-inf")  # every class listed one by one
    gnn.log_probs(Z, y, top=top)
    gt.check("masked throughout")
