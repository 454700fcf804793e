"""Typed, 8-bit and last-layer calls on matrices of more than 2^31 elements.

Products: whole numbers of at most 2 and contractions of 64, so that every sum of Y and dX (at most 256) is exact in bf16, and
every partial sum of dW in fp32 (rows of a part times 4 stay under 2^24, and so do the results, which are looked at); dW then
takes one rounding to bf16, as the reference does.  Results are compared bit for bit with fp32 products of the same whole numbers.
Scores: sampled rows (first, last, around element 2^31) against 64 bits with test_gpu_log_probs' tolerances."""
import numpy as np
import pytest

from test_gpu_log_probs import exact, near

pytestmark = pytest.mark.gpu

N, K, M = 35_000_000, 64, 64  # 2.24e9 elements
STEP = 2_500_000


@pytest.fixture(scope="module")
def gnn():
    from paper_2412_06354_b200 import gnn as g
    g.load()
    return g


def whole(rows, cols, seed, dtype):
    import torch
    g = torch.Generator("cuda").manual_seed(seed)
    out = torch.empty(rows, cols, dtype=dtype, device="cuda")
    for a in range(0, rows, STEP):
        b = min(a + STEP, rows)
        out[a:b] = torch.randint(-2, 3, (b - a, cols), generator=g, device="cuda", dtype=torch.int8).to(dtype)
    return out


def test_segments(gnn):
    import torch
    ptr = [1000, 5_000_001, 5_000_001, 20_000_000, 34_999_000]
    G = len(ptr) - 1
    X, W = whole(N, K, 1, torch.bfloat16), whole(G * K, M, 2, torch.bfloat16).view(G, K, M)
    p = torch.tensor(ptr, device="cuda")
    Y = gnn.linear_segments(X, p, W)
    sums = torch.zeros(G, K, M, device="cuda", dtype=torch.float64)
    for g in range(G):
        for a in range(ptr[g], ptr[g + 1], STEP):
            b = min(a + STEP, ptr[g + 1])
            assert torch.equal(Y[a:b].float(), X[a:b].float() @ W[g].float()), (g, a)
    assert not bool(Y[:ptr[0]].any()) and not bool(Y[ptr[-1]:].any())
    dY = Y
    dY[:] = whole(N, M, 3, torch.bfloat16)
    dX, dW = gnn.linear_segments_backward(X, p, W, dY)
    for g in range(G):
        for a in range(ptr[g], ptr[g + 1], STEP):
            b = min(a + STEP, ptr[g + 1])
            assert torch.equal(dX[a:b].float(), dY[a:b].float() @ W[g].float().t()), (g, a)
            sums[g] += (X[a:b].float().t() @ dY[a:b].float()).double()
    assert float(sums.abs().max()) < 2 ** 24
    assert torch.equal(dW, sums.float().to(torch.bfloat16))
    assert not bool(dX[:ptr[0]].any()) and not bool(dX[ptr[-1]:].any())


def test_8_bits(gnn):
    import torch
    X = whole(N, K, 4, torch.bfloat16)
    X[:, 0] = 2  # every row's largest: scale 2 / 127
    q, s = gnn.quantize_rows(X)
    steps = torch.tensor([-127, -64, 0, 64, 127], device="cuda", dtype=torch.int8)  # 63.5 steps: to the even one
    for a in range(0, N, STEP):
        assert torch.equal(q[a:a + STEP], steps[(X[a:a + STEP] + 2).long()])
    assert bool((s == torch.tensor(2.0, device="cuda") / 127).all())
    wq = torch.randint(-127, 128, (M, K), device="cuda", dtype=torch.int8)
    one = torch.ones(M, device="cuda")
    del X
    Y = gnn.linear_i8(q, s, wq, one, dtype=torch.float32)
    for a in range(0, N, STEP):
        assert torch.equal(Y[a:a + STEP], (q[a:a + STEP].float() @ wq.float().t()) * s[a:a + STEP, None])  # sums under 2^24: one rounding


@pytest.mark.parametrize("C", [45, 1000, 30011])
def test_log_probs(gnn, C):
    import torch
    n = 2_300_000_000 // C
    g = torch.Generator("cuda").manual_seed(C)
    Z = torch.empty(n, C, dtype=torch.bfloat16, device="cuda")
    step = 50_000_000 // C
    for a in range(0, n, step):
        Z[a:a + step] = torch.randn(min(step, n - a), C, generator=g, device="cuda")
    label = torch.randint(0, C, (n,), generator=g, device="cuda", dtype=torch.int32)
    logp, H, lse, tl, ti = gnn.log_probs(Z, label, top=3)
    dl = torch.ones(n, device="cuda")
    mid = 2 ** 31 // C
    rows = torch.tensor([0, 1, n // 3, mid - 1, mid, mid + 1, n - 2, n - 1], device="cuda")
    z, y = Z[rows].cpu(), label[rows].cpu()
    rl, lp, rp, rh = exact(z, y)
    near(lse[rows], rl, 2e-6 + 2.0 ** -23 * rl.abs(), "lse")
    near(logp[rows], rp, 2e-6 + 2.0 ** -22 * rp.abs(), "logp")
    near(H[rows], rh, 2e-6 * (1.0 + rh) + 2e-6 * rh, "entropy")
    want = np.argsort(-z.double().numpy(), axis=1, kind="stable")[:, :3].astype(np.int32)
    assert np.array_equal(ti[rows].cpu().numpy(), want)
    dZ = gnn.log_probs_backward(Z, label, lse, dlogp=dl)
    p = torch.exp(lp)
    ref = -p
    ref[torch.arange(len(rows)), y.long()] += 1.0
    room = 2.0 * (4e-6 + 2.0 ** -22 * rl.abs()[:, None] + 2.0 ** -22 * lp.abs()) * p + 2.0 ** -23 * ref.abs() + 1e-38
    near(dZ[rows], ref, room + 2.0 ** -8 * (ref.abs() + room), "dZ")


@pytest.mark.parametrize("dtype,K,M", [("bf16", 8192, 8192), ("bf16", 8191, 24), ("bf16", 40, 8190), ("f32", 2048, 2048), ("f32", 2047, 20), ("f32", 33, 2046)])
def test_widest_matrices(gnn, dtype, K, M):
    """The largest K and M that are taken, and their neighbours: whole numbers again, sums under 2^15, one rounding to bf16."""
    import torch
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    sizes = [3, 0, 150, 140]
    ptr = torch.tensor([0, 3, 3, 153, 293], device="cuda")
    X, W, dY = whole(293, K, 5, t), whole(4 * K, M, 6, t).view(4, K, M), whole(293, M, 7, t)
    Y = gnn.linear_segments(X, ptr, W)
    dX, dW = gnn.linear_segments_backward(X, ptr, W, dY)
    a = 0
    for g, n in enumerate(sizes):
        x, w, dy = (v.double() for v in (X[a:a + n], W[g], dY[a:a + n]))
        assert torch.equal(Y[a:a + n], (x @ w).to(t)), g
        assert torch.equal(dX[a:a + n], (dy @ w.t()).to(t)), g
        assert torch.equal(dW[g], (x.t() @ dy).to(t)), g
        a += n


@pytest.mark.parametrize("n", [5, 200])
def test_longest_8_bit_sums(gnn, n):
    """K = 131071: random values (sums far under 2^24, one rounding) and one row of the extremes (a sum of nearly 2^31, rounded to 24 bits)."""
    import torch
    K, M = 131071, 70
    g = torch.Generator("cuda").manual_seed(n)
    x = torch.randint(-3, 4, (n, K), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-3, 4, (M, K), generator=g, device="cuda", dtype=torch.int8)
    x[0], w[0] = -128, -128
    Y = gnn.linear_i8(x, torch.ones(n, device="cuda"), w, torch.ones(M, device="cuda"), dtype=torch.float32)
    assert torch.equal(Y, (x.double() @ w.double().t()).float())
