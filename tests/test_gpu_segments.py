"""GPU parity of the dense transform with a weight per segment: Y = act(X W[g] + b[g]), dX = dY W[g]^T, dW[g] = X_g^T dY_g
against products in 64 bits.

Tolerance: fp32 1e-5 * S (S: the sum of the terms' absolute values), as for the plain dense transform.  bf16: the fp32 sum
(1e-5 * S) plus the one rounding of the result, eps / 2 = 2^-8 of its value (and of what the sum may be off)."""
import numpy as np
import pytest

from util import bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gnn():
    from paper_2412_06354_b200 import gnn as g
    g.load()
    return g


def close(got, ref, S, what):
    import torch
    assert got.shape == ref.shape, what
    err = (got.double().cpu() - ref).abs()
    bound = 1e-5 * S
    if got.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (ref.abs() + bound)
    bad = ~(err <= bound)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} out of tolerance, worst {float((err - bound).max()):.3e}"


def data(dtype, sizes, K, M, lead=0, tail=0, seed=1):
    """-> (X, seg_ptr, W, bias, dY) on the CPU; rows before and behind the segments hold what must not be read into results"""
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    N, G = lead + sum(sizes) + tail, len(sizes)
    ptr = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64) + lead)
    X = torch.randn(N, K, generator=g).to(dt)
    W = (torch.randn(G, K, M, generator=g) * (2.0 / (K + M)) ** 0.5).to(dt)
    b = torch.randn(G, M, generator=g) * 0.1
    dY = torch.randn(N, M, generator=g).to(dt)
    for t in (X, dY):
        if lead:
            t[:lead] = float("nan")
        if tail:
            t[N - tail:] = float("inf")
    return X, ptr, W, b, dY


def forward_ref(X, ptr, W, b, relu):
    import torch
    N, M = X.shape[0], W.shape[2]
    Y, S = torch.zeros(N, M, dtype=torch.float64), torch.zeros(N, M, dtype=torch.float64)
    for g in range(W.shape[0]):
        r = slice(int(ptr[g]), int(ptr[g + 1]))
        x, w = X[r].double(), W[g].double()
        Y[r] = x @ w
        S[r] = x.abs() @ w.abs()
        if b is not None:
            Y[r] += b[g].double()
            S[r] += b[g].double().abs()
    return (Y.clamp_min(0.0) if relu else Y), S


def backward_ref(X, ptr, W, dY):
    import torch
    dX, SX = torch.zeros(X.shape, dtype=torch.float64), torch.zeros(X.shape, dtype=torch.float64)
    dW, SW = torch.zeros(W.shape, dtype=torch.float64), torch.zeros(W.shape, dtype=torch.float64)
    for g in range(W.shape[0]):
        r = slice(int(ptr[g]), int(ptr[g + 1]))
        x, w, d = X[r].double(), W[g].double(), dY[r].double()
        dX[r], SX[r] = d @ w.t(), d.abs() @ w.abs().t()
        dW[g], SW[g] = x.t() @ d, x.abs().t() @ d.abs()
    return dX, SX, dW, SW


def status(ws):
    import torch
    torch.cuda.synchronize()
    return int(ws[:4].view(torch.int32).item())


#        sizes, K, M, lead, tail
CASES = [
    ([1], 8, 8, 0, 0), ([1], 1, 1, 0, 0), ([1, 1, 1], 64, 64, 0, 0), ([0, 5, 0, 0, 3, 0], 64, 48, 0, 0),
    # ends of the 128-row tiles and of the 64-row slices of dW; rows of no segment on both sides
    ([127, 1, 128, 129, 63, 64, 65, 0, 191], 128, 128, 0, 0), ([300, 7, 0, 200], 96, 72, 5, 40), ([40], 64, 64, 128, 1), ([0, 0], 32, 32, 10, 10),
    # widths that divide nothing, one column, one feature, several blocks of columns and of features
    ([50, 200, 33], 100, 47, 0, 3), ([17, 90], 33, 1, 0, 0), ([130, 20], 1, 130, 0, 0), ([100, 60, 5], 257, 328, 2, 0), ([150, 0, 90], 520, 300, 0, 0),
    # a long contraction (bf16: 32 slices), one row each of many segments
    ([70, 140], 1040, 136, 0, 0), ([1] * 40, 64, 96, 0, 0),
    # long segments: dW from several parts, cut at odd rows
    ([9000, 1, 12000, 0, 4000], 64, 64, 0, 0), ([20011], 40, 72, 7, 9), ([3, 15000, 2], 256, 256, 0, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_products_in_64_bits(gnn, dtype, case):
    import torch
    sizes, K, M, lead, tail = CASES[case]
    X, ptr, W, b, dY = data(dtype, sizes, K, M, lead, tail, seed=case)
    Xd, pd, Wd, bd, dYd = (t.cuda() for t in (X, ptr, W, b, dY))
    Y, ws = gnn.linear_segments(Xd, pd, Wd, return_ws=True)
    assert status(ws) == 0
    ref, S = forward_ref(X, ptr, W, None, False)
    close(Y, ref, S, "Y")
    ref, S = forward_ref(X, ptr, W, b, True)
    ws.fill_(255)  # whatever the workspace holds
    close(gnn.linear_segments(Xd, pd, Wd, bias=bd, relu=True, ws=ws), ref, S, "relu(Y + b)")
    dX, dW, ws = gnn.linear_segments_backward(Xd, pd, Wd, dYd, return_ws=True)
    assert status(ws) == 0
    rX, SX, rW, SW = backward_ref(X, ptr, W, dY)
    close(dX, rX, SX, "dX")
    close(dW, rW, SW, "dW")
    ws.fill_(255)
    dX2, dW2 = gnn.linear_segments_backward(Xd, pd, Wd, dYd, ws=ws)
    assert np.array_equal(bits(dX), bits(dX2)) and np.array_equal(bits(dW), bits(dW2)), "not bit-reproducible"
    only, none = gnn.linear_segments_backward(None, pd, Wd, dYd, want_dW=False)
    assert none is None and np.array_equal(bits(dX), bits(only))
    none, only = gnn.linear_segments_backward(Xd, pd, Wd, dYd, want_dX=False)
    assert none is None and np.array_equal(bits(dW), bits(only))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_segments_and_empty_ones(gnn, dtype):
    """More segments than one step of the 32-way search holds, two thirds of them empty."""
    import torch
    rng = np.random.default_rng(5)
    sizes = [int(n) if rng.random() < 1 / 3 else 0 for n in rng.integers(1, 200, 1500)]
    X, ptr, W, b, dY = data(dtype, sizes, 24, 40, 0, 0)
    Xd, pd, Wd, bd, dYd = (t.cuda() for t in (X, ptr, W, b, dY))
    ref, S = forward_ref(X, ptr, W, b, False)
    close(gnn.linear_segments(Xd, pd, Wd, bias=bd), ref, S, "Y")
    dX, dW = gnn.linear_segments_backward(Xd, pd, Wd, dYd)
    rX, SX, rW, SW = backward_ref(X, ptr, W, dY)
    close(dX, rX, SX, "dX")
    close(dW, rW, SW, "dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_segment_never_meets_anothers_values(gnn, dtype):
    """NaN and infinities in the rows, weights and biases of one segment stay in its results."""
    import torch
    sizes = [100, 90, 200]
    X, ptr, W, b, dY = data(dtype, sizes, 96, 80)
    for t in (X, dY):
        t[100:190] = float("nan")
        t[150] = float("inf")
    W[1] = float("nan")
    b[1] = float("-inf")
    Xd, pd, Wd, bd, dYd = (t.cuda() for t in (X, ptr, W, b, dY))
    Y = gnn.linear_segments(Xd, pd, Wd, bias=bd, relu=True)
    dX, dW = gnn.linear_segments_backward(Xd, pd, Wd, dYd)
    clean = [t.clone() for t in (X, W, b, dY)]
    for t in (clean[0], clean[3]):
        t[100:190] = 0.0
    clean[1][1] = 0.0
    clean[2][1] = 0.0
    ref, S = forward_ref(clean[0], ptr, clean[1], clean[2], True)
    rX, SX, rW, SW = backward_ref(clean[0], ptr, clean[1], clean[3])
    keep = torch.cat([torch.arange(0, 100), torch.arange(190, 390)])
    close(Y[keep.cuda()], ref[keep], S[keep], "Y")
    close(dX[keep.cuda()], rX[keep], SX[keep], "dX")
    for g in (0, 2):
        close(dW[g], rW[g], SW[g], "dW")
    assert bool(Y[100:190].isnan().all()) and bool(dX[100:190].isnan().all()) and bool(dW[1].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows_no_segments(gnn, dtype):
    import torch
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    W = torch.ones(3, 16, 24, dtype=dt, device="cuda")
    ptr = torch.zeros(4, dtype=torch.int64, device="cuda")
    X = torch.empty(0, 16, dtype=dt, device="cuda")
    dY = torch.empty(0, 24, dtype=dt, device="cuda")
    assert gnn.linear_segments(X, ptr, W).shape == (0, 24)
    dX, dW = gnn.linear_segments_backward(X, ptr, W, dY)
    assert dX.shape == (0, 16) and bool((dW == 0).all())
    X, dY = torch.full((7, 16), float("nan"), dtype=dt, device="cuda"), torch.full((7, 24), float("nan"), dtype=dt, device="cuda")
    Y = gnn.linear_segments(X, ptr[:1], W[:0])
    assert bool((Y == 0).all())
    dX, dW = gnn.linear_segments_backward(X, ptr[:1], W[:0], dY)
    assert bool((dX == 0).all()) and dW.shape == (0, 16, 24)


def test_fp32_sums_of_one_sign(gnn):
    """Terms of one sign, where the tensor cores' cut-off sums drift furthest: 2048 features forward, 40,000 rows in dW."""
    import torch
    g = torch.Generator().manual_seed(3)
    X = torch.rand(300, 2048, generator=g) + 0.5
    W = torch.rand(2, 2048, 64, generator=g) + 0.5
    ptr = torch.tensor([0, 130, 300])
    ref, S = forward_ref(X, ptr, W, None, False)
    close(gnn.linear_segments(X.cuda(), ptr.cuda(), W.cuda()), ref, S, "Y")
    X = torch.rand(40000, 32, generator=g) + 0.5
    dY = torch.rand(40000, 64, generator=g) + 0.5
    ptr = torch.tensor([0, 1, 40000])
    dX, SX, dW, SW = backward_ref(X, ptr, W[:, :32].contiguous(), dY)
    got = gnn.linear_segments_backward(X.cuda(), ptr.cuda(), W[:, :32].contiguous().cuda(), dY.cuda())
    close(got[0], dX, SX, "dX")
    close(got[1], dW, SW, "dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_streams_and_replayed_graphs(gnn, dtype):
    """Two calls at once on two streams, and two captured graphs replayed in turn with new inputs and new segment bounds."""
    import torch
    sizes = [400, 0, 111, 700]
    sets = [data(dtype, s, 100, 72, seed=q) for q, s in enumerate([sizes, sizes[::-1]])]
    dev = [[t.cuda() for t in s] for s in sets]
    want = [gnn.linear_segments(x, p, w, bias=b, relu=True) for x, p, w, b, _ in dev]
    want_b = [gnn.linear_segments_backward(x, p, w, d) for x, p, w, b, d in dev]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got, got_b = [None, None], [None, None]
    for _ in range(5):
        for q, s in enumerate(streams):
            with torch.cuda.stream(s):
                x, p, w, b, d = dev[q]
                got[q] = gnn.linear_segments(x, p, w, bias=b, relu=True)
                got_b[q] = gnn.linear_segments_backward(x, p, w, d)
        torch.cuda.synchronize()
        for q in range(2):
            assert np.array_equal(bits(got[q]), bits(want[q]))
            assert all(np.array_equal(bits(a), bits(b)) for a, b in zip(got_b[q], want_b[q]))
    live = [t.clone() for t in dev[0]]
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x, p, w, b, d = live
            out = (gnn.linear_segments(x, p, w, bias=b, relu=True), *gnn.linear_segments_backward(x, p, w, d))
        graphs.append((g, out))
    for q in (0, 1, 0):
        for t, s in zip(live, dev[q]):
            t.copy_(s)
        for g, out in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, out in graphs:
            assert np.array_equal(bits(out[0]), bits(want[q]))
            assert all(np.array_equal(bits(a), bits(b)) for a, b in zip(out[1:], want_b[q]))


def test_gradients_against_differences(gnn):
    """<dY, Y(X + h V)> in fp32 changes by h <dX, V>, and the same for W: the product is linear in each, so that any h serves."""
    import torch
    X, ptr, W, b, dY = data("f32", [60, 0, 77], 40, 24, seed=9)
    Xd, pd, Wd, dYd = (t.cuda() for t in (X, ptr, W, dY))
    dX, dW = gnn.linear_segments_backward(Xd, pd, Wd, dYd)
    g = torch.Generator().manual_seed(4)
    for base, grad, call in ((X, dX, lambda v: gnn.linear_segments(v, pd, Wd)), (W, dW, lambda v: gnn.linear_segments(Xd, pd, v))):
        V = torch.randn(base.shape, generator=g)
        h = 0.5
        up, down = (call((base + s * h * V).cuda()).double().cpu() for s in (1, -1))
        slope = float((dY.double() * (up - down)).sum()) / (2 * h)
        want = float((grad.double().cpu() * V.double()).sum())
        # each Y is off by at most 1e-5 of its terms' absolute sum (under 1e-5 * K * |x||w|), summed with |dY| over both calls
        room = 1e-5 * float((dY.double().abs() * (up.abs() + down.abs() + 40)).sum()) / (2 * h) + 1e-5 * float((grad.double().cpu().abs() * V.abs().double()).sum() + 40)
        assert abs(slope - want) <= room


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,M", [(64, 64), (128, 200), (300, 128)])
def test_rows_by_consecutive_ranges(gnn, dtype, K, M):
    """Rows enough for every SM, few segments: ends of ranges and of segments in all places, segments of one row and none among
    long ones, rows of no segment on both sides."""
    import torch
    sizes = [9000, 1, 0, 127, 14001, 1, 1, 5000, 0, 33, 12800]
    X, ptr, W, b, dY = data(dtype, sizes, K, M, lead=77, tail=1203, seed=K)
    Xd, pd, Wd, bd, dYd = (t.cuda() for t in (X, ptr, W, b, dY))
    Y, ws = gnn.linear_segments(Xd, pd, Wd, bias=bd, relu=True, return_ws=True)
    assert status(ws) == 0
    ref, S = forward_ref(X, ptr, W, b, True)
    close(Y, ref, S, "relu(Y + b)")
    dX, dW, ws = gnn.linear_segments_backward(Xd, pd, Wd, dYd, return_ws=True)
    assert status(ws) == 0
    rX, SX, rW, SW = backward_ref(X, ptr, W, dY)
    close(dX, rX, SX, "dX")
    close(dW, rW, SW, "dW")


@pytest.mark.parametrize("K,M", [(520, 200), (1030, 300)])
def test_long_contractions_by_tiles_of_256_rows(gnn, K, M):
    """Weights too many to stay in shared memory, rows enough for every SM: second halves of a tile full, cut, of one row, missing."""
    import torch
    sizes = [20000, 128, 129, 300, 1, 255, 256, 257, 0, 385, 18000]
    X, ptr, W, b, dY = data("bf16", sizes, K, M, lead=3, tail=70, seed=K)
    Xd, pd, Wd, bd, dYd = (t.cuda() for t in (X, ptr, W, b, dY))
    Y, ws = gnn.linear_segments(Xd, pd, Wd, bias=bd, relu=True, return_ws=True)
    assert status(ws) == 0
    ref, S = forward_ref(X, ptr, W, b, True)
    close(Y, ref, S, "relu(Y + b)")
    Wt = W.transpose(1, 2).contiguous()  # dX with a contraction of K
    dX, _, ws = gnn.linear_segments_backward(None, pd, Wt.cuda(), Xd, want_dW=False, return_ws=True)
    assert status(ws) == 0
    ref, S = forward_ref(X, ptr, W, None, False)
    close(dX, ref, S, "dX")
