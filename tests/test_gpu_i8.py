"""GPU parity of the dense transform in 8 bits: the rounding of rows against exact quotients, the product against int64.

The integers are equal.  The scale is one rounding off max / 127 (2^-24).  Y: fp32 takes the rounding of the sum to 24 bits, of
the two scales' product, of their product with the sum and of adding the bias: four roundings of 2^-24 each, on |sum| sx sw and
on the result; bf16 one more of 2^-8."""
import numpy as np
import pytest

from util import bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gnn():
    from paper_2412_06354_b200 import gnn as g
    g.load()
    return g


def rounded(X):
    """-> (q int64, scale float64 of fp32) by exact quotients: ratios of fp32 numbers this far from a tie are told apart in 64 bits"""
    import torch
    x = X.double()
    top = x.abs().amax(1) if X.shape[1] else torch.zeros(X.shape[0], dtype=torch.float64)
    scale = (top / 127.0).float().double()
    finite = torch.isfinite(top)
    q = torch.zeros_like(x)
    ok = finite & (scale > 0)
    q[ok] = torch.round(x[ok] / scale[ok][:, None])
    scale[~finite] = float("nan")
    return q.long(), scale


def check_rows(gnn, X, what):
    import torch
    q, scale = gnn.quantize_rows(X.cuda())
    rq, rs = rounded(X)
    assert q.dtype == torch.int8 and torch.equal(q.long().cpu(), rq), what
    assert torch.equal(scale.double().cpu().nan_to_num(-1.0), rs.nan_to_num(-1.0)), what
    return q, scale


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,K", [(1, 1), (3, 7), (5, 8), (33, 16), (100, 24), (1000, 64), (257, 100), (129, 128), (70, 256), (9, 500), (40, 512), (17, 1024), (5, 2048), (3, 4104), (2, 9000)])
def test_rows_to_8_bits(gnn, dtype, n, K):
    import torch
    g = torch.Generator().manual_seed(n * 10007 + K)
    X = (torch.randn(n, K, generator=g) * torch.exp(4 * torch.randn(n, 1, generator=g))).to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
    check_rows(gnn, X, "random")


def test_ties_and_their_neighbours(gnn):
    """Halves of the step, the next fp32 numbers beside them, both signs, at several scales."""
    import torch
    rows = []
    for step in (1.0, 2.0 ** -20, 3.0, 1.0 / 3.0, 2.0 ** -60):
        s = np.float32(step)
        base = (np.arange(-127, 127) + 0.5).astype(np.float32) * s
        rows.append(np.concatenate([base, np.nextafter(base, np.float32(np.inf)), np.nextafter(base, np.float32(-np.inf)), np.array([127 * s, -127 * s], np.float32)]))
    check_rows(gnn, torch.from_numpy(np.stack(rows).astype(np.float32)), "ties")


def test_smallest_and_largest_rows(gnn):
    import torch
    X = torch.zeros(12, 64)
    X[1, 3] = 1e-45           # scale rounds to zero
    X[2] = torch.linspace(-1, 1, 64) * 1e-43  # scale below the normal numbers
    X[3] = torch.linspace(-1, 1, 64) * 1e-37
    X[4] = torch.linspace(-1, 1, 64) * 3.4e38
    X[5] = -0.0
    X[6, 7] = float("inf")
    X[7, 9] = float("nan")
    X[8] = float("-inf")
    X[9] = 5.0
    X[10, 63] = -3.0
    X[11] = torch.randn(64, generator=torch.Generator().manual_seed(1)) * 1e-31
    q, scale = check_rows(gnn, X, "extremes")
    assert bool(scale[6:9].isnan().all()) and bool((q[6:9] == 0).all()) and float(scale[0]) == 0.0
    Y = gnn.linear_i8(q, scale, q[9:11].contiguous(), scale[9:11].contiguous())
    assert bool(Y[6:9].isnan().all()) and bool((Y[0] == 0).all())
    check_rows(gnn, X.bfloat16(), "extremes, bf16")


def product_ref(q, sx, w, sw, b, relu):
    import torch
    acc = q.double().cpu() @ w.double().cpu().t()  # exact: under 2^53
    y = acc * sx.double().cpu()[:, None] * sw.double().cpu()[None]
    room = y.abs() * 4
    if b is not None:
        y = y + b.double().cpu()
        room = room + y.abs()
    return (y.clamp_min(0.0) if relu else y), room * 2.0 ** -24


SHAPES = [(1, 1, 1), (1, 16, 8), (1, 1024, 1024), (3, 37, 5), (8, 48, 100), (9, 16, 8), (9, 1, 1), (17, 33, 3), (127, 128, 64), (128, 144, 65), (129, 256, 256), (300, 100, 47), (1000, 512, 328),
          (64, 4096, 264), (700, 80, 1030), (20000, 64, 128), (2, 100, 70000 // 64), (40001, 1100, 300), (38100, 1024, 256), (40000, 256, 250)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,K,M", SHAPES)
def test_product_against_whole_numbers(gnn, dtype, n, K, M):
    import torch
    g = torch.Generator().manual_seed(n + 31 * K + 1009 * M)
    q = torch.randint(-128, 128, (n, K), generator=g, dtype=torch.int8)
    w = torch.randint(-128, 128, (M, K), generator=g, dtype=torch.int8)
    sx, sw = torch.rand(n, generator=g) + 0.1, torch.rand(M, generator=g) + 0.1
    b = torch.randn(M, generator=g) * 100
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    dev = [t.cuda() for t in (q, sx, w, sw)]
    for bias, relu in ((None, False), (b, True)):
        Y, ws = gnn.linear_i8(*dev, bias=None if bias is None else bias.cuda(), relu=relu, dtype=dt, return_ws=True)
        torch.cuda.synchronize()
        assert Y.dtype == dt and int(ws[:4].view(torch.int32).item()) == 0
        ref, room = product_ref(q, sx, w, sw, bias, relu)
        if dtype == "bf16":
            room = room + 2.0 ** -8 * (ref.abs() + room)
        err = (Y.double().cpu() - ref).abs()
        assert bool((err <= room).all()), f"{float((err - room).max()):.3e}"
        ws.fill_(255)
        again = gnn.linear_i8(*dev, bias=None if bias is None else bias.cuda(), relu=relu, dtype=dt, ws=ws)
        assert np.array_equal(bits(Y), bits(again))


@pytest.mark.parametrize("n", [4, 200])
def test_largest_sums_are_exact(gnn, n):
    """128 * 128 * 131071 is the last sum inside int32; one more feature is refused."""
    import torch
    K = 131071
    q = torch.full((n, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((16, K), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    one, ones = torch.ones(n, device="cuda"), torch.ones(16, device="cuda")
    Y = gnn.linear_i8(q, one, w, ones)
    want = torch.full((16,), float(np.float32(128 * 128 * K)))
    want[1] = float(np.float32(-128 * 127 * K))
    assert torch.equal(Y.cpu(), want.expand(n, 16))
    big = torch.zeros(n, K + 1, dtype=torch.int8, device="cuda")
    with pytest.raises(gnn.GnnError) as e:
        gnn.linear_i8(big, one, torch.zeros(16, K + 1, dtype=torch.int8, device="cuda"), ones)
    assert e.value.status == 5


def test_no_rows(gnn):
    import torch
    q, s = gnn.quantize_rows(torch.empty(0, 32, device="cuda"))
    assert q.shape == (0, 32) and s.shape == (0,)
    w = torch.zeros(8, 32, dtype=torch.int8, device="cuda")
    assert gnn.linear_i8(q, s, w, torch.ones(8, device="cuda")).shape == (0, 8)


@pytest.mark.parametrize("n", [1, 500])
def test_replayed_graph_and_second_stream(gnn, n):
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    w, sw = gnn.quantize_rows(torch.randn(72, 100, generator=g, device="cuda"))
    xs = [torch.randn(n, 100, generator=g, device="cuda").bfloat16() for _ in range(3)]
    call = lambda x: gnn.linear_i8(*gnn.quantize_rows(x), w, sw, relu=True, dtype=torch.bfloat16)
    want = [call(x) for x in xs]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = call(xs[1])
    same = call(xs[2])
    torch.cuda.synchronize()
    assert np.array_equal(bits(other), bits(want[1])) and np.array_equal(bits(same), bits(want[2]))
    live = xs[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(live)
    for x, y in zip(xs, want):
        live.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(bits(out), bits(y))


@pytest.mark.parametrize("K", [64, 61])
def test_scales_with_few_digits(gnn, K):
    """Rows of the smallest subnormals: the scale is a few units of 2^-149, rounded down by up to a third, and the quotient of the
    largest value passes 127."""
    import torch
    unit = torch.arange(1, 401, dtype=torch.float64)[:, None] * (1 - 2 * (torch.arange(K, dtype=torch.float64) % 2)) * torch.linspace(0, 1, K, dtype=torch.float64).flip(0)
    X = (unit.round() * 2.0 ** -149).float()
    q, scale = gnn.quantize_rows(X.cuda())
    rq, rs = rounded(X)
    assert int(rq.abs().max()) > 127  # the oracle's quotients do pass it
    assert torch.equal(q.long().cpu(), rq.clamp(-127, 127))
    assert torch.equal(scale.double().cpu(), rs)
