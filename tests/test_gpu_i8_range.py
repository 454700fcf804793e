"""The 8-bit product over the whole range of its scales: rows up to the largest fp32 number, scales from the subnormal numbers up.

Tolerance: the sum to 24 bits, its product with the row's scale, scale and bias in one more: three roundings of 2^-24, the first two on
|sum| sx sw, the last on the result; bf16 one more of 2^-8; results under the normal numbers half a unit of 2^-149 (bf16 2^-134) each."""
import numpy as np
import pytest

from util import bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gnn():
    from paper_2412_06354_b200 import gnn as g
    g.load()
    return g


def reference(q, sx, w, sw, b, relu):
    """-> result in 64 bits, room of three roundings"""
    import torch
    term = (q.double() @ w.double().t()) * sx.double()[:, None] * sw.double()[None]
    y = term + (b.double() if b is not None else 0.0)
    return (y.clamp_min(0.0) if relu else y), 2.0 ** -24 * (2 * term.abs() + y.abs()) * 1.0001 + 2.0 ** -149


def check(gnn, q, sx, w, sw, b, relu, dtype):
    import torch
    Y = gnn.linear_i8(q.cuda(), sx.cuda(), w.cuda(), sw.cuda(), bias=None if b is None else b.cuda(), relu=relu, dtype=dtype)
    ref, room = reference(q, sx, w, sw, b, relu)
    if dtype == torch.bfloat16:
        room = room + 2.0 ** -8 * (ref.abs() + room) + 2.0 ** -134
    got, most = Y.double().cpu(), torch.finfo(dtype).max * (1 + 2.0 ** -9)
    over = ref.abs() > most  # no number of the type: infinite
    assert bool((got[over] == ref[over].sign() * float("inf")).all())
    err = (got - ref).abs()
    bad = ~over & ~((err <= room) | (got.isinf() & (ref.abs() + room >= torch.finfo(dtype).max)))
    assert not bool(bad.any()), f"{int(bad.sum())} off, first {got[bad][0]} for {ref[bad][0]}"
    return Y


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [5, 300])
@pytest.mark.parametrize("K", [256, 1000])
def test_scales_of_every_size(gnn, dtype, n, K):
    """Row scales from 2^-149 to the largest, channel scales that bring the products back, sums of every size, 0 among them."""
    import torch
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(n + K)
    q = torch.randint(-127, 128, (n, K), generator=g, dtype=torch.int8)
    w = torch.randint(-127, 128, (72, K), generator=g, dtype=torch.int8)
    q[::5] = 127
    w[:8] = 127
    w[8:16] = 0
    w[16:24, 1:] = 0
    sx = torch.ldexp(torch.rand(n, generator=g) + 0.5, torch.randint(-149, 128, (n,), generator=g))
    sx[:4] = torch.tensor([2.6e36, 2.0 ** 96, 2.0 ** 96 * (1 + 2.0 ** -23), 3e38])
    b = torch.randn(72, generator=g) * 10.0
    for lo, hi in ((-149, -100), (-60, -20), (-20, 20), (60, 128)):
        sw = torch.ldexp(torch.rand(72, generator=g) + 0.5, torch.randint(lo, hi, (72,), generator=g))
        check(gnn, q, sx, w, sw, None, False, dt)
        check(gnn, q, sx, w, sw, b, True, dt)


@pytest.mark.parametrize("n", [3, 200])
def test_large_rows_from_rows_to_8_bits(gnn, n):
    """Features of 1e36 and 3e38 with weights under 0.02: finite results."""
    import torch
    g = torch.Generator().manual_seed(n)
    X = torch.rand(n, 256, generator=g) * 1e36
    X[0] = 1e36
    X[1] = 3.4e38
    X[2] = torch.randn(256, generator=g)
    q, s = gnn.quantize_rows(X.cuda())
    w, sw = gnn.quantize_rows((torch.randn(40, 256, generator=g) * 0.01).cuda())
    Y = check(gnn, q.cpu(), s.cpu(), w.cpu(), sw.cpu(), None, False, torch.float32)
    assert bool(Y[0].isfinite().all()) and float(Y[0].abs().max()) > 1e34
    other = gnn.linear_i8(q[2:].contiguous(), s[2:].contiguous(), w, sw)  # rows keep their bits whatever lies beside them
    assert np.array_equal(bits(other), bits(Y[2:]))


def test_a_row_alone_gets_the_bits_of_the_batch(gnn):
    import torch
    g = torch.Generator().manual_seed(4)
    q = torch.randint(-127, 128, (64, 512), generator=g, dtype=torch.int8).cuda()
    w = torch.randint(-127, 128, (96, 512), generator=g, dtype=torch.int8).cuda()
    sx = torch.ldexp(torch.rand(64, generator=g) + 0.5, torch.randint(-149, 128, (64,), generator=g)).cuda()
    sw = torch.ldexp(torch.rand(96, generator=g) + 0.5, torch.randint(-90, 40, (96,), generator=g)).cuda()
    b = torch.randn(96, generator=g).cuda()
    Y = gnn.linear_i8(q, sx, w, sw, bias=b)
    for i in range(64):
        assert np.array_equal(bits(gnn.linear_i8(q[i:i + 1].contiguous(), sx[i:i + 1].clone(), w, sw, bias=b)), bits(Y[i:i + 1])), i


def test_scales_that_are_not_numbers(gnn):
    """A row's NaN or infinite scale stays in its row, a channel's in its column."""
    import torch
    q, w = torch.ones(20, 64, dtype=torch.int8), torch.ones(16, 64, dtype=torch.int8)
    for n in (4, 20):
        sx, sw = torch.ones(n), torch.ones(16)
        sx[1], sx[2], sx[3], sw[5], sw[6] = float("nan"), float("inf"), 1e35, float("nan"), float("inf")
        Y = gnn.linear_i8(q[:n].contiguous().cuda(), sx.cuda(), w.cuda(), sw.cuda()).cpu()
        assert bool(Y[1].isnan().all()) and bool(Y[:, 5].isnan().all())
        keep = [m for m in range(16) if m not in (5, 6)]
        assert bool((Y[2][keep] == float("inf")).all()) and float(Y[3, 6]) == float("inf") and bool((Y[0][keep] == 64).all())
        assert bool((Y[3][keep] == float(np.float32(64) * np.float32(1e35))).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,K,M", [(40000, 1040, 264), (38111, 64, 250), (700, 96, 1030)])
def test_large_scales_in_every_kind_of_tile(gnn, dtype, n, K, M):
    """Tiles of 256 rows, ranges of rows, several blocks of columns, rows that do not start on 16 bytes: every third row's scale is large."""
    import torch
    g = torch.Generator().manual_seed(M)
    q = torch.randint(-127, 128, (n, K), generator=g, dtype=torch.int8)
    w = torch.randint(-127, 128, (M, K), generator=g, dtype=torch.int8)
    sx = torch.rand(n, generator=g) + 0.5
    sx[::3] *= 2.0 ** 120
    sx[n // 2: n // 2 + 64] = 1.0  # boxes without one
    sw = (torch.rand(M, generator=g) + 0.5) * 2.0 ** -30
    check(gnn, q, sx, w, sw, torch.randn(M, generator=g), False, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
