"""Log probabilities of scores far from zero: masks of -1e9 or -1e30, whole rows of them, scores shifted by a constant.

Tolerances.  As in test_gpu_log_probs.py: sums 2e-6 of 1 + s, a rounding 2^-24 of its value, |d| 2^-23 for the exponent's argument, which the
2e-6 holds as long as the classes that count are within a few tens of the largest; nothing grows with the scores but the rounding of lse itself."""
import numpy as np
import pytest

from test_gpu_log_probs import best, exact, near
from util import bits

pytestmark = pytest.mark.gpu

# rows by a thread, by a warp, by a block, by a cluster, by parts
SHAPES = [(4200, 47), (20, 47), (12, 900), (8, 5000), (4, 60000), (1, 600000)]
FAR = [-1e4, -65504.0, -1.1e6, -2.0 ** 24, -2.0 ** 24 - 4, -1e9, -2.0 ** 30, -2.0 ** 30 - 128, -1e10, -2.0 ** 33 - 1024, -1e15, -1e20, -1e30, -9e36, -1.1e37, -3e38, 1e6, 1e10, 1e30, 1.1e37, 3e38]


@pytest.fixture(scope="module")
def gnn():
    from paper_2412_06354_b200 import gnn as g
    g.load()
    return g


def check(gnn, Z, label, top, what):
    import torch
    d = Z.cuda()
    logp, H, lse, tl, ti = gnn.log_probs(d, label.cuda(), top=top)
    rl, rlp, rp, rh = exact(Z, label)
    near(lse, rl, 2e-6 + 2.0 ** -23 * rl.abs().nan_to_num(posinf=0.0), what + " lse")
    near(logp, rp, 2e-6 + 2.0 ** -22 * rp.abs().nan_to_num(posinf=0.0), what + " logp")
    near(H, rh, 2e-6 * (1.0 + rh) + 2e-6 * rh, what + " entropy")
    idx = best(Z, top)
    assert np.array_equal(ti.cpu().numpy(), idx), what + " best classes"
    lp = rlp.gather(1, torch.from_numpy(idx).long())
    near(tl, lp, 2e-6 + 2.0 ** -22 * lp.abs().nan_to_num(posinf=0.0), what + " their log p")


@pytest.mark.parametrize("n,C", SHAPES)
def test_scores_shifted_by_a_constant(gnn, n, C):
    """Eighths around a constant at which they are exact, threads' maxima that rise: the same log p and entropy wherever they lie."""
    import torch
    g = torch.Generator().manual_seed(C + 1)
    near_zero = torch.randint(-40, 41, (min(n, 64), C), generator=g).float() / 8
    label = torch.randint(0, C, (near_zero.shape[0],), generator=g, dtype=torch.int32)
    for shift in (100.0, -1000.0, 3e4, -1e5, 2.0 ** 18):
        check(gnn, near_zero + shift, label, min(5, C), f"{shift}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", SHAPES)
def test_masks_of_any_size(gnn, dtype, n, C):
    """A value far from zero throughout a row, in its first half, in its last, everywhere but in one place."""
    import torch
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(C)
    base = torch.randn(min(n, 8), C, generator=g).to(dt)
    label = torch.randint(0, C, (n,), generator=g, dtype=torch.int32)
    rows = max(1, n // 4)
    for v in FAR:
        kinds = torch.stack([base[0]] * 4)
        kinds[0] = v
        kinds[1, : C // 2] = v
        kinds[2, C // 2:] = v
        kinds[3, : C - 1] = v
        for Z in ([kinds.repeat(rows, 1)] if n >= 4 else [k[None] for k in kinds]):
            check(gnn, Z, label[: Z.shape[0]], min(5, C), f"{v}")


@pytest.mark.parametrize("n,C", SHAPES)
def test_scores_around_the_border_of_exact_differences(gnn, n, C):
    """Whole numbers on both sides of 2^24, 2^25 and 2^30 where steps of 2 to 128 are left: the classes within a few steps of the largest count."""
    import torch
    g = torch.Generator().manual_seed(C + 2)
    steps = torch.randint(-20, 1, (min(n, 64), C), generator=g).float()
    label = torch.randint(0, C, (steps.shape[0],), generator=g, dtype=torch.int32)
    for top in (2.0 ** 20 + 6, 2.0 ** 24, 2.0 ** 24 + 6, 2.0 ** 25, 2.0 ** 30, 2.0 ** 30 + 256, -(2.0 ** 20) - 2, -(2.0 ** 24) + 7, -(2.0 ** 24) - 2, -(2.0 ** 30) + 64, -(2.0 ** 30) - 128):
        unit = float(np.spacing(np.float32(abs(top))))
        check(gnn, top + unit * steps, label, min(5, C), f"{top}")


@pytest.mark.parametrize("steps", [(9e36, 1.1e37, 2e37, 3e37), (-5e37, -1e37, 0.0, 1.0), (-1e38, -1e20, -1e10, -1.0), (-2e6, -1e6, 1e6, 2e6), (1.0, 2e6, 1e12, 3e38), (-2.0 ** 30 - 128, -2.0 ** 30, -2.0 ** 24 - 2, -2.0 ** 24 + 1), (2.0 ** 24 - 1, 2.0 ** 24 + 2, 2.0 ** 30, 2.0 ** 30 + 128)])
@pytest.mark.parametrize("C", [900, 16384, 170000])
def test_maxima_that_rise_from_far_to_far(gnn, C, steps):
    """Every thread meets the four values one after the other, in rising order."""
    import torch
    Z = torch.full((3, C), steps[0])
    Z[1:] = -3.4e38
    for q in range(4):
        Z[1, q * (C // 4):(q + 1) * (C // 4)] = steps[q]
        Z[2, q * (C // 4): q * (C // 4) + 5] = steps[q]
    check(gnn, Z, torch.tensor([0, C - 1, 1], dtype=torch.int32), 3, f"{steps}")


def test_a_far_row_leaves_the_others_alone(gnn):
    import torch
    g = torch.Generator().manual_seed(8)
    for n, C in ((4100, 47), (16, 47), (16, 900), (4, 70000)):
        Z = torch.randn(n, C, generator=g)
        other = Z.clone()
        other[1] = -1e30
        a, b = (gnn.log_probs(z.cuda(), None, top=3) for z in (Z, other))
        keep = torch.cat([torch.arange(0, 1), torch.arange(2, n)]).cuda()
        for x, y in zip(a[1:], b[1:]):
            assert np.array_equal(bits(x[keep]), bits(y[keep]))


@pytest.mark.parametrize("C", [60000, 1200000, 3000001])
def test_parts_whose_maxima_lie_farther_apart_than_a_number_holds(gnn, C):
    """The lowest value throughout and one score from which it is farther away than the largest fp32 number, so that the difference of
    two parts' maxima is -inf (the longest rows have more parts than the joining block has lanes per warp and turn)."""
    import torch
    for big in (1e32, 3e38):
        for at in (0, C // 2, C - 1):
            Z = torch.full((1, C), torch.finfo(torch.float32).min)
            Z[0, at] = big
            logp, H, lse, tl, ti = gnn.log_probs(Z.cuda(), torch.tensor([at], dtype=torch.int32, device="cuda"), top=2)
            assert float(logp) == 0.0 and float(H) == 0.0 and float(lse) == float(torch.tensor(big)) and ti[0].tolist() == [at, 1 if at == 0 else 0]
            assert float(tl[0, 0]) == 0.0 and float(tl[0, 1]) == float("-inf")  # -6.4e38 and less: no fp32 number
