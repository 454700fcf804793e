"""Log probabilities of scores far from zero.

Tolerances.  As in test_gpu_log_probs.py: sums 2e-6 of 1 + s, a rounding 2^-24 of its value, |d| 2^-23 for the exponent's argument, which the
2e-6 holds as long as the classes that count are within a few tens of the largest; nothing grows with the scores but the rounding of lse itself."""
import numpy as np
import pytest

from test_gpu_log_probs import best, exact, near
from util import bits

pytestmark = pytest.mark.gpu

# rows by a thread, by a warp, by a block, by a cluster, by parts
SHAPES = [(4200, 47), (20, 47), (12, 900), (8, 5000), (4, 60000), (1, 600000)]

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
