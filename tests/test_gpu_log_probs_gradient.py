"""The gradient of log probabilities and entropy where it is easily lost: large incoming gradients, scores far from zero, nearly sure rows.

Tolerances.  p = exp(lp) off by |lp| 2^-23 + 2^-22 of itself (the exponent's argument, the exponential) and by what lp is off by;
three roundings of 2^-24 behind it."""
import numpy as np
import pytest

from test_gpu_log_probs import exact, near
from util import bits

pytestmark = pytest.mark.gpu

# a chunk in several rows, rows of several chunks, blocks per row
SHAPES = [(50, 5), (30, 47), (9, 1000), (5, 5000), (2, 60001)]


@pytest.fixture(scope="module")
def gnn():
    from paper_2412_06354_b200 import gnn as g
    g.load()
    return g


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", SHAPES)
def test_masked_classes_get_zero_however_large_the_gradients(gnn, dtype, n, C):
    """Gradients of the entropy from 1 to 1e30: exact zeros at -inf and at the type's lowest value, the others scale with them."""
    import torch
    g = torch.Generator().manual_seed(C)
    Z = torch.randn(n, C, generator=g)
    masked = torch.rand(n, C, generator=g) < 0.3
    masked[:, 0] = False
    label = torch.zeros(n, dtype=torch.int32)
    for low in (float("-inf"), torch.finfo({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]).min):
        z = Z.masked_fill(masked, low).to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]).cuda()
        _, H, lse, _, _ = gnn.log_probs(z, label.cuda())
        call = lambda h: gnn.log_probs_backward(z, label.cuda(), lse, dlogp=None, entropy=H, dentropy=torch.full((n,), h, device="cuda"))
        one = call(1.0)
        for h in (1.0, 2.0 ** 30, 2.0 ** 100):  # powers of two: the same digits
            d = call(h)
            assert bool((d.cpu()[masked] == 0).all())
            assert np.array_equal(bits((d.double() / h).to(d.dtype)), bits(one))
