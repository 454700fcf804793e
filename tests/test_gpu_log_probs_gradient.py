"""The gradient of log probabilities and entropy where it is easily lost: large incoming gradients, scores far from zero, nearly sure rows.

Tolerances.  p = exp(lp) off by |lp| 2^-23 + 2^-22 of itself (the exponent's argument, the exponential) and by what lp is off by.  The label's
1 - p by expm1 is off by one unit of the last bit, 2^-23 of itself, its product and the difference by 2^-24 each: 2^-22 of the result."""
import numpy as np
import pytest

from test_gpu_canaries import guarded  # noqa: F401  (the fixture)
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


def in_two_numbers(gnn, Z, label, dl, dh):
    """-> the gradient by lse and lse_rest, and the forward pass's outputs"""
    z, y = Z.cuda(), label.cuda()
    logp, H, lse, tl, ti, rest = gnn.log_probs(z, y, top=1, return_rest=True)
    dev = lambda t: None if t is None else t.cuda()
    return gnn.log_probs_backward(z, y, lse, dlogp=dev(dl), entropy=H, dentropy=dev(dh), lse_rest=rest), (logp, H, lse, tl, ti, rest)


def reference(Z, label, dl, dh):
    """-> gradient in 64 bits, log p, and what the errors are relative to"""
    import torch
    rl, lp, _, rh = exact(Z, label)
    p = torch.exp(lp)
    fin = torch.where(p > 0, lp, torch.zeros_like(lp))
    known = (label >= 0) & (rl > float("-inf"))
    gg = torch.where(known, dl.double(), torch.zeros_like(rl))
    hh = dh.double()
    ref = -p * (gg[:, None] + hh[:, None] * (fin + rh[:, None]))
    hit = torch.arange(len(label))[known]
    ref[hit, label[known].long()] += gg[known]
    ref[rl == float("-inf")] = 0.0
    return ref, fin, p * (gg.abs()[:, None] + hh.abs()[:, None] * (fin.abs() + rh[:, None] + 1.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", SHAPES)
@pytest.mark.parametrize("shift", [0.0, 1e3, -1e4, 1e6, -1e9, 1e25])
def test_scores_far_from_zero(gnn, dtype, n, C, shift):
    """The bound has no part that grows with the scores: log p is off by the forward pass's 2e-6 and its own |log p| 2^-22."""
    import torch
    g = torch.Generator().manual_seed(C)
    Z = (torch.randn(n, C, generator=g) * 2.5 + shift).to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
    Z[torch.rand(n, C, generator=g) < 0.2] = float("-inf")
    Z[0] = float("-inf")
    Z[1] = shift
    label = torch.randint(-1, C, (n,), generator=g, dtype=torch.int32)
    dl, dh = torch.randn(n, generator=g), torch.randn(n, generator=g)
    got, _ = in_two_numbers(gnn, Z, label, dl, dh)
    ref, lp, size = reference(Z, label, dl, dh)
    room = 2.0 * (4e-6 + 2.0 ** -22 * lp.abs()) * size + 2.0 ** -22 * ref.abs() + 1e-38
    if dtype == "bf16":
        room = room + 2.0 ** -8 * (ref.abs() + room)
    near(got, ref, room, "dZ")


@pytest.mark.parametrize("n,C", SHAPES)
@pytest.mark.parametrize("shift", [0.0, 1000.0])
def test_nearly_sure_labels_keep_their_gradient(gnn, n, C, shift):
    """A label ahead by 5 to 60: its gradient, 1 - p, is right in its leading digits far below 2^-24."""
    import torch
    g = torch.Generator().manual_seed(C + 3)
    Z = torch.randint(-8, 9, (n, C), generator=g).float() / 8  # exact with the shift too
    label = torch.arange(n, dtype=torch.int32) % C
    rows = torch.arange(n)
    ahead = torch.linspace(5, 60, n).round() + float(int(np.log(C)))
    Z[rows, label.long()] += ahead
    Z += shift
    dl = torch.ones(n)
    got, (logp, H, lse, _, _, rest) = in_two_numbers(gnn, Z, label, dl, None)
    d = Z.double() - Z.double().amax(1, keepdim=True)
    others = d.exp()
    others[rows, label.long()] = 0.0
    s = others.sum(1)
    ref = -others / (1 + s)[:, None]
    ref[rows, label.long()] = s / (1 + s)
    room = (80 * 2.0 ** -23 + 4e-6) * ref.abs() + 1e-37  # as for log p of such rows; below the normal numbers zeros
    near(got, ref, room, "dZ")
    near(rest.double().cpu() + lse.double().cpu(), Z.double().amax(1) + torch.log1p(s), (80 * 2.0 ** -23 + 4e-6) * torch.log1p(s) + 2.0 ** -50 * (shift + 80), "lse in two numbers")
    # the entropy's gradient: p (log p + H), of which the terms are as exact as log p and H are
    dh = torch.ones(n)
    got, _ = in_two_numbers(gnn, Z, torch.full((n,), -1, dtype=torch.int32), dl, dh)
    t = (others * d).sum(1)
    H64 = torch.log1p(s) - t / (1 + s)
    lp64 = d - torch.log1p(s)[:, None]
    ref = -lp64.exp() * (lp64 + H64[:, None])
    near(got, ref, 3.0 * (80 * 2.0 ** -23 + 4e-6) * lp64.exp() * (lp64.abs() + H64[:, None]) + 1e-37, "dZ of the entropy")


def test_against_differences_far_from_zero(gnn):
    """logp and entropy of fp32 scores around 4096, moved by +-h along a direction that keeps them exact."""
    import torch
    g = torch.Generator().manual_seed(11)
    Z = torch.randint(-512, 513, (40, 23), generator=g).float() / 256 + 4096.0
    V = torch.randint(-8, 9, (40, 23), generator=g).float() / 8
    label = torch.randint(0, 23, (40,), generator=g, dtype=torch.int32)
    dl, dh = torch.randn(40, generator=g), torch.randn(40, generator=g)
    dZ, _ = in_two_numbers(gnn, Z, label, dl, dh)
    h = 2.0 ** -6

    def value(z):
        logp, H, _, _, _ = gnn.log_probs(z.cuda(), label.cuda())
        return float((logp.double().cpu() * dl.double() + H.double().cpu() * dh.double()).sum())

    slope = (value(Z + h * V) - value(Z - h * V)) / (2 * h)
    want = float((dZ.double().cpu() * V.double()).sum())
    # third derivatives of lse and H along V are under 10 |V|^3 a row: h^2 / 6 of that; the values' own error 4e-6 a row over h
    room = float(((dl.abs() + dh.abs()) * (10 * h * h / 6 * V.abs().amax(1) ** 3 + 4e-6 / h)).sum())
    assert abs(slope - want) <= room


@pytest.mark.parametrize("n,C", [(4200, 47), (300, 47), (20, 900), (5, 60000), (1, 600000)])
def test_the_other_outputs_are_the_same(gnn, n, C):
    """With and without the rest; the rest of rows that have none is 0; the gradient in place; a replayed graph."""
    import torch
    g = torch.Generator().manual_seed(C)
    Z = torch.randn(n, C, generator=g) + 300.0
    Z[0] = float("-inf")
    Z[-1, 0] = float("nan") if n > 1 else 1.0
    z, y = Z.cuda(), torch.randint(-1, C, (n,), generator=g, dtype=torch.int32).cuda()
    plain = gnn.log_probs(z, y, top=3)
    *same, rest = gnn.log_probs(z, y, top=3, return_rest=True)
    for a, b in zip(plain, same):
        assert np.array_equal(bits(a), bits(b))
    assert float(rest[0]) == 0.0 and (n == 1 or float(rest[-1]) == 0.0)
    one = torch.ones(n, device="cuda")
    call = lambda: gnn.log_probs_backward(z, y, same[2], dlogp=one, entropy=same[1], dentropy=one, lse_rest=rest)
    want = call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    out.fill_(-1.0)
    graph.replay()
    torch.cuda.synchronize()
    assert np.array_equal(bits(out), bits(want))
    lib = gnn.load()
    p = lambda t: t.data_ptr()
    assert lib.gnn_log_probs_rest_backward(p(z), p(y), p(same[2]), p(rest), p(same[1]), p(one), p(one), n, C, gnn.F32, p(z), gnn._stream()) == 0
    torch.cuda.synchronize()
    assert np.array_equal(bits(z), bits(want))


def test_a_rest_that_does_not_fit_is_refused(gnn):
    import torch
    z, s = torch.zeros(6, 8, device="cuda"), torch.zeros(6, device="cuda")
    for bad, error in ((torch.zeros(5, device="cuda"), ValueError), (s.double(), TypeError), (torch.zeros(6), ValueError), (torch.zeros(12, device="cuda")[::2], TypeError)):
        with pytest.raises(error):
            gnn.log_probs_backward(z, None, s, entropy=s, dentropy=s, lse_rest=bad)
    logp, H, lse, tl, ti, rest = gnn.log_probs(torch.empty(0, 9, device="cuda"), None, top=3, return_rest=True)
    assert rest.shape == (0,) and gnn.log_probs_backward(torch.empty(0, 9, device="cuda"), None, lse, lse_rest=rest).shape == (0, 9)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(1, 1), (7, 33), (13, 3), (5000, 47), (50, 2049), (3, 40001)])
def test_guard_bands(guarded, dtype, n, C):  # noqa: F811
    import torch
    gnn, gt = guarded
    Z = torch.randn(n, C, device="cuda").to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
    y = torch.randint(-2, C + 2, (n,), device="cuda", dtype=torch.int32)
    y[-1] = C - 1
    logp, H, lse, _, _, rest = gnn.log_probs(Z, y, top=1, return_rest=True)
    gt.check("forward")
    d = torch.ones(n, device="cuda")
    gnn.log_probs_backward(Z, y, lse.clone(), dlogp=d, entropy=H.clone(), dentropy=d, lse_rest=rest.clone())
    gt.check("gradient")


def test_last_layer_with_scores_far_from_zero(gnn):
    """Typed last layer -> log probabilities -> their gradient -> the layer's gradients, with a bias that moves a type's scores by thousands:
    each step against 64 bits from the step before, and rows of the gradient that add up to nothing."""
    import torch
    g = torch.Generator().manual_seed(21)
    ptr = torch.tensor([0, 700, 700, 1500])
    X, W = torch.randn(1500, 64, generator=g), torch.randn(3, 64, 47, generator=g) * 0.3
    b = torch.tensor([0.0, 5.0, -3000.0])[:, None] + torch.randn(3, 47, generator=g)
    label = torch.randint(-1, 47, (1500,), generator=g, dtype=torch.int32)
    Xd, Wd, pd, y = X.cuda(), W.cuda(), ptr.cuda(), label.cuda()
    Z = gnn.linear_segments(Xd, pd, Wd, bias=b.cuda())
    logp, H, lse, _, _, rest = gnn.log_probs(Z, y, return_rest=True)
    dl, dh = torch.full((1500,), -1.0), torch.full((1500,), -0.01)
    dZ = gnn.log_probs_backward(Z, y, lse, dlogp=dl.cuda(), entropy=H, dentropy=dh.cuda(), lse_rest=rest)
    ref, lp, size = reference(Z.cpu(), label, dl, dh)
    room = 2.0 * (4e-6 + 2.0 ** -22 * lp.abs()) * size + 2.0 ** -22 * ref.abs() + 1e-38
    near(dZ, ref, room, "dZ")
    assert bool((dZ.double().sum(1).abs().cpu() <= room.sum(1)).all())
    dX, dW = gnn.linear_segments_backward(Xd, pd, Wd, dZ)
    d = dZ.double().cpu()
    for s in range(3):
        r = slice(int(ptr[s]), int(ptr[s + 1]))
        x, w = X[r].double(), W[s].double()
        near(dX[r], d[r] @ w.t(), 1e-5 * (d[r].abs() @ w.abs().t()), "dX")
        near(dW[s], x.t() @ d[r], 1e-5 * (x.t().abs() @ d[r].abs()), "dW")
