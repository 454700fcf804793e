"""GPU parity of the class log probabilities, their entropy, the best classes and the gradient, against 64 bits.

Tolerances.  The exponentials are fp32: the argument's rounding and that of the product with log2(e) move e^d by up to
|d| 2^-23 + 2^-22 of its value, and |d| e^d is under 1, so that each of the sums of n terms is off by at most 2^-21 of itself plus the
summation's n/256 * 2^-24 (parts of at most a few hundred terms, then their sums): under 2e-6 of 1 + s for what is tested.  lse: that
plus two roundings of 2^-24 |lse|.  log p: the same and the rounding of z - m.  Entropy: log1p(s) and t / (1 + s) each off by
2e-6 of themselves, at least of 1 together.  Gradients: p is off by |log p| 2^-23 + 2^-22 + what lse carries (2^-24 |lse|) of
itself, the rest three roundings."""
import numpy as np
import pytest

from util import bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gnn():
    from paper_2412_06354_b200 import gnn as g
    g.load()
    return g


def exact(Z, label):
    """-> lse, log p of all classes, logp, entropy in 64 bits; a row of nothing but -inf: -inf, -inf and 0.  log p is (z - m) - log sum:
    m + log sum would swallow the sum of a row at the type's lowest value."""
    import torch
    z = Z.double()
    m = z.amax(1)
    none = m == float("-inf")
    safe = torch.where(none, torch.zeros_like(m), m)
    e = torch.exp(z - safe[:, None])
    lse = safe + torch.log(e.sum(1))
    lse[none] = float("-inf")
    lp = (z - safe[:, None]) - torch.where(none, torch.zeros_like(m), torch.log(e.sum(1)))[:, None]
    p = torch.exp(lp)
    H = -(torch.where(p > 0, p * lp, torch.zeros_like(p))).sum(1)
    logp = None
    if label is not None:
        known = (label >= 0) & (label < Z.shape[1])
        logp = torch.where(known, lp.gather(1, torch.where(known, label, torch.zeros_like(label)).long()[:, None])[:, 0], torch.zeros_like(m))
    return lse, lp, logp, H


def best(Z, k):
    """indices by (value, lower index), with numpy's stable sort"""
    z = Z.double().numpy()
    return np.argsort(-z, axis=1, kind="stable")[:, :k].astype(np.int32)


def scores(n, C, dtype, seed, scale=2.5, masked=0.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    Z = torch.randn(n, C, generator=g) * scale
    if masked:
        Z[torch.rand(n, C, generator=g) < masked] = float("-inf")
    label = torch.randint(-1, C, (n,), generator=g, dtype=torch.int32)
    return Z.to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]), label


def near(got, ref, room, what):
    import torch
    got = got.double().cpu()
    same = (got == ref) | ((got - ref).abs() <= room)
    assert bool(same.all()), f"{what}: {int((~same).sum())} off, worst {float((got - ref).abs()[~same].max()):.3e}"


def check(gnn, Z, label, top, what=""):
    import torch
    d = Z.cuda()
    logp, H, lse, tl, ti = gnn.log_probs(d, None if label is None else label.cuda(), top=top)
    rl, rlp, rp, rh = exact(Z, label)
    near(lse, rl, 2e-6 + 2.0 ** -23 * rl.abs().nan_to_num(posinf=0.0), what + " lse")
    if label is None:
        assert logp is None
    else:
        near(logp, rp, 2e-6 + 2.0 ** -22 * rp.abs().nan_to_num(posinf=0.0), what + " logp")
    near(H, rh, 2e-6 * (1.0 + rh) + 2e-6 * rh, what + " entropy")
    if top:
        idx = best(Z, top)
        assert np.array_equal(ti.cpu().numpy(), idx), what + " best classes"
        lp = rlp.gather(1, torch.from_numpy(idx).long())
        near(tl, lp, 2e-6 + 2.0 ** -22 * lp.abs().nan_to_num(posinf=0.0), what + " their log p")
    again = gnn.log_probs(d, None if label is None else label.cuda(), top=top)
    for a, b in zip((logp, H, lse, tl, ti), again):
        if a is not None:
            assert np.array_equal(bits(a), bits(b)), what + " not bit-reproducible"


SHAPES = [(1, 1), (1, 2), (3, 7), (100, 8), (1000, 47), (33, 33), (65, 100), (257, 128), (20, 129), (300, 256), (50, 1000), (9, 1024), (9, 1025), (40, 5001), (5, 20000), (1, 33000), (2, 170001),
          (700, 9000), (1, 1000003), (20000, 3), (5000, 64), (3000, 200)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", SHAPES)
def test_against_64_bits(gnn, dtype, n, C):
    Z, label = scores(n, C, dtype, n * 7 + C)
    for top in {0, 1, min(5, C), min(32, C)}:
        check(gnn, Z, label if top else None, top, f"top {top}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", [(60, 5), (60, 47), (60, 300), (20, 3000), (7, 70000)])
def test_masked_classes_and_rows(gnn, dtype, n, C):
    """Most classes at -inf, rows with one class left, rows with none, more listed classes than are left."""
    import torch
    Z, label = scores(n, C, dtype, C, masked=0.7)
    Z[0] = float("-inf")
    Z[1] = float("-inf")
    Z[1, C - 1] = -5.0
    Z[2] = float("-inf")
    Z[2, 0] = torch.finfo(Z.dtype).min
    Z[3] = torch.finfo(Z.dtype).min  # masked by the lowest value: all equal
    Z[4] = torch.finfo(Z.dtype).min
    Z[4, C // 2] = 1.0
    label[:5] = C - 1
    label[5], label[6] = C, -7  # no class
    check(gnn, Z, label, min(C, 20))


@pytest.mark.parametrize("C", [47, 300, 40000])
def test_ties_take_the_lower_index(gnn, C):
    import torch
    g = torch.Generator().manual_seed(C)
    Z = torch.randint(-2, 3, (40, C), generator=g).float()
    Z[Z == 0] = torch.where(torch.rand(int((Z == 0).sum()), generator=g) < 0.5, 0.0, -0.0)
    Z[0] = 0.0
    Z[1] = torch.arange(C).float()             # ascending: every class enters the list
    Z[2] = -torch.arange(C).float()
    Z[3] = -0.0
    check(gnn, Z, None, 32)
    check(gnn, Z.bfloat16(), None, 7)


@pytest.mark.parametrize("C", [30, 900, 50000])
def test_nearly_sure_rows_keep_their_digits(gnn, C):
    """A class ahead by 5 to 60: log p and entropy far below 2^-24 of the largest term are right in their leading digits."""
    import torch
    Z, label = scores(24, C, "f32", C, scale=0.5)
    lead = torch.arange(24) % C
    Z[torch.arange(24), lead] += torch.linspace(5, 60, 24) + float(np.log(C))
    label = lead.int()
    logp, H, lse, tl, ti = gnn.log_probs(Z.cuda(), label.cuda(), top=1)
    z = Z.double()
    others = (z - z.amax(1, keepdim=True)).exp()
    others[torch.arange(24), lead] = 0.0
    s = others.sum(1)
    t = (others * torch.where(others > 0, others.log(), torch.zeros_like(others))).sum(1)
    for got, ref in ((logp, -torch.log1p(s)), (tl[:, 0], -torch.log1p(s)), (H, torch.log1p(s) - t / (1 + s))):
        # relative: the spread of d (up to 70) in the exponent, |d| 2^-23, and the sums' 2e-6
        near(got, ref, (70 * 2.0 ** -23 + 4e-6) * ref.abs() + 1e-44, "sure row")
    assert np.array_equal(ti[:, 0].cpu().numpy(), lead.int().numpy())


@pytest.mark.parametrize("C", [5, 200, 5000, 60000])
def test_not_a_number_stays_in_its_row(gnn, C):
    import torch
    Z, label = scores(8, C, "f32", C)
    bad = Z.clone()
    bad[2, C // 2] = float("nan")
    bad[4] = float("nan")
    bad[6, C - 1] = float("inf")
    label[:] = 0
    got = gnn.log_probs(bad.cuda(), label.cuda(), top=4)
    want = gnn.log_probs(Z.cuda(), label.cuda(), top=4)
    rows = torch.tensor([2, 4, 6])
    rest = torch.tensor([0, 1, 3, 5, 7])
    for a, b in zip(got, want):
        assert np.array_equal(bits(a[rest.cuda()]), bits(b[rest.cuda()]))
    for a in got[:4]:
        assert bool(a[rows.cuda()].isnan().all())
    idx = got[4].cpu()
    assert bool(((idx >= 0) & (idx < C)).all()) and all(len(set(r.tolist())) == 4 for r in idx)
    assert int(idx[6, 0]) == C - 1 and idx[2].tolist() == best(Z.index_fill(1, torch.tensor([C // 2]), float("-inf")), 4)[2].tolist()


GRAD_SHAPES = [(1, 1), (1, 7), (3, 8), (5, 9), (100, 47), (33, 64), (20, 1000), (7, 4097), (2, 100001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,C", GRAD_SHAPES)
@pytest.mark.parametrize("which", ["logp", "entropy", "both"])
def test_gradient(gnn, dtype, n, C, which):
    import torch
    Z, label = scores(n, C, dtype, n + C, masked=0.2 if C > 4 else 0.0)
    if n > 2:
        Z[0] = float("-inf")
        label[0] = 0
    g = torch.Generator().manual_seed(C)
    dl = torch.randn(n, generator=g) if which != "entropy" else None
    dh = torch.randn(n, generator=g) if which != "logp" else None
    _, H, lse, _, _ = gnn.log_probs(Z.cuda(), label.cuda())
    dev = lambda t: None if t is None else t.cuda()
    got = gnn.log_probs_backward(Z.cuda(), label.cuda(), lse, dlogp=dev(dl), entropy=H, dentropy=dev(dh))
    rl, lp, _, rh = exact(Z, label)
    none = rl == float("-inf")
    p = torch.exp(lp)
    known = (label >= 0) & ~none
    gg = torch.where(known, dl.double() if dl is not None else torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64))
    hh = dh.double() if dh is not None else torch.zeros(n, dtype=torch.float64)
    inner = gg[:, None] + hh[:, None] * (torch.where(p > 0, lp, torch.zeros_like(lp)) + rh[:, None])
    ref = torch.where(p > 0, -p * inner, torch.zeros_like(p))
    size = p * (gg.abs()[:, None] + hh.abs()[:, None] * (torch.where(p > 0, lp, torch.zeros_like(lp)).abs() + rh[:, None] + 1.0))
    hit = torch.arange(n)[known]
    ref[hit, label[known].long()] += gg[known]
    # p and log p: what the forward pass's lse is off by (2e-6 + 2^-23 |lse|), the exponent's |log p| 2^-23 + 2^-22; three roundings
    off = 4e-6 + 2.0 ** -22 * torch.where(none, torch.zeros_like(rl), rl).abs()[:, None] + 2.0 ** -22 * torch.where(p > 0, lp.abs(), torch.zeros_like(lp))
    room = 2.0 * off * size + 2.0 ** -23 * ref.abs() + 1e-38
    if dtype == "bf16":
        room = room + 2.0 ** -8 * (ref.abs() + room) + 1e-38
    near(got, ref, room, "dZ")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_of_a_row_with_nothing_to_choose(gnn, dtype):
    """All classes at -inf or at the type's lowest value (whose lse has no digits left for the classes): zeros, other rows as ever."""
    import torch
    Z, label = scores(6, 50, dtype, 5)
    label[:] = 3
    want = Z.clone()
    Z[1], Z[4] = float("-inf"), torch.finfo(Z.dtype).min
    one = torch.ones(6, device="cuda")
    out = []
    for z in (Z, want):
        _, H, lse, _, _ = gnn.log_probs(z.cuda(), label.cuda())
        out.append(gnn.log_probs_backward(z.cuda(), label.cuda(), lse, dlogp=one, entropy=H, dentropy=one))
    assert bool((out[0][[1, 4]] == 0).all())
    rest = [0, 2, 3, 5]
    assert np.array_equal(bits(out[0][rest]), bits(out[1][rest]))


def test_gradient_against_differences(gnn):
    """logp and entropy of fp32 scores, moved by +-h along a direction."""
    import torch
    Z, label = scores(40, 23, "f32", 3, scale=1.0)
    g = torch.Generator().manual_seed(2)
    dl, dh, V = torch.randn(40, generator=g), torch.randn(40, generator=g), torch.randn(40, 23, generator=g)
    _, H, lse, _, _ = gnn.log_probs(Z.cuda(), label.cuda())
    dZ = gnn.log_probs_backward(Z.cuda(), label.cuda(), lse, dlogp=dl.cuda(), entropy=H, dentropy=dh.cuda()).double().cpu()
    h = 2.0 ** -6

    def value(z):
        logp, H, _, _, _ = gnn.log_probs(z.cuda(), label.cuda())
        return float((logp.double().cpu() * dl.double() + H.double().cpu() * dh.double()).sum())

    slope = (value(Z + h * V) - value(Z - h * V)) / (2 * h)
    want = float((dZ * V.double()).sum())
    # third derivatives of lse and H along V are under 10 |V|^3 a row: h^2 / 6 of that; the values' own error 4e-6 a row over h
    room = float(((dl.abs() + dh.abs()) * (10 * h * h / 6 * V.abs().amax(1) ** 3 + 4e-6 / h)).sum())
    assert abs(slope - want) <= room


@pytest.mark.parametrize("n,C", [(300, 47), (5, 60000), (200, 20000), (5000, 47)])
def test_replayed_graph_and_second_stream(gnn, n, C):
    import torch
    zs = [scores(n, C, "bf16", q)[0].cuda() for q in range(3)]
    label = torch.zeros(n, dtype=torch.int32, device="cuda")
    one = torch.ones(n, device="cuda")

    def call(z):
        logp, H, lse, tl, ti = gnn.log_probs(z, label, top=5)
        return logp, H, lse, tl, ti, gnn.log_probs_backward(z, label, lse, dlogp=one, entropy=H, dentropy=one)

    want = [call(z) for z in zs]
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        other = call(zs[1])
    same = call(zs[2])
    torch.cuda.synchronize()
    for got, ref in ((other, want[1]), (same, want[2])):
        assert all(np.array_equal(bits(a), bits(b)) for a, b in zip(got, ref))
    live = zs[0].clone()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = call(live)
        graphs.append((g, out))
    for z, ref in zip(zs, want):
        live.copy_(z)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(np.array_equal(bits(a), bits(b)) for a, b in zip(out, ref))


def test_no_rows_and_gradient_in_place(gnn):
    import torch
    logp, H, lse, tl, ti = gnn.log_probs(torch.empty(0, 9, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), top=3)
    assert logp.shape == H.shape == lse.shape == (0,) and tl.shape == ti.shape == (0, 3)
    assert gnn.log_probs_backward(torch.empty(0, 9, device="cuda"), None, lse).shape == (0, 9)
    Z, label = scores(50, 33, "f32", 1)
    z, y = Z.cuda(), label.cuda()
    _, H, lse, _, _ = gnn.log_probs(z, y)
    one = torch.ones(50, device="cuda")
    want = gnn.log_probs_backward(z, y, lse, dlogp=one)
    lib = gnn.load()
    assert lib.gnn_log_probs_backward(z.data_ptr(), y.data_ptr(), lse.data_ptr(), None, one.data_ptr(), None, 50, 33, gnn.F32, z.data_ptr(), gnn._stream()) == 0
    torch.cuda.synchronize()
    assert np.array_equal(bits(z), bits(want))
