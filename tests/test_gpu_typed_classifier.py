"""The typed layer, the propagate, the last layer and the log probabilities run together, as a classifier of the nodes of a
heterogeneous graph uses them: a training step's loss and gradients against automatic differentiation in 64 bits, the same step
replayed from a captured graph, and the answer of the trained layers in 8 bits."""
import numpy as np
import pytest

from paper_2412_06354_b200 import synth
from util import bits, to_dev

pytestmark = pytest.mark.gpu

SIZES, K, H, CLASSES, BETA = [900, 0, 1300, 801], 40, 64, 23, 0.02


@pytest.fixture(scope="module")
def setup():
    import torch
    from paper_2412_06354_b200 import gnn
    gnn.load()
    n = sum(SIZES)
    src, dst = synth.rmat(12, n, 12000, 41, symmetric=True)
    g = gnn.coo_to_csr(n, to_dev(src), to_dev(dst))
    gen = torch.Generator().manual_seed(7)
    t = {"X": torch.randn(n, K, generator=gen), "W1": torch.randn(len(SIZES), K, H, generator=gen) * 0.15, "b1": torch.randn(len(SIZES), H, generator=gen) * 0.1,
         "W2": torch.randn(H, CLASSES, generator=gen) * 0.15, "label": torch.randint(-1, CLASSES, (n,), generator=gen, dtype=torch.int32)}
    kinds = torch.repeat_interleave(torch.arange(len(SIZES), dtype=torch.int32), torch.tensor(SIZES))
    ptr = gnn.graph_ptr_from_ids(kinds.cuda(), len(SIZES))
    assert ptr.tolist() == np.concatenate([[0], np.cumsum(SIZES)]).tolist()
    return gnn, g, src, dst, ptr, t


def step(gnn, g, ptr, X, W1, b1, W2, label):
    """loss rows and gradients of sum over labelled nodes of -log p(label) / n - BETA * entropy / n"""
    import torch
    n = X.shape[0]
    h = gnn.linear_segments(X, ptr, W1, bias=b1, relu=True)
    a = gnn.propagate_fused(g, h, None, "mean")
    z = gnn.linear(a, W2)
    logp, ent, lse, _, _ = gnn.log_probs(z, label)
    dz = gnn.log_probs_backward(z, label, lse, dlogp=torch.full((n,), -1.0 / n, device="cuda"), entropy=ent, dentropy=torch.full((n,), -BETA / n, device="cuda"))
    da, dW2 = gnn.linear_backward(a, W2, dz)
    dh, _ = gnn.propagate_fused_backward(g, da, "mean")
    dp, _ = gnn.row_epilogue_backward(h, dh)
    db1 = gnn.reduce_nodes(ptr, dp, "sum")
    _, dW1 = gnn.linear_segments_backward(X, ptr, W1, dp, want_dX=False)
    return logp, ent, dW1, db1, dW2


def test_training_step_against_automatic_differentiation(setup):
    import torch
    gnn, g, src, dst, ptr, t = setup
    d = {k: v.cuda() for k, v in t.items()}
    got = step(gnn, g, ptr, **d)
    p = {k: v.double().requires_grad_(k in ("W1", "b1", "W2")) for k, v in t.items() if k != "label"}
    n = t["X"].shape[0]
    kinds = torch.repeat_interleave(torch.arange(len(SIZES)), torch.tensor(SIZES))
    h = torch.relu(torch.cat([p["X"][kinds == q] @ p["W1"][q] + p["b1"][q] for q in range(len(SIZES))]))
    deg = torch.zeros(n, dtype=torch.float64).index_add_(0, torch.from_numpy(dst).long(), torch.ones(len(dst), dtype=torch.float64))
    a = torch.zeros(n, H, dtype=torch.float64).index_add(0, torch.from_numpy(dst).long(), h[torch.from_numpy(src).long()]) / deg.clamp_min(1.0)[:, None]
    lp = torch.log_softmax(a @ p["W2"], 1)
    known = t["label"] >= 0
    logp = torch.where(known, lp.gather(1, t["label"].clamp_min(0).long()[:, None])[:, 0], torch.zeros(n, dtype=torch.float64))
    ent = -(lp.exp() * lp).sum(1)
    (-(logp.sum() / n) - BETA * ent.sum() / n).backward()
    # norm-wise: each of the five passes is within 1e-5 of its terms, of which a gradient adds up a few thousand of both signs
    for name, x, ref in (("logp", got[0], logp), ("entropy", got[1], ent), ("dW1", got[2], p["W1"].grad), ("db1", got[3], p["b1"].grad), ("dW2", got[4], p["W2"].grad)):
        err = float((x.double().cpu() - ref.detach()).norm() / ref.detach().norm())
        assert err <= 5e-5, f"{name}: {err:.2e}"
    assert bool((got[2][1] == 0).all()) and bool((got[3][1] == 0).all())  # a type without nodes


def test_the_step_replayed_from_a_graph(setup):
    import torch
    gnn, g, src, dst, ptr, t = setup
    d = {k: v.cuda() for k, v in t.items()}
    want = step(gnn, g, ptr, **d)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(gnn, g, ptr, **d)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(np.array_equal(bits(a), bits(b)) for a, b in zip(out, want))
    d["X"].mul_(-1.0)
    graph.replay()
    fresh = step(gnn, g, ptr, **d)
    torch.cuda.synchronize()
    assert all(np.array_equal(bits(a), bits(b)) for a, b in zip(out, fresh))


def test_the_answer_in_8_bits(setup):
    """The last layer in 8 bits: scores within what two roundings of 1 / 254 of each row's and channel's largest value move them."""
    import torch
    gnn, g, src, dst, ptr, t = setup
    d = {k: v.cuda() for k, v in t.items()}
    h = gnn.linear_segments(d["X"], ptr, d["W1"], bias=d["b1"], relu=True)
    a = gnn.propagate_fused(g, h, None, "mean")
    wq, ws = gnn.quantize_rows(d["W2"].t().contiguous())  # once
    aq, as_ = gnn.quantize_rows(a)
    z = gnn.linear_i8(aq, as_, wq, ws)
    a64, w64 = a.double().cpu(), d["W2"].double().cpu()
    # |x q-error| <= scale / 2 per feature: sum |a| ws/2 + |w| as/2 + as ws / 4, and fp32 roundings of the whole
    room = a64.abs().sum(1, keepdim=True) * ws.double().cpu() / 2 + as_.double().cpu()[:, None] * w64.abs().sum(0) / 2 + H * as_.double().cpu()[:, None] * ws.double().cpu() / 4
    ref = a64 @ w64
    assert bool(((z.double().cpu() - ref).abs() <= room * (1 + 1e-6) + 1e-5 * ref.abs() + 1e-30).all())
    _, _, lse, top_logp, top_idx = gnn.log_probs(z, top=3, want_entropy=False)
    best = torch.sort(z.cpu(), dim=1, descending=True, stable=True).indices[:, :3]
    assert torch.equal(top_idx.cpu().long(), best)
    # one node at a time gives the same integers and the same scores
    one = [gnn.linear_i8(*gnn.quantize_rows(a[i:i + 1]), wq, ws) for i in (0, 5, 900)]
    assert all(np.array_equal(bits(o[0]), bits(z[i])) for o, i in zip(one, (0, 5, 900)))
