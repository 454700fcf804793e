"""Cases of the typed dense transform, the 8-bit dense transform and the class log probabilities.

``run`` computes an operator in elementary torch operations where ``own`` is false, and through the library where it is
true.  Outputs are whole tensors.  Sizes follow the workloads of the benchmark and the tests (170,000 nodes of 128 features,
100,000 nodes of 256, layers of 100 -> 47) and round numbers around them.
"""
import math

import torch

own = False

_F32, _BF16 = torch.float32, torch.bfloat16
_DT = {"f32": _F32, "bf16": _BF16}


def listed():
    return [
        # answering for one node of each of eight types: latency, and the weights read once
        {"name": "segments_one_row_each", "op": "segments", "N": 8, "G": 8, "K": 256, "M": 256, "dtype": "bf16", "even": True, "relu": False},
        # a typed layer over a citation-scale graph, forward
        {"name": "segments_nodes", "op": "segments", "N": 170000, "G": 12, "K": 128, "M": 128, "dtype": "bf16", "even": False, "relu": True},
        # the typed last layer in fp32, widths that divide nothing
        {"name": "segments_nodes_odd_f32", "op": "segments", "N": 170000, "G": 7, "K": 100, "M": 47, "dtype": "f32", "even": False, "relu": False},
        # wide typed layer with many types: bound by the products
        {"name": "segments_wide", "op": "segments", "N": 65536, "G": 64, "K": 1024, "M": 1024, "dtype": "bf16", "even": False, "relu": True},
        # training: gradients of a typed layer
        {"name": "segments_grad", "op": "segments_grad", "N": 100000, "G": 12, "K": 256, "M": 256, "dtype": "bf16", "even": False},
        # the same in fp32, a smaller layer
        {"name": "segments_grad_f32", "op": "segments_grad", "N": 40000, "G": 5, "K": 128, "M": 64, "dtype": "f32", "even": False},
        # serving one node with 8-bit weights: latency
        {"name": "i8_one_row", "op": "i8", "N": 1, "K": 1024, "M": 1024, "dtype": "bf16", "relu": True},
        # serving all nodes of a citation-scale graph with 8-bit weights
        {"name": "i8_nodes", "op": "i8", "N": 170000, "K": 256, "M": 256, "dtype": "bf16", "relu": True},
        # a wide 8-bit layer in fp32 features: bound by the products
        {"name": "i8_wide_f32", "op": "i8", "N": 16384, "K": 2048, "M": 2048, "dtype": "f32", "relu": False},
        # node classification: log probability of the label, entropy and the five best classes
        {"name": "log_probs_classes", "op": "log_probs", "N": 170000, "C": 47, "dtype": "f32", "top": 5, "masked": False},
        # ranking all nodes as answers to 256 queries, answers known already masked out
        {"name": "log_probs_entities", "op": "log_probs", "N": 256, "C": 170000, "dtype": "bf16", "top": 10, "masked": True},
        # training against many classes, with an entropy term
        {"name": "log_probs_grad", "op": "log_probs_grad", "N": 2048, "C": 50000, "dtype": "bf16", "masked": True},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["segments", "segments", "segments_grad", "i8", "i8", "log_probs", "log_probs", "log_probs_grad"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("segments", "segments_grad"):
        wide = 1024 if dtype == "bf16" else 256
        K, M = _spread(rng, 8, wide), _spread(rng, 8, wide)
        if rng.random() < 0.6:
            K, M = (K + 7) // 8 * 8, (M + 7) // 8 * 8
        G = _spread(rng, 1, 64)
        top = min(170000, int((6.0e10 if op == "segments" else 3.0e10) / (K * M)), int(4.0e7 / max(K, M)))
        case = {"op": op, "N": _spread(rng, min(G, top), top), "G": G, "K": K, "M": M, "dtype": dtype, "even": rng.random() < 0.3}
        if op == "segments":
            case["relu"] = rng.random() < 0.5
        return case
    if op == "i8":
        K, M = _spread(rng, 8, 2048), _spread(rng, 8, 2048)
        if rng.random() < 0.6:
            K = (K + 15) // 16 * 16
        top = min(170000, int(6.0e10 / (K * M)), int(4.0e7 / max(K, M)))
        return {"op": op, "N": _spread(rng, 1, top), "K": K, "M": M, "dtype": dtype, "relu": rng.random() < 0.5}
    C = _spread(rng, 2, 170000)
    N = _spread(rng, 1, min(170000, max(1, int(4.0e7 / C))))
    case = {"op": op, "N": N, "C": C, "dtype": dtype, "masked": C >= 16 and rng.random() < 0.5}
    if op == "log_probs":
        case["top"] = rng.randint(0, min(C // 2, 20))
    return case


def work(case):
    N, s = case["N"], 4 if case["dtype"] == "f32" else 2
    if case["op"] in ("segments", "segments_grad"):
        G, K, M = case["G"], case["K"], case["M"]
        if case["op"] == "segments":
            return {"bytes": s * (N * K + G * K * M + N * M) + 4 * G * M, "flops": 2 * N * K * M}
        return {"bytes": s * (2 * N * K + 2 * G * K * M + N * M), "flops": 4 * N * K * M}
    if case["op"] == "i8":
        K, M = case["K"], case["M"]
        return {"bytes": N * K * (s + 1) + K * M + N * M * s, "flops": 2 * N * K * M}
    C = case["C"]
    if case["op"] == "log_probs":
        return {"bytes": N * (C * s + 16 + 8 * case["top"]), "flops": 8 * N * C}
    return {"bytes": N * (2 * C * s + 20), "flops": 8 * N * C}


# ---------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _scale(x):
    """What one step of an 8-bit row stands for (a true quotient: dividing by a number would multiply by its reciprocal)."""
    top = x.abs().amax(1)
    return top / torch.full_like(top, 127.0)


def _sizes(case, seed):
    """Rows of each type: even, or ragged as the node types of a graph are, with one type in six empty."""
    N, G = case["N"], case["G"]
    if case["even"] or G == 1:
        return [N // G + (1 if g < N % G else 0) for g in range(G)]
    cpu = torch.Generator()
    cpu.manual_seed(seed)
    part = torch.rand(G, generator=cpu, dtype=torch.float64).clamp_(1e-3, 0.999).log_().neg_().pow_(1.5)
    part[torch.rand(G, generator=cpu) < 1.0 / 6.0] = 0.0
    if float(part.sum()) == 0.0:
        part[0] = 1.0
    cut = (part.cumsum(0) / part.sum() * N).round().long().tolist()
    return [b - a for a, b in zip([0] + cut[:-1], cut)]


def prepare(case, seed):
    gen = _generator(seed)
    dt = _DT[case["dtype"]]
    N, op = case["N"], case["op"]
    st = {"case": case}
    if op in ("segments", "segments_grad"):
        G, K, M = case["G"], case["K"], case["M"]
        sizes = _sizes(case, seed)
        ptr = [0]
        for n in sizes:
            ptr.append(ptr[-1] + n)
        st["ptr"] = ptr
        st["seg_ptr"] = torch.tensor(ptr, dtype=torch.int64, device="cuda")
        st["X"] = _normal(gen, (N, K), dt)
        st["W"] = _normal(gen, (G, K, M), dt, (2.0 / (K + M)) ** 0.5)
        if op == "segments":
            st["bias"] = _normal(gen, (G, M), _F32, 0.1)
        else:
            st["dY"] = _normal(gen, (N, M), dt)
    elif op == "i8":
        K, M = case["K"], case["M"]
        st["X"] = _normal(gen, (N, K), dt)
        W = _normal(gen, (M, K), _F32, (2.0 / (K + M)) ** 0.5)  # a row for each output channel
        st["wscale"] = _scale(W)
        st["Wq"] = torch.round(W.double() / st["wscale"].double()[:, None]).to(torch.int8)
        st["bias"] = _normal(gen, (M,), _F32, 0.1)
    else:
        C = case["C"]
        st["Z"] = _normal(gen, (N, C), dt, 2.5)
        label = torch.randint(0, C, (N,), generator=gen, device="cuda", dtype=torch.int32)
        rows = torch.arange(N, device="cuda")
        if case["masked"]:  # classes that cannot be the answer
            keep = st["Z"][rows, label.long()].clone()
            st["Z"].masked_fill_(torch.rand((N, C), generator=gen, device="cuda") < 0.1, float("-inf"))
            st["Z"][rows, label.long()] = keep
        label[torch.rand(N, generator=gen, device="cuda") < 0.1] = -1  # nodes without a label
        st["label"] = label
        if op == "log_probs_grad":  # what the forward pass left
            st["lse"], st["entropy"] = _statistics(st["Z"])
            st["dlogp"] = -(1.0 + 0.1 * torch.randn(N, generator=gen, device="cuda"))
            st["dentropy"] = -0.01 * (1.0 + 0.1 * torch.randn(N, generator=gen, device="cuda"))
    return st


# ---------------------------------------------------------------- plain forms
def _statistics(Z):
    """log sum exp and entropy of each row, in 32 bits."""
    z = Z.float()
    m = z.amax(1, keepdim=True)
    e = (z - m).exp()
    s = e.sum(1)
    lse = m[:, 0] + s.log()
    logp = z - lse[:, None]
    H = -(e / s[:, None] * logp.masked_fill(z == float("-inf"), 0.0)).sum(1)
    return lse, H


def _plain_segments(st):
    X, W, b, ptr = st["X"], st["W"], st["bias"], st["ptr"]
    Y = torch.empty((X.shape[0], W.shape[2]), dtype=X.dtype, device=X.device)
    for g in range(W.shape[0]):
        lo, hi = ptr[g], ptr[g + 1]
        if hi > lo:
            y = X[lo:hi].float() @ W[g].float() + b[g]
            Y[lo:hi] = y.clamp_min(0.0) if st["case"]["relu"] else y
    return Y


def _plain_segments_grad(st):
    X, W, dY, ptr = st["X"], st["W"], st["dY"], st["ptr"]
    dX, dW = torch.empty_like(X), torch.zeros_like(W)
    for g in range(W.shape[0]):
        lo, hi = ptr[g], ptr[g + 1]
        if hi > lo:
            d = dY[lo:hi].float()
            dX[lo:hi] = d @ W[g].float().t()
            dW[g] = X[lo:hi].float().t() @ d
    return dX, dW


def _plain_i8(st):
    x = st["X"].float()
    scale = _scale(x)
    # 64 bits where a quotient may lie next to a half
    q = torch.round(x.double() / scale.double().clamp_min(1e-300)[:, None]).to(torch.int8)
    acc = (q.double() @ st["Wq"].double().t()).float()  # sums of products pass 24 bits
    y = acc * (scale[:, None] * st["wscale"][None, :]) + st["bias"]
    if st["case"]["relu"]:
        y = y.clamp_min(0.0)
    return q, scale, y.to(st["X"].dtype)


def _plain_log_probs(st):
    Z, label, k = st["Z"], st["label"], st["case"]["top"]
    z = Z.float()
    lse, H = _statistics(Z)
    picked = z.gather(1, label.clamp_min(0).long()[:, None])[:, 0] - lse
    logp = torch.where(label >= 0, picked, torch.zeros_like(picked))
    out = {"logp": logp, "entropy": H, "lse": lse}
    if k > 0:
        # a key that orders by value, then by the lower index (-0 counts as 0)
        bits = (z + 0.0).view(torch.int32).long()
        order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))
        key = order * (1 << 32) + (0xFFFFFFFF - torch.arange(z.shape[1], device=z.device))
        idx = 0xFFFFFFFF - (key.topk(k, dim=1).values & 0xFFFFFFFF)
        out["top_logp"] = z.gather(1, idx) - lse[:, None]
        out["top_idx"] = idx.int()
    return out


def _plain_log_probs_grad(st):
    z, label = st["Z"].float(), st["label"]
    logp = z - st["lse"][:, None]
    p = logp.exp()
    dlogp = torch.where(label >= 0, st["dlogp"], torch.zeros_like(st["dlogp"]))
    d = -p * (dlogp[:, None] + st["dentropy"][:, None] * (logp.masked_fill(z == float("-inf"), 0.0) + st["entropy"][:, None]))
    rows = torch.arange(z.shape[0], device=z.device)
    d[rows, label.clamp_min(0).long()] += dlogp
    return d.to(st["Z"].dtype)


_PLAIN = {"segments": _plain_segments, "segments_grad": _plain_segments_grad, "i8": _plain_i8, "log_probs": _plain_log_probs,
          "log_probs_grad": _plain_log_probs_grad}


# ---------------------------------------------------------------- the library's calls
def _own(st):
    from paper_2412_06354_b200 import gnn
    case, op = st["case"], st["case"]["op"]
    if op == "segments":
        return gnn.linear_segments(st["X"], st["seg_ptr"], st["W"], bias=st["bias"], relu=case["relu"])
    if op == "segments_grad":
        return gnn.linear_segments_backward(st["X"], st["seg_ptr"], st["W"], st["dY"])
    if op == "i8":
        q, scale = gnn.quantize_rows(st["X"])
        return q, scale, gnn.linear_i8(q, scale, st["Wq"], st["wscale"], bias=st["bias"], relu=case["relu"], dtype=st["X"].dtype)
    if op == "log_probs":
        logp, entropy, lse, top_logp, top_idx = gnn.log_probs(st["Z"], st["label"], top=case["top"])
        out = {"logp": logp, "entropy": entropy, "lse": lse}
        if case["top"] > 0:
            out["top_logp"], out["top_idx"] = top_logp, top_idx
        return out
    return gnn.log_probs_backward(st["Z"], st["label"], st["lse"], st["dlogp"], entropy=st["entropy"], dentropy=st["dentropy"])


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------- 64 bits
def _exact_row_blocks(Z, per=1 << 24):
    step = max(1, per // Z.shape[1])
    for lo in range(0, Z.shape[0], step):
        yield lo, min(Z.shape[0], lo + step)


def exact(case, seed):
    st = prepare(case, seed)
    op, f64 = case["op"], torch.float64
    if op in ("segments", "segments_grad"):
        X, W = st["X"], st["W"]
        owner = torch.repeat_interleave(torch.arange(case["G"]), torch.tensor(_sizes(case, seed)))
        first = "segments" == op
        Y = torch.zeros((case["N"], case["M"] if first else case["K"]), dtype=f64, device="cuda")
        dW = torch.zeros(W.shape, dtype=f64, device="cuda")
        for g in owner.unique().tolist():
            rows = (owner == g).nonzero()[:, 0].to("cuda")
            if first:
                Y[rows] = torch.einsum("nk,km->nm", X[rows].to(f64), W[g].to(f64)) + st["bias"][g].to(f64)
            else:
                d = st["dY"][rows].to(f64)
                Y[rows] = torch.einsum("nm,km->nk", d, W[g].to(f64))
                dW[g] = torch.einsum("nk,nm->km", X[rows].to(f64), d)
        if first:
            return torch.relu(Y) if case["relu"] else Y
        return Y, dW
    if op == "i8":
        x = st["X"].to(f64)
        top = x.abs().max(dim=1).values
        scale = torch.div(top, torch.full_like(top, 127.0))
        stored = scale.to(_F32).to(f64)  # what the values are divided by
        q = torch.where(stored[:, None] > 0, x / torch.where(stored > 0, stored, torch.ones_like(stored))[:, None], torch.zeros_like(x)).round()
        y = torch.einsum("nk,mk->nm", q, st["Wq"].to(f64)) * stored[:, None] * st["wscale"].to(f64)[None] + st["bias"].to(f64)
        return q.to(torch.int8), scale, torch.relu(y) if case["relu"] else y
    Z, label = st["Z"], st["label"].long()
    N, C = Z.shape
    if op == "log_probs":
        k = case["top"]
        out = {n: torch.zeros(N, dtype=f64, device="cuda") for n in ("logp", "entropy", "lse")}
        if k > 0:
            out["top_logp"] = torch.zeros((N, k), dtype=f64, device="cuda")
            out["top_idx"] = torch.zeros((N, k), dtype=torch.int32, device="cuda")
        for lo, hi in _exact_row_blocks(Z):
            z = Z[lo:hi].to(f64)
            lse = torch.logsumexp(z, dim=1)
            lp = z - lse[:, None]
            out["lse"][lo:hi] = lse
            out["entropy"][lo:hi] = -torch.special.xlogy(lp.exp(), lp.exp()).sum(1)
            known = label[lo:hi] >= 0
            out["logp"][lo:hi][known] = lp[known, label[lo:hi][known]]
            if k > 0:
                v, i = torch.sort(z, dim=1, descending=True, stable=True)
                out["top_logp"][lo:hi] = v[:, :k] - lse[:, None]
                out["top_idx"][lo:hi] = i[:, :k].int()
        return out
    d = torch.zeros((N, C), dtype=f64, device="cuda")
    for lo, hi in _exact_row_blocks(Z):
        z = Z[lo:hi].to(f64)
        lp = z - st["lse"][lo:hi].to(f64)[:, None]
        p = lp.exp()
        known = label[lo:hi] >= 0
        g = torch.where(known, st["dlogp"][lo:hi].to(f64), torch.zeros(hi - lo, dtype=f64, device="cuda"))
        part = -p * g[:, None]
        part[known, label[lo:hi][known]] += g[known]
        slope = torch.where(p > 0, p * (lp + st["entropy"][lo:hi].to(f64)[:, None]), torch.zeros_like(p))
        d[lo:hi] = part - st["dentropy"][lo:hi].to(f64)[:, None] * slope
    return d
