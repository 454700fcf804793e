"""What the typed, 8-bit and last-layer calls refuse, seen on the host before any launch (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2412_06354_b200 import gnn

P = C.c_void_p(0x1000)    # on 16 bytes, never read
ODD = C.c_void_p(0x1004)
BIG = 1 << 40
INVALID, SMALL, UNSUPPORTED = 1, 4, 5


@pytest.fixture(scope="module")
def lib():
    return gnn.load()


def segments(lib, X=P, ptr=P, W=P, N=10, G=2, K=8, M=8, dtype=gnn.F32, Y=P, ws=P, n=BIG):
    return lib.gnn_linear_segments(X, ptr, W, N, G, K, M, dtype, None, 0, Y, ws, n, None)


def segments_backward(lib, X=P, ptr=P, W=P, dY=P, N=10, G=2, K=8, M=8, dtype=gnn.F32, dX=P, dW=P, ws=P, n=BIG):
    return lib.gnn_linear_segments_backward(X, ptr, W, dY, N, G, K, M, dtype, dX, dW, ws, n, None)


def i8(lib, xq=P, sx=P, wq=P, sw=P, N=10, K=8, M=8, dtype=gnn.F32, Y=P, ws=P, n=BIG):
    return lib.gnn_linear_i8(xq, sx, wq, sw, N, K, M, dtype, None, 0, Y, ws, n, None)


def probs(lib, Z=P, label=P, N=10, Cn=50, dtype=gnn.F32, top=3, logp=P, H=P, lse=P, tl=P, ti=P, ws=P, n=BIG):
    return lib.gnn_log_probs(Z, label, N, Cn, dtype, top, logp, H, lse, tl, ti, ws, n, None)


def probs_backward(lib, Z=P, label=P, lse=P, H=P, dlogp=P, dH=P, N=10, Cn=50, dtype=gnn.F32, dZ=P):
    return lib.gnn_log_probs_backward(Z, label, lse, H, dlogp, dH, N, Cn, dtype, dZ, None)


@pytest.mark.parametrize("call", [segments, segments_backward])
def test_segments(lib, call):
    for bad in (dict(N=-1), dict(G=-1), dict(K=0), dict(M=0), dict(dtype=2), dict(ptr=None), dict(X=None), dict(W=None), dict(X=ODD), dict(W=ODD), dict(ws=ODD)):
        assert call(lib, **bad) == INVALID, bad
    for bad in (dict(ws=None), dict(n=255)):
        assert call(lib, **bad) == SMALL, bad
    for bad in (dict(K=2049), dict(M=2049), dict(K=8193, dtype=gnn.BF16), dict(G=1 << 24, K=256, dtype=gnn.BF16)):
        assert call(lib, **bad) == UNSUPPORTED, bad
    back = int(call is segments_backward)
    need = lib.gnn_linear_segments_workspace(10, 2, 8, 8, gnn.F32, back)
    assert need > 256 and call(lib, n=need - 1) == SMALL
    assert b"bytes needed" in lib.gnn_last_error_string()


def test_segments_outputs(lib):
    assert segments(lib, Y=None) == INVALID and segments(lib, Y=ODD) == INVALID
    assert segments_backward(lib, dY=None) == INVALID
    for bad in (dict(dX=ODD), dict(dW=ODD), dict(dY=ODD)):
        assert segments_backward(lib, **bad) == INVALID, bad


def test_segments_workspace(lib):
    ws = lib.gnn_linear_segments_workspace
    assert ws(1000, 4, 64, 64, gnn.BF16, 0) == 256                           # rows on 16 bytes as they are
    assert ws(1000, 4, 100, 47, gnn.BF16, 0) >= 2 * (1000 * 104 + 400 * 48)  # padded copies
    assert ws(1000, 4, 64, 64, gnn.F32, 0) >= 6 * 256 * 64                   # three terms of the weights
    assert ws(1000, 4, 64, 64, gnn.F32, 1) > ws(1000, 4, 64, 64, gnn.F32, 0)
    assert ws(-1, 4, 64, 64, gnn.F32, 0) == 0 and ws(5, 4, 0, 64, gnn.F32, 1) == 0


def test_quantize_rows(lib):
    call = lambda X=P, N=4, K=8, dtype=gnn.F32, q=P, s=P: lib.gnn_quantize_rows(X, N, K, dtype, q, s, None)
    for bad in (dict(N=-1), dict(K=0), dict(dtype=5), dict(X=None), dict(q=None), dict(s=None), dict(X=ODD), dict(q=ODD)):
        assert call(**bad) == INVALID, bad
    assert call(N=0) == 0


@pytest.mark.parametrize("N", [3, 100])
def test_linear_i8(lib, N):
    for bad in (dict(N=-1), dict(K=0), dict(M=0), dict(dtype=7), dict(xq=None), dict(sx=None), dict(wq=None), dict(sw=None), dict(Y=None), dict(xq=ODD), dict(wq=ODD), dict(Y=ODD), dict(ws=ODD)):
        assert i8(lib, **{"N": N, **bad}) == INVALID, bad
    assert i8(lib, N=N, K=131072) == UNSUPPORTED
    assert i8(lib, N=N, ws=None) == SMALL and i8(lib, N=N, n=lib.gnn_linear_i8_workspace(N, 8, 8) - 1) == SMALL


def test_log_probs(lib):
    for bad in (dict(N=-1), dict(Cn=0), dict(dtype=3), dict(top=-1), dict(top=51), dict(label=None), dict(Z=None), dict(tl=None), dict(ti=None), dict(Z=ODD)):
        assert probs(lib, **bad) == INVALID, bad
    assert probs(lib, top=33) == UNSUPPORTED
    need = lib.gnn_log_probs_workspace(2, 1 << 20, 3, gnn.F32)
    assert need > 0
    for bad in (dict(ws=None), dict(n=need - 1), dict(ws=ODD)):
        assert probs(lib, N=2, Cn=1 << 20, **bad) == SMALL, bad
    assert lib.gnn_log_probs_workspace(2, 100, 33, gnn.F32) == 0


def test_log_probs_backward(lib):
    for bad in (dict(N=-1), dict(Cn=0), dict(dtype=3), dict(label=None), dict(H=None), dict(Z=None), dict(lse=None), dict(dZ=None), dict(Z=ODD), dict(dZ=ODD)):
        assert probs_backward(lib, **bad) == INVALID, bad


def test_the_binding_takes_device_tensors_only():
    x = torch.zeros(4, 8)
    ptr = torch.zeros(3, dtype=torch.int64)
    W = torch.zeros(2, 8, 8)
    s = torch.zeros(4)
    for call in (lambda: gnn.linear_segments(x, ptr, W), lambda: gnn.linear_segments_backward(x, ptr, W, x), lambda: gnn.quantize_rows(x),
                 lambda: gnn.linear_i8(x.to(torch.int8), s, x.to(torch.int8), s), lambda: gnn.log_probs(x), lambda: gnn.log_probs_backward(x, None, s)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(TypeError):
        gnn.linear_i8(x.to(torch.int8), s, x.to(torch.int8), s, dtype=torch.float16)
