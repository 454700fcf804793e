"""Shapes, types and layouts that the binding of the typed, 8-bit and last-layer calls refuses before it calls the library."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gnn():
    from paper_2412_06354_b200 import gnn as g
    g.load()
    return g


def test_arguments_that_do_not_fit_one_another(gnn):
    import torch
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")
    X, ptr, W, dY = z(6, 8), z(3, dt=torch.int64), z(2, 8, 16), z(6, 16)
    q, s = z(6, 8, dt=torch.int8), z(6)
    w, sw = z(16, 8, dt=torch.int8), z(16)
    y = z(6, dt=torch.int32)
    value = [lambda: gnn.linear_segments(X, z(4, dt=torch.int64), W), lambda: gnn.linear_segments(X, ptr, z(2, 9, 16)), lambda: gnn.linear_segments(X, ptr, z(8, 16)),
             lambda: gnn.linear_segments(X, ptr, W, bias=z(16)), lambda: gnn.linear_segments_backward(X, ptr, W, z(6, 8)), lambda: gnn.linear_segments_backward(z(5, 8), ptr, W, dY),
             lambda: gnn.linear_i8(q, z(5), w, sw), lambda: gnn.linear_i8(q, s, z(16, 9, dt=torch.int8), sw), lambda: gnn.linear_i8(q, s, w, s), lambda: gnn.linear_i8(q, s, w, sw, bias=s),
             lambda: gnn.quantize_rows(z(6)), lambda: gnn.log_probs(z(6)), lambda: gnn.log_probs(X, z(5, dt=torch.int32)), lambda: gnn.log_probs(X, y, top=9), lambda: gnn.log_probs(X, y, top=-1),
             lambda: gnn.log_probs_backward(X, y, z(5)), lambda: gnn.log_probs_backward(X, y, s, dlogp=z(7)), lambda: gnn.log_probs(X, y.cpu()), lambda: gnn.linear_segments(X, ptr, W, bias=torch.zeros(2, 16))]
    types = [lambda: gnn.linear_segments(X, ptr.int(), W), lambda: gnn.linear_segments(X, ptr, W.bfloat16()), lambda: gnn.linear_segments(X.half(), ptr, W.half()),
             lambda: gnn.linear_segments(X, ptr, W, bias=z(2, 16, dt=torch.float64)), lambda: gnn.linear_segments_backward(X, ptr, W, dY.bfloat16()), lambda: gnn.quantize_rows(X.half()),
             lambda: gnn.linear_i8(X, s, w, sw), lambda: gnn.linear_i8(q, s.double(), w, sw), lambda: gnn.log_probs(X.half()), lambda: gnn.log_probs(X, y.long()),
             lambda: gnn.log_probs_backward(X, y, s.double()), lambda: gnn.linear_segments(X, ptr, W, ws=z(100000)), lambda: gnn.linear_segments(X, ptr, W.transpose(1, 2).contiguous(), bias=z(16, 2).t())]
    layout = [lambda: gnn.linear_segments(z(8, 6).t(), ptr, W), lambda: gnn.linear_segments(X, ptr, z(2, 16, 8).transpose(1, 2)), lambda: gnn.quantize_rows(z(6, 16)[:, :8]),
              lambda: gnn.linear_i8(q, s, z(8, 16, dt=torch.int8).t(), sw), lambda: gnn.log_probs(z(6, 9)[:, :8]), lambda: gnn.linear_segments_backward(None, ptr, W, dY)]
    for call in value:
        with pytest.raises(ValueError):
            call()
    for call in types:
        with pytest.raises((TypeError, ValueError)):
            call()
    for call in layout:
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(gnn.GnnError) as e:
        gnn.linear_segments(z(49)[1:].view(6, 8), ptr, W)  # four bytes off 16
    assert e.value.status == 1
    with pytest.raises(gnn.GnnError) as e:
        gnn.linear_segments(X, ptr, W, ws=z(256, dt=torch.uint8))
    assert e.value.status == 4
    with pytest.raises(gnn.GnnError) as e:
        gnn.log_probs(z(2, 64), top=33)
    assert e.value.status == 5
