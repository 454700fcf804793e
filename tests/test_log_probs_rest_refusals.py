"""What the log probabilities' calls with lse in two numbers refuse, seen on the host before any launch (no GPU needed)."""
import pytest

from paper_2412_06354_b200 import gnn
from test_dense_refusals import BIG, INVALID, ODD, P, SMALL, UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    return gnn.load()


def test_forward(lib):
    def call(Z=P, label=P, N=10, C=50, dtype=gnn.F32, top=3, logp=P, H=P, lse=P, rest=P, tl=P, ti=P, ws=P, n=BIG):
        return lib.gnn_log_probs_rest(Z, label, N, C, dtype, top, logp, H, lse, rest, tl, ti, ws, n, None)
    for rest in (P, None):
        for bad in (dict(N=-1), dict(C=0), dict(dtype=3), dict(top=-1), dict(top=51), dict(label=None), dict(Z=None), dict(tl=None), dict(ti=None), dict(Z=ODD)):
            assert call(rest=rest, **bad) == INVALID, bad
    assert call(top=33) == UNSUPPORTED and call(N=0) == 0
    need = lib.gnn_log_probs_workspace(2, 1 << 20, 3, gnn.F32)
    assert call(N=2, C=1 << 20, n=need - 1) == SMALL


def test_backward(lib):
    def call(Z=P, label=P, lse=P, rest=P, H=P, dlogp=P, dH=P, N=10, C=50, dtype=gnn.F32, dZ=P):
        return lib.gnn_log_probs_rest_backward(Z, label, lse, rest, H, dlogp, dH, N, C, dtype, dZ, None)
    for rest in (P, None):
        for bad in (dict(N=-1), dict(C=0), dict(dtype=3), dict(label=None), dict(H=None), dict(Z=None), dict(lse=None), dict(dZ=None), dict(Z=ODD), dict(dZ=ODD)):
            assert call(rest=rest, **bad) == INVALID, bad
    assert call(N=0) == 0
