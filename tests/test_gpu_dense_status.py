"""The status word of the dense calls' workspaces: 0 after every call that ran, calls without rows among them."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gnn():
    from paper_2412_06354_b200 import gnn as g
    g.load()
    return g


def status(ws):
    import torch
    torch.cuda.synchronize()
    return int(ws[:4].view(torch.int32).item())


@pytest.mark.parametrize("n", [0, 1, 40])
def test_written_whatever_the_workspace_held(gnn, n):
    import torch
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")
    junk = lambda: torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
    ptr, W = z(3, dt=torch.int64), z(2, 32, 16)
    ws = junk()
    gnn.linear_i8(z(n, 32, dt=torch.int8), z(n), z(16, 32, dt=torch.int8), z(16), ws=ws)
    assert status(ws) == 0
    ws = junk()
    gnn.linear_segments(z(n, 32), ptr, W, ws=ws)
    assert status(ws) == 0
    ws = junk()
    gnn.linear_segments_backward(z(n, 32), ptr, W, z(n, 16), ws=ws)
    assert status(ws) == 0
