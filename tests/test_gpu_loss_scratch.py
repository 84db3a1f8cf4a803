"""The handle's scratch of the losses: what calls of growing sizes leave behind, and graphs recorded before it grew."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import Domino  # noqa: E402
from test_gpu_token_loss import d, inputs  # noqa: E402,F401


def held(calls):
    """Device bytes of a handle after the losses of these sizes (rows off 16-byte boundaries: the weight is laid out anew)."""
    d = Domino(0)  # noqa: F811
    before = d.info()["device_bytes"]
    for T, V, D in calls:
        h, w, y, _, _ = inputs(T, V, D)
        d.token_loss(h, w, y)
    torch.cuda.synchronize()
    n = d.info()["device_bytes"] - before
    d.close()
    return n


def test_outgrown_scratch_is_given_back(d):  # noqa: F811
    """At most a quarter more than the largest call needs."""
    sizes = [(64, 20000 + 800 * i, 1001) for i in range(8)]
    need = held(sizes[-1:])
    assert need >= 2 * sizes[-1][1] * 1008
    assert held(sizes) <= 1.25 * need
    assert held([(64, 1000, 1001)] + sizes[-1:]) <= 1.25 * need


def test_a_recorded_graph_keeps_its_scratch():
    d = Domino(0)  # noqa: F811
    h, w, y, mask, c = inputs(70, 900, 65, density=0.5)
    loss, lse = d.token_loss(h, w, y, mask)
    dh, dw = d.token_loss_grad(h, w, y, lse, c, mask)
    out = [torch.empty_like(t) for t in (loss, lse, dh, dw)]
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        d.token_loss(h, w, y, mask, out=(out[0], out[1]))
        d.token_loss_grad(h, w, y, out[1], c, mask, out=(out[2], out[3]))
    for V in (5000, 9000, 30000):                       # the scratch grows, and is used
        H, W, Y, _, _ = inputs(64, V, 1001)
        d.token_loss(H, W, Y)
    for t in out:
        t.fill_(7)
    g.replay()
    torch.cuda.synchronize()
    for a, b in zip(out, (loss, lse, dh, dw)):
        assert torch.equal(a, b)
    del g
    d.close()
