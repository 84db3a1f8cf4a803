"""A teacher's list for distill_loss and distill_grad: logits of -inf in it."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from loss_reference import INF, Distill, assert_within  # noqa: E402
from test_gpu_distill import d, inputs  # noqa: E402,F401


@pytest.mark.parametrize("teacher", ["f32", "bf16"])
@pytest.mark.parametrize("density", [None, 0.5])
def test_teacher_logits_of_minus_infinity(d, teacher, density):  # noqa: F811
    """They are no entries, wherever they stand: in all of a row's places, beside others, before an equal id."""
    x, t, ids, mask, c = inputs(12, 3000, 20, "f32", density, teacher=teacher)
    g = torch.Generator("cuda").manual_seed(3)
    t[torch.rand(t.shape, generator=g, device="cuda") < 0.3] = -INF
    t[7] = -INF                                # nothing is left
    t[8], t[8, 11] = -INF, 0.5                 # one entry
    t[9, 2:4], ids[9, 3] = 1.0, ids[9, 2]
    t[9, 2] = -INF                             # the second of two equal ids counts
    ref = Distill(x, t.masked_fill(t == -INF, 0.0), ids.masked_fill(t == -INF, -1), 1.5, mask, c)
    loss, lse = d.distill_loss(x, t, ids, 1.5, mask)
    dx = d.distill_grad(x, t, ids, 1.5, lse, c, mask)
    for name, got in (("lse", lse), ("loss", loss), ("dlogits", dx)):
        assert_within(got, getattr(ref, name), ref.tol[name], name)
    assert loss[7] == 0 and not dx[7].any()
