"""distill_loss and distill_grad of logits whose quotient by the temperature is far from a whole number of units in the last
place: the log-sum-exp and the differences from it are made of the same rounded quotients."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from loss_reference import pack  # noqa: E402
from test_gpu_distill import TYPES, d  # noqa: E402,F401

SIZES = [1.0, 1e3, 1e6, 1e9, 1e20, torch.finfo(torch.float32).max]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tau", [0.7, 1.5, 3.0])
def test_one_allowed_token(d, dtype, tau):  # noqa: F811
    """q is 1 there, whatever its logit: no divergence and no gradient."""
    T, V = 2 * len(SIZES), 5000
    x = torch.zeros(T, V, dtype=TYPES[dtype], device="cuda")
    at = torch.arange(T, device="cuda") * 401 + 3
    value = torch.tensor([s * k for s in SIZES for k in (1, -0.93)], device="cuda").to(TYPES[dtype])
    x[torch.arange(T, device="cuda"), at] = value.clamp(-torch.finfo(TYPES[dtype]).max, torch.finfo(TYPES[dtype]).max)
    bits = torch.zeros(T, V, dtype=torch.bool, device="cuda")
    bits[torch.arange(T, device="cuda"), at] = True
    c = torch.ones(T, device="cuda")
    ok = x.float().abs().amax(1) / tau < torch.finfo(torch.float32).max     # the quotient is a number
    loss, lse = d.distill_loss(x, torch.zeros(T, 1, device="cuda"), at.int()[:, None], tau, pack(bits))
    dx = d.distill_grad(x, torch.zeros(T, 1, device="cuda"), at.int()[:, None], tau, lse, c, pack(bits))
    assert ok.sum() >= T - 2
    assert not loss[ok].any() and not dx[ok].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tau", [1.5, 3.0])
def test_gradients_stay_within_their_weight(d, dtype, tau):  # noqa: F811
    """|q - p| <= 1, as lse is no smaller than the largest quotient: also where every logit is the type's lowest."""
    T, V = len(SIZES) + 1, 3000
    g = torch.Generator("cuda").manual_seed(2)
    x = torch.randn(T, V, generator=g, device="cuda").clamp(-3, 3) / 3
    x = (x * torch.tensor(SIZES + [1.0], device="cuda")[:, None]).to(TYPES[dtype])
    x = x.clamp(-torch.finfo(TYPES[dtype]).max, torch.finfo(TYPES[dtype]).max)
    x[-1] = torch.finfo(TYPES[dtype]).min
    ids = torch.arange(T, device="cuda").int()[:, None] * 7
    loss, lse = d.distill_loss(x, torch.zeros(T, 1, device="cuda"), ids, tau)
    dx = d.distill_grad(x, torch.zeros(T, 1, device="cuda"), ids, tau, lse, torch.ones(T, device="cuda"))
    assert torch.isfinite(lse).all()
    assert float(dx.abs().max()) <= tau * (1 + 2.0 ** -8)
