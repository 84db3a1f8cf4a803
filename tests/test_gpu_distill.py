"""domino_distill_loss and domino_distill_grad against their definitions in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import Domino, DominoError  # noqa: E402
from paper_2403_06988_gb300 import _binding as B  # noqa: E402
from loss_reference import INF, Distill, assert_within, pack  # noqa: E402

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def d():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2403_06988_gb300 import build
    build.build()
    d = Domino(0)
    yield d
    assert d.device_error() == 0
    d.close()


def inputs(T, V, K, dtype="f32", density=None, seed=0, teacher="f32"):
    g = torch.Generator("cuda").manual_seed(1000 * T + 10 * V + K + seed)
    x = (torch.randn(T, V, generator=g, device="cuda") * 3).to(TYPES[dtype])
    ids = torch.rand(T, V, generator=g, device="cuda").topk(min(K, V), dim=1).indices.int()
    if K > V:
        ids = torch.cat([ids, torch.full((T, K - V), -1, dtype=torch.int32, device="cuda")], 1)
    t = (torch.randn(T, K, generator=g, device="cuda") * 2).to(TYPES[teacher])
    bits = None
    if density is not None:
        bits = torch.rand(T, V, generator=g, device="cuda") < density
        bits.scatter_(1, ids[:, :max(1, K // 2)].long().clamp(min=0), True)
        if T > 3:
            bits[1] = False                        # nothing allowed
            bits[2] = False
            bits[2, int(ids[2, 0])] = True         # one token
    if T > 6 and K > 2:
        ids[4, 1:] = -1                            # one entry
        ids[5] = -1                                # none
        ids[6, 2] = ids[6, 0]                      # the same id twice
    c = torch.randn(T, generator=g, device="cuda") / T
    return x, t, ids, None if bits is None else pack(bits), c


def check(d, x, t, ids, tau, mask, c, what):
    ref = Distill(x, t, ids, tau, mask, c)
    loss, lse = d.distill_loss(x, t, ids, tau, mask)
    dx = d.distill_grad(x, t, ids, tau, lse, c, mask)
    for name, got in (("lse", lse), ("loss", loss), ("dlogits", dx)):
        assert_within(got, getattr(ref, name), ref.tol[name], f"{what}: {name}")
    return ref, dx


@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (1, 7, 3), (2, 31, 40), (9, 1003, 16), (7, 4096, 1024), (40, 33000, 64),
                                   (400, 5001, 5), (1, 150001, 513)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("density", [None, 0.01, 0.8])
def test_loss_and_gradient(d, T, V, K, dtype, density):
    x, t, ids, mask, c = inputs(T, V, K, dtype, density)
    check(d, x, t, ids, 1.5, mask, c, f"{T} x {V}, {K}")


@pytest.mark.parametrize("tau", [0.25, 1.0, 8.0])
def test_temperatures_and_bf16_teacher(d, tau):
    x, t, ids, mask, c = inputs(20, 3000, 30, "bf16", 0.3, teacher="bf16")
    check(d, x, t, ids, tau, mask, c, f"temperature {tau}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off,pad,to_off,to_pad", [(1, 2, 1, 2), (0, 5, 3, 1), (8, 0, 0, 8)])
def test_strides_and_alignment(d, dtype, off, pad, to_off, to_pad):
    T, V = 12, 2500
    x, t, ids, mask, c = inputs(T, V, 20, dtype, 0.5)
    ref = Distill(x, t, ids, 2.0, mask, c)

    def apart(v, off, pad):
        big = torch.full((T, off + V + pad), float("nan"), dtype=v.dtype, device="cuda")
        big[:, off:off + V] = v
        return big[:, off:off + V]
    xs = apart(x, off, pad)
    loss, lse = d.distill_loss(xs, t, ids, 2.0, mask)
    out = apart(torch.zeros_like(x), to_off, to_pad)
    d.distill_grad(xs, t, ids, 2.0, lse, c, mask, out=out)
    for name, got in (("lse", lse), ("loss", loss), ("dlogits", out)):
        assert_within(got, getattr(ref, name), ref.tol[name], name)
    base = out._base
    assert torch.isnan(base[:, :to_off]).all() and torch.isnan(base[:, to_off + V:]).all()


@pytest.mark.parametrize("T", [2, 300])
def test_in_place(d, T):
    x, t, ids, mask, c = inputs(T, 20001, 48, "bf16", 0.3)
    _, lse = d.distill_loss(x, t, ids, 2.0, mask)
    want = d.distill_grad(x, t, ids, 2.0, lse, c, mask)
    y = x.clone()
    d.distill_grad(y, t, ids, 2.0, lse, c, mask, out=y)
    assert torch.equal(y, want)


@pytest.mark.parametrize("value", [float("nan"), INF, -INF, 3e38])
def test_masked_places_hold_anything(d, value):
    x, t, ids, mask, c = inputs(20, 3000, 12, "f32", 0.4)
    ref = Distill(x, t, ids, 1.0, mask, c)
    from loss_reference import unpack
    x2 = x.masked_fill(~unpack(mask, 3000), value)
    loss, lse = d.distill_loss(x2, t, ids, 1.0, mask)
    dx = d.distill_grad(x2, t, ids, 1.0, lse, c, mask)
    for name, got in (("lse", lse), ("loss", loss), ("dlogits", dx)):
        assert_within(got, getattr(ref, name), ref.tol[name], name)


@pytest.mark.parametrize("ban", [-INF, -1e10, torch.finfo(torch.float32).min])
def test_banned_tokens(d, ban):
    """Logits of -inf, or of the type's lowest value, beside ordinary ones."""
    x, t, ids, _, c = inputs(8, 5000, 10)
    x[:, 100:4000] = ban
    x[torch.arange(8, device="cuda")[:, None], ids.clamp(min=0).long()] = 1.0
    x[3, int(ids[3, 1])] = -INF           # an entry that the student bans
    loss, lse = d.distill_loss(x, t, ids, 2.0)
    dx = d.distill_grad(x, t, ids, 2.0, lse, c)
    ref = Distill(x.clamp(min=-200.0).masked_fill(x == -INF, -INF), t, ids, 2.0, None, c)
    for name, got in (("lse", lse), ("loss", loss), ("dlogits", dx)):
        assert_within(got, getattr(ref, name), ref.tol[name], name)


def test_gradient_against_differences(d):
    x, t, ids, mask, c = inputs(12, 200, 9, "f32", 0.6)
    ref, dx = check(d, x, t, ids, 2.0, mask, c, "differences")
    g = torch.Generator("cuda").manual_seed(5)
    for _ in range(4):
        e = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64)
        s = 1e-5
        up, down = (Distill(x.double() + k * s * e, t, ids, 2.0, mask).loss for k in (1, -1))
        rise = float(((up - down) * c.double()).sum()) / (2 * s)
        got = float((dx.double() * e).sum())
        assert abs(got - rise) <= float((ref.tol["dlogits"] * e.abs()).sum()) + 1e-7


def test_same_bits_again_and_on_another_stream(d):
    x, t, ids, mask, c = inputs(5, 60000, 100, "bf16", 0.3)
    a = d.distill_loss(x, t, ids, 1.0, mask)
    ga = d.distill_grad(x, t, ids, 1.0, a[1], c, mask)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = d.distill_loss(x, t, ids, 1.0, mask)
        gb = d.distill_grad(x, t, ids, 1.0, b[1], c, mask)
    s.synchronize()
    for p, q in zip(a + (ga,), b + (gb,)):
        assert torch.equal(p, q)


def test_no_rows_and_bad_ids():
    d = Domino(0)
    x, t, ids, _, c = inputs(4, 100, 5)
    loss, lse = d.distill_loss(x[:0], t[:0], ids[:0])
    assert loss.shape == (0,) and d.distill_grad(x[:0], t[:0], ids[:0], 1.0, lse, c[:0]).shape == (0, 100)
    good = ids.clone()
    ids[2, 3], good[2, 3] = 100, -1
    loss, lse = d.distill_loss(x, t, ids)
    assert d.device_error() == 4
    d.distill_grad(x, t, ids, 1.0, lse, c)
    assert d.device_error() == 4
    ref = Distill(x, t, good, 1.0)
    assert_within(loss, ref.loss, ref.tol["loss"], "loss")
    d.close()


def test_refusals(d):
    x, t, ids, mask, c = inputs(4, 100, 5, density=0.5)
    with pytest.raises(TypeError):
        d.distill_loss(x.double(), t, ids)
    with pytest.raises(TypeError):
        d.distill_loss(x, t, ids.long())
    with pytest.raises(ValueError):
        d.distill_loss(x, t, ids[:, :3].contiguous())
    with pytest.raises(ValueError):
        d.distill_loss(x, t, ids, mask=mask[:2])
    for tau in (0.0, -1.0, INF, float("nan"), 1e-39):
        with pytest.raises(DominoError) as e:
            d.distill_loss(x, t, ids, tau)
        assert e.value.status == -1
    _, lse = d.distill_loss(x, t, ids)
    wide = torch.empty(4, 200, device="cuda")
    with pytest.raises(DominoError) as e:    # in place, but with another stride
        B.domino_distill_grad(d.h, wide, 0, 4, 200, 100, None, t, 0, ids, 5, 1.0, lse, c, wide, 100)
    assert e.value.status == -1
    many = torch.zeros(4, 1025, device="cuda")
    with pytest.raises(DominoError) as e:
        d.distill_loss(x, many, many.int())
    assert e.value.status == -1
