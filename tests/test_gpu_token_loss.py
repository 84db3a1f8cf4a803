"""domino_token_loss and domino_token_loss_grad against their definitions in 64 bits: sizes around the edges of tiles
(128 rows, 256 tokens, 64 values), rows without a target or with nothing allowed, strides and alignments, several
pieces of the vocabulary, differences, repeatability, other streams."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import Domino, DominoError  # noqa: E402
from paper_2403_06988_gb300 import _binding as B  # noqa: E402
from loss_reference import INF, TokenLoss, assert_within, pack  # noqa: E402


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


def inputs(T, V, D, seed=0, density=None, spread=2.0):
    g = torch.Generator("cuda").manual_seed(1000 * T + 10 * V + D + seed)
    h = torch.randn(T, D, generator=g, device="cuda").bfloat16()
    w = (torch.randn(V, D, generator=g, device="cuda") * spread / D ** 0.5).bfloat16()
    y = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    mask = None
    if density is not None:
        bits = torch.rand(T, V, generator=g, device="cuda") < density
        bits[torch.arange(T, device="cuda"), y.long()] = True
        if T > 4:
            bits[1] = False                                   # nothing allowed
            bits[2, int(y[2])] = False                        # the target excluded
            bits[3] = False
            bits[3, int(y[3])] = True                         # the target alone
        mask = pack(bits)
    if T > 6:
        y[5], y[6] = -1, -100
    c = torch.randn(T, generator=g, device="cuda") / T
    return h, w, y, mask, c


def check(d, h, w, y, mask, c, what):
    ref = TokenLoss(h, w, y, mask, c)
    loss, lse = d.token_loss(h, w, y, mask)
    dh, dw = d.token_loss_grad(h, w, y, lse, c, mask)
    for name, got in (("lse", lse), ("loss", loss), ("dhidden", dh), ("dweight", dw)):
        assert_within(got, getattr(ref, name), ref.tol[name], f"{what}: {name}")
    return ref, (loss, lse, dh, dw)


SIZES = [(1, 1, 1), (1, 257, 64), (2, 31, 7), (3, 1000, 63), (7, 256, 65), (127, 255, 128), (128, 511, 200),
         (129, 1003, 72), (300, 5000, 512), (257, 2049, 1000), (33, 40000, 96)]


@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("density", [None, 0.02, 0.7])
def test_loss_and_gradient(d, T, V, D, density):
    check(d, *inputs(T, V, D, density=density), f"{T} x {V} x {D}")


@pytest.mark.parametrize("T,V,D", [(2, 33001, 517), (3, 9000, 1904), (3, 33001, 517), (4, 5000, 2048), (4, 33001, 517)])
@pytest.mark.parametrize("density", [None, 0.02, 0.7])
def test_few_rows_of_a_large_weight(d, T, V, D, density):
    check(d, *inputs(T, V, D, density=density), f"{T} x {V} x {D}")


def test_several_pieces_of_the_vocabulary(d):
    """G of 2100 x 65600 tokens passes what is kept at a time; the last piece is short."""
    check(d, *inputs(2100, 65600, 64, density=0.3), "pieces")


def test_many_row_tiles(d):
    check(d, *inputs(2500, 700, 40), "row tiles")


@pytest.mark.parametrize("off,pad", [(0, 8), (1, 0), (3, 5), (8, 3)])
def test_strides_and_alignment(d, off, pad):
    T, V, D = 70, 700, 104
    h, w, y, mask, c = inputs(T, V, D, density=0.5)

    def apart(x):
        big = torch.full((x.shape[0], off + D + pad), float("nan"), dtype=x.dtype, device="cuda")
        big[:, off:off + D] = x
        return big[:, off:off + D]
    ref = TokenLoss(h, w, y, mask, c)
    loss, lse = d.token_loss(apart(h), apart(w), y, mask)
    out = (apart(torch.zeros_like(h)), apart(torch.zeros_like(w)))
    dh, dw = d.token_loss_grad(apart(h), apart(w), y, lse, c, mask, out=out)
    for name, got in (("lse", lse), ("loss", loss), ("dhidden", dh), ("dweight", dw)):
        assert_within(got, getattr(ref, name), ref.tol[name], f"offset {off}, pad {pad}: {name}")
    for o in out:   # nothing beside the rows was written
        base = o._base
        assert torch.isnan(base[:, :off]).all() and torch.isnan(base[:, off + D:]).all()


def test_rows_without_a_gradient_do_not_touch_others(d):
    """Padding may hold anything, and its weight may be anything."""
    h, w, y, mask, c = inputs(40, 600, 48, density=0.4)
    ref = TokenLoss(h, w, y, mask, c)
    h2, c2 = h.clone(), c.clone()
    for row in (1, 2, 5, 6):
        h2[row] = float("nan")
        c2[row] = INF
    _, lse = d.token_loss(h, w, y, mask)
    dh, dw = d.token_loss_grad(h2, w, y, lse, c2, mask)
    assert_within(dw, ref.dweight, ref.tol["dweight"], "dweight")
    assert_within(dh, ref.dhidden, ref.tol["dhidden"], "dhidden")
    assert not dh[[1, 2, 5, 6]].any()


def test_nan_stays_in_its_row(d):
    h, w, y, mask, c = inputs(9, 300, 32)
    h[4] = float("nan")
    loss, lse = d.token_loss(h, w, y, mask)
    assert torch.isnan(loss[4]) and torch.isnan(lse[4])
    keep = torch.tensor([0, 1, 2, 3, 7, 8], device="cuda")
    ref = TokenLoss(h[keep], w, y[keep])
    assert_within(loss[keep], ref.loss, ref.tol["loss"], "other rows")


@pytest.mark.parametrize("size", [1e4, 1e9, 1e15])
def test_large_logits(d, size):
    """Two tokens share the maximum: the loss is ln 2 for one of them, whatever the logits' size."""
    h = torch.zeros(3, 8, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(500, 8, dtype=torch.bfloat16, device="cuda")
    h[:, 0] = 1.0
    w[:, 0] = -size
    w[[17, 400], 0] = size
    y = torch.tensor([17, 400, -1], dtype=torch.int32, device="cuda")
    loss, lse = d.token_loss(h, w, y)
    x = float(w[17, 0])
    assert (lse.double() - x).abs().max() <= 1.0 + 2.0 ** -23 * x
    want = float(lse[0]) - x
    assert loss[0] == want and loss[1] == want and loss[2] == 0
    assert 0.0 <= want <= 0.7 + 2.0 ** -23 * x


def test_gradient_against_differences(d):
    h, w, y, mask, c = inputs(24, 90, 16, density=0.6)
    _, (_, _, dh, dw) = check(d, h, w, y, mask, c, "differences")
    ref = TokenLoss(h, w, y, mask, c)
    g = torch.Generator("cuda").manual_seed(5)
    fin = torch.isfinite(TokenLoss(h, w, y, mask).loss)

    def total(hh, ww):
        return float((TokenLoss(hh, ww, y, mask).loss * c.double())[fin].sum())
    for _ in range(4):
        eh = torch.randn(h.shape, generator=g, device="cuda", dtype=torch.float64)
        ew = torch.randn(w.shape, generator=g, device="cuda", dtype=torch.float64)
        s = 1e-5
        rise = (total(h.double() + s * eh, w.double() + s * ew) - total(h.double() - s * eh, w.double() - s * ew)) / (2 * s)
        got = float((dh.double() * eh).sum() + (dw.double() * ew).sum())
        bound = float((ref.tol["dhidden"] * eh.abs()).sum() + (ref.tol["dweight"] * ew.abs()).sum()) + 1e-7
        assert abs(got - rise) <= bound


def test_same_bits_again_and_on_another_stream(d):
    h, w, y, mask, c = inputs(300, 3000, 264, density=0.3)
    first = d.token_loss(h, w, y, mask)
    grads = d.token_loss_grad(h, w, y, first[1], c, mask)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        again = d.token_loss(h, w, y, mask)
        grads2 = d.token_loss_grad(h, w, y, again[1], c, mask)
    s.synchronize()
    for a, b in zip(first + grads, again + grads2):
        assert torch.equal(a, b)


def test_graph_replay(d):
    h, w, y, mask, c = inputs(64, 1500, 128, density=0.3)
    loss, lse = d.token_loss(h, w, y, mask)
    dh, dw = d.token_loss_grad(h, w, y, lse, c, mask)
    out = [torch.empty_like(t) for t in (loss, lse, dh, dw)]
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        d.token_loss(h, w, y, mask, out=(out[0], out[1]))
        d.token_loss_grad(h, w, y, out[1], c, mask, out=(out[2], out[3]))
    for _ in range(2):
        for t in out:
            t.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, (loss, lse, dh, dw)):
            assert torch.equal(a, b)


def test_no_rows(d):
    h, w, y, mask, c = inputs(4, 100, 24)
    loss, lse = d.token_loss(h[:0], w, y[:0])
    dh, dw = d.token_loss_grad(h[:0], w, y[:0], lse, c[:0])
    assert loss.shape == (0,) and dh.shape == (0, 24) and not dw.any()


def test_targets_beyond_the_vocabulary():
    d = Domino(0)
    h, w, y, _, c = inputs(8, 100, 24)
    ref = TokenLoss(h, w, torch.where(torch.arange(8, device="cuda") == 3, -1, y), None, c)
    y[3] = 100
    loss, lse = d.token_loss(h, w, y)
    assert d.device_error() == 4
    dh, dw = d.token_loss_grad(h, w, y, lse, c)
    assert d.device_error() == 4
    assert_within(loss, ref.loss, ref.tol["loss"], "loss")
    assert_within(dw, ref.dweight, ref.tol["dweight"], "dweight")
    d.close()


def test_refusals(d):
    h, w, y, mask, c = inputs(8, 100, 24, density=0.5)
    with pytest.raises(TypeError):
        d.token_loss(h, w.float(), y)
    with pytest.raises(TypeError):
        d.token_loss(h, w, y.long())
    with pytest.raises(ValueError):
        d.token_loss(h, w[:, :20], y)
    with pytest.raises(ValueError):
        d.token_loss(h, w, y, mask[:, :2].contiguous())
    with pytest.raises(ValueError):
        d.token_loss(h.T, w, y)
    with pytest.raises(DominoError) as e:
        d.token_loss(h.float(), w.float(), y)
    assert e.value.status == -3
    loss = torch.empty(8, device="cuda")
    for bad in (dict(hs=23), dict(rows=-1), dict(dim=0), dict(V=0), dict(V=(1 << 24) + 1), dict(dtype=2), dict(loss=None)):
        a = dict(hs=24, rows=8, dim=24, V=100, dtype=B.DTYPE_BF16, loss=loss)
        a.update(bad)
        with pytest.raises(DominoError) as e:
            B.domino_token_loss(d.h, h, a["hs"], w, 24, a["dtype"], a["rows"], a["dim"], a["V"], None, y, a["loss"])
        assert e.value.status == -1


def test_capture_needs_room_first():
    """The first call at a larger size grows the handle's scratch, which a capture does not allow."""
    d = Domino(0)
    h, w, y, _, _ = inputs(64, 1000, 64)
    loss = torch.empty(64, device="cuda")
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        loss.zero_()
        with pytest.raises(DominoError) as e:
            d.token_loss(h, w, y, out=(loss, loss))
    assert e.value.status == -1
    torch.cuda.synchronize()
    d.close()


@pytest.mark.parametrize("T,V,D", [(1, 300, 1029), (2, 6000, 517), (4, 90, 3), (3, 20000, 261), (5, 300, 1029), (200, 900, 261)])
@pytest.mark.parametrize("off", [0, 1, 6])
def test_odd_widths_at_every_offset(d, T, V, D, off):
    """Rows that begin at every even byte of a 16-byte block; nothing beside the gradients is written."""
    h, w, y, mask, c = inputs(T, V, D, density=0.5)
    ref = TokenLoss(h, w, y, mask, c)

    def inside(x):
        base = torch.full((x.numel() + off + 64,), float("nan"), dtype=x.dtype, device="cuda")
        view = base[off:off + x.numel()].view(x.shape)
        view.copy_(x)
        return base, view
    (_, hv), (_, wv) = inside(h), inside(w)
    loss, lse = d.token_loss(hv, wv, y, mask)
    (bh, dh), (bw, dw) = inside(torch.zeros_like(h)), inside(torch.zeros_like(w))
    d.token_loss_grad(hv, wv, y, lse, c, mask, out=(dh, dw))
    for name, got in (("lse", lse), ("loss", loss), ("dhidden", dh), ("dweight", dw)):
        assert_within(got, getattr(ref, name), ref.tol[name], name)
    for base, x in ((bh, h), (bw, w)):
        assert torch.isnan(base[:off]).all() and torch.isnan(base[off + x.numel():]).all()


@pytest.mark.parametrize("T", [3, 40])
def test_weights_of_masked_tokens_hold_anything_forward(d, T):
    """The loss is over the allowed tokens alone."""
    h, w, y, mask, _ = inputs(T, 700, 64, density=0.3)
    bits = torch.zeros(T, 700, dtype=torch.bool, device="cuda")
    bits[:, ::2] = True
    y = (y // 2 * 2).clamp(max=698)
    mask = pack(bits)
    ref = TokenLoss(h, w, y, mask)
    w2 = w.clone()
    w2[1::2] = float("nan")
    loss, lse = d.token_loss(h, w2, y, mask)
    assert_within(lse, ref.lse, ref.tol["lse"], "lse")
    assert_within(loss, ref.loss, ref.tol["loss"], "loss")
