"""The norm's gradient where a strip has several rows: values that make every sum exact, so that dx and dweight are known to
the bit; and which calls give the same bits for rows at any alignment."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_norm import TYPES, d, inputs  # noqa: E402,F401


def rows_for(D):
    """At least four rows a strip, strips that differ by a row: at most 32 strips an SM, 16 beyond 512 columns, 8 beyond 1024,
    4 beyond 2048."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    most = sms * (32 if D <= 512 else 16 if D <= 1024 else 8 if D <= 2048 else 4)
    return 4 * most + most // 3 | 1


def whole(T, D, dtype):
    """h, weight, rstd, dy, dsum: whole numbers of few bits, rstd a half, one or two."""
    g = torch.Generator("cuda").manual_seed(T + D)

    def numbers(lo, hi, *shape):
        return torch.randint(lo, hi + 1, shape, generator=g, device="cuda").to(TYPES[dtype])
    rstd = 2.0 ** torch.randint(-1, 2, (T,), generator=g, device="cuda").float()
    return numbers(-4, 4, T, D), numbers(-2, 2, D), rstd, numbers(-4, 4, T, D), numbers(-8, 8, T, D)


def exact(h, w, rstd, dy, dsum):
    """Sums of g h stay below 2^19 and those of dy h rstd below 2^23 with steps of a half: exact in fp32 in any order.  The
    mean is rounded (a quotient of 64 bits of whole numbers below 2^24, then of 32: as if at once), g - h c is exact in 64 bits
    and rounded once, rstd is a power of two, dsum's addition is rounded, and the result to its type."""
    T, D = h.shape
    dx, dw = torch.empty_like(h), torch.zeros(D, dtype=torch.float64, device="cuda")
    for lo in range(0, T, 4096):
        i = slice(lo, lo + 4096)
        hd, r = h[i].double(), rstd[i].double()[:, None]
        g = dy[i].double() * w.double()
        c = ((g * hd).sum(1, keepdim=True) / D).float().double() * r * r
        x = (g - hd * c).float().double() * r
        if dsum is not None:
            x = (x + dsum[i].double()).float()
        dx[i] = x.float().to(h.dtype)
        dw += (dy[i].double() * hd * r).sum(0)
    return dx, dw.float().to(h.dtype)


def apart(t, off):
    """t with rows off 16-byte boundaries where `off` is not 0."""
    if not off:
        return t
    big = torch.empty(t.shape[0], t.shape[1] + off + 2 - (t.shape[1] + off) % 2, dtype=t.dtype, device="cuda")
    view = big[:, off:off + t.shape[1]]
    view.copy_(t)
    return view


# one, two and four vectors a thread, strips that share a CTA and that do not, rows of more than 8192
WIDTHS = [24, 96, 255, 333, 512, 1000, 1024, 2048, 4096, 8192, 8200]


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("dsum", [False, True])
def test_gradient_of_several_rows_a_strip(d, D, dtype, off, dsum):  # noqa: F811
    h, w, rstd, dy, ds = whole(rows_for(D), D, dtype)
    ds = ds if dsum else None
    dx, dw = exact(h, w, rstd, dy, ds)
    got, got_w = d.norm_grad(apart(h, off), w, rstd, apart(dy, off), None if ds is None else apart(ds, off))
    assert torch.equal(got_w, dw)
    assert torch.equal(got, dx)


def test_gradient_of_many_rows_a_strip(d):  # noqa: F811
    for dtype in ("bf16", "f32"):
        h, w, rstd, dy, ds = whole(200001, 40, dtype)        # 200001 x 32 in halves: below 2^24
        dx, dw = exact(h, w, rstd, dy, ds)
        got, got_w = d.norm_grad(h, w, rstd, dy, ds)
        assert torch.equal(got_w, dw) and torch.equal(got, dx)


@pytest.mark.parametrize("D", [96, 512, 1000, 4096, 8192])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("over", ["dy", "dsum"])
def test_in_place_with_several_rows_a_strip(d, D, dtype, off, over):  # noqa: F811
    h, w, rstd, dy, ds = whole(rows_for(D), D, dtype)
    dx, dw = exact(h, w, rstd, dy, ds)
    a, b = apart(dy, off), apart(ds, off)
    into = a if over == "dy" else b
    got, got_w = d.norm_grad(apart(h, off), w, rstd, a, b, out=(into, None))
    assert got.data_ptr() == into.data_ptr()
    assert torch.equal(got_w, dw) and torch.equal(into, dx)


@pytest.mark.parametrize("T,D", [(50, 264), (50, 1032), (9, 4096), (3, 16400)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bits_at_any_alignment(d, T, D, dtype):  # noqa: F811
    """The norm's, in its type and in codes, and the gradient's but for bf16 rows of up to 8192 columns."""
    x, r, w, dy, ds = inputs(T, D, dtype)
    y, h, rstd = d.norm(x, w, r)
    q, scales, _ = d.norm8(x, w, r)
    dx, dw = d.norm_grad(h, w, rstd, dy, ds)
    for off in (1, 3, 5):
        for a, b in zip(d.norm(apart(x, off), w, apart(r, off)), (y, h, rstd)):
            assert torch.equal(a, b)
        q2, scales2, _ = d.norm8(apart(x, off), w, apart(r, off))
        assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(scales2, scales)
        if dtype == "f32" or D > 8192:
            dx2, dw2 = d.norm_grad(apart(h, off), w, rstd, apart(dy, off), apart(ds, off))
            assert torch.equal(dx2, dx) and torch.equal(dw2, dw)
