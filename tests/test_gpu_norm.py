"""domino_norm, domino_norm8 and domino_norm_grad against their definitions in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import Domino, DominoError  # noqa: E402
from paper_2403_06988_gb300 import _binding as B  # noqa: E402
from norm8_reference import Codes, Norm, assert_within, decode  # noqa: E402

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# one row and value; rows of a warp, of shared CTAs, of one, two and four vectors a thread; long rows; odd widths
SIZES = [(1, 1), (1, 4096), (3, 7), (5, 64), (130, 65), (33, 129), (7, 333), (64, 1000), (9, 1024), (40, 2049), (6, 4096), (31, 4103),
         (5, 8192), (3, 8200), (4, 12345), (2, 16384), (3, 16392), (2, 40001)]


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


def inputs(T, D, dtype, seed=0):
    """x, residual, weight, dy, dsum."""
    g = torch.Generator("cuda").manual_seed(T * 31 + D + seed)
    loud = 1.0 + 30.0 * (torch.rand(D, generator=g, device="cuda") < 0.01)

    def rows(size):
        return (torch.randn(T, D, generator=g, device="cuda") * loud * size).to(TYPES[dtype])
    w = (1.0 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(TYPES[dtype])
    return rows(0.5), rows(2.0), w, rows(1e-3), rows(1e-3)


def check_codes(q, scales, y, rel, block, what):
    ref = Codes(y, block, rel)
    assert_within(scales, ref.scales, ref.tol_scales, what + " scales")
    assert_within(decode(q), ref.units, ref.tol, what + " codes")


@pytest.mark.parametrize("T,D", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
def test_norm(d, T, D, dtype, residual):
    x, r, w, _, _ = inputs(T, D, dtype)
    r = r if residual else None
    ref = Norm(x, w, r)
    y, h, rstd = d.norm(x, w, r)
    assert torch.equal(h, ref.sum) and (residual or h.data_ptr() == x.data_ptr())
    assert_within(rstd, ref.rstd, ref.tol["rstd"], "rstd")
    assert_within(y, ref.y, ref.tol["y"], "y")
    q, scales, h8 = d.norm8(x, w, r)
    assert torch.equal(h8, ref.sum) and q.dtype == torch.float8_e4m3fn and q.stride(0) % 16 == 0
    check_codes(q, scales, ref.y, ref.rel_y, 1, "norm8")


@pytest.mark.parametrize("T,D", SIZES + [(700, 512), (2000, 96)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dsum", [False, True])
def test_gradient(d, T, D, dtype, dsum):
    x, _, w, dy, ds = inputs(T, D, dtype)
    ds = ds if dsum else None
    _, _, rstd = d.norm(x, w)
    ref = Norm(x, w, None, dy=dy, dsum=ds)
    dx, dw = d.norm_grad(x, w, rstd, dy, ds)
    assert_within(dx, ref.dx, ref.tol["dx"], "dx")
    assert_within(dw, ref.dweight, ref.tol["dweight"], "dweight")


@pytest.mark.parametrize("T,D", [(3, 40), (2, 300)])
def test_gradient_against_differences(d, T, D):
    """Of sum(dy y) + sum(dsum sum), in 64 bits, along random directions: central differences, error of third order."""
    x, r, w, dy, ds = (t.double() for t in inputs(T, D, "f32"))
    g = torch.Generator("cuda").manual_seed(5)
    y, h, rstd = d.norm(x.float(), w.float(), r.float())
    dx, dw = d.norm_grad(h, w.float(), rstd, dy.float(), ds.float())

    def value(x, r, w):
        h = x + r
        return (dy * h * ((h * h).mean(1, keepdim=True) + 1e-6) ** -0.5 * w).sum() + (ds * h).sum()
    for which in range(3):
        e = torch.randn(w.shape if which == 2 else x.shape, generator=g, device="cuda").double()
        step = 1e-4
        args = [[x, r, w], [x, r, w]]
        args[0][which], args[1][which] = args[0][which] + step * e, args[1][which] - step * e
        rise = (value(*args[0]) - value(*args[1])) / (2 * step)
        got = ((dw if which == 2 else dx).double() * e).sum()
        size = float(((dw if which == 2 else dx).double().abs() * e.abs()).sum())
        # fp32 results (norm's 60 roundings or so), the inputs' rounding in h, step^2 for the third derivative
        assert abs(float(got - rise)) <= size * (200 * 2.0 ** -24 + 100 * step * step) + 1e-12


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off,pad", [(0, 8), (1, 0), (3, 6), (8, 8)])
@pytest.mark.parametrize("D", [72, 1031])
def test_strides_and_alignment(d, dtype, off, pad, D):
    """Rows apart and off 16-byte boundaries give the bits of rows that are not, and nothing beside them is written."""
    T = 20
    x, r, w, dy, ds = inputs(T, D, dtype)

    def apart(t):
        big = torch.full((T, off + D + pad), float("nan"), dtype=t.dtype, device="cuda")
        big[:, off:off + D] = t
        return big[:, off:off + D]
    wide = torch.full((off + D,), float("nan"), dtype=w.dtype, device="cuda")
    wide[off:] = w
    y, h, rstd = d.norm(x, w, r)
    out = (apart(torch.zeros_like(x)), apart(torch.zeros_like(x)), torch.empty(T, device="cuda"))
    d.norm(apart(x), wide[off:], apart(r), out=out)
    assert all(torch.equal(a, b) for a, b in zip(out, (y, h, rstd)))
    q, scales, _ = d.norm8(x, w, r)
    q2, scales2, _ = d.norm8(apart(x), wide[off:], apart(r))
    assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(scales, scales2)
    dx, dw = d.norm_grad(h, w, rstd, dy, ds)
    dx2, dw2 = apart(torch.zeros_like(x)), wide.clone()
    d.norm_grad(apart(h), wide[off:], rstd, apart(dy), apart(ds), out=(dx2, dw2[off:]))
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2[off:])
    for o in (out[0], out[1], dx2):
        assert torch.isnan(o._base[:, :off]).all() and torch.isnan(o._base[:, off + D:]).all()


@pytest.mark.parametrize("T,D", [(20, 72), (9, 1031), (3, 4096), (2, 16400)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(d, T, D, dtype):
    x, r, w, dy, ds = inputs(T, D, dtype)
    y, h, rstd = d.norm(x, w, r)
    q, scales, _ = d.norm8(x, w, r)
    for k in range(2):
        a, b = x.clone(), r.clone()
        into = (a, b)[k]
        y2, h2, _ = d.norm(a, w, b, out=(None, into, None))
        assert h2.data_ptr() == into.data_ptr() and torch.equal(h2, h) and torch.equal(y2, y)
        a, b = x.clone(), r.clone()
        q2, s2, h2 = d.norm8(a, w, b, out=(None, None, (a, b)[k]))
        assert torch.equal(h2, h) and torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s2, scales)
    dx, dw = d.norm_grad(h, w, rstd, dy, ds)
    for k in range(2):
        a, b = dy.clone(), ds.clone()
        dx2, dw2 = d.norm_grad(h, w, rstd, a, b, out=((a, b)[k], None))
        assert torch.equal(dx2, dx) and torch.equal(dw2, dw)


def test_codes_leave_the_rest_of_their_rows(d):
    x, _, w, _, _ = inputs(6, 37, "f32")
    big = torch.full((6, 64), 0x55, dtype=torch.uint8, device="cuda")
    q = big.view(torch.float8_e4m3fn)[:, :37]
    d.norm8(x, w, out=(q, None, None))
    assert (big[:, 37:] == 0x55).all()
    assert torch.equal(q.float(), d.norm8(x, w)[0].float())


def test_small_and_large_values(d):
    """Rows of zeros (with eps: zeros), of the largest values whose squares are finite, and of very small ones."""
    x = torch.zeros(4, 200, device="cuda")
    x[1], x[2], x[3, 7] = 1e18, 1e-30, -3.0
    w = torch.ones(200, device="cuda")
    ref = Norm(x, w)
    y, _, rstd = d.norm(x, w)
    assert_within(y, ref.y, ref.tol["y"], "y")
    q, scales, _ = d.norm8(x, w)
    assert not decode(q)[0].any()
    check_codes(q, scales, ref.y, ref.rel_y, 1, "norm8")
    assert (decode(q)[1] == 448).all() and decode(q)[3, 7] == -448


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_widest_rows(d, dtype):
    T, D = 3, 1 << 20
    x, r, w, dy, ds = inputs(T, D, dtype)
    ref = Norm(x, w, r, dy=dy, dsum=ds)
    y, h, rstd = d.norm(x, w, r)
    assert torch.equal(h, ref.sum)
    assert_within(y, ref.y, ref.tol["y"], "y")
    q, scales, _ = d.norm8(x, w, r)
    check_codes(q, scales, ref.y, ref.rel_y, 1, "norm8")
    dx, dw = d.norm_grad(h, w, rstd, dy, ds)
    assert_within(dx, ref.dx, ref.tol["dx"], "dx")
    assert_within(dw, ref.dweight, ref.tol["dweight"], "dweight")


def test_no_rows(d):
    x, r, w, dy, _ = inputs(3, 24, "bf16")
    y, h, rstd = d.norm(x[:0], w, r[:0])
    assert y.shape == h.shape == (0, 24) and rstd.shape == (0,)
    q, scales, _ = d.norm8(x[:0], w)
    assert q.shape == (0, 24) and scales.shape == (0, 1)
    dx, dw = d.norm_grad(x[:0], w, rstd, dy[:0])
    assert dx.shape == (0, 24) and not dw.any()


def test_offsets_beyond_32_bits(d):
    """Rows whose offsets pass 2^32 bytes and 2^31 values."""
    T, D = 140000, 16384
    x = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda")
    x[T - 1], x[131072, :8192] = 2.0, 4.0
    w = torch.full((D,), 0.5, dtype=torch.bfloat16, device="cuda")
    q, scales, _ = d.norm8(x, w, None, 0.25)
    last = 2.0 * 0.5 * (4.0 + 0.25) ** -0.5
    assert (q[T - 1].float() == 448).all() and abs(float(scales[T - 1, 5]) * 448 - last) < 1e-6
    assert (q[131072, :8192].float() == 448).all() and not q[131072, 8192:].float().any() and not q[131071].float().any()
    rstd = torch.ones(T, device="cuda")
    dx, dw = d.norm_grad(x, w, rstd, x, out=(x, None))
    # g h / dim = 0.5 * 4 = 2: dx = 0.5 * 2 - 2 * 2
    assert (dx[T - 1] == -3.0).all() and dw[0] == 4.0 + 16.0 and dw[D - 1] == 4.0 and not dx[5].any()


def test_graph_and_another_stream(d):
    x, r, w, dy, ds = inputs(300, 520, "bf16")

    def call(out=None, **k):
        o = out or [None] * 8
        y, h, rstd = d.norm(x, w, r, out=tuple(o[:3]), **k)
        dx, dw = d.norm_grad(h, w, rstd, dy, ds, out=tuple(o[3:5]), **k)
        q, s, h8 = d.norm8(x, w, r, out=tuple(o[5:8]), **k)
        return [y, h, rstd, dx, dw, q, s, h8]
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = call(stream=s)
    s.synchronize()
    out = [torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda") for t in want]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call(out)
    d.token_loss(*(torch.zeros(n, 1001, dtype=torch.bfloat16, device="cuda") for n in (64, 30000)),
                 torch.zeros(64, dtype=torch.int32, device="cuda"))      # the scratch grows
    for t in out:
        t.view(torch.uint8).fill_(7)
    g.replay()
    torch.cuda.synchronize()
    for t in (got, out):
        for a, b in zip(t, want):
            assert torch.equal(a.float(), b.float())
    del g


def test_refusals(d):
    x, r, w, dy, ds = inputs(5, 24, "bf16")
    rstd = torch.ones(5, device="cuda")
    with pytest.raises(TypeError):
        d.norm(x, w.float())
    with pytest.raises(TypeError):
        d.norm(x.half(), w.half())
    with pytest.raises(TypeError):
        d.norm(x, w, r.float())
    with pytest.raises(ValueError):
        d.norm(x, w[:23])
    with pytest.raises(ValueError):
        d.norm(x, w, r[:4])
    with pytest.raises(ValueError):
        d.norm(x.T, w[:5])
    with pytest.raises(ValueError):
        d.norm(x, w, out=(None, r, None))                     # no residual: sum is x
    with pytest.raises(ValueError):
        d.norm8(x, w, out=(torch.empty(5, 25, device="cuda").to(torch.float8_e4m3fn)[:, :24], None, None))
    with pytest.raises(ValueError):
        d.norm_grad(x, w, rstd[:4], dy)
    with pytest.raises(TypeError):
        d.norm_grad(x, w, rstd, None)
    with pytest.raises(RuntimeError, match="requires a gradient"):
        d.norm(x, w.clone().requires_grad_())
    for eps in (-1e-6, float("nan"), float("inf")):
        with pytest.raises(DominoError) as e:
            d.norm(x, w, eps=eps)
        assert e.value.status == -1
    y = torch.empty_like(x)
    for rows, dim, xs, ys in ((-1, 24, 24, 24), (5, 0, 24, 24), (5, 24, 23, 24), (5, 24, 24, 23), (5, (1 << 20) + 1, 1 << 21, 1 << 21)):
        with pytest.raises(DominoError) as e:
            B.domino_norm(d.h, x, xs, None, 0, w, B.DTYPE_BF16, rows, dim, 1e-6, y, ys)
        assert e.value.status == -1
    with pytest.raises(DominoError) as e:                     # a residual without a place for the sum
        B.domino_norm(d.h, x, 24, r, 24, w, B.DTYPE_BF16, 5, 24, 1e-6, y, 24)
    assert e.value.status == -1
    with pytest.raises(DominoError) as e:                     # the sum over x, rows elsewhere
        B.domino_norm(d.h, x, 24, r, 24, w, B.DTYPE_BF16, 2, 24, 1e-6, y, 24, x, 48)
    assert e.value.status == -1
    with pytest.raises(DominoError) as e:
        B.domino_norm_grad(d.h, x, 24, w, rstd, dy, 24, ds, 24, B.DTYPE_BF16, 2, 24, ds, 48, w)
    assert e.value.status == -1
    for p, stride in ((8, 32), (16, 24), (16, 16)):           # codes off 16-byte boundaries, rows too close
        with pytest.raises(DominoError) as e:
            B.domino_norm8(d.h, x, 24, None, 0, w, B.DTYPE_BF16, 5, 24, 1e-6, y.data_ptr() + p, stride, rstd)
        assert e.value.status == -1
