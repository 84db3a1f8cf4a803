"""domino_embed (exact) and domino_embed_grad against 64-bit sums."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import Domino, DominoError  # noqa: E402
from paper_2403_06988_gb300 import _binding as B  # noqa: E402
from loss_reference import assert_within, embed_grad  # noqa: E402

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


def tokens(n, V, seed=0, hot=True):
    g = torch.Generator("cuda").manual_seed(n * 31 + V + seed)
    t = torch.randint(0, V, (n,), generator=g, device="cuda").int()
    if hot and n > 20:     # one token takes a third of the list, another a tenth
        u = torch.rand(n, generator=g, device="cuda")
        t[u < 0.3] = V // 2
        t[(u > 0.3) & (u < 0.4)] = V - 1
        t[u > 0.97] = -1
    return t


def values(n, D, dtype, seed=0):
    g = torch.Generator("cuda").manual_seed(n + 7 * D + seed)
    return torch.randn(n, D, generator=g, device="cuda").to(TYPES[dtype])


CASES = [(1, 5, 1), (1, 1, 4096), (3, 100, 8), (31, 1000, 33), (33, 7, 64), (500, 32000, 333), (1025, 40, 1000),
         (5000, 128256, 256), (40000, 300, 24)]


@pytest.mark.parametrize("n,V,D", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lookup(d, n, V, D, dtype):
    t, w = tokens(n, V), values(V, D, dtype)
    want = torch.where((t >= 0)[:, None], w[t.long().clamp(min=0)].float() * 3.7, torch.zeros((), device="cuda"))
    assert torch.equal(d.embed(t, w, 3.7), want.to(w.dtype))


@pytest.mark.parametrize("n,V,D", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("add", [False, True])
def test_gradient(d, n, V, D, dtype, add):
    t, g = tokens(n, V), values(n, D, dtype)
    into = values(V, D, dtype, seed=1) if add else None
    want, tol = embed_grad(t, g, V, 0.3, into)
    before = into.clone() if add else None
    got = d.embed_grad(t, g, V, 0.3, into=into)
    assert_within(got, want, tol, f"{n} of {V} x {D}")
    if add:    # rows of tokens that do not occur are not touched
        other = torch.ones(V, dtype=torch.bool, device="cuda")
        other[t[t >= 0].long()] = False
        assert torch.equal(got[other], before[other])


@pytest.mark.parametrize("n,V", [(300, 1), (70000, 3), (4096, 1 << 20), (140000, 129)])
def test_gradient_long_runs_and_large_vocabularies(d, n, V):
    """Whole numbers: every order of additions gives the same sums."""
    t = tokens(n, V, hot=False)
    g = torch.randint(-4, 5, (n, 16), device="cuda").float()
    want, _ = embed_grad(t, g, V, 1.0)
    assert torch.equal(d.embed_grad(t, g, V).double(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off,pad", [(1, 0), (3, 6), (8, 8)])
def test_strides_and_alignment(d, dtype, off, pad):
    n, V, D = 200, 50, 72
    t, w, g = tokens(n, V), values(V, D, dtype), values(n, D, dtype)

    def apart(x):
        big = torch.full((x.shape[0], off + D + pad), float("nan"), dtype=x.dtype, device="cuda")
        big[:, off:off + D] = x
        return big[:, off:off + D]
    out = apart(torch.zeros_like(g))
    assert torch.equal(d.embed(t, apart(w), 2.0, out=out), d.embed(t, w, 2.0))
    dw = apart(torch.zeros_like(w))
    d.embed_grad(t, apart(g), V, 2.0, into=dw)
    assert torch.equal(dw, d.embed_grad(t, g, V, 2.0, into=torch.zeros_like(w)))
    for o in (out, dw):
        assert torch.isnan(o._base[:, :off]).all() and torch.isnan(o._base[:, off + D:]).all()


def test_gradient_against_differences(d):
    """The lookup is linear: sum(grad * embed(W + E)) - sum(grad * embed(W)) = sum(dweight * E)."""
    n, V, D = 100, 30, 16
    t, w, e, g = tokens(n, V), values(V, D, "f32"), values(V, D, "f32", 3), values(n, D, "f32", 4)
    rise = ((d.embed(t, w + e, 0.5).double() - d.embed(t, w, 0.5).double()) * g.double()).sum()
    dw = d.embed_grad(t, g, V, 0.5)
    size = float((g.abs().double().sum() * (w.abs().max() + e.abs().max())))
    assert abs(float((dw.double() * e.double()).sum() - rise)) <= 2.0 ** -20 * size


def test_same_bits_again_and_on_another_stream(d):
    t, g = tokens(9000, 2000), values(9000, 72, "f32")
    a = d.embed_grad(t, g, 2000)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = d.embed_grad(t, g, 2000)
    s.synchronize()
    assert torch.equal(a, b)


def test_rows_beyond_32_bits(d):
    """A table and a list of gradients whose offsets pass 2^32 bytes and 2^31 values."""
    V, D = 140000, 16384
    w = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    t = torch.tensor([0, V - 1, 131072, V - 1], dtype=torch.int32, device="cuda")
    w[131072:] = 1.0
    out = d.embed(t, w, 2.0)
    assert (out[0] == 0).all() and (out[1:] == 2).all()
    g = torch.ones(4, D, dtype=torch.bfloat16, device="cuda")
    d.embed_grad(t, g, V, into=w)
    assert (w[0] == 1).all() and (w[V - 1] == 3).all() and (w[131072] == 2).all() and (w[V - 2] == 1).all()


def test_no_tokens_and_bad_tokens():
    d = Domino(0)
    t, w = tokens(5, 40, hot=False), values(40, 12, "bf16")
    assert d.embed(t[:0], w).shape == (0, 12)
    assert not d.embed_grad(t[:0], w[:0], 40).any()
    t[1] = 40
    out = d.embed(t, w)
    assert d.device_error() == 4 and not out[1].any() and torch.equal(out[0], w[int(t[0])])
    dw = d.embed_grad(t, w[:5], 40)
    assert d.device_error() == 4
    good = t.clone()
    good[1] = -1
    assert torch.equal(dw, d.embed_grad(good, w[:5], 40)) and d.device_error() == 0
    d.close()


def test_refusals(d):
    t, w = tokens(5, 40, hot=False), values(40, 12, "bf16")
    with pytest.raises(TypeError):
        d.embed(t.long(), w)
    with pytest.raises(TypeError):
        d.embed(t, w.double())
    with pytest.raises(ValueError):
        d.embed(t, w.T)
    with pytest.raises(ValueError):
        d.embed(t, w, out=w[:4].clone())
    with pytest.raises(ValueError):
        d.embed_grad(t, w[:4], 40)
    out = torch.empty(5, 12, dtype=torch.bfloat16, device="cuda")
    for args in ((-1, 12, 40, 12, 12), (5, 11, 40, 12, 12), (5, 12, 0, 12, 12), (5, 12, 40, 0, 12), (5, 12, 40, 12, 11)):
        n, ws, V, D, os_ = args
        with pytest.raises(DominoError) as e:
            B.domino_embed(d.h, t, n, w, ws, B.DTYPE_BF16, V, D, 1.0, out, os_)
        assert e.value.status == -1
    with pytest.raises(DominoError) as e:
        B.domino_embed_grad(d.h, t, 5, w, 12, B.DTYPE_BF16, 40, 12, 1.0, 2, w, 12)
    assert e.value.status == -1


@pytest.mark.parametrize("n,V,D", [(3, 9, 3), (40, 12, 257), (700, 50, 515), (64, 7, 2055)])
def test_bf16_rows_at_every_offset(d, n, V, D):
    """Odd widths: consecutive rows begin at every even byte of a 16-byte block; nothing beside them is written."""
    t, w, g = tokens(n, V), values(V, D, "bf16"), values(n, D, "bf16")
    want = torch.where((t >= 0)[:, None], w[t.long().clamp(min=0)].float() * 1.5, torch.zeros((), device="cuda"))
    guard = torch.full((n * D + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    for off in (0, 3, 8):
        guard.fill_(7.0)
        out = guard[off:off + n * D].view(n, D)
        d.embed(t, w, 1.5, out=out)
        assert torch.equal(out, want.bfloat16())
        assert (guard[:off] == 7).all() and (guard[off + n * D:] == 7).all()
    big = torch.full((V * D + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    into = big[5:5 + V * D].view(V, D)
    into.copy_(w)
    ref, tol = embed_grad(t, g, V, 0.5, w)
    assert_within(d.embed_grad(t, g, V, 0.5, into=into), ref, tol, "into")
    assert (big[:5] == 7).all() and (big[5 + V * D:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("off,stride", [(0, 40), (1, 33), (3, 37)])
def test_table_rows_apart_are_cleared(d, dtype, off, stride):
    """accumulate = 0 with rows that do not follow each other: every row is written, nothing between them."""
    n, V, D = 30, 300, 33
    t, g = tokens(n, V), values(n, D, dtype)
    want, tol = embed_grad(t, g, V, 2.0)
    base = torch.full((V * stride + 16,), 7.0, dtype=TYPES[dtype], device="cuda")
    dw = base[off:off + V * stride].view(V, stride)[:, :D]
    code = B.DTYPE_BF16 if dtype == "bf16" else B.DTYPE_F32
    for count in (n, 0):
        B.domino_embed_grad(d.h, t, count, g, D, code, V, D, 2.0, 0, dw.data_ptr(), stride)
        assert_within(dw, want if count else torch.zeros_like(want), tol if count else torch.zeros_like(tol), "table")
        rest = base.clone()
        rest[off:off + V * stride].view(V, stride)[:, :D] = 7.0
        assert (rest == 7.0).all()
