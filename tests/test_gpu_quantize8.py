"""domino_quantize8 against its definition in 64 bits; domino_logits8 against that of codes, and exactly on whole numbers."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import DominoError  # noqa: E402
from paper_2403_06988_gb300 import _binding as B  # noqa: E402
from norm8_reference import assert_within, logits8  # noqa: E402
from test_gpu_norm import TYPES, check_codes, d  # noqa: E402,F401


def matrix(R, D, dtype, seed=0):
    g = torch.Generator("cuda").manual_seed(R * 31 + D + seed)
    x = torch.randn(R, D, generator=g, device="cuda")
    x *= torch.exp(3 * torch.randn(R, 1, generator=g, device="cuda"))
    return x.to(TYPES[dtype])


@pytest.mark.parametrize("R,D", [(1, 1), (1, 128), (3, 7), (128, 128), (129, 130), (301, 1001), (64, 4096), (1000, 96), (2, 20000), (257, 384)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [1, 128])
def test_quantize(d, R, D, dtype, block):  # noqa: F811
    x = matrix(R, D, dtype)
    q, scales = d.quantize8(x, block)
    assert scales.shape == (-(-R // block), -(-D // 128)) and q.stride(0) % 16 == 0
    check_codes(q, scales, x.double(), 0.0, block, "quantize8")
    off = torch.full((R * (D + 3) + 5,), float("nan"), dtype=x.dtype, device="cuda")[5:].view(R, D + 3)[:, :D]
    off.copy_(x)
    q2, s2 = d.quantize8(off, block)
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s2, scales)


def test_exact_codes(d):  # noqa: F811
    """Every code of a block whose largest value is 448 comes out as itself, ties to even, zeros with the least scale."""
    every = torch.arange(256, device="cuda").to(torch.uint8).view(torch.float8_e4m3fn).float()
    x = torch.nan_to_num(every, nan=448.0).view(2, 128)
    q, scales = d.quantize8(x)
    assert torch.equal(q.float(), x) and (scales == 1).all()
    x = torch.zeros(2, 200, device="cuda")
    x[0, 0], x[0, 1], x[0, 2], x[0, 3] = 448.0, 17.0, 19.0, 2.0 ** -10      # 16 | 18 | 20: ties; half the smallest: 0
    q, scales = d.quantize8(x)
    assert q[0, :4].float().tolist() == [448.0, 16.0, 20.0, 0.0]
    assert torch.equal(scales[1], torch.full((2,), 2.0 ** -100, device="cuda") / torch.full((2,), 448.0, device="cuda"))
    assert not q[1].float().any()


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("size", [3e38, 1e30, 1e-25, 1e-36])
def test_sizes_of_values(d, size, block):  # noqa: F811
    """Up to the largest; blocks below 2^-100 keep its scale, and their codes get small."""
    x = matrix(130, 260, "f32").clamp(-1, 1) * size
    check_codes(*d.quantize8(x, block), x.double(), 0.0, block, "quantize8")


def test_offsets_beyond_32_bits(d):  # noqa: F811
    R, D = 140000, 16384
    x = torch.zeros(R, D, dtype=torch.bfloat16, device="cuda")
    x[R - 1, D - 1], x[131073, 5] = 2.0, -4.0
    for block in (1, 128):
        q, scales = d.quantize8(x, block)
        assert q[R - 1, D - 1].float() == 448 and q[131073, 5].float() == -448
        assert scales[(R - 1) // block, 127] == 2.0 / 448 and scales[131073 // block, 0] == 4.0 / 448
        assert int((q.view(torch.uint8) != 0).sum()) == 2
        del q


def test_refusals(d):  # noqa: F811
    x = matrix(5, 24, "bf16")
    with pytest.raises(ValueError):
        d.quantize8(x, 2)
    with pytest.raises(TypeError):
        d.quantize8(x.half())
    with pytest.raises(ValueError):
        d.quantize8(x.T)
    with pytest.raises(ValueError):
        d.quantize8(x, out=(None, torch.empty(4, 1, device="cuda")))
    assert d.quantize8(x[:0])[0].shape == (0, 24)
    out, s = torch.empty(5, 32, dtype=torch.uint8, device="cuda"), torch.empty(5, 1, device="cuda")
    for rows, dim, xs, block, p, stride in ((-1, 24, 24, 1, 0, 32), (5, 0, 24, 1, 0, 32), (5, 24, 23, 1, 0, 32), (5, 24, 24, 64, 0, 32),
                                            (5, 24, 24, 1, 8, 32), (5, 24, 24, 1, 0, 24), (5, 24, 24, 1, 0, 16)):
        with pytest.raises(DominoError) as e:
            B.domino_quantize8(d.h, x, xs, B.DTYPE_BF16, rows, dim, block, out.data_ptr() + p, stride, s)
        assert e.value.status == -1


# ---- logits ----------------------------------------------------------------------
def operands(d, T, V, D, seed=0):  # noqa: F811
    g = torch.Generator("cuda").manual_seed(T + 7 * V + D + seed)
    h = torch.randn(T, D, generator=g, device="cuda") * (1 + 20 * (torch.rand(D, generator=g, device="cuda") < 0.01))
    w = torch.randn(V, D, generator=g, device="cuda") * 2 / D ** 0.5
    return (*d.quantize8(h), *d.quantize8(w, 128))


# one token to several tiles of rows, each shape of tiles, widths and vocabularies off every boundary, one block and several
SIZES = [(1, 1, 1), (1, 1000, 64), (1, 32000, 1024), (3, 129, 200), (8, 5000, 128), (33, 4001, 333), (64, 40000, 520), (128, 1111, 96),
         (129, 50000, 130), (20, 25001, 272), (100, 45000, 130), (200, 20000, 1152), (256, 24000, 256), (257, 9000, 384), (300, 33001, 144), (513, 3001, 260)]


@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits(d, T, V, D, dtype):  # noqa: F811
    q, s, wq, ws = operands(d, T, V, D)
    want, tol = logits8(q, s, wq, ws, TYPES[dtype])
    got = d.logits8(q, s, wq, ws, TYPES[dtype])
    assert got.stride(0) * got.element_size() % 16 == 0
    assert_within(got, want, tol, f"{T} x {V} x {D}")
    # rows that are not on 16-byte boundaries, and nothing beside them
    base = torch.full((T * (V + 3) + 9,), 7.0, dtype=TYPES[dtype], device="cuda")
    out = base[5:5 + T * (V + 3)].view(T, V + 3)[:, :V]
    d.logits8(q, s, wq, ws, out=out)
    assert torch.equal(out, got)
    out.fill_(7.0)
    assert (base == 7.0).all()


@pytest.mark.parametrize("T,V,D", [(1, 300, 128), (5, 1000, 1000), (64, 20000, 300), (256, 20001, 513), (390, 2000, 777)])
def test_whole_numbers_are_exact(d, T, V, D):  # noqa: F811
    """Codes -8 .. 8 and scales that are powers of two: every sum is a whole number of steps, in fp32 without a rounding."""
    g = torch.Generator("cuda").manual_seed(T + V + D)
    wide = -(-D // 16) * 16
    q = torch.randint(-8, 9, (T, wide), generator=g, device="cuda").float().to(torch.float8_e4m3fn)[:, :D]
    wq = torch.randint(-8, 9, (V, wide), generator=g, device="cuda").float().to(torch.float8_e4m3fn)[:, :D]
    nb = -(-D // 128)
    s = 2.0 ** torch.randint(-3, 3, (T, nb), generator=g, device="cuda").float()
    ws = 2.0 ** torch.randint(-3, 3, (-(-V // 128), nb), generator=g, device="cuda").float()
    want, _ = logits8(q, s, wq, ws, torch.float32)
    assert torch.equal(d.logits8(q, s, wq, ws).double(), want)


def test_a_row_that_is_no_number_stays_alone(d):  # noqa: F811
    T, V, D = 40, 3000, 200
    q, s, wq, ws = operands(d, T, V, D)
    want = d.logits8(q, s, wq, ws)
    q[7, 3] = float("nan")
    got = d.logits8(q, s, wq, ws)
    assert torch.isnan(got[7]).all()
    keep = torch.arange(T, device="cuda") != 7
    assert torch.equal(got[keep], want[keep])


@pytest.mark.parametrize("T,V,D", [(4, 600, 40), (140, 30000, 136)])
def test_columns_beyond_the_last_are_not_read(d, T, V, D):  # noqa: F811
    q, s, wq, ws = operands(d, T, V, D)
    want = d.logits8(q, s, wq, ws)

    def within(t):
        big = torch.full((t.shape[0], t.shape[1] // 16 * 16 + 32), 0x7F, dtype=torch.uint8, device="cuda")   # no number
        big[:, :t.shape[1]] = t.view(torch.uint8)
        return big.view(torch.float8_e4m3fn)[:, :t.shape[1]]
    assert torch.equal(d.logits8(within(q), s, within(wq), ws), want)


def test_logits_graph_and_another_stream(d):  # noqa: F811
    q, s, wq, ws = operands(d, 130, 20000, 264)
    want = d.logits8(q, s, wq, ws)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = d.logits8(q, s, wq, ws, stream=st)
    st.synchronize()
    assert torch.equal(got, want)
    g, out = torch.cuda.CUDAGraph(), torch.zeros_like(want)
    with torch.cuda.graph(g, stream=st):
        d.logits8(q, s, wq, ws, out=out)
    out.fill_(7)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    del g


def test_logits_refusals(d):  # noqa: F811
    q, s, wq, ws = operands(d, 5, 300, 40)
    with pytest.raises(TypeError):
        d.logits8(q.float(), s, wq, ws)
    with pytest.raises(TypeError):
        d.logits8(q, s, wq, ws, torch.float16)
    with pytest.raises(ValueError):
        d.logits8(q, s, wq[:, :39], ws)
    with pytest.raises(ValueError):
        d.logits8(q, s[:4], wq, ws)
    with pytest.raises(ValueError):
        d.logits8(q, s, wq, ws[:2])
    with pytest.raises(ValueError):
        d.logits8(q.float().to(torch.float8_e4m3fn).reshape(-1).view(5, 40), s, wq, ws)     # rows of 40 bytes
    with pytest.raises(ValueError):
        d.logits8(q, s, wq, ws, out=torch.empty(5, 299, device="cuda"))
    assert d.logits8(q[:0], s[:0], wq, ws).shape == (0, 300)
    out = torch.empty(5, 300, device="cuda")
    good = dict(hidden_dev=q.data_ptr(), hidden_stride=48, weight_dev=wq.data_ptr(), weight_stride=48, rows=5, dim=40, n_tokens=300,
                dtype=0, logits_stride=300)
    for bad in ({"hidden_stride": 40}, {"hidden_stride": 32}, {"weight_stride": 40}, {"rows": -1}, {"dim": 0}, {"n_tokens": 0},
                {"dtype": 2}, {"logits_stride": 299}, {"hidden_dev": q.data_ptr() + 8}, {"weight_dev": None}):
        a = {**good, **bad}
        with pytest.raises(DominoError) as e:
            B.domino_logits8(d.h, a["hidden_dev"], a["hidden_stride"], s, a["weight_dev"], a["weight_stride"], ws, a["rows"], a["dim"],
                             a["n_tokens"], a["dtype"], out, a["logits_stride"])
        assert e.value.status == -1, bad
    with pytest.raises(DominoError) as e:
        B.domino_logits8(d.h, q.data_ptr(), 48, s, wq.data_ptr(), 48, ws, (1 << 31) - 1, 40, 300, 0, out, 300)
    assert e.value.status == -3
