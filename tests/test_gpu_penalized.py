"""domino_mask_logits_penalized and domino_mask_sample_penalized: the penalised logits are formed here in fp32 on the host, every
step rounded, and decoded by the oracle."""
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import DominoError  # noqa: E402
from paper_2403_06988_gb300 import _binding as B  # noqa: E402
from test_gpu_norm import TYPES, d  # noqa: E402,F401

NT = os.cpu_count() or 1
NAMES = ("history", "lengths", "prompt_lengths", "repetition", "presence", "frequency", "bias_ids", "bias_values")


class Case:
    """Inputs of one call (`args`, device tensors), the masks and the penalised logits (host)."""

    def __init__(self, batch, V, L, n_bias, dtype, density=0.5, seed=0, hot=True, drop=(), pad=0, equal_bias=False):
        rng = np.random.default_rng(seed * 1000 + batch + V + L + n_bias)
        self.V, W = V, (V + 31) // 32
        x = torch.from_numpy((rng.standard_normal((batch, V + pad)) * 3).astype(np.float32)).to(TYPES[dtype])
        self.logits = x.cuda()[:, :V]
        u = rng.random((batch, L))
        hist = np.minimum(((V + 1.0) ** u - 1.0 if hot else u * V).astype(np.int64), V - 1).astype(np.int32)
        hist[rng.random((batch, L)) < 0.05] = -1
        a = {"history": hist, "lengths": rng.integers(0, L + 1, batch).astype(np.int32)}
        a["lengths"][-1] = L
        a["prompt_lengths"] = (a["lengths"] * rng.random(batch)).astype(np.int32)
        a["repetition"] = (1 + rng.random(batch)).astype(np.float32)
        a["repetition"][0] = 0.75
        a["presence"], a["frequency"] = (rng.random(batch).astype(np.float32) for _ in range(2))
        ids = np.stack([rng.permutation(V)[:n_bias] if n_bias <= V else rng.integers(0, V, n_bias) for _ in range(batch)]).astype(np.int32)
        if equal_bias and n_bias:
            ids = np.minimum(ids, max(1, n_bias // 3)).astype(np.int32)
        if n_bias and L:     # biases of tokens that are in the history too
            for b in range(batch):
                n = min(n_bias // 2, L)
                ids[b, :n] = np.where(hist[b, :n] >= 0, hist[b, :n], ids[b, :n])
        ids[rng.random(ids.shape) < 0.1] = -1
        values = (rng.standard_normal(ids.shape) * 5).astype(np.float32)
        values[rng.random(ids.shape) < 0.1] = -np.inf
        a["bias_ids"], a["bias_values"] = ids, values
        for name in drop:
            a[name] = None
        if not n_bias:
            a["bias_ids"] = a["bias_values"] = None
        self.host = a
        self.args = {n: None if v is None else torch.from_numpy(v).cuda() for n, v in a.items()}
        bits = np.zeros((batch, W * 32), np.uint8)
        bits[:, :V] = rng.random((batch, V)) < density
        if batch > 2:
            bits[1] = 0                                # nothing allowed
        self.bits = bits
        self.mask_host = np.packbits(bits, axis=1, bitorder="little").view("<u4")
        self.mask = torch.from_numpy(self.mask_host.view(np.int32)).cuda()
        self.x = self.penalise(x[:, :V].float().numpy())

    def penalise(self, x):
        a, V = self.host, self.V
        x = x.copy()
        for b in range(x.shape[0]):
            if a["history"] is not None:
                h = a["history"][b]
                h = h[:len(h) if a["lengths"] is None else a["lengths"][b]]
                prompt = 0 if a["prompt_lengths"] is None else a["prompt_lengths"][b]
                seen, new = (np.bincount(t[t >= 0], minlength=V) for t in (h, h[prompt:]))
                rep, pres, freq = (np.float32(default if a[n] is None else a[n][b]) for n, default in
                                   (("repetition", 1), ("presence", 0), ("frequency", 0)))
                row = x[b]
                row = np.where(seen > 0, np.where(row > 0, row / rep, row * rep), row).astype(np.float32)
                row = np.where(new > 0, row - freq * new.astype(np.float32), row).astype(np.float32)
                x[b] = np.where(new > 0, row - pres, row).astype(np.float32)
            if a["bias_ids"] is not None:
                done = set()
                for t, v in zip(a["bias_ids"][b], a["bias_values"][b]):
                    if t >= 0 and int(t) not in done:
                        done.add(int(t))
                        x[b, t] = np.float32(x[b, t] + v)
        return x

    def want(self, masked=True):
        import oracle
        m = self.mask_host
        if not masked:
            bits = np.zeros_like(self.bits)
            bits[:, :self.V] = 1
            m = np.packbits(bits, axis=1, bitorder="little").view("<u4")
        # a banned token (-inf) has no part in the sum; the oracle's logits are finite
        allowed = np.unpackbits(m.view(np.uint8), axis=1, bitorder="little")[:, :self.V].astype(bool)
        allowed &= self.x > -np.inf
        full = np.zeros((len(m), m.shape[1] * 32), np.uint8)
        full[:, :self.V] = allowed
        m = np.packbits(full, axis=1, bitorder="little").view("<u4")
        x = np.where(self.x > -np.inf, self.x, 0).astype(np.float32)
        return x, m, oracle.mask_logits(x, m, want_logprobs=True, n_threads=NT)

    def check(self, got, masked=True):
        _, _, (arg, lse, lp) = self.want(masked)
        g_arg, g_lse, g_lp = got
        assert (g_arg.cpu().numpy() == arg).all()
        # the sum: V / 512 terms one after the other a thread and some 30 merges, each term 2^x with its own error of 2^-22,
        # the logarithm; the maximum added
        tol = (self.V / 512 + 40) * 2.0 ** -24 + 2.0 ** -20
        lse = lse.astype(np.float64)
        fin = np.isfinite(lse)
        for g, w in ((g_lse, lse), (g_lp, lp.astype(np.float64))):
            if g is None:
                continue
            g = g.cpu().numpy().astype(np.float64)
            f = np.isfinite(w)
            assert (np.isfinite(g) == f).all() and (g[~f] == -np.inf).all()
            allowed_off = tol + np.abs(w[f]) * 2.0 ** -23 + (np.abs(lse[fin]).max(initial=0) if w.ndim == 2 else 0) * 2.0 ** -23
            assert (np.abs(g[f] - w[f]) <= allowed_off).all()


SIZES = [(1, 1, 0, 0), (1, 1, 3, 1), (1, 32000, 500, 16), (3, 50, 1, 3), (5, 1000, 63, 1), (4, 50001, 1023, 7), (24, 8000, 200, 300), (7, 128256, 4096, 64),
         (160, 3001, 100, 5), (2, 70000, 9000, 1024), (3, 40, 300, 60), (310, 66000, 20, 2), (153, 20011, 700, 30), (161, 31, 5, 2), (177, 129, 0, 0)]


@pytest.mark.parametrize("batch,V,L,n_bias", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_greedy(d, batch, V, L, n_bias, dtype):  # noqa: F811
    c = Case(batch, V, L, n_bias, dtype)
    before = c.logits.clone()
    c.check(d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args))
    got = d.mask_logits_penalized(c.logits, mask=c.mask, **c.args)
    assert got[2] is None
    c.check(got)
    arg, lse, _ = d.mask_logits_penalized(c.logits, mask=c.mask, want_lse=False, **c.args)
    assert lse is None and torch.equal(arg, got[0])
    c.check(d.mask_logits_penalized(c.logits, want_logprobs=True, **c.args), masked=False)
    assert torch.equal(c.logits, before)


@pytest.mark.parametrize("batch,V,L,n_bias", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_draws(d, batch, V, L, n_bias, dtype):  # noqa: F811
    import oracle
    c = Case(batch, V, L, n_bias, dtype, seed=1)
    x, m, _ = c.want()
    got = d.mask_sample_penalized(c.logits, 0.7, 11, 1 << 33, mask=c.mask, **c.args)
    assert (got.cpu().numpy() == oracle.mask_sample(x, m, 0.7, 11, 1 << 33)).all()


@pytest.mark.parametrize("drop", [(n,) for n in NAMES[1:6]] + [NAMES[:6], ("bias_ids", "bias_values"), NAMES])
def test_what_is_not_given_penalises_nothing(d, drop):  # noqa: F811
    c = Case(6, 3000, 90, 4, "f32", seed=2, drop=drop)
    got = d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args)
    c.check(got)
    if drop == NAMES:
        plain = [torch.empty_like(t) for t in got]
        B.domino_mask_logits_noalloc(c.logits.data_ptr(), B.DTYPE_F32, 6, 3000, 3000, c.mask, *plain)
        assert all(torch.equal(a, b) for a, b in zip(got, plain))


@pytest.mark.parametrize("pad", [0, 1, 3, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_apart(d, pad, dtype):  # noqa: F811
    c = Case(5, 9001, 300, 9, dtype, seed=3, pad=pad)
    c.check(d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args))


@pytest.mark.parametrize("batch,V", [(6, 700), (3, 50001), (200, 5000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties_go_to_the_lowest_token(d, batch, V, dtype):  # noqa: F811
    """Few different logits, and penalties that are whole: changed and other tokens tie at the top."""
    c = Case(batch, V, 80, 9, dtype, seed=14, density=0.6)
    c.logits = c.logits.float().round().clamp(-2, 1).to(c.logits.dtype)
    c.host["repetition"][:], c.host["presence"][:], c.host["frequency"][:] = 1.0, 1.0, 0.0
    c.host["presence"][::2] = 0.0
    c.host["bias_values"] = np.sign(c.host["bias_values"]).astype(np.float32)
    c.args = {n: None if v is None else torch.from_numpy(v).cuda() for n, v in c.host.items()}
    c.x = c.penalise(c.logits.float().cpu().numpy())
    c.check(d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args))
    arg, _, _ = d.mask_logits_penalized(c.logits, mask=c.mask, want_lse=False, **c.args)
    assert (arg.cpu().numpy() == c.want()[2][0]).all()


def test_of_equal_biases_the_first_counts(d):  # noqa: F811
    c = Case(4, 2000, 50, 700, "f32", seed=4, equal_bias=True, density=0.9)
    c.check(d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args))


@pytest.mark.parametrize("V,L", [(128256, 60000), (200000, 150000), (40000, 300000)])
def test_histories_longer_than_shared_memory(d, V, L):  # noqa: F811
    """Rows in several parts, most of whose tokens change."""
    c = Case(3, V, L, 20, "bf16", seed=5, hot=False)
    c.check(d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args))


def test_one_token_many_times(d):  # noqa: F811
    """Counts beyond 16 bits, in the prompt and after it."""
    c = Case(2, 500, 200000, 0, "f32", seed=6, density=1.0)
    h = c.host["history"]
    h[:] = 123
    c.host["lengths"][:], c.host["prompt_lengths"][:] = (200000, 200000), (70000, 200000)
    c.args = {n: None if v is None else torch.from_numpy(v).cuda() for n, v in c.host.items()}
    c.x = c.penalise(c.logits.float().cpu().numpy())
    assert c.x[0, 123] < -1000
    c.check(d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args))


def test_all_tokens_changed_and_all_banned(d):  # noqa: F811
    c = Case(3, 1024, 5, 1024, "f32", seed=7, density=1.0)
    c.host["bias_ids"][:] = np.arange(1024)
    c.host["bias_values"][0] = -np.inf
    c.args = {n: None if v is None else torch.from_numpy(v).cuda() for n, v in c.host.items()}
    c.x = c.penalise(c.logits.cpu().numpy())
    got = d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args)
    assert int(got[0][0]) == -1 and float(got[1][0]) == -np.inf and (got[2][0] == -np.inf).all()
    c.check(got)


def test_masked_places_are_not_used(d):  # noqa: F811
    """No numbers, infinities and the lowest values where the mask allows nothing, in the history and outside of it."""
    c = Case(5, 4000, 400, 30, "f32", seed=8)
    want = d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args)
    off = torch.from_numpy(c.bits[:, :4000] == 0).cuda()
    for bad in (float("nan"), float("inf"), -float("inf"), -3.4e38):
        x = torch.where(off, torch.full_like(c.logits, bad), c.logits)
        got = d.mask_logits_penalized(x, mask=c.mask, want_logprobs=True, **c.args)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(d.mask_sample_penalized(x, 1.0, 3, 4, mask=c.mask, **c.args),
                           d.mask_sample_penalized(c.logits, 1.0, 3, 4, mask=c.mask, **c.args))
    c = Case(5, 4001, 400, 30, "f32", seed=9)
    full = c.mask.clone()
    full[:, -1] |= -2            # bits at or beyond V are ignored
    a, b = (d.mask_logits_penalized(c.logits, mask=m, want_logprobs=True, **c.args) for m in (c.mask, full))
    assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_bad_tokens_and_lengths(d):  # noqa: F811
    c = Case(4, 1000, 60, 8, "f32", seed=10, density=1.0)
    assert d.device_error() == 0
    want = d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args)
    for name, at in (("history", (3, 5)), ("bias_ids", (2, 1))):
        good, bad = dict(c.args), dict(c.args)
        good[name], bad[name] = c.args[name].clone(), c.args[name].clone()
        good[name][at], bad[name][at] = -1, 1000
        if name == "bias_ids":
            bad[name][at] = 2 ** 31 - 1
        a = d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **good)
        assert d.device_error() == 0
        b = d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **bad)
        assert d.device_error() == B.DEVERR_BAD_TOKEN and all(torch.equal(u, v) for u, v in zip(a, b))
    far = c.args["lengths"].clone()
    far[3] = 61                  # the row's is 60
    got = d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **{**c.args, "lengths": far})
    assert d.device_error() == B.DEVERR_BAD_TOKEN and all(torch.equal(u, v) for u, v in zip(got, want))
    far[3] = -5
    none = c.args["lengths"].clone()
    none[3] = 0
    a, b = (d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **{**c.args, "lengths": t}) for t in (none, far))
    assert d.device_error() == B.DEVERR_BAD_TOKEN and all(torch.equal(u, v) for u, v in zip(a, b))


def test_beyond_a_rows_length_nothing_is_read(d):  # noqa: F811
    c = Case(4, 1000, 60, 0, "f32", seed=11)
    want = d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **c.args)
    h = c.args["history"].clone()
    h[torch.arange(60, device="cuda")[None] >= c.args["lengths"][:, None]] = 2 ** 30
    got = d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, **{**c.args, "history": h})
    assert all(torch.equal(u, v) for u, v in zip(got, want)) and d.device_error() == 0


def test_offsets_beyond_32_bits(d):  # noqa: F811
    """Logits and histories whose offsets pass 2^32 bytes and 2^31 values."""
    batch, V = 33000, 66000
    x = torch.zeros(batch, V, dtype=torch.bfloat16, device="cuda")
    x[-1, 5], x[-1, 65999] = 4.0, 3.0
    h = torch.full((batch, 66000), -1, dtype=torch.int32, device="cuda")
    h[-1, 65999] = 5
    arg, lse, _ = d.mask_logits_penalized(x, h, repetition=torch.full((batch,), 2.0, device="cuda"))
    assert int(arg[-1]) == 65999 and not arg[:-1].any()
    want = np.log(65998 + np.exp(3.0) + np.exp(2.0))
    assert abs(float(lse[-1]) - want) < 1e-4 and abs(float(lse[0]) - np.log(66000)) < 1e-4


def test_graph_and_another_stream(d):  # noqa: F811
    c = Case(9, 30000, 700, 20, "bf16", seed=12)

    def call(out=(None, None, None), tokens=None, **k):
        return [*d.mask_logits_penalized(c.logits, mask=c.mask, want_logprobs=True, out=out, **c.args, **k),
                d.mask_sample_penalized(c.logits, 0.9, 5, 6, mask=c.mask, out=tokens, **c.args, **k)]
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = call(stream=s)
    s.synchronize()
    out = [torch.empty_like(t) for t in want]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call(tuple(out[:3]), out[3])
    for t in out:
        t.fill_(7)
    g.replay()
    torch.cuda.synchronize()
    for t in (got, out):
        assert all(torch.equal(a, b) for a, b in zip(t, want))
    del g


def test_refusals(d):  # noqa: F811
    c = Case(4, 500, 20, 5, "f32", seed=13)

    def call(**k):
        return d.mask_logits_penalized(c.logits, mask=c.mask, **{**c.args, **k})
    for k in ({"history": c.args["history"].long()}, {"repetition": c.args["repetition"].double()}, {"lengths": 3}):
        with pytest.raises(TypeError):
            call(**k)
    for k in ({"history": c.args["history"][:3]}, {"lengths": c.args["lengths"][:3]}, {"bias_ids": None}, {"bias_values": None},
              {"bias_values": c.args["bias_values"][:, :4].contiguous()}, {"history": c.args["history"][:, ::2]},
              {"repetition": c.args["repetition"].cpu()}):
        with pytest.raises(ValueError):
            call(**k)
    with pytest.raises(ValueError):
        d.mask_logits_penalized(c.logits, mask=c.mask[:, :15])
    with pytest.raises(TypeError):
        d.mask_logits_penalized(c.logits.half())
    many = torch.zeros(4, 1025, dtype=torch.int32, device="cuda")
    with pytest.raises(DominoError) as e:
        call(bias_ids=many, bias_values=many.float())
    assert e.value.status == -1
    for t in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(DominoError) as e:
            d.mask_sample_penalized(c.logits, t, 0, 0, mask=c.mask, **c.args)
        assert e.value.status == -1
    arg = torch.empty(4, dtype=torch.int32, device="cuda")
    for V, stride, p in ((0, 500, {}), (500, 499, {}), (500, 500, {"history_len": -1}), (500, 500, {"history_len": 3}),
                         (500, 500, {"n_bias": 3}), (500, 500, {"n_bias": -1}), (500, 500, {"lengths_dev": c.logits.data_ptr() + 2})):
        with pytest.raises(DominoError) as e:
            B.domino_mask_logits_penalized(d.h, c.logits.data_ptr(), 0, 4, stride, V, B.penalties(**p), c.mask, arg)
        assert e.value.status == -1
    with pytest.raises(DominoError) as e:
        B.domino_mask_logits_penalized(d.h, c.logits.data_ptr(), 0, 4, 500, 500, None, c.mask, arg)
    assert e.value.status == -1
    with pytest.raises(DominoError) as e:
        B.domino_mask_logits_penalized(d.h, c.logits.data_ptr(), 0, 4, 500, 500, B.penalties(c.args["history"], (1 << 30) + 1), c.mask, arg)
    assert e.value.status == -3
    empty = d.mask_logits_penalized(c.logits[:0], c.args["history"][:0])
    assert empty[0].shape == (0,)
