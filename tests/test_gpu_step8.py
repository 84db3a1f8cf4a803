"""The norm, 8-bit logits and the decode under penalties as a server runs them with the mask step, and the norm with the token
loss and the embedding as a training step does: each result against what it was made from, eagerly and from a CUDA graph."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import Domino, synth  # noqa: E402
from loss_reference import unpack  # noqa: E402
from norm8_reference import Norm, assert_within, logits8  # noqa: E402
from test_gpu_norm import check_codes  # noqa: E402

DIM, STEPS, ROOM = 200, 6, 16


class Server:
    """One table at both ends, a mixing matrix for the model's blocks; greedy under the key/value grammar (V = 1024)."""

    def __init__(self, batch=24, seed=3):
        self.w = synth.workload(1)
        self.d = Domino.from_parts(self.w.automaton, self.w.vocab, device=0)
        self.V = self.w.vocab.n_tokens
        g = torch.Generator("cuda").manual_seed(seed)
        self.table = (torch.randn(self.V, DIM, generator=g, device="cuda") * 0.5).bfloat16()
        self.mix = (torch.randn(DIM, DIM, generator=g, device="cuda") / DIM ** 0.5).bfloat16()
        self.gain = (1 + 0.1 * torch.randn(DIM, generator=g, device="cuda")).bfloat16()
        self.codes = self.d.quantize8(self.table, 128)
        states, _ = self.w.initial_configs(batch=batch)
        self.states = torch.from_numpy(states).cuda()
        self.last = torch.randint(0, self.V, (batch,), generator=g, device="cuda").int()
        self.stream = torch.zeros(batch, DIM, dtype=torch.bfloat16, device="cuda")
        self.history = torch.full((batch, ROOM), -1, dtype=torch.int32, device="cuda")
        self.history[:, 0] = self.last
        self.length = torch.ones(batch, dtype=torch.int32, device="cuda")
        self.prompt = torch.ones(batch, dtype=torch.int32, device="cuda")
        self.rep, self.pres, self.freq = (torch.full((batch,), v, device="cuda") for v in (1.3, 0.4, 0.2))
        self.ids = torch.randint(0, self.V, (batch, 3), generator=g, device="cuda").int()
        self.values = torch.randn(batch, 3, generator=g, device="cuda") * 4

    def step(self):
        d = self.d
        block = d.embed(self.last, self.table) @ self.mix
        q, s, total = d.norm8(block, self.gain, self.stream)
        logits = d.logits8(q, s, *self.codes)
        mask, _ = d.step_mask(self.states)
        seen, count = self.history.clone(), self.length.clone()
        token, lse, lp = d.mask_logits_penalized(logits, self.history, self.length, self.prompt, self.rep, self.pres, self.freq,
                                                 self.ids, self.values, mask, want_logprobs=True)
        self.kept = dict(block=block, before=self.stream.clone(), q=q, s=s, total=total, logits=logits, mask=mask, seen=seen,
                         count=count, token=token, lse=lse, lp=lp)
        self.stream.copy_(total)
        d.advance(self.states, None, token)
        self.history.scatter_(1, self.length.long()[:, None], token[:, None])
        self.length += 1
        self.last.copy_(token)
        return token

    def penalised(self, k):
        """The step's penalised logits, -inf where the mask allows nothing: fp32, on the host."""
        x, seen, count = k["logits"].cpu().numpy().copy(), k["seen"].cpu().numpy(), k["count"].cpu().numpy()
        ids, values = self.ids.cpu().numpy(), self.values.cpu().numpy()
        for b in range(len(x)):
            h = seen[b, :count[b]]
            n, c = (np.bincount(t[t >= 0], minlength=self.V) for t in (h, h[1:]))
            row = np.where(n > 0, np.where(x[b] > 0, x[b] / np.float32(1.3), x[b] * np.float32(1.3)), x[b]).astype(np.float32)
            row = np.where(c > 0, row - np.float32(0.2) * c.astype(np.float32), row).astype(np.float32)
            row = np.where(c > 0, row - np.float32(0.4), row).astype(np.float32)
            for i in range(3):
                if ids[b, i] not in ids[b, :i]:
                    row[ids[b, i]] = np.float32(row[ids[b, i]] + values[b, i])
            x[b] = row
        return np.where(unpack(k["mask"], self.V).cpu().numpy(), x, -np.inf)


def test_decode_steps():
    m = Server()
    for _ in range(STEPS):
        m.step()
        k = m.kept
        ref = Norm(k["block"], m.gain, k["before"])
        assert torch.equal(k["total"], ref.sum)
        check_codes(k["q"], k["s"], ref.y, ref.rel_y, 1, "norm8")
        want, tol = logits8(k["q"], k["s"], *m.codes, torch.float32)
        assert_within(k["logits"], want, tol, "logits")
        x = m.penalised(k)
        token = np.where(np.isinf(x.max(1)), -1, x.argmax(1))
        assert (k["token"].cpu().numpy() == token).all() and (token >= 0).all()
        wide = x.astype(np.float64)
        lse = np.log(np.exp(wide - wide.max(1, keepdims=True)).sum(1)) + wide.max(1)
        assert np.abs(k["lse"].cpu().numpy() - lse).max() < 1e-5 and np.isinf(k["lp"].cpu().numpy()).sum() == np.isinf(x).sum()
    assert m.d.device_error() == 0
    m.d.close()


def test_decode_steps_from_a_graph():
    eager, m = Server(), Server()
    want = [eager.step().clone() for _ in range(STEPS)]
    kept = [t.clone() for t in (m.states, m.last, m.stream, m.history, m.length)]
    m.step()                                   # warm, and put back
    for t, old in zip((m.states, m.last, m.stream, m.history, m.length), kept):
        t.copy_(old)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        token = m.step()
    for w in want:
        g.replay()
        assert torch.equal(token, w)
    torch.cuda.synchronize()
    assert torch.equal(m.stream, eager.stream) and torch.equal(m.states, eager.states)
    del g
    for s in (eager, m):
        assert s.d.device_error() == 0
        s.d.close()


def test_two_handles_at_once():
    """Two servers on two streams, their steps interleaved, decode what each alone does."""
    alone = []
    for seed in (5, 6):
        m = Server(seed=seed)
        alone.append([m.step().clone() for _ in range(STEPS)])
        m.d.close()
    torch.cuda.synchronize()
    servers, streams = [Server(seed=s) for s in (5, 6)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(STEPS):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(servers[i].step().clone())
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[i], alone[i]))
        servers[i].d.close()


def train_inputs(T=300, V=2000, D=264):
    g = torch.Generator("cuda").manual_seed(9)
    x, r = ((torch.randn(T, D, generator=g, device="cuda") * s).bfloat16() for s in (1.0, 2.0))
    gain = (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).bfloat16()
    w = (torch.randn(V, D, generator=g, device="cuda") / D ** 0.5).bfloat16()
    y = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    c = torch.full((T,), 1.0 / T, device="cuda")
    ds = (torch.randn(T, D, generator=g, device="cuda") * 1e-4).bfloat16()
    return x, r, gain, w, y, c, ds


def train_step(d, x, r, gain, w, y, c, ds):
    h, total, rstd = d.norm(x, gain, r)
    loss, lse = d.token_loss(h, w, y)
    dh, dw = d.token_loss_grad(h, w, y, lse, c)
    dx, dgain = d.norm_grad(total, gain, rstd, dh, ds)
    return loss, dw, dx, dgain


def test_training_step():
    """The gradients of the mean loss and of sum(ds (x + r)) against autograd in 64 bits: norms within the roundings of h, G, dh
    (each 2^-9 to 2^-8 of a value) and of the results."""
    d = Domino(0)
    x, r, gain, w, y, c, ds = train_inputs()
    loss, dw, dx, dgain = train_step(d, x, r, gain, w, y, c, ds)
    leaves = [t.double().requires_grad_() for t in ((x.float() + r.float()).bfloat16(), gain, w)]
    total, g64, w64 = leaves
    h = total * ((total * total).mean(1, keepdim=True) + 1e-6) ** -0.5 * g64
    z = (h @ w64.T).log_softmax(1)
    value = -z.gather(1, y.long()[:, None])[:, 0]
    (value.mean() + (ds.double() * total).sum()).backward()
    # a logit: D products of h, off by 2^-9 at random, and w: sqrt(D) 2^-9 |h w|, some 0.01 at most
    assert float((loss.double() - value.detach()).abs().max()) < 0.03
    for got, leaf in ((dx, total), (dgain, g64), (dw, w64)):
        assert float((got.double() - leaf.grad).norm() / leaf.grad.norm()) < 2.0 ** -6
    d.close()


def test_training_step_from_a_graph():
    d = Domino(0)
    a = train_inputs()
    want = [t.clone() for t in train_step(d, *a)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = train_step(d, *a)
    for _ in range(2):
        for t in got:
            t.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, want))
    del g
    d.close()


@pytest.mark.parametrize("fill", [None, 0xAB])
def test_outputs_are_not_the_current_streams(monkeypatch, fill):
    """Calls with stream= given: what they make comes from that stream's memory."""
    monkeypatch.setattr(Domino, "fill_byte", fill)
    d = Domino(0)
    x, r, gain, w, _, _, ds = train_inputs()
    _, total, rstd = d.norm(x, gain, r)
    q, s = d.quantize8(x)
    wq, ws = d.quantize8(w, 128)
    logits = d.logits8(q, s, wq, ws).contiguous()
    hist = torch.randint(0, 2000, (300, 9), device="cuda").int()
    rep = torch.full((300,), 1.5, device="cuda")
    calls = {
        "norm": lambda **k: d.norm(x, gain, r, **k),
        "norm8": lambda **k: d.norm8(x, gain, r, **k),
        "norm_grad": lambda **k: d.norm_grad(total, gain, rstd, ds, **k),
        "quantize8": lambda **k: d.quantize8(x, **k),
        "logits8": lambda **k: (d.logits8(q, s, wq, ws, **k),),
        "penalized": lambda **k: d.mask_logits_penalized(logits, hist, repetition=rep, want_logprobs=True, **k),
        "draw": lambda **k: (d.mask_sample_penalized(logits, 0.8, 1, 2, hist, repetition=rep, **k),),
    }
    st = torch.cuda.Stream()
    for name, call in calls.items():
        want = call()
        torch.cuda.synchronize()
        used = [torch.empty(o.untyped_storage().nbytes(), dtype=torch.uint8, device="cuda") for o in want for _ in range(2)]
        places = {u.data_ptr() for u in used}
        del used
        got = call(stream=st)
        assert not places & {o.data_ptr() for o in got}, name
        st.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a.float(), b.float()), name
    d.close()
