"""Calls with stream= given: outputs that they make come from that stream's memory, not from what the current stream has
just given back and may still be using."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2403_06988_gb300 import Domino, synth  # noqa: E402
from test_gpu_token_loss import d, inputs  # noqa: E402,F401


@pytest.mark.parametrize("fill", [None, 0xAB])
@pytest.mark.parametrize("as_int", [False, True])
def test_outputs_are_not_the_current_streams(d, monkeypatch, fill, as_int):  # noqa: F811
    monkeypatch.setattr(Domino, "fill_byte", fill)
    h, w, y, mask, c = inputs(300, 3000, 264, density=0.3)
    logits = (h.float() @ w.float().T).contiguous()
    ids = logits.topk(7, dim=1).indices.int()
    teacher = torch.randn(300, 7, device="cuda")
    t = y.clamp(min=0)
    want = {"token_loss": d.token_loss(h, w, y, mask)}
    lse = want["token_loss"][1]
    want["distill_loss"] = d.distill_loss(logits, teacher, ids, 2.0, mask)
    dlse = want["distill_loss"][1]
    s = torch.cuda.Stream()
    stream = s.cuda_stream if as_int else s
    calls = {
        "token_loss": lambda **k: d.token_loss(h, w, y, mask, **k),
        "token_loss_grad": lambda **k: d.token_loss_grad(h, w, y, lse, c, mask, **k),
        "distill_loss": lambda **k: d.distill_loss(logits, teacher, ids, 2.0, mask, **k),
        "distill_grad": lambda **k: (d.distill_grad(logits, teacher, ids, 2.0, dlse, c, mask, **k),),
        "embed": lambda **k: (d.embed(t, w, 2.0, **k),),
        "embed_grad": lambda **k: (d.embed_grad(t, h, 3000, 2.0, **k),),
    }
    for name, call in calls.items():
        want = call()
        torch.cuda.synchronize()
        # blocks of the outputs' sizes that this stream has used and given back
        used = [torch.empty_like(o) for o in want for _ in range(2)]
        places = {u.data_ptr() for u in used}
        for u in used:
            u.zero_()
        del used, u
        got = call(stream=stream)
        assert not places & {o.data_ptr() for o in got}, name
        s.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), name
        del got


def test_walk_and_decode_outputs_too(monkeypatch):
    monkeypatch.setattr(Domino, "fill_byte", None)
    w = synth.workload(1)
    d = Domino.from_parts(w.automaton, w.vocab, device=0)  # noqa: F811
    states = torch.full((64,), w.automaton.start, dtype=torch.int32, device="cuda")
    logits = torch.randn(64, w.vocab.n_tokens, device="cuda")
    mask, _ = d.step_mask(states)
    table_next, table_mask = d.precompute_table()
    s = torch.cuda.Stream()
    calls = [lambda **k: d.step_mask(states, want_next=True, **k),
             lambda **k: d.mask_logits(logits, mask, want_logprobs=True, **k),
             lambda **k: (d.mask_sample(logits, mask, 1.0, 1, 2, **k),),
             lambda **k: d.step_decode(states, None, logits, want_logprobs=True, **k),
             lambda **k: d.opportunistic_step(logits, states, **k),
             lambda **k: d.mask_logits_table(logits, table_mask, states, want_logprobs=True, **k),
             lambda **k: d.precompute_table(**k)]
    for i, call in enumerate(calls):
        want = call()
        torch.cuda.synchronize()
        used = [torch.empty_like(o) for o in want for _ in range(3)]
        places = {u.data_ptr() for u in used}
        del used
        got = call(stream=s)
        assert not places & {o.data_ptr() for o in got}, i
        s.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), i
        del got
    d.close()
