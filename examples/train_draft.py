"""Trains a small model on sequences that a grammar allows, under the grammar's masks, and distills a narrower draft
model from it (the kind of model whose proposals speculative decoding verifies).

The data are random walks through the grammar (mask, draw, update) with a fixed preference for each pair of tokens.
Both models predict the next token from the last one: hidden = embed(last) @ mix, logits = hidden @ table.T, with one
table at both ends.  The library computes the lookup, the masked losses and their gradients; torch the small products
and the optimizer's arithmetic.

    python examples/train_draft.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2403_06988_gb300 import Domino, synth  # noqa: E402


def walks(d, start, batch, length, preference, seed):
    """(last tokens, next tokens, masks) of `batch` walks of `length` tokens, one position after the other."""
    V = preference.shape[0]
    states = torch.full((batch,), start, dtype=torch.int32, device="cuda")
    last = torch.full((batch,), -1, dtype=torch.int32, device="cuda")
    lasts, nexts, masks = [], [], []
    for i in range(length):
        mask, _ = d.step_mask(states)
        logits = torch.where((last >= 0)[:, None], preference[last.long().clamp(min=0)], torch.zeros(V, device="cuda"))
        token = d.mask_sample(logits, mask, 1.0, seed, i)
        lasts.append(last), nexts.append(token), masks.append(mask)
        d.advance(states, None, token)
        last = token
    return torch.cat(lasts), torch.cat(nexts), torch.cat(masks)


class Model:
    def __init__(self, d, V, dim, seed):
        g = torch.Generator("cuda").manual_seed(seed)
        self.d, self.V, self.scale = d, V, 1.0
        self.table = torch.randn(V, dim, generator=g, device="cuda") * 0.3      # fp32, rounded for the products
        self.mix = torch.randn(dim, dim, generator=g, device="cuda") / dim ** 0.5
        self.moments = [torch.zeros_like(p) for p in (self.table, self.table, self.mix, self.mix)]
        self.steps = 0

    def hidden(self, last):
        self.w, self.m = self.table.bfloat16(), self.mix.bfloat16()
        self.x = self.d.embed(last, self.w, self.scale)
        return self.x @ self.m

    def update(self, last, dhidden, dweight, rate=0.02):
        """Adam, with the gradients of both ends of the table."""
        dmix = self.x.T @ dhidden
        self.d.embed_grad(last, dhidden @ self.m.T, self.V, self.scale, into=dweight)
        self.steps += 1
        for p, g, a, b in ((self.table, dweight, *self.moments[:2]), (self.mix, dmix, *self.moments[2:])):
            g = g.float()
            a.mul_(0.9).add_(g, alpha=0.1)
            b.mul_(0.99).addcmul_(g, g, value=0.01)
            p -= rate * (a / (1 - 0.9 ** self.steps)) / ((b / (1 - 0.99 ** self.steps)).sqrt() + 1e-8)


def run(steps=60, batch=64, length=32, top=16, temperature=2.0):
    """(training losses, divergences, agreement before, agreement after): the last two are the shares of positions where
    the draft's greedy token under the mask is the model's."""
    w = synth.workload(1)                        # the 16-state key/value grammar, 1024 tokens
    V = w.vocab.n_tokens
    d = Domino.from_parts(w.automaton, w.vocab, device=0)
    preference = torch.randn(V, V, generator=torch.Generator("cuda").manual_seed(1), device="cuda") * 2
    last, target, masks = walks(d, w.automaton.start, batch, length, preference, seed=7)
    share = torch.full((len(target),), 1.0 / len(target), device="cuda")

    model, losses = Model(d, V, 128, 2), []
    for _ in range(steps):
        h = model.hidden(last)
        loss, lse = d.token_loss(h, model.w, target, masks)
        dh, dw = d.token_loss_grad(h, model.w, target, lse, share, masks)
        model.update(last, dh, dw)
        losses.append(loss.mean())

    teacher = model.hidden(last) @ model.w.T
    top_logits, ids = teacher.float().topk(top, dim=1)
    ids = ids.int()
    chosen, _, _ = d.mask_logits(teacher, masks, n_tokens=V)
    draft, divergences, agreement = Model(d, V, 32, 3), [], []
    for step in range(steps + 1):
        h = draft.hidden(last)
        logits = h @ draft.w.T
        if step in (0, steps):
            agreement.append((d.mask_logits(logits, masks, n_tokens=V)[0] == chosen).float().mean())
        loss, lse = d.distill_loss(logits, top_logits, ids, temperature, masks)
        divergences.append(loss.mean())
        if step < steps:
            dl = d.distill_grad(logits, top_logits, ids, temperature, lse, share, masks, out=logits)
            draft.update(last, dl @ draft.w, dl.T @ h)
    assert d.device_error() == 0
    d.close()
    return [float(x) for x in losses], [float(x) for x in divergences], float(agreement[0]), float(agreement[1])


if __name__ == "__main__":
    losses, divergences, before, after = run(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
    print(f"model: masked cross entropy {losses[0]:.3f} -> {losses[-1]:.3f}")
    print(f"draft: divergence from the model's top logits {divergences[0]:.3f} -> {divergences[-1]:.3f}")
    print(f"draft's greedy token is the model's: {100 * before:.1f} % -> {100 * after:.1f} % of positions")
