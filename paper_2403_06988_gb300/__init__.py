"""DOMINO constrained decoding hot path on GB300 (sm_103a).

The compute lives in libdomino.so (C ABI in include/domino.h, kernels in
csrc/).  `_binding` exposes every entry point under its C name; `Domino`
below is a thin holder of one handle that allocates output tensors with torch
and forwards to those entry points.  There is no CPU fallback: without a
built libdomino.so the binding raises ImportError, and compute calls on a
handle created without a GPU raise DominoError(E_NO_DEVICE).
"""
from __future__ import annotations

import os
from typing import Optional, Tuple

from . import _binding as B
from ._binding import DominoError, DTYPE_BF16, DTYPE_F32  # noqa: F401


_CALLS = None


def _calls():
    """The extension that the losses, the embedding, the norm, 8-bit operands and the decode under penalties are called
    through (csrc/calls.cpp), bound to the loaded library."""
    global _CALLS
    if _CALLS is None:
        import ctypes

        import torch  # noqa: F401  (its libraries, before the extension's)
        from . import build
        if not os.path.exists(build.CALLS) or build.calls_built_for_another():
            raise ImportError("_loss_calls.so is not built for this torch; run __graft_entry__.build() or "
                              "python -m paper_2403_06988_gb300.build")
        from . import _loss_calls as c
        c.bind(*(ctypes.cast(getattr(B.lib(), "domino_" + n), ctypes.c_void_p).value
                 for n in ("token_loss", "token_loss_grad", "distill_loss", "distill_grad", "embed", "embed_grad", "norm",
                           "norm8", "norm_grad", "quantize8", "logits8", "mask_logits_penalized", "mask_sample_penalized")))
        _CALLS = c
    return _CALLS


class Domino:
    """One library handle: a vocabulary plus a scanner (+ bracket rules).

    fill_byte: None (default), or a byte value that every output buffer this
    holder allocates is filled with before the call that writes it.  A word a
    kernel leaves unwritten then keeps that pattern (0xAB bytes, say) instead
    of whatever the allocator handed back, so an exact comparison catches it.
    A debugging aid; it costs one fill per output.
    """

    fill_byte: Optional[int] = None

    def __init__(self, device: int = 0):
        self.device = device
        self.h = B.domino_create(device)

    def close(self):
        if self.h:
            B.domino_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- loads ---------------------------------------------------------------
    def load_vocab(self, vocab) -> None:
        B.domino_load_vocab(self.h, vocab.data, vocab.offsets, vocab.n_tokens, vocab.eos_id)

    def load_automaton(self, a) -> None:
        B.domino_load_automaton(self.h, a.delta, a.n_states, a.live, a.accepting, a.start, a.rules, None,
                                a.max_depth)

    @staticmethod
    def from_parts(automaton, vocab, device: int = 0) -> "Domino":
        d = Domino(device)
        d.load_vocab(vocab)
        d.load_automaton(automaton)
        return d

    def info(self) -> dict:
        return B.domino_get_info(self.h)

    def _empty(self, shape, dtype, device, stream=None, zero=False):
        """An output of a call on `stream`.  Where that is not torch's current one, it is made on it (not from a block that
        the current stream has given back and may still be using), and stays in use until what the current stream does
        with it has ended."""
        import torch
        if stream is not None:
            now, to = torch.cuda.current_stream(device), B._stream(stream)
            if to != now.cuda_stream:
                to = 0 if to == 1 else to     # cudaStreamLegacy: the default stream's other name
                with torch.cuda.stream(torch.cuda.ExternalStream(to, device)):
                    t = self._empty(shape, dtype, device, None, zero)
                if t.numel():
                    t.record_stream(now)
                return t
        t = torch.empty(shape, dtype=dtype, device=device)
        if zero:
            t.zero_()
        elif self.fill_byte is not None and t.numel():
            t.view(torch.uint8).fill_(self.fill_byte)
        return t

    # -- compute (torch tensors on this handle's device) -----------------------
    def step_mask(self, states, stacks=None, want_next: bool = False, out_mask=None, out_next=None,
                  stream=None):
        import torch
        b = states.shape[0]
        mask, nxt = out_mask, out_next
        if mask is None or (want_next and nxt is None):
            V, W = B.sizes(self.h)
            if mask is None:
                mask = self._empty((b, W), torch.int32, states.device, stream)
            if want_next and nxt is None:
                nxt = self._empty((b, V), torch.int32, states.device, stream)
        B.domino_step_mask(self.h, states, stacks, b, mask, nxt, stream)
        return mask, nxt

    def step_decode(self, states, stacks, logits, want_logprobs: bool = False, advance: bool = False, out_mask=None,
                    stream=None):
        """Mask step fused with the masked greedy decode: returns (mask, argmax, lse, logprobs or None).
        advance: states (and stacks) are then updated in place by the decoded tokens."""
        import torch
        b = states.shape[0]
        dtype = DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_F32
        if dtype == DTYPE_F32 and logits.dtype != torch.float32:
            raise TypeError("logits must be float32 or bfloat16")
        if logits.stride(1) != 1:
            raise ValueError("logits rows must be contiguous")
        dev = states.device
        mask, lp = out_mask, None
        if mask is None or want_logprobs:
            V, W = B.sizes(self.h)
            if mask is None:
                mask = self._empty((b, W), torch.int32, dev, stream)
            if want_logprobs:
                lp = self._empty((b, V), torch.float32, dev, stream)
        argmax = self._empty(b, torch.int32, dev, stream)
        lse = self._empty(b, torch.float32, dev, stream)
        B.domino_step_decode(self.h, states, stacks, b, logits.data_ptr(), dtype, logits.stride(0), mask, argmax, lse,
                             lp, states if advance else None, stacks if advance else None, stream)
        return mask, argmax, lse, lp

    def precompute_table(self, want_next: bool = True, want_mask: bool = True, stream=None):
        import torch
        info = self.info()
        dev = f"cuda:{self.device}"
        nxt = self._empty((info["n_states"], info["n_tokens"]), torch.int32, dev, stream) if want_next else None
        mask = self._empty((info["n_states"], info["n_words"]), torch.int32, dev, stream) if want_mask else None
        B.domino_precompute_table(self.h, nxt, mask, stream)
        return nxt, mask

    def mask_logits(self, logits, mask, want_lse: bool = True, want_logprobs: bool = False, n_tokens: Optional[int]
                    = None, out=None, stream=None) -> Tuple:
        import torch
        b = logits.shape[0]
        if n_tokens is None and want_logprobs and (out is None or out[2] is None):
            n_tokens = B.sizes(self.h)[0]
        dtype = DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_F32
        if dtype == DTYPE_F32 and logits.dtype != torch.float32:
            raise TypeError("logits must be float32 or bfloat16")
        if logits.stride(1) != 1:
            raise ValueError("logits rows must be contiguous")
        argmax, lse, lp = out if out is not None else (None, None, None)
        if argmax is None:
            argmax = self._empty(b, torch.int32, logits.device, stream)
        if want_lse and lse is None:
            lse = self._empty(b, torch.float32, logits.device, stream)
        if want_logprobs and lp is None:
            lp = self._empty((b, n_tokens), torch.float32, logits.device, stream)
        B.domino_mask_logits(self.h, logits.data_ptr(), dtype, b, logits.stride(0), mask, argmax,
                             lse if want_lse else None, lp if want_logprobs else None, stream)
        return argmax, (lse if want_lse else None), (lp if want_logprobs else None)

    def advance(self, states, stacks, tokens, states_out=None, stacks_out=None, stream=None):
        b = states.shape[0]
        so = states if states_out is None else states_out
        wo = stacks if stacks_out is None else stacks_out
        B.domino_advance(self.h, states, stacks, tokens, b, so, wo, stream)
        return so, wo

    def mask_sample(self, logits, mask, temperature: float, seed: int, offset: int, stream=None):
        """Gumbel-max draw per row from softmax(logits / T) over the allowed tokens (-1: none allowed)."""
        import torch
        b = logits.shape[0]
        dtype = DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_F32
        if logits.stride(1) != 1:
            raise ValueError("logits rows must be contiguous")
        tokens = self._empty(b, torch.int32, logits.device, stream)
        B.domino_mask_sample(self.h, logits, dtype, b, logits.stride(0), mask, temperature, seed, offset, tokens,
                             stream)
        return tokens

    def opportunistic_step(self, logits, states, stacks=None, stream=None):
        """Greedy tokens via opportunistic masking; returns (tokens, number of fallback rows as a tensor)."""
        import torch
        b = logits.shape[0]
        dtype = DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_F32
        if logits.stride(1) != 1:
            raise ValueError("logits rows must be contiguous")
        W = B.sizes(self.h)[1]
        scratch = self._empty((b, W), torch.int32, logits.device, stream)
        tokens = self._empty(b, torch.int32, logits.device, stream)
        n_fb = self._empty(1, torch.int32, logits.device, stream, zero=True)
        B.domino_opportunistic_step(self.h, logits, dtype, b, logits.stride(0), states, stacks, scratch, tokens, n_fb,
                                    stream)
        return tokens, n_fb

    def mask_logits_table(self, logits, table_mask, states, want_lse: bool = True, want_logprobs: bool = False,
                          stream=None) -> Tuple:
        """Table-driven mask + decode: row b's mask is table_mask[states[b]] (DFA only)."""
        import torch
        b = logits.shape[0]
        dtype = DTYPE_BF16 if logits.dtype == torch.bfloat16 else DTYPE_F32
        if logits.stride(1) != 1:
            raise ValueError("logits rows must be contiguous")
        argmax = self._empty(b, torch.int32, logits.device, stream)
        lse = self._empty(b, torch.float32, logits.device, stream) if want_lse else None
        lp = self._empty((b, B.sizes(self.h)[0]), torch.float32, logits.device, stream) if want_logprobs else None
        B.domino_mask_logits_table(self.h, logits, dtype, b, logits.stride(0), table_mask, states, argmax, lse, lp,
                                   stream)
        return argmax, lse, lp

    def advance_table(self, table_next, states, tokens, states_out=None, stream=None):
        """Table-driven update: states_out[b] = table_next[states[b], tokens[b]] (DFA only)."""
        so = states if states_out is None else states_out
        B.domino_advance_table(self.h, table_next, states, tokens, states.shape[0], so, stream)
        return so

    # -- losses over the vocabulary, the embedding (no loaded vocabulary needed) -----
    # Their gradients are calls of their own; autograd does not see them.  Tensors that require a gradient are refused in grad
    # mode (RuntimeError): pass detach(), or call under torch.no_grad().
    def _result(self, name, r):
        if type(r) is int:
            B._check(name, r)
        return r

    def _fill(self, out, rows, cols, dtype, like, stream):
        """`out`, or with fill_byte the filled tensor that the call would otherwise make itself."""
        if out is not None or self.fill_byte is None:
            return out
        return self._empty(rows if cols is None else (rows, cols), dtype, like.device, stream)

    def _losses(self, out, like, stream):
        import torch
        loss, lse = out if out is not None else (None, None)
        if self.fill_byte is None:
            return loss, lse
        n = like.shape[0]
        return tuple(self._fill(o, n, None, torch.float32, like, stream) for o in (loss, lse))

    def token_loss(self, hidden, weight, targets, mask=None, out=None, stream=None) -> Tuple:
        """Cross entropy of `targets` under the masked softmax of hidden @ weight.T, the logits never kept: (loss,
        lse), fp32 [rows].  hidden [rows, dim], weight [n_tokens, dim] bf16; targets int32 (below 0: none); mask as
        step_mask's or None.  out: (loss, lse) to write to."""
        loss, lse = self._losses(out, hidden, stream)
        return self._result("domino_token_loss", _calls().token_loss(
            self.h, self.device, hidden, weight, targets, mask, loss, lse, None if stream is None else B._stream(stream)))

    def token_loss_grad(self, hidden, weight, targets, lse, grad_loss, mask=None, out=None, stream=None) -> Tuple:
        """(dhidden, dweight) of sum(grad_loss * loss), lse as token_loss returned it; in the inputs' type."""
        dh, dw = out if out is not None else (None, None)
        if self.fill_byte is not None:
            dh = self._fill(dh, *hidden.shape, hidden.dtype, hidden, stream)
            dw = self._fill(dw, *weight.shape, weight.dtype, weight, stream)
        return self._result("domino_token_loss_grad", _calls().token_loss_grad(
            self.h, self.device, hidden, weight, targets, lse, grad_loss, mask, dh, dw,
            None if stream is None else B._stream(stream)))

    def distill_loss(self, logits, teacher, ids, temperature: float = 1.0, mask=None, out=None, stream=None) -> Tuple:
        """Divergence of the teacher's top logits (teacher, ids [rows, k]; ids below 0: no entry) from the masked
        softmax of logits / temperature, times temperature^2: (loss, lse), fp32 [rows]."""
        loss, lse = self._losses(out, logits, stream)
        return self._result("domino_distill_loss", _calls().distill_loss(
            self.h, self.device, logits, teacher, ids, temperature, mask, loss, lse,
            None if stream is None else B._stream(stream)))

    def distill_grad(self, logits, teacher, ids, temperature: float, lse, grad_loss, mask=None, out=None, stream=None):
        """d sum(grad_loss * loss) / d logits, in the logits' type; out may be `logits` itself."""
        if self.fill_byte is not None:
            out = self._fill(out, *logits.shape, logits.dtype, logits, stream)
        return self._result("domino_distill_grad", _calls().distill_grad(
            self.h, self.device, logits, teacher, ids, temperature, lse, grad_loss, mask, out,
            None if stream is None else B._stream(stream)))

    def embed(self, tokens, weight, scale: float = 1.0, out=None, stream=None):
        """scale * weight[tokens], zeros for tokens below 0: [n, dim] of the weight's type."""
        if self.fill_byte is not None:
            out = self._fill(out, tokens.numel(), weight.shape[-1], weight.dtype, weight, stream)
        return self._result("domino_embed", _calls().embed(
            self.h, self.device, tokens, weight, scale, out, None if stream is None else B._stream(stream)))

    def embed_grad(self, tokens, grad, n_tokens: int, scale: float = 1.0, into=None, stream=None):
        """Gradient of the table [n_tokens, dim]: scale * the sums of grad's rows by token.  into: a gradient that the
        sums are added to (the loss's, for a table that is its weight too)."""
        out = into
        if self.fill_byte is not None:
            out = self._fill(into, n_tokens, grad.shape[-1], grad.dtype, grad, stream)
        return self._result("domino_embed_grad", _calls().embed_grad(
            self.h, self.device, tokens, grad, n_tokens, scale, out, into is not None,
            None if stream is None else B._stream(stream)))

    # -- norm, 8-bit operands, decode under penalties (no loaded vocabulary needed; as above, autograd does not see them) ---
    def _fill_codes(self, out, rows, cols, like, stream):
        """_fill of codes: rows on 16-byte boundaries."""
        import torch
        if out is not None or self.fill_byte is None:
            return out
        return self._empty((rows, -(-cols // 16) * 16), torch.float8_e4m3fn, like.device, stream)[:, :cols]

    def norm(self, x, weight, residual=None, eps: float = 1e-6, out=None, stream=None) -> Tuple:
        """Root-mean-square norm of x + residual: (y, sum, rstd).  x, residual [rows, dim], weight [dim], y and sum of one
        type, bf16 or fp32; rstd fp32 [rows].  Without a residual sum is x itself.  out: (y, sum, rstd) to write to; its
        sum may be x or residual."""
        y, h, rstd = out if out is not None else (None, None, None)
        if self.fill_byte is not None:
            import torch
            y = self._fill(y, *x.shape, x.dtype, x, stream)
            h = self._fill(h, *x.shape, x.dtype, x, stream) if residual is not None else h
            rstd = self._fill(rstd, x.shape[0], None, torch.float32, x, stream)
        return self._result("domino_norm", _calls().norm(
            self.h, self.device, x, weight, residual, eps, y, h, rstd, None if stream is None else B._stream(stream)))

    def norm8(self, x, weight, residual=None, eps: float = 1e-6, out=None, stream=None) -> Tuple:
        """norm with y as logits8 takes it: (codes, scales, sum).  codes float8_e4m3fn [rows, dim], its rows on 16-byte
        boundaries; scales fp32 [rows, ceil(dim / 128)]."""
        q, sc, h = out if out is not None else (None, None, None)
        if self.fill_byte is not None:
            import torch
            q = self._fill_codes(q, *x.shape, x, stream)
            sc = self._fill(sc, x.shape[0], -(-x.shape[1] // 128), torch.float32, x, stream)
            h = self._fill(h, *x.shape, x.dtype, x, stream) if residual is not None else h
        return self._result("domino_norm8", _calls().norm8(
            self.h, self.device, x, weight, residual, eps, q, sc, h, None if stream is None else B._stream(stream)))

    def norm_grad(self, sum, weight, rstd, dy, dsum=None, out=None, stream=None) -> Tuple:
        """(dx, dweight): dx the gradient of x and of the residual alike, from dy and the gradient dsum of the sum's other
        uses; sum and rstd as norm returned them.  out: (dx, dweight) to write to; its dx may be dy or dsum."""
        dx, dw = out if out is not None else (None, None)
        if self.fill_byte is not None:
            dx = self._fill(dx, *sum.shape, sum.dtype, sum, stream)
            dw = self._fill(dw, sum.shape[1], None, sum.dtype, sum, stream)
        return self._result("domino_norm_grad", _calls().norm_grad(
            self.h, self.device, sum, weight, rstd, dy, dsum, dx, dw, None if stream is None else B._stream(stream)))

    def quantize8(self, x, block: int = 1, out=None, stream=None) -> Tuple:
        """(codes, scales) of a matrix: a scale for each 1 x 128 values (block 1, hidden states) or 128 x 128 (block 128, a
        weight); see norm8."""
        q, sc = out if out is not None else (None, None)
        if self.fill_byte is not None:
            import torch
            q = self._fill_codes(q, *x.shape, x, stream)
            sc = self._fill(sc, x.shape[0] if block == 1 else -(-x.shape[0] // 128), -(-x.shape[1] // 128), torch.float32, x, stream)
        return self._result("domino_quantize8", _calls().quantize8(
            self.h, self.device, x, block, q, sc, None if stream is None else B._stream(stream)))

    def logits8(self, codes, scales, weight_codes, weight_scales, dtype=None, out=None, stream=None):
        """hidden @ weight.T of codes: [rows, n_tokens] in dtype (fp32 unless bf16 is asked for), rows on 16-byte boundaries.
        codes, scales: the hidden states', by norm8 or quantize8; weight_codes, weight_scales: by quantize8(weight, 128)."""
        if out is None and self.fill_byte is not None:
            import torch
            made = torch.float32 if dtype is None else dtype
            n, per = weight_codes.shape[0], 16 // made.itemsize
            out = self._empty((codes.shape[0], -(-n // per) * per), made, codes.device, stream)[:, :n]
        return self._result("domino_logits8", _calls().logits8(
            self.h, self.device, codes, scales, weight_codes, weight_scales, dtype, out,
            None if stream is None else B._stream(stream)))

    def mask_logits_penalized(self, logits, history=None, lengths=None, prompt_lengths=None, repetition=None, presence=None,
                              frequency=None, bias_ids=None, bias_values=None, mask=None, want_lse: bool = True,
                              want_logprobs: bool = False, out=None, stream=None) -> Tuple:
        """mask_logits of logits under penalties for what each row has said, and biases: (argmax, lse or None, logprobs or
        None).  history int32 [rows, n], the prompt's prompt_lengths tokens and then the generated ones, lengths of it in
        use (below 0: no token): a token in it has its logit divided by repetition (multiplied where it is not above 0); of
        those beyond the prompt one that occurs c times loses frequency * c + presence.  bias_values are added to the
        logits of bias_ids [rows, k] (below 0: none).  lengths, prompt_lengths int32 and the penalties fp32 [rows]; what is
        None penalises nothing.  mask as step_mask's or None.  The logits are not changed."""
        argmax, lse, lp = out if out is not None else (None, None, None)
        if self.fill_byte is not None:
            import torch
            n = logits.shape[0]
            argmax = self._fill(argmax, n, None, torch.int32, logits, stream)
            lse = self._fill(lse, n, None, torch.float32, logits, stream) if want_lse else None
            lp = self._fill(lp, *logits.shape, torch.float32, logits, stream) if want_logprobs else None
        return self._result("domino_mask_logits_penalized", _calls().mask_logits_penalized(
            self.h, self.device, logits, history, lengths, prompt_lengths, repetition, presence, frequency, bias_ids, bias_values,
            mask, argmax, None if not want_lse else True if lse is None else lse,
            None if not want_logprobs else True if lp is None else lp, None if stream is None else B._stream(stream)))

    def mask_sample_penalized(self, logits, temperature: float, seed: int, offset: int, history=None, lengths=None,
                              prompt_lengths=None, repetition=None, presence=None, frequency=None, bias_ids=None,
                              bias_values=None, mask=None, out=None, stream=None):
        """mask_sample of logits under mask_logits_penalized's penalties and biases."""
        if self.fill_byte is not None:
            import torch
            out = self._fill(out, logits.shape[0], None, torch.int32, logits, stream)
        return self._result("domino_mask_sample_penalized", _calls().mask_sample_penalized(
            self.h, self.device, logits, history, lengths, prompt_lengths, repetition, presence, frequency, bias_ids, bias_values,
            mask, temperature, seed, offset, out, None if stream is None else B._stream(stream)))

    def device_error(self, stream=None) -> int:
        return B.domino_get_device_error(self.h, stream)
