"""What the text head makes of residual rows: final RMSNorm, 8-bit vocabulary
product, log probabilities.

The stack calls end at the fp32 residual stream.  ``AnswerHead`` holds the
head's weights in 8 bits (made once from bf16 by the library's quantiser) with
the buffers of one pass, and runs the three calls over any number of rows, in
passes of ``max_rows``.  It allocates nothing and never synchronises after its
construction.  Passes share the buffers, so two calls that may overlap need a
head each (they may share the weights: ``sharing``).  Keep a head, its outputs
and its rows until the stream has passed their last call: torch does not see the
library's streams and would give their memory away.
"""
from __future__ import annotations

import dataclasses
from typing import Optional

import torch

from . import binding


@dataclasses.dataclass
class Answers:
    """Device results for a number of rows; what is None is not computed."""
    token_logprobs: Optional[torch.Tensor] = None   # fp32 [rows, n_tokens]
    entropy: Optional[torch.Tensor] = None          # fp32 [rows]
    top_logprobs: Optional[torch.Tensor] = None     # fp32 [rows, top_k]
    top_tokens: Optional[torch.Tensor] = None       # int32 [rows, top_k]


class AnswerHead:
    """gain: bf16 [hidden] of the final norm; weight: bf16 [vocab, hidden]; bias: bf16 [vocab] or None.

    weight may also be (int8 [vocab, hidden], fp32 [vocab]) as hs_quantize_rows
    made it.  logits: torch.float32, bfloat16 or float16, the type in which the
    product hands its rows on."""

    def __init__(self, ctx, gain, weight, bias=None, eps: float = 1e-6, max_rows: int = 128, top_k: int = 0,
                 logits=torch.float32):
        if max_rows < 1:
            raise ValueError(f"max_rows is {max_rows}")
        self.ctx, self.gain, self.bias, self.eps = ctx, gain, bias, eps
        self.max_rows, self.top_k = max_rows, top_k
        device = gain.device
        if isinstance(weight, tuple):
            self.w, self.w_scale = weight
        else:
            self.w = torch.empty(weight.shape, dtype=torch.int8, device=device)
            self.w_scale = torch.empty(weight.shape[0], dtype=torch.float32, device=device)
            torch.cuda.synchronize(device)
            binding.hs_quantize_rows(ctx, weight, self.w, self.w_scale)
            torch.cuda.synchronize(device)
        self.vocab, self.hidden = self.w.shape
        self.q = torch.empty((max_rows, self.hidden), dtype=torch.int8, device=device)
        self.q_scale = torch.empty(max_rows, dtype=torch.float32, device=device)
        self.logits = torch.empty((max_rows, self.vocab), dtype=logits, device=device)
        self.ws = torch.empty(max(1, binding.hs_logprobs_workspace_size(max_rows, self.vocab, top_k)),
                              dtype=torch.uint8, device=device)

    def sharing(self, max_rows: Optional[int] = None, top_k: Optional[int] = None) -> "AnswerHead":
        """A head with the same weights and buffers of its own."""
        return AnswerHead(self.ctx, self.gain, (self.w, self.w_scale), self.bias, self.eps,
                          self.max_rows if max_rows is None else max_rows, self.top_k if top_k is None else top_k,
                          self.logits.dtype)

    def outputs(self, rows: int, n_tokens: int = 0) -> Answers:
        """Buffers for `rows` rows with n_tokens given tokens each and this head's alternatives."""
        def new(*shape, dtype=torch.float32):
            return torch.empty(shape, dtype=dtype, device=self.q.device)
        out = Answers(entropy=new(rows))
        if n_tokens:
            out.token_logprobs = new(rows, n_tokens)
        if self.top_k:
            out.top_logprobs, out.top_tokens = new(rows, self.top_k), new(rows, self.top_k, dtype=torch.int32)
        return out

    def __call__(self, y, out: Answers, tokens=None, cu_budget: int = 256, stream=None) -> None:
        """y: fp32 (bf16, fp16) [rows, hidden] residual rows -> out; tokens: int32 [rows, n_tokens] or None."""
        if y.dim() != 2 or y.shape[1] != self.hidden:
            raise ValueError(f"y has shape {tuple(y.shape)}, expected (rows, {self.hidden})")
        rows = y.shape[0]
        for name, t in (("tokens", tokens), *vars(out).items()):
            if t is not None and t.shape[:1] != (rows,):
                raise ValueError(f"{name} has {t.shape[0] if t.shape else 'no'} rows, y {rows}")
        for first in range(0, rows, self.max_rows):
            part = slice(first, min(first + self.max_rows, rows))
            n = part.stop - first
            q, q_scale, z = self.q[:n], self.q_scale[:n], self.logits[:n]
            binding.hs_quantize_rows(self.ctx, y[part], q, q_scale, self.gain, self.eps, cu_budget, stream)
            binding.hs_linear_i8(self.ctx, q, q_scale, self.w, self.w_scale, z, self.bias, cu_budget, stream)
            given = {k: t[part] for k, t in vars(out).items() if t is not None}
            binding.hs_logprobs(self.ctx, z, None if tokens is None else tokens[part], cu_budget=cu_budget,
                                stream=stream, workspace=self.ws, **given)
