"""Beam search over a paged cache whose beams share what they have in common.

``BeamSearch`` prefills the prompts, one sequence each, and lets every request's beams
list the prompt's pages.  A step reserves a position for each beam (the partly filled
last page of beams that share it is copied), decodes all beams behind their shared
prefix, takes the head's logits and selects the best continuations of every request;
then each beam takes the pages of its parent.  The selection and the decoding run on
the device, the pages' bookkeeping on the host, which reads the selection back
once a step.

A beam that has ended, or stands for no continuation, stays in the batch while any other
goes on; it proposes its own score, or nothing, and takes a position a step like the others.
"""
from __future__ import annotations

import dataclasses
from typing import Callable, List

import numpy as np
import torch

from . import binding
from .answer import AnswerHead
from .device_data import DeviceCache


@dataclasses.dataclass
class Beam:
    tokens: List[int]    # the continuation, its end token included
    score: float         # its log probability; -inf: there is none
    finished: bool


class BeamSearch:
    """shape, weights: the stack as for the decode step; head: an AnswerHead of at least groups * beams rows.

    embed(tokens, out): writes the bf16 rows of int32 tokens into out, on torch's current stream.
    max_groups prompts of at most max_prompt positions in all their rows, max_new steps.
    The search runs on `stream` (default: the context's SHARED stream of cu_budget); calls must not overlap."""

    def __init__(self, ctx, shape, weights, head: AnswerHead, embed: Callable, beams: int, max_groups: int,
                 max_prompt: int, max_new: int, end_token: int = -1, page: int = 64, n_pages: int = 0,
                 cu_budget: int = 256, stream=None):
        if not 1 <= beams <= 64:
            raise ValueError(f"{beams} beams, expected 1 to 64")
        if max_groups < 1 or max_prompt < 1 or max_new < 1:
            raise ValueError(f"{max_groups} groups, prompts of {max_prompt}, {max_new} steps")
        if head.max_rows < max_groups * beams:
            raise ValueError(f"the head takes {head.max_rows} rows, {max_groups * beams} needed")
        self.ctx, self.shape, self.weights, self.head, self.embed = ctx, shape, weights, head, embed
        self.beams, self.max_groups, self.max_prompt, self.max_new = beams, max_groups, max_prompt, max_new
        self.end_token, self.cu_budget = end_token, cu_budget
        self.stream = binding.hs_context_stream(ctx, cu_budget) if stream is None else stream
        rows, n_layers = max_groups * beams, len(weights)
        self.max_pos = max_prompt + max_new
        per_seq = -(-self.max_pos // page)
        self.pages = binding.Pages(n_pages or rows * per_seq, page, rows, per_seq)
        device = head.q.device
        self.torch_stream = torch.cuda.ExternalStream(self.stream, device=device)
        self.cache = DeviceCache(n_layers, n_pages or rows * per_seq, page, shape.n_kv_heads, shape.head_dim, device)

        def new(*size, dtype=torch.float32, pinned=False):
            return torch.empty(size, dtype=dtype, device=None if pinned else device, pin_memory=pinned)
        self.x = new(rows, shape.hidden, dtype=torch.bfloat16)
        self.y = new(max(rows, max_groups * max_prompt), shape.hidden)
        self.last = new(max_groups, shape.hidden)
        self.scores = [new(max_groups, beams) for _ in range(2)]
        # What a selection leaves, and where the host reads it: parents, tokens, and finished flags of two steps.
        self.left, self.left_host = (new(10 * rows, dtype=torch.uint8, pinned=p) for p in (False, True))

        def parts(left):
            ints = left[:8 * rows].view(torch.int32).view(2, max_groups, beams)
            return ints[0], ints[1], list(left[8 * rows:].view(2, max_groups, beams))
        self.parents, self.tokens, self.finished = parts(self.left)
        self.host = parts(self.left_host)
        self.zero = torch.zeros((max_groups, 1), device=device)
        self.ws = new(max(binding.hs_workspace_size_paged(shape, max_groups * max_prompt, max_groups, self.max_pos, page),
                          binding.hs_workspace_size_prefix(shape, rows, self.max_pos, page, self.max_pos, self.max_pos)),
                      dtype=torch.uint8)
        self.select_ws = new(max(binding.hs_beam_select_workspace_size(max_groups, beams, head.vocab, beams),
                                 binding.hs_beam_select_workspace_size(max_groups, 1, head.vocab, beams)),
                             dtype=torch.uint8)
        self.groups, self.ready = 0, False  # ready: the pages hold what the history says, and no more
        self.steps, self.at, self.history = 0, 0, []
        torch.cuda.synchronize(device)

    def _kv(self, table):
        return (*self.cache.as_arg(), table)

    def _seqs(self, g: int) -> List[int]:
        return list(range(g * self.beams, (g + 1) * self.beams))

    def start(self, x, offsets) -> None:
        """x: bf16 [T, hidden] prompt rows on the device, as torch's current stream leaves them; offsets: host
        [groups + 1], no prompt empty.  Ends the search before and selects every group's first tokens."""
        groups = len(offsets) - 1
        lengths = [int(b) - int(a) for a, b in zip(offsets, offsets[1:])]
        if not 1 <= groups <= self.max_groups or min(lengths) < 1 or max(lengths) > self.max_prompt:
            raise ValueError(f"prompts of {lengths} positions: 1 to {self.max_groups} of 1 to {self.max_prompt}")
        if x.shape != (int(offsets[-1]), self.shape.hidden) or int(offsets[0]) != 0:
            raise ValueError(f"x has shape {tuple(x.shape)}, the offsets end at {int(offsets[-1])}")
        if x.dtype != torch.bfloat16 or x.device != self.x.device or not x.is_contiguous():
            raise ValueError(f"x is {x.dtype} on {x.device} with strides {x.stride()}: contiguous bfloat16 rows on "
                             f"{self.x.device} expected")
        self.torch_stream.wait_stream(torch.cuda.current_stream(x.device))
        self.groups, self.ready = 0, False
        self.pages.release(list(range(self.max_groups * self.beams)))
        self.steps, self.at = 0, 0
        firsts = [g * self.beams for g in range(groups)]
        self.pages.reserve(firsts, lengths)
        table, _ = self.pages.table(firsts)
        y = self.y[:x.shape[0]]
        binding.hs_shared_stage_forward(self.ctx, self.shape, self.weights, x, y, offsets, [0] * groups,
                                        self._kv(table), self.cu_budget, self.stream, self.ws)
        with torch.cuda.stream(self.torch_stream):
            for g in range(groups):
                self.last[g].copy_(y[int(offsets[g + 1]) - 1])
        self.history = [[[] for _ in range(self.beams)] for _ in range(groups)]
        z = self.head.product(self.last[:groups], self.cu_budget, self.stream)
        self._select(z, self.zero[:groups], None)
        # Every beam starts from its prompt.
        for g in range(groups):
            self.pages.fork(self._seqs(g), [g * self.beams] * self.beams)
        self.groups, self.ready = groups, True

    def step(self) -> bool:
        """One more token for every beam; False once each of them has ended or stands for no continuation, or
        max_new tokens are there.

        A step that runs out of pages changes nothing; after any other failure the results stay and the
        search cannot go on."""
        if not self.ready:
            raise ValueError("no search has been started, or its last step failed")
        if self.steps >= self.max_new or not self._goes_on():
            return False
        n = self.groups * self.beams
        seqs = list(range(n))
        copies = self.pages.reserve(seqs, [1] * n)
        self.ready = False
        if copies[0]:
            binding.hs_cache_copy(self.ctx, self.cache.as_arg(), *copies, cu_budget=self.cu_budget, stream=self.stream)
        table, lens = self.pages.table(seqs)
        kv_lens = lens - 1
        prefix = [min(self.pages.shared(self._seqs(g)), int(kv_lens[self._seqs(g)].min())) for g in range(self.groups)]
        x, y = self.x[:n], self.y[:n]
        with torch.cuda.stream(self.torch_stream):
            # (Where there is no continuation any token will do.)
            self.embed(self.tokens[:self.groups].view(n).clamp(min=0), x)
        binding.hs_downstream_decode_step_prefix(
            self.ctx, self.shape, self.weights, x, y, self._kv(table), kv_lens,
            [g * self.beams for g in range(self.groups + 1)], prefix, self.cu_budget, self.stream, self.ws)
        z = self.head.product(y, self.cu_budget, self.stream)
        parents = self._select(z, self.scores[self.at][:self.groups], self.finished[self.at][:self.groups])
        for g in range(self.groups):
            first = g * self.beams
            self.pages.fork(self._seqs(g), [first + max(int(p), 0) for p in parents[g]])
        self.ready = True
        return True

    def _goes_on(self) -> bool:
        """Whether any beam of the last selection proposes something new."""
        parents, _, finished = self.host
        return bool(((parents[:self.groups] >= 0) & (finished[self.at][:self.groups] == 0)).any())

    def _select(self, z, scores, finished) -> np.ndarray:
        """The best continuations into the other buffers; their parents, and everything else, on the host too."""
        g, to = scores.shape[0], 1 - self.at
        binding.hs_beam_select(
            self.ctx, z, scores, self.scores[to][:g], self.parents[:g], self.tokens[:g],
            finished=finished if self.end_token >= 0 else None, out_finished=self.finished[to][:g],
            end_token=self.end_token, cu_budget=self.cu_budget, stream=self.stream, workspace=self.select_ws)
        # A copy that is waited for: torch remembers the stream of any other until the pinned memory is given back,
        # and by then the context may have closed it.
        with torch.cuda.stream(self.torch_stream):
            self.left_host.copy_(self.left)
        parents, tokens = (h[:g].numpy() for h in self.host[:2])
        self.history = [[self._continued(i, int(parents[i, j]), int(tokens[i, j])) for j in range(self.beams)]
                        for i in range(g)]
        self.at, self.steps = to, self.steps + 1
        return parents

    def _continued(self, group: int, parent: int, token: int) -> List[int]:
        if parent < 0:
            return []
        before = self.history[group][parent]
        ended = bool(before) and before[-1] == self.end_token
        return before if ended else before + [token]

    def results(self) -> List[List[Beam]]:
        """Every group's beams, best first; no groups before a start and after one that failed."""
        self.torch_stream.synchronize()
        scores = self.scores[self.at][:self.groups].cpu().numpy()
        finished = self.host[2][self.at][:self.groups].numpy()
        return [[Beam(list(self.history[g][j]), float(scores[g, j]), bool(finished[g, j])) for j in range(self.beams)]
                for g in range(self.groups)]
