"""Answering from a pruned prefill: the caches of a plan's layers and the loop's calls.

Marshalling only, as in :mod:`.binding`: the layers, the caches, the eviction and the choice of
the tokens run in the HIP library.  Embedding and output head are the caller's."""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from . import binding as mv


class Answer:
    """Tokens after a pruned prefill, one per sample and step.

    ``prefill`` runs the plan and leaves every layer's keys and values in a 4-bit cache (S rows up
    to the pruning step, the kept rows behind it); ``step`` runs the layers on one new token a
    sample, adds the attention that the cached rows get to their weights and, with a ``budget``,
    evicts every layer down to that many rows a head (positions below ``first_pos`` and the last
    ``n_recent`` ones stay).  Nothing is allocated and nothing waits on the device in a step.  A
    prefill leaves no weights: the first eviction goes by the attention of the first token alone.

    The plan's rotary table has to cover the prompt's and the answer's positions (``rope_len`` of
    S + room at least) and its context the workspace (``Context(...,
    min_bytes=Answer.workspace_bytes(...))``).  ``room``: the longest answer."""

    @staticmethod
    def workspace_bytes(B: int, S: int, D: int, H: int, F: int, room: int) -> int:
        nbytes = mv.load().mvla_decode_workspace_bytes(B, 1, D, H, F, -(-(S + room) // 32) * 32)
        if nbytes == 0:
            raise mv.MvlaError(-1, "mvla_decode_workspace_bytes")
        return nbytes

    def __init__(self, plan: mv.PrefillPlan, room: int, budget: Optional[int] = None,
                 first_pos: int = 0, n_recent: int = 0):
        assert room >= 1 and (budget is None or budget >= 1) and n_recent >= 0
        if plan.rope[0].shape[0] < plan.S + room:    # (later positions would be rotated as the last one of the table)
            raise ValueError(f"the plan's rotary table (rope_len) has {plan.rope[0].shape[0]} positions, an answer of "
                             f"{room} tokens needs {plan.S + room}")
        self.plan, self.room, self.budget = plan, room, budget
        self.first_pos, self.n_recent = first_pos, n_recent
        B, L, cfg, dev = plan.B, plan.L, plan.cfg, plan.ctx.device
        i32 = dict(dtype=torch.int32, device=dev)
        self.rows = [plan.S if l < plan.p else plan.S_kept for l in range(L)]
        # a step adds its row before it evicts, so a budget needs one row more than it keeps
        most = [r + room if budget is None else max(r, min(budget, r + room)) + 1 for r in self.rows]
        # (a step's rows are in the caches when its eviction asks for workspace: too late to refuse)
        if plan.ctx.workspace.numel() < self.workspace_bytes(B, max(most), cfg.D, cfg.H, cfg.F, 0):
            raise mv.MvlaError(-2, "Answer")
        with self._on_stream():
            self.caches = [mv.Cache4.empty(B, cfg.H, cfg.dh, m, dev) for m in most]
            self._cache_array = (mv.Cache4C * L)(*[c._c for c in self.caches])
            self.length, self._other = torch.zeros(L, B, **i32), torch.zeros(L, B, **i32)
            self._start = torch.tensor(self.rows, **i32)[:, None].expand(L, B).contiguous()
            self._recent = torch.zeros(B, **i32)
            if budget is not None:
                self._budgets = [min(budget, c.capacity) for c in self.caches]
                self._kept = [torch.empty(B, cfg.H, b, **i32) for b in self._budgets]
            self._h = [torch.empty(B, 1, cfg.D, dtype=torch.bfloat16, device=dev) for _ in range(2)]
        self._h_array = (C.c_void_p * 2)(*[t.data_ptr() for t in self._h])
        self._bound = None       # by layer, what its length cannot exceed; None before the prefill

    def _on_stream(self):
        """The context's stream, for what torch does between the library's calls on it."""
        return torch.cuda.stream(self.plan.ctx.stream)

    def prefill(self, x: torch.Tensor, pos: torch.Tensor, key_bias: Optional[torch.Tensor] = None,
                **options):
        """The plan's pruned prefill; returns the kept tokens' hidden states [B, S', D].  An action
        iteration's cold start prunes nothing and does not fit: smoothed steps count from 2."""
        if options.get("smooth_step", 0) == 1:
            raise ValueError("a cold start leaves every layer unpruned: its rows do not fit an answer's caches")
        y = self.plan.run(x, pos, key_bias, caches=self._cache_array, **options)
        with self._on_stream():
            self.length.copy_(self._start)
        self._bound = list(self.rows)
        self._taken = 0
        return y

    def step(self, x: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
        """One new token a sample: x bf16 [B, 1, D], pos int32 [B, 1] (below rope_len).  Returns the
        last layer's output [B, 1, D], which the next step overwrites."""
        plan, ctx = self.plan, self.plan.ctx
        if self._bound is None:
            raise RuntimeError("no prefill has filled the caches")
        if self._taken >= self.room:
            raise RuntimeError(f"the answer has taken its {self.room} steps")
        B = plan.B
        assert mv._dev(x, torch.bfloat16).shape == (B, 1, plan.cfg.D)
        assert mv._dev(pos, torch.int32).shape == (B, 1)
        bound = [b + 1 for b in self._bound]
        with self._on_stream():
            self.length += 1
        y = C.c_void_p()
        try:
            mv._check(mv.load().mvla_decode_step(
                ctx.handle, C.byref(plan.cfg), plan._layer_array, self._cache_array, plan.L,
                x.data_ptr(), pos.data_ptr(), B, 1, None, self.length.data_ptr(), max(bound), 1,
                self._h_array, C.byref(y)), "mvla_decode_step")
        except mv.MvlaError:
            with self._on_stream():
                self.length -= 1     # (refused before anything ran: the answer is where it was)
            raise
        self._taken += 1
        self._bound = bound
        if self.budget is not None:
            if self.n_recent:
                with self._on_stream():
                    torch.sub(pos[:, 0], self.n_recent - 1, out=self._recent)
            for l, cache in enumerate(self.caches):
                ctx.cache_evict(cache, cache, self.length[l], self._budgets[l], self.first_pos,
                                self._recent if self.n_recent else None, self._bound[l],
                                out=(self._kept[l], self._other[l]))
                self._bound[l] = min(self._bound[l], self._budgets[l])
            self.length, self._other = self._other, self.length
        return next(t for t in self._h if t.data_ptr() == y.value)
