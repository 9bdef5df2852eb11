"""Beam search over paged caches, the calls of a step in their order: the best continuations, block tables and pages, every layer's new rows and attention.
Allocation glue around the C-ABI calls, as in runner.py: no arithmetic of the method happens here.

``python -m paper_2508_07101_amd.beam_runner`` runs a few steps over drawn prompts and logits and prints what a step takes.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as cb


class BeamRunner:
    """A paged cache of several layers, shared by groups of ``width`` rows each, and the steps of a search on it.

    A prompt comes in by ``admit``, ``append`` for each layer, and ``spread``.  A step is ``select`` from the last tokens' logits and ``fork`` (or ``step``, which is both), then
    ``layer`` for each layer in order.  ``parents`` and ``tokens`` are what ``select`` chose, for the caller's own account; ``scores`` and ``ended`` belong to the rows as they are now.
    Everything is enqueued on the current stream; nothing here waits for the GPU.  A row that has ended keeps its tokens and gets no new one (its slot is -1).
    A group that found no page keeps its rows (``granted`` is 0).  With ``hold`` it keeps all that belongs to them: ``fork`` puts its scores and ends back, its ``parents`` are
    the rows themselves and its ``tokens`` -1, so that the same logits make the same choice in a later step, which finds pages or waits again (for ever with rows of ``16 * max_pages`` tokens); a caller's account that follows
    ``parents`` and ``tokens`` is right either way, and a captured step needs no host in between.  That is what a pool that may run out wants.  Without it ``scores``, ``ended``,
    ``parents`` and ``tokens`` of such a group are the chosen ones', which its rows do not have: it can be finished, but a further step would go on from scores of other rows.
    ``finish`` gives the pages of whole groups back.
    """

    def __init__(self, params: cb.CusaParams, width: int, schedule: Sequence[int], n_pages: int, max_pages: int, vocab: int, end_token: int = -1, device="cuda",
                 hold: bool = False):
        b, g = params.batch, params.n_kv_heads
        self.params, self.width, self.schedule, self.end_token, self.n_pages, self.hold = params, width, list(schedule), end_token, n_pages, hold

        def ints(*shape):
            return torch.zeros(shape, dtype=torch.int32, device=device)

        self.pool = cb.PagePool.empty(b, max_pages, n_pages, device)
        self.lens, self.kept, self.parents, self.tokens, self.ended, self.granted = ints(b), ints(b), ints(b), ints(b), ints(b), ints(b // width)
        self.scores = torch.full((b,), float("-inf"), device=device)
        self.old_scores, self.old_ended, self.none = torch.empty_like(self.scores), ints(b), ints(b) - 1     # (with hold: before the choice)
        self.slots = torch.full((b,), -1, dtype=torch.int64, device=device)
        self.copies, self.tok_start = ints(b, 4), ints(b + 1)
        self.own = torch.arange(b, dtype=torch.int32, device=device) % width     # every row its own parent
        self.first = (self.own == 0).to(torch.int32)
        self.idx, self.cnt = ints(b, params.budget), ints(b)
        shape, self.max_len = (n_pages, g, 16, params.head_dim), 16 * max_pages
        # zeros, not whatever memory holds: rows of a page behind a sequence's end are read as parts of tiles
        self.kvs = [cb.KvCache(torch.zeros(shape, dtype=torch.bfloat16, device=device), torch.zeros(shape, dtype=torch.bfloat16, device=device), self.lens,
                               self.max_len, self.pool.block_table) for _ in self.schedule]
        self.shared = cb.SharedPages.empty(b, width, self.max_len, n_pages, device)
        self.plan_ws, self.fork_ws = cb.alloc_plan_workspace(b, device), cb.alloc_fork_workspace(self.pool)
        self.pages_ws = cb.alloc_pages_workspace(b, self.max_len, device)
        self.beam_ws = cb.alloc_beam_workspace(b, vocab, width, device)
        self.attn_ws = cb.alloc_beam_attn_workspace(params, self.max_len, self.shared, device)
        self.select_ws = cb.alloc_workspace(params, self.max_len, device) if cb.LAYER_SELECT in self.schedule or cb.LAYER_SPARSE in self.schedule else None
        self.copy = cb.KvCopy(params, self.kvs)

    def admit(self, add: torch.Tensor, slots: torch.Tensor):
        """Room for the prompts of groups that hold nothing: add[g] tokens of group g, 0 for the others; slots of their rows, packed in order of the groups.  Returns tok_start,
        by rows of the batch: a group without room has no rows."""
        prompts = torch.zeros_like(self.lens)
        prompts[:: self.width] = add
        self.kept.copy_(self.lens)
        cb.kv_plan(self.lens, self.kept, prompts, self.lens, self.tok_start, slots, self.plan_ws, self.pool)
        return self.tok_start

    def append(self, layer: int, slots: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor):
        cb.kv_append(self.params, self.kvs[layer], slots, k_new, v_new)

    def spread(self, new: torch.Tensor):
        """The admitted prompts become those of all rows of their groups; new: int32 or bool [groups], which groups these are.  Their search starts with one beam:
        the first selection takes its continuations from the logits of the group's first row.  A group whose prompt found no room has no tokens and stays as it was."""
        new = (new != 0) & (self.lens[:: self.width] > 0)
        rows = new.to(torch.int32).repeat_interleave(self.width)
        self._fork(torch.where(rows != 0, torch.zeros_like(self.own), self.own), None, False)
        start = torch.where(self.first != 0, torch.zeros_like(self.scores), torch.full_like(self.scores, float("-inf")))
        self.scores.copy_(torch.where(rows != 0, start, self.scores))
        self.ended.copy_(torch.where(rows != 0, torch.zeros_like(self.ended), self.ended))

    def select(self, logits: torch.Tensor):
        """The width best continuations of every group: parents, tokens, and the rows' next scores and ends.  logits [rows, vocab]."""
        shape = (self.params.batch // self.width, self.width)
        ended = self.ended if self.end_token >= 0 else None
        if self.hold:
            self.old_scores.copy_(self.scores)
            self.old_ended.copy_(self.ended)
        cb.beam_select(logits, self.scores, self.width, self.scores.view(shape), self.parents.view(shape), self.tokens.view(shape), self.beam_ws, ended,
                       None if ended is None else ended.view(shape), self.end_token)

    def fork(self):
        """The caches follow the choice: tables by parents, a slot for every row's token, pages that two rows would write to copied in all layers, and
        the list of pages that the layers' attention goes by."""
        self._fork(self.parents, self.ended, True)
        if self.hold:
            refused = self.granted.view(-1, 1) == 0
            for now, old in ((self.scores, self.old_scores), (self.ended, self.old_ended), (self.parents, self.own), (self.tokens, self.none)):
                now, old = now.view(-1, self.width), old.view(-1, self.width)
                now.copy_(torch.where(refused, old, now))
        self.copy.run(self.copies)
        self.list_pages()

    def step(self, logits: torch.Tensor):
        self.select(logits)
        self.fork()

    def list_pages(self):
        cb.shared_pages(self.pool.block_table, self.lens, self.max_len, self.n_pages, self.shared, self.pages_ws)

    def layer(self, layer: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, out: torch.Tensor):
        """The rows' new tokens into the layer's cache, and their attention: q [rows, H, 128], k_new and v_new [rows, G, 128]; in a sparse layer over what the last selection
        layer chose for each row."""
        kv, kind = self.kvs[layer], self.schedule[layer]
        cb.kv_append(self.params, kv, self.slots, k_new, v_new)
        if kind == cb.LAYER_SELECT:
            cb.select(self.params, q.contiguous(), kv, self.idx, self.cnt, self.select_ws)
        if kind == cb.LAYER_SPARSE:
            cb.sparse_attn(self.params, q.contiguous(), kv, self.idx, self.cnt, out, self.select_ws)
        else:
            cb.beam_attn(self.params, q, kv, self.shared, out, self.attn_ws)

    def finish(self, over: torch.Tensor):
        """The pages of groups go back; over: int32 or bool [groups]."""
        rows = over.to(torch.int32).repeat_interleave(self.width)
        self._fork(torch.where(rows != 0, torch.full_like(self.own, -1), self.own), None, False)
        self.scores.copy_(torch.where(rows != 0, torch.full_like(self.scores, float("-inf")), self.scores))

    def _fork(self, parents, ended, grow):
        cb.kv_fork(self.pool, self.width, self.lens, parents, self.lens, self.slots, self.copies, self.fork_ws, ended, grow, granted=self.granted)


def demo(groups: int = 4, width: int = 4, prompt: int = 4000, vocab: int = 32000, steps: int = 8, device: Optional[str] = "cuda"):
    """Drawn prompts and logits; returns the rows' final lengths and the milliseconds of a step."""
    rows = groups * width
    params = cb.make_params(rows, 32, 8, 1024, 256)
    schedule = [cb.LAYER_FULL, cb.LAYER_SELECT] + [cb.LAYER_SPARSE] * 6
    max_pages = (prompt + steps) // 16 + 2
    r = BeamRunner(params, width, schedule, groups * max_pages + rows * (steps // 16 + 3), max_pages, vocab, device=device)
    gen = torch.Generator(device=device)
    gen.manual_seed(1)

    def qkv(n):
        x = torch.randn((n, 48, 128), generator=gen, device=device).to(torch.bfloat16)     # a fused projection's
        return x[:, :32], x[:, 32:40], x[:, 40:]

    slots = torch.empty(groups * prompt, dtype=torch.int64, device=device)
    r.admit(torch.full((groups,), prompt, dtype=torch.int32, device=device), slots)
    for i in range(len(schedule)):
        _, k, v = qkv(groups * prompt)
        r.append(i, slots, k, v)
    r.spread(torch.ones(groups, dtype=torch.int32, device=device))
    q, k, v = qkv(rows)
    out = torch.empty((rows, 32, 128), dtype=torch.bfloat16, device=device)
    logits = (torch.randn((rows, vocab), generator=gen, device=device) * 3).to(torch.bfloat16)
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for step in range(steps):
        if step == 1:                                                            # (the first one loads the kernels)
            start.record()
        r.step(logits)
        for i in range(len(schedule)):
            r.layer(i, q, k, v, out)
    stop.record()
    torch.cuda.synchronize()
    return r.lens.tolist(), start.elapsed_time(stop) / max(steps - 1, 1)


if __name__ == "__main__":
    lengths, ms = demo()
    print(f"rows of {lengths} tokens after 8 steps, {ms:.3f} ms a step of 8 layers")
