"""Decoding with trees of drafted tokens, the calls of a step in their order: room for the trees, masks and positions, every layer's new rows and
attention, the accepted branch.  Allocation glue around the C-ABI calls, as in runner.py: no arithmetic of the method happens here.

``python -m paper_2508_07101_amd.tree_runner`` runs a few steps over drawn prompts and trees and prints what a step takes.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as cb


class TreeRunner:
    """A paged cache of several layers and the speculative steps on it.

    A step is ``draft`` (or ``room`` and ``trees``), then ``layer`` for each layer in order, then ``accept``.  Prompts come in by ``admit`` (and ``append`` for each
    layer).  Everything is enqueued on the current stream; nothing here waits for the GPU.  A sequence whose new tokens find no room has no rows:
    ``tok_start`` tells, and a caller whose pool may run out looks at it after ``draft`` (or ``admit``), before it packs the rows of q, K and V.
    Places of the batch may be empty.  A sequence ends when its entry of ``keep`` is set to 0: the next plan takes its pages back.
    """

    def __init__(self, params: cb.CusaParams, schedule: Sequence[int], n_pages: int, max_pages: int, max_tokens: int, max_nodes: int, device="cuda"):
        b, g = params.batch, params.n_kv_heads
        self.params, self.schedule, self.max_nodes = params, list(schedule), max_nodes

        def ints(*shape):
            return torch.zeros(shape, dtype=torch.int32, device=device)

        self.pool = cb.PagePool.empty(b, max_pages, n_pages, device)
        self.lens, self.keep, self.first, self.kept = ints(b), ints(b), ints(b), ints(b)   # lens: with pages and rows; keep: of these, what stays
        self.tok_start = ints(b + 1)
        self.slots = torch.full((max_tokens,), -1, dtype=torch.int64, device=device)
        self.masks = torch.zeros((max_tokens, cb.mask_words(max_nodes)), dtype=torch.int64, device=device)
        self.positions = ints(max_tokens)
        self.rows = torch.arange(max_tokens, dtype=torch.int32, device=device)
        self.idx, self.cnt = ints(b, params.budget), ints(b)
        shape, self.max_len = (n_pages, g, 16, params.head_dim), 16 * max_pages
        # zeros, not whatever memory holds: rows of a page behind a sequence's end are read as parts of tiles
        self.kvs = [cb.KvCache(torch.zeros(shape, dtype=torch.bfloat16, device=device), torch.zeros(shape, dtype=torch.bfloat16, device=device), self.lens,
                               self.max_len, self.pool.block_table) for _ in self.schedule]
        # the selection scores the tree's first node over the tokens up to it
        self.first_kvs = [cb.KvCache(kv.k, kv.v, self.first, kv.max_seq_len, kv.block_table) for kv in self.kvs]
        self.plan_ws = cb.alloc_plan_workspace(b, device)
        self.tree_ws = cb.alloc_tree_workspace(params, self.max_len, max_tokens, max_nodes, device)
        self.select_ws = cb.alloc_workspace(params, self.max_len, device) if cb.LAYER_SELECT in self.schedule else None
        self.commit = cb.KvCommit(params, self.kvs)

    def admit(self, add: torch.Tensor, slots: torch.Tensor):
        """Room for add[b] more tokens that stay (prompts, or what follows of one): slots of their rows, packed in order of the sequences."""
        cb.kv_plan(self.lens, self.keep, add, self.lens, self.tok_start, slots, self.plan_ws, self.pool)
        self.keep.copy_(self.lens)

    def append(self, layer: int, slots: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor):
        cb.kv_append(self.params, self.kvs[layer], slots, k_new, v_new)

    def room(self, nodes: torch.Tensor, n: int) -> torch.Tensor:
        """Room for nodes[b] drafted tokens of sequence b (max_nodes at most), n of all at most; what the step before did not accept goes back.  Returns tok_start: a sequence
        without room has no rows."""
        if n > self.slots.numel():
            raise ValueError(f"{n} drafted tokens, room for {self.slots.numel()}")
        cb.kv_plan(self.lens, self.keep, nodes, self.lens, self.tok_start, self.slots[:n], self.plan_ws, self.pool)
        torch.minimum(self.keep + 1, self.lens, out=self.first)
        return self.tok_start

    def trees(self, parents: torch.Tensor) -> torch.Tensor:
        """The trees of the sequences that have room, by their nodes' parents, packed as tok_start says.  Returns the positions."""
        n = parents.numel()
        cb.tree_masks(self.keep, self.tok_start, parents, self.masks[:n], self.positions[:n], self.max_nodes)
        self.tree = cb.Tree(self.tok_start, self.masks[:n], self.max_nodes)
        return self.positions[:n]

    def draft(self, nodes: torch.Tensor, parents: torch.Tensor) -> torch.Tensor:
        """room and trees in one, without a look at what was granted: the parents are packed as they were asked for, nodes[b] of sequence b, and those of
        sequences without room are left out (by torch, some 30 to 60 us of a step in which the GPU waits for the host; where nothing can be refused, and in
        a captured step, room and trees do without).  Returns the positions, packed as tok_start says (what is behind the last row is not defined)."""
        n = parents.numel()
        start = self.room(nodes, n)
        if n > 0:
            asked = nodes.clamp(min=0)
            ahead = asked.cumsum(0, dtype=torch.int32) - asked - start[:-1]       # rows of sequences without room before each one's own
            rows = self.rows[:n]
            own = torch.searchsorted(start[1:], rows, right=True, out_int32=True).clamp(max=len(ahead) - 1)
            parents = parents[(rows + ahead[own]).clamp(max=n - 1)]
        return self.trees(parents)

    def layer(self, layer: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, out: torch.Tensor):
        """The nodes' rows into the layer's cache, and their attention: over the whole prefix, or in a sparse layer over what the last selection
        layer chose for the trees' first nodes."""
        kv, kind = self.kvs[layer], self.schedule[layer]
        if q.shape[0] == 0:
            return
        cb.kv_append(self.params, kv, self.slots[: q.shape[0]], k_new, v_new)
        if kind == cb.LAYER_SELECT:
            rows = self.tok_start[:-1].clamp(max=q.shape[0] - 1)
            cb.select(self.params, q[rows].contiguous(), self.first_kvs[layer], self.idx, self.cnt, self.select_ws)
        sparse = kind == cb.LAYER_SPARSE
        cb.tree_attn(self.params, q, kv, self.tree, out, self.tree_ws, self.idx if sparse else None, self.cnt if sparse else None)

    def accept(self, path: torch.Tensor, n_path: torch.Tensor):
        """The accepted nodes of each tree, ascending (path [batch, most], n_path of them): their rows move together in all layers.  A sequence that had no
        room has no nodes to accept, whatever n_path says: behind its tokens, its table names pages that may be another one's by now."""
        self.commit.run(self.keep, path, torch.minimum(n_path, self.lens - self.keep), self.kept)
        self.keep.copy_(self.kept)


def demo(batch: int = 4, prompt: int = 4000, nodes: int = 32, steps: int = 8, device: Optional[str] = "cuda"):
    """Drawn prompts, trees and accepted branches; returns the sequences' final lengths and the milliseconds of a step."""
    params = cb.make_params(batch, 32, 8, 1024, 256)
    schedule = [cb.LAYER_FULL, cb.LAYER_SELECT] + [cb.LAYER_SPARSE] * 6
    max_pages = (prompt + nodes * (steps + 1)) // 16 + 2
    r = TreeRunner(params, schedule, batch * max_pages, max_pages, batch * nodes, nodes, device)
    gen = torch.Generator(device=device)
    gen.manual_seed(1)

    def rows(n):
        qkv = torch.randn((n, 48, 128), generator=gen, device=device).to(torch.bfloat16)   # a fused projection's
        return qkv[:, :32], qkv[:, 32:40], qkv[:, 40:]

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=device)

    slots = torch.empty(batch * prompt, dtype=torch.int64, device=device)
    r.admit(ints([prompt] * batch), slots)
    for i in range(len(schedule)):
        _, k, v = rows(batch * prompt)
        r.append(i, slots, k, v)
    parents = ints(([-1] + [(j - 1) // 2 for j in range(1, nodes)]) * batch)     # two candidates behind each node
    branch = [0]
    while 2 * branch[-1] + 2 < nodes:
        branch.append(2 * branch[-1] + 2)
    path, taken, most = ints([branch] * batch), ints([len(branch)] * batch), ints([nodes] * batch)
    q, k, v = rows(batch * nodes)
    out = torch.empty((batch * nodes, 32, 128), dtype=torch.bfloat16, device=device)
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for step in range(steps):
        if step == 1:                                                            # (the first one loads the kernels)
            start.record()
        r.room(most, len(parents))                                               # (there are pages for all steps: nothing is refused)
        r.trees(parents)
        for i in range(len(schedule)):
            r.layer(i, q, k, v, out)
        r.accept(path, taken)
    stop.record()
    torch.cuda.synchronize()
    return r.keep.tolist(), start.elapsed_time(stop) / max(steps - 1, 1)


if __name__ == "__main__":
    lengths, ms = demo()
    print(f"sequences of {lengths} tokens after 8 steps, {ms:.3f} ms a step of 8 layers")
