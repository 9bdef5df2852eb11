"""A search whose logits and K and V rows follow from what each row has read, so that two runs of it can be compared wherever one of them had to wait."""
import zlib

import numpy as np
import torch

import beam_reference as ref
import tree_reference
from paper_2508_07101_amd import binding as cb
from paper_2508_07101_amd.beam_runner import BeamRunner

VOCAB, END, H, G = 60, 7, 4, 2


def i32(v, device="cpu"):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=device)


def runner(width, groups, n_pages, device, **more):
    return BeamRunner(cb.make_params(groups * width, H, G, 64, 16), width, [cb.LAYER_FULL], n_pages, 12, VOCAB, END, device, **more)


def _number(x):
    return zlib.crc32(repr(x).encode())


def _rows(stories, device):
    """K and V rows of tokens: a number for each, that of everything up to it."""
    x = torch.tensor([_number(("kv", s)) % 251 for s in stories], dtype=torch.float32, device=device)
    return x.to(torch.bfloat16)[:, None, None].expand(-1, G, 128).contiguous()


def logits_of(stories, width, device):
    """Each row's, from its group and what it has read."""
    return torch.tensor(np.stack([np.random.default_rng(_number((b // width, s))).standard_normal(VOCAB) * 3 for b, s in enumerate(stories)]), dtype=torch.float32, device=device)


class Story:
    def __init__(self, r, prompts):
        """The prompts of groups that hold nothing come in; 0: none."""
        self.r, self.width, self.device = r, r.width, r.scores.device
        self.stories = [()] * len(r.lens)
        self.admit(prompts)

    def admit(self, prompts):
        r = self.r
        slots = torch.full((max(1, sum(prompts)),), -1, dtype=torch.int64, device=self.device)
        starts = r.admit(i32(prompts, self.device), slots).tolist()
        read = [tuple(range(i + 1)) for g, n in enumerate(prompts) for i in range(starts[g * self.width + 1] - starts[g * self.width])]
        if read:
            x = _rows(read, self.device)
            r.append(0, slots[: len(read)], x, x)
        r.spread(i32([int(n > 0) for n in prompts], self.device))
        for b in range(len(self.stories)):
            if prompts[b // self.width]:
                self.stories[b] = tuple(range(int(r.lens[b])))

    def step(self, do):
        """One step, by `do`, which takes the logits; the account goes by what the runner chose.  Groups that it was made for."""
        r = self.r
        do(logits_of(self.stories, self.width, self.device))
        parents, tokens, slots, granted = r.parents.tolist(), r.tokens.tolist(), r.slots.tolist(), r.granted.tolist()
        told = list(self.stories)
        for b, p in enumerate(parents):
            self.stories[b] = told[b // self.width * self.width + p] + ((tokens[b],) if tokens[b] >= 0 else ()) if p >= 0 else ()
        x = _rows(self.stories, self.device)
        q = torch.zeros((len(told), H, 128), dtype=torch.bfloat16, device=self.device)
        r.layer(0, q, x, x, torch.empty_like(q))
        assert all(s < 0 for b, s in enumerate(slots) if not granted[b // self.width])
        return granted

    def group(self, g):
        """All that a group's search is: scores, ends, what its rows have read and what their tables name."""
        r, rows = self.r, range(g * self.width, (g + 1) * self.width)
        lens, cached = r.lens.tolist(), []
        for b in rows:
            pos = torch.arange(lens[b], device=self.device)
            cached.append(r.kvs[0].k[r.pool.block_table[b].long()[pos // 16], :, pos % 16].float().cpu().tolist())
        return [r.scores[rows.start: rows.stop].tolist(), r.ended[rows.start: rows.stop].tolist(), [lens[b] for b in rows], [self.stories[b] for b in rows], cached]


def plain_calls(monkeypatch):
    """The runner's calls from their plain statements, on the CPU."""
    def kv_plan(held, keep, add, lens, tok_start, slots, ws, pool):
        got = tree_reference.plan(held.tolist(), keep.tolist(), add.tolist(), len(slots), pool.block_table.shape[1] * 16, pool.block_table.numpy(), pool.ring.numpy(), pool.state.tolist())
        for t, x in zip((lens, tok_start, slots, pool.block_table, pool.ring, pool.state), got):
            t.copy_(torch.as_tensor(np.asarray(x)))

    def kv_fork(pool, width, held, parents, lens, slots, copies, ws, ended, grow, granted):
        got = ref.fork(width, held.tolist(), parents.tolist(), None if ended is None else ended.tolist(), grow, pool.block_table.numpy(), pool.ring.numpy(), pool.state.tolist(),
                       pool.block_table.numpy())
        for t, x in zip((lens, slots, copies, pool.block_table, pool.ring, pool.state, granted), got):
            t.copy_(torch.as_tensor(np.asarray(x)))

    def beam_select(logits, scores, width, out_scores, parents, tokens, ws, ended=None, out_ended=None, end_token=-1):
        over = None if ended is None else ended.tolist()
        best = ref.select(logits.double().numpy(), scores.tolist(), over, width, out_scores.shape[1], end_token)
        for g, found in enumerate(best):
            for i in range(out_scores.shape[1]):
                v, b, t = found[i] if i < len(found) else (float("-inf"), -1, -1)
                out_scores[g, i], parents[g, i], tokens[g, i] = v, b, t
                if out_ended is not None:
                    out_ended[g, i] = int(b >= 0 and (over[g * width + b] != 0 or t == end_token))

    def kv_append(params, kv, slots, k_new, v_new):
        for s, k, v in zip(slots.tolist(), k_new, v_new):
            if s >= 0:
                kv.k[s // 16, :, s % 16], kv.v[s // 16, :, s % 16] = k, v

    class KvCopy:
        def __init__(self, params, kvs):
            self.kvs = kvs

        def run(self, copies):
            for kv in self.kvs:
                for f, t, n, _ in copies.tolist():
                    if n:
                        kv.k[t, :, :n], kv.v[t, :, :n] = kv.k[f, :, :n], kv.v[f, :, :n]

    for name, f in dict(kv_plan=kv_plan, kv_fork=kv_fork, beam_select=beam_select, kv_append=kv_append, KvCopy=KvCopy, shared_pages=lambda *a: None, beam_attn=lambda *a: None).items():
        monkeypatch.setattr(cb, name, f)
    monkeypatch.setattr(cb, "alloc_beam_attn_workspace", lambda *a: torch.empty(256, dtype=torch.uint8))


def waits_and_goes_on(make, step_of, rounds=24):
    """Three searches in a pool that runs out, and in one that does not: a group's i-th step that found its pages leaves what its i-th step leaves there.  make(n_pages) gives a
    runner, step_of(runner) what makes a step of the logits.  Returns how often a group had to wait."""
    width, groups, prompts = 4, 3, [30, 17, 45]
    ample = Story(make(200), prompts)
    do, want = step_of(ample.r), [[] for _ in range(groups)]
    for _ in range(rounds):
        assert ample.step(do) == [1] * groups
        for g in range(groups):
            want[g].append(ample.group(g))
    tight = Story(make(19), prompts)
    do, steps, waited, after = step_of(tight.r), [0] * groups, 0, 0
    for i in range(rounds):
        before = [tight.group(g) for g in range(groups)]
        granted = tight.step(do)
        for g in range(groups):
            rows = slice(g * width, (g + 1) * width)
            if granted[g]:
                assert i < 12 or g != 0 or tight.r.lens.tolist()[rows] == [0] * width
                if tight.r.lens.tolist()[rows] != [0] * width:
                    assert tight.group(g) == want[g][steps[g]], (i, g)
                steps[g] += 1
                after += waited > 0 and steps[g] < i + 1
            else:
                assert tight.group(g) == before[g], (i, g)
                assert tight.r.parents.tolist()[rows] == list(range(width)) and tight.r.tokens.tolist()[rows] == [-1] * width
                waited += 1
        if i == 11:                                              # one search is over: its pages are the others'
            tight.r.finish(i32([1, 0, 0], tight.device))
            for b in range(width):
                tight.stories[b] = ()
    assert after > 0                                             # (a group that had waited went on)
    return waited
