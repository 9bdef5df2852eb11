"""Searches as a user's program makes them, step by step, against a host's own account of every row's tokens; and steps in a captured graph."""
import math

import numpy as np
import pytest
import torch

import beam_reference as ref
from paper_2508_07101_amd import binding as cb
from paper_2508_07101_amd.beam_runner import BeamRunner, demo

pytestmark = pytest.mark.gpu
DEV = "cuda"
VOCAB, END = 3001, 7


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


class Account:
    """Every row's K and V of every layer, as the search's own history has them."""

    def __init__(self, rows, layers):
        self.kv = [[None] * rows for _ in range(layers)]         # [layer][row] -> (k [n, G, 128], v)
        self.tokens = [[] for _ in range(rows)]

    def follow(self, r, parents, tokens, granted, width):
        old, told = [list(x) for x in self.kv], [list(x) for x in self.tokens]
        for b in range(len(self.tokens)):
            g = b // width
            if granted[g]:
                src = g * width + parents[b] if parents[b] >= 0 else None
                for i in range(len(self.kv)):
                    self.kv[i][b] = None if src is None else old[i][src]
                self.tokens[b] = [] if src is None else told[src] + [tokens[b]]


def _run(H, G, width, groups, schedule, steps, n_pages, prompts, seed, samples=1.0):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    rows = groups * width
    params = cb.make_params(rows, H, G, 64, 16)
    r = BeamRunner(params, width, schedule, n_pages, 24, VOCAB, END, DEV)
    acc = Account(rows, len(schedule))

    def qkv(n):
        x = torch.randn((n, H + 2 * G, 128), generator=gen, device=DEV).to(torch.bfloat16)
        return x[:, :H], x[:, H: H + G], x[:, H + G:]

    slots = torch.empty(max(1, sum(prompts)), dtype=torch.int64, device=DEV)
    r.admit(_i32(prompts), slots)
    at = np.concatenate([[0], np.cumsum(prompts)])
    for i in range(len(schedule)):
        _, k, v = qkv(max(1, sum(prompts)))
        r.append(i, slots, k, v)
        for b in range(rows):
            g = b // width
            acc.kv[i][b] = (k[at[g]: at[g + 1]], v[at[g]: at[g + 1]])
    r.spread(_i32([1] * groups))
    assert r.lens.tolist() == [prompts[b // width] for b in range(rows)] and r.granted.tolist() == [1] * groups
    scores, ended, refused = r.scores.cpu().numpy(), np.zeros(rows, dtype=np.int64), 0
    assert all((s == 0.0) if b % width == 0 else s == -math.inf for b, s in enumerate(scores))
    for step in range(steps):
        logits = (torch.randn((rows, VOCAB), generator=gen, device=DEV) * 4 * samples).to(torch.bfloat16)
        if step == 2:
            logits[:, END] = logits.amax() + 1                   # (beams end)
        want = ref.select(logits.double().cpu().numpy(), scores, ended, width, width, END)
        print("step", step, flush=True)
        r.step(logits)
        torch.cuda.synchronize()
        parents, tokens, granted, now = r.parents.tolist(), r.tokens.tolist(), r.granted.tolist(), r.ended.tolist()
        for g, best in enumerate(want):
            got = r.scores.view(groups, width)[g].tolist()
            for j in range(width):
                v = best[j][0] if j < len(best) else -math.inf
                assert got[j] == v or abs(got[j] - v) <= 2.0 ** -17 + 2.0 ** -24 * abs(v)
        refused += granted.count(0)
        acc.follow(r, parents, tokens, granted, width)
        scores, ended = r.scores.cpu().numpy(), r.ended.cpu().numpy().copy()
        q0 = qkv(rows)[0]
        for i, kind in enumerate(schedule):
            q, k, v = qkv(rows)
            out = torch.full((rows, H, 128), 7.0, dtype=torch.bfloat16, device=DEV)
            r.layer(i, q, k, v, out)
            torch.cuda.synchronize()
            lens = r.lens.tolist()
            for b in range(rows):
                if acc.kv[i][b] is not None and granted[b // width] and not now[b]:
                    acc.kv[i][b] = tuple(torch.cat([x, y[b: b + 1]]) for x, y in zip(acc.kv[i][b], (k, v)))
                n = 0 if acc.kv[i][b] is None else len(acc.kv[i][b][0])
                assert lens[b] == n, (step, i, b)
                if n == 0:
                    assert not out[b].any()
                    continue
                kk, vv = (x.transpose(0, 1).double() for x in acc.kv[i][b])
                # what the row's table names is what its history says
                pos = torch.arange(n, device=DEV)
                page = r.pool.block_table[b].long()[pos // 16]
                assert torch.equal(r.kvs[i].k[page, :, pos % 16].transpose(0, 1).double(), kk) and torch.equal(r.kvs[i].v[page, :, pos % 16].transpose(0, 1).double(), vv)
                if kind == cb.LAYER_SPARSE:
                    own = r.idx[b, : int(r.cnt[b])].long()
                    assert len(own) == min(n, params.budget)
                    kk, vv = kk[:, own], vv[:, own]
                wanted, mass = ref.attention(q[b], kk, vv, 128 ** -0.5)
                # (weights of the sparse kernel are rounded to bf16, those of few rows are not)
                tol = (2.0 ** -7 + 2.0 ** -11) * mass + 2.0 ** -8 * wanted.abs() + 1e-30
                assert ((out[b].double() - wanted).abs() <= tol).all(), (step, i, b)
        # every page is held by rows of one group or free
        first, free = r.pool.state.tolist()
        held = {}
        table = r.pool.block_table.cpu().numpy()
        for b, n in enumerate(r.lens.tolist()):
            for j in range(ref.pages(n)):
                held.setdefault(int(table[b, j]), set()).add((b // width, j))
        assert all(len(x) == 1 for x in held.values())
        queued = [int(r.pool.ring[(first + i) % n_pages]) for i in range(free)]
        assert sorted(list(held) + queued) == list(range(n_pages))
    r.finish(_i32([1] * groups))
    torch.cuda.synchronize()
    assert r.lens.tolist() == [0] * rows and r.pool.state.tolist()[1] == n_pages
    return refused


@pytest.mark.parametrize("H,G,width,groups", [(8, 2, 4, 3), (32, 8, 3, 2), (4, 4, 1, 2), (16, 2, 12, 1)])
def test_searches(H, G, width, groups):
    schedule = [cb.LAYER_FULL, cb.LAYER_SELECT, cb.LAYER_SPARSE]
    assert _run(H, G, width, groups, schedule, 8, 400, [150, 16, 33][:groups], H + width) == 0


def test_a_search_whose_pool_runs_out():
    """A group that gets no page keeps its rows; the others go on."""
    assert 0 < _run(8, 2, 4, 3, [cb.LAYER_FULL], 6, 19, [95, 80, 31], 5) < 18


def test_a_step_in_a_graph_serves_every_step():
    """Selection, tables, copies, list and layers captured once and replayed, with the program's own work between; the same as step by step."""
    width, groups, H, G = 4, 3, 8, 2
    rows, schedule = width * groups, [cb.LAYER_FULL, cb.LAYER_FULL]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    params = cb.make_params(rows, H, G, 64, 16)
    prompts = [40, 100, 7]
    runners = [BeamRunner(params, width, schedule, 120, 12, VOCAB, END, DEV) for _ in range(2)]
    x = torch.randn((sum(prompts), 2 * G, 128), generator=gen, device=DEV).to(torch.bfloat16)
    for r in runners:
        slots = torch.empty(sum(prompts), dtype=torch.int64, device=DEV)
        r.admit(_i32(prompts), slots)
        for i in range(2):
            r.append(i, slots, x[:, :G], x[:, G:])
        r.spread(_i32([1] * groups))
    logits = torch.zeros((rows, VOCAB), dtype=torch.bfloat16, device=DEV)
    qkv = torch.zeros((2, rows, H + 2 * G, 128), dtype=torch.bfloat16, device=DEV)
    outs = [torch.zeros((2, rows, H, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]

    def step(r, out):
        r.step(logits)
        for i in range(2):
            r.layer(i, qkv[i][:, :H], qkv[i][:, H: H + G], qkv[i][:, H + G:], out[i])

    def draw():
        logits.copy_(torch.randn((rows, VOCAB), generator=gen, device=DEV) * 4)
        qkv.copy_(torch.randn(qkv.shape, generator=gen, device=DEV))

    draw()
    for r, out in zip(runners, outs):                            # (kernels are loaded before the capture)
        step(r, out)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        step(runners[1], outs[1])
    for _ in range(20):
        draw()
        step(runners[0], outs[0])
        graph.replay()
        torch.cuda.synchronize()
        a, b = runners
        for name in ("lens", "scores", "parents", "tokens", "ended", "slots", "copies", "granted"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
        assert torch.equal(a.pool.state, b.pool.state) and torch.equal(a.pool.ring, b.pool.ring) and torch.equal(outs[0], outs[1])


def test_groups_that_come_and_go():
    """A group ends and another takes its place while the others' rows share pages."""
    width, groups, H, G = 2, 3, 4, 2
    params = cb.make_params(width * groups, H, G, 64, 16)
    r = BeamRunner(params, width, [cb.LAYER_FULL], 40, 10, VOCAB, END, DEV)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    slots = torch.empty(200, dtype=torch.int64, device=DEV)
    kv = torch.randn((200, 2 * G, 128), generator=gen, device=DEV).to(torch.bfloat16)

    def admit(add):
        r.admit(_i32(add), slots)
        r.append(0, slots, kv[:, :G], kv[:, G:])
        r.spread(_i32([int(n > 0) for n in add]))

    def steps(n):
        for _ in range(n):
            r.step((torch.randn((6, VOCAB), generator=gen, device=DEV) * 4).to(torch.bfloat16))
            x = torch.randn((6, H + 2 * G, 128), generator=gen, device=DEV).to(torch.bfloat16)
            r.layer(0, x[:, :H], x[:, H: H + G], x[:, H + G:], torch.empty((6, H, 128), dtype=torch.bfloat16, device=DEV))

    admit([60, 0, 17])
    steps(5)
    before = r.lens.tolist()
    assert before[2:4] == [0, 0] and before[0] == 65
    admit([0, 30, 0])
    assert r.lens.tolist() == [before[0], before[1], 30, 30, before[4], before[5]]
    steps(3)
    r.finish(_i32([1, 0, 0]))
    steps(2)
    assert r.lens.tolist()[:2] == [0, 0] and r.parents.tolist()[:2] == [-1, -1] and r.lens.tolist()[2] == 35
    admit([90, 0, 0])
    steps(2)
    assert r.lens.tolist()[0] == 92
    r.finish(_i32([1, 1, 1]))
    torch.cuda.synchronize()
    assert sorted(int(r.pool.ring[(r.pool.state.tolist()[0] + i) % 40]) for i in range(40)) == list(range(40)) and r.pool.state.tolist()[1] == 40


def test_the_example_runs():
    lengths, ms = demo(groups=2, width=3, prompt=500, vocab=1000, steps=3)
    assert lengths == [503] * 6 and ms > 0
