"""Speculative steps as a user's program makes them: prompts, drafts, layers and accepted branches against a host's own account of every row."""
import numpy as np
import pytest
import torch

import tree_reference as ref
from paper_2508_07101_amd import binding as cb
from paper_2508_07101_amd.tree_runner import TreeRunner, demo

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("H,G,nodes", [(32, 8, 20), (8, 2, 70), (4, 4, 1)])
def test_steps_over_prompts_drafts_and_branches(H, G, nodes):
    rng = np.random.default_rng(H + nodes)
    B, schedule = 3, [cb.LAYER_FULL, cb.LAYER_SELECT, cb.LAYER_SPARSE]
    params = cb.make_params(B, H, G, 128, 32)
    r = TreeRunner(params, schedule, 200, 40, B * nodes, nodes, DEV)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(5)

    def rows(n):
        qkv = torch.randn((n, H + 2 * G, 128), generator=gen, device=DEV).to(torch.bfloat16)
        return qkv[:, :H], qkv[:, H: H + G], qkv[:, H + G:]

    prompts = [300, 0, 45]
    slots = torch.empty(sum(prompts), dtype=torch.int64, device=DEV)
    r.admit(_i32(prompts), slots)
    at = np.concatenate([[0], np.cumsum(prompts)])
    cached = []                                              # [layer][sequence] -> K, V of the tokens that stay
    for i in range(len(schedule)):
        _, k, v = rows(sum(prompts))
        r.append(i, slots, k, v)
        cached.append([[k[at[b]: at[b + 1]], v[at[b]: at[b + 1]]] for b in range(B)])
    for step in range(4):
        n = [nodes, int(rng.integers(1, nodes + 1)), 0 if step == 1 else nodes]
        parents = [[int(rng.integers(-1, j)) if j else -1 for j in range(c)] for c in n]
        start = np.concatenate([[0], np.cumsum(n)])
        base = [len(cached[0][b][0]) for b in range(B)]
        bits, depth = zip(*[ref.masks(p, cb.mask_words(nodes)) for p in parents])
        positions = r.draft(_i32(n), _i32(sum(parents, [])))
        assert positions.tolist() == [base[b] + d for b in range(B) for d in depth[b]]
        new = []
        for i, kind in enumerate(schedule):
            q, k, v = rows(sum(n))
            out = torch.full((sum(n), H, 128), 7.0, dtype=torch.bfloat16, device=DEV)
            print("step", step, "layer", i, n, flush=True)
            r.layer(i, q, k, v, out)
            torch.cuda.synchronize()
            new.append((k, v))
            for b in range(B):
                if not n[b]:
                    continue
                own = slice(start[b], start[b + 1])
                seen = torch.arange(base[b], device=DEV)
                if kind == cb.LAYER_SPARSE:
                    seen = r.idx[b, : int(r.cnt[b])].long()
                    assert len(seen) == min(base[b] + 1, params.budget) and base[b] in seen.tolist()
                    seen = seen[seen < base[b]]
                kk, vv = (torch.cat([c[seen], x[own]]).transpose(0, 1).double() for c, x in zip(cached[i][b], (k, v)))
                want, mass = ref.attention(q[own], kk, vv, len(seen), n[b], ref.allowed(bits[b], n[b]), 128 ** -0.5)
                ref.assert_attention(out[own], want, mass, f"step {step} layer {i} sequence {b}")
        path, taken = np.zeros((B, 8), dtype=np.int32), []
        for b in range(B):
            m = int(rng.integers(0, min(8, n[b]) + 1))
            path[b, :m] = np.sort(rng.choice(n[b], size=m, replace=False)) if m else 0
            taken.append(m)
            for i, (k, v) in enumerate(new):
                for j, x in enumerate((k, v)):
                    cached[i][b][j] = torch.cat([cached[i][b][j], x[start[b] + torch.as_tensor(path[b, :m].astype(np.int64), device=DEV)]])
        r.accept(_i32(path), _i32(taken))
        assert r.keep.tolist() == [a + t for a, t in zip(base, taken)]
    for i in range(len(schedule)):
        for b in range(B):
            pos = torch.arange(len(cached[i][b][0]), device=DEV)
            for x, want in zip((r.kvs[i].k, r.kvs[i].v), cached[i][b]):
                assert torch.equal(ref.cache_rows(x, r.pool.block_table, b, pos), want.transpose(0, 1).double())
    # every page is held once or free
    first, free = r.pool.state.tolist()
    held = [p for b, length in enumerate(r.lens.tolist()) for p in r.pool.block_table[b, : ref.pages(length)].tolist()]
    queued = [int(r.pool.ring[(first + i) % 200]) for i in range(free)]
    assert sorted(held + queued) == list(range(200))


def test_the_example_runs():
    lengths, ms = demo(batch=2, prompt=500, nodes=15, steps=3)
    assert lengths == [500 + 3 * 4] * 2 and ms > 0
