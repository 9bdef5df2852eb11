"""Page plans that give back: no new tokens at all, and few among thousands of sequences."""
import numpy as np
import pytest
import torch

import tree_reference as ref
from paper_2508_07101_amd import binding as cb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("batch", [1, 64, 1024, 1025, 3000])
@pytest.mark.parametrize("tokens", [0, 3, 5000])
def test_pages_come_back_whatever_is_asked_for(batch, tokens):
    print("plan", batch, tokens, flush=True)
    rng = np.random.default_rng(batch + tokens)
    held = rng.integers(0, 100, batch)
    keep = np.where(rng.random(batch) < 0.4, 0, np.maximum(held - rng.integers(0, 40, batch), 0))
    add = np.zeros(batch, dtype=np.int64)
    if tokens:
        add[-1], keep[-1] = 3, held[-1]
    used = [ref.pages(int(h)) for h in held]
    n_pages, max_pages = sum(used) + 4, 8
    perm = rng.permutation(n_pages)
    table = np.full((batch, max_pages), -1)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = perm[at: at + u]
        at += u
    ring = np.full(n_pages, -1)
    ring[(n_pages - 2 + np.arange(4)) % n_pages] = perm[at:]
    state = [n_pages - 2, 4]
    want = ref.plan(held, keep, add, tokens, max_pages * 16, table, ring, state)
    lens, pool = _i32(held), cb.PagePool(_i32(table), _i32(ring), _i32(state))
    start, slots = torch.zeros(batch + 1, dtype=torch.int32, device=DEV), torch.full((tokens,), 77, dtype=torch.int64, device=DEV)
    cb.kv_plan(lens, _i32(keep), _i32(add), lens, start, slots, cb.alloc_plan_workspace(batch), pool)
    torch.cuda.synchronize()
    got = (lens.tolist(), start.tolist(), slots.tolist(), pool.block_table.cpu().numpy(), pool.ring.cpu().numpy(), pool.state.tolist())
    for g, w in zip(got, want):
        assert np.array_equal(np.asarray(g), np.asarray(w))


def test_contiguous_sequences_without_new_tokens():
    held = np.arange(2000) % 90
    lens, start = _i32(held), torch.full((2001,), 5, dtype=torch.int32, device=DEV)
    cb.kv_plan(lens, _i32(held // 2), _i32([0] * 2000), lens, start, torch.empty(0, dtype=torch.int64, device=DEV), cb.alloc_plan_workspace(2000), capacity=100)
    torch.cuda.synchronize()
    assert lens.tolist() == (held // 2).tolist() and not start.any()
