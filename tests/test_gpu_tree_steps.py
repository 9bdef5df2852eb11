"""Steps at their edges: nothing drafted, sequences without room, empty places of the batch."""
import numpy as np
import pytest
import torch

import tree_reference as ref
from paper_2508_07101_amd import binding as cb
from paper_2508_07101_amd.tree_runner import TreeRunner

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def _rows(n, H, G, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    qkv = torch.randn((n, H + 2 * G, 128), generator=gen, device=DEV).to(torch.bfloat16)
    return qkv[:, :H], qkv[:, H: H + G], qkv[:, H + G:]


def _started(prompts, n_pages, max_pages, max_tokens, max_nodes, schedule, H=8, G=2, budget=32):
    """A runner with its prompts in, and the prompts' K and V rows by layer."""
    r = TreeRunner(cb.make_params(len(prompts), H, G, budget, 8), schedule, n_pages, max_pages, max_tokens, max_nodes, DEV)
    slots = torch.empty(sum(prompts), dtype=torch.int64, device=DEV)
    r.admit(_i32(prompts), slots)
    kept = []
    for i in range(len(schedule)):
        _, k, v = _rows(sum(prompts), H, G, 100 + i)
        r.append(i, slots, k, v)
        kept.append((k, v))
    return r, kept


def test_a_step_in_which_nothing_is_drafted():
    """Sequences only give back what the step before did not accept, then go on."""
    r, _ = _started([40, 17], 12, 6, 40, 20, [cb.LAYER_FULL, cb.LAYER_SELECT, cb.LAYER_SPARSE])
    r.draft(_i32([20, 20]), _i32([-1] + list(range(19)) + [-1] + list(range(19))))
    r.accept(_i32([[0], [0]]), _i32([1, 0]))
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    assert r.draft(_i32([0, 0]), none).numel() == 0
    q, k, v = _rows(0, 8, 2, 1)
    out = torch.empty((0, 8, 128), dtype=torch.bfloat16, device=DEV)
    for i in range(3):
        r.layer(i, q, k, v, out)
    r.accept(_i32([[0], [0]]), _i32([0, 0]))
    torch.cuda.synchronize()
    assert r.lens.tolist() == r.keep.tolist() == [41, 17] and r.tok_start.tolist() == [0, 0, 0]
    assert r.pool.state.tolist()[1] == 12 - 3 - 2
