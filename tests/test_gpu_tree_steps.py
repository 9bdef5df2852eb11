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


@pytest.mark.parametrize("split", [False, True])
def test_trees_of_the_others_where_one_finds_no_room(split):
    """Sequences of 16, 17, 0 and 33 tokens ask for 64, 3, 0 and 15 nodes with two free pages: the first is refused, the others need none.  The parents
    are packed as they were asked for (draft), or as they were granted (room, then trees)."""
    H, G, schedule = 8, 2, [cb.LAYER_FULL, cb.LAYER_SELECT, cb.LAYER_SPARSE]
    prompts, asked = [16, 17, 0, 33], [64, 3, 0, 15]
    r, kept = _started(prompts, 1 + 2 + 3 + 2, 8, 100, 64, schedule)
    rng = np.random.default_rng(2)
    parents = [[int(rng.integers(-1, j)) if j else -1 for j in range(n)] for n in asked]
    granted = [0, 3, 0, 15]
    if split:
        assert r.room(_i32(asked), sum(asked)).tolist() == [0, 0, 3, 3, 18]
        positions = r.trees(_i32(parents[1] + parents[3]))
    else:
        positions = r.draft(_i32(asked), _i32(sum(parents, [])))
    assert r.tok_start.tolist() == [0, 0, 3, 3, 18] and r.lens.tolist() == [16, 20, 0, 48]
    bits, depth = zip(*[ref.masks(p, 1) for p in parents])
    assert positions[:18].tolist() == [17 + d for d in depth[1]] + [33 + d for d in depth[3]]
    assert r.masks[:18].cpu().numpy().view(np.uint64).tolist() == np.concatenate([bits[1], bits[3]]).tolist()
    q, k, v = _rows(18, H, G, 7)
    at = np.concatenate([[0], np.cumsum(prompts)])
    for i, kind in enumerate(schedule):
        out = torch.full((18, H, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        r.layer(i, q, k, v, out)
        torch.cuda.synchronize()
        for b, own in ((1, slice(0, 3)), (3, slice(3, 18))):
            old = [x[at[b]: at[b + 1]] for x in kept[i]]
            seen = torch.arange(prompts[b], device=DEV)
            if kind == cb.LAYER_SPARSE:
                seen = r.idx[b, : int(r.cnt[b])].long()
                seen = seen[seen < prompts[b]]
            kk, vv = (torch.cat([c[seen], x[own]]).transpose(0, 1).double() for c, x in zip(old, (k, v)))
            want, mass = ref.attention(q[own], kk, vv, len(seen), granted[b], ref.allowed(bits[b], granted[b]), 128 ** -0.5)
            ref.assert_attention(out[own], want, mass, f"layer {i} sequence {b}")


def test_more_nodes_than_the_runner_has_rows_for_change_nothing():
    r, _ = _started([16, 17], 8, 8, 10, 64, [cb.LAYER_FULL])
    state = r.pool.state.tolist()
    with pytest.raises(ValueError, match="room for 10"):
        r.draft(_i32([6, 6]), _i32([-1] * 12))
    assert r.pool.state.tolist() == state and r.lens.tolist() == [16, 17]


def test_a_sequence_without_room_accepts_nothing():
    """The second sequence gives its two pages back, the first one gets them, the second one is refused and accepts three nodes all the same: its table
    still names the pages, and the first one's rows in them stay as they are."""
    r, _ = _started([16, 16], 4, 8, 100, 64, [cb.LAYER_FULL, cb.LAYER_FULL])
    chain = list(range(-1, 63))
    r.draft(_i32([0, 20]), _i32(chain[:20]))
    r.accept(_i32([[0], [0]]), _i32([0, 0]))
    r.draft(_i32([0, 0]), torch.empty(0, dtype=torch.int32, device=DEV))
    r.draft(_i32([20, 64]), _i32(chain[:20] + chain))
    assert r.tok_start.tolist() == [0, 20, 20] and r.pool.block_table[0, 1:3].tolist() == r.pool.block_table[1, 1:3].tolist()
    new = [_rows(20, 8, 2, 50 + i)[1:] for i in range(2)]
    before = []
    for i, (k, v) in enumerate(new):
        r.append(i, r.slots[:20], k, v)
        before.append((r.kvs[i].k.clone(), r.kvs[i].v.clone()))
    r.accept(_i32([[1, 4, 0], [3, 4, 5]]), _i32([2, 3]))
    torch.cuda.synchronize()
    page = int(r.pool.block_table[0, 1])
    for kv, new_rows, old in zip(r.kvs, new, before):
        for x, rows, want in zip((kv.k, kv.v), new_rows, old):
            want[page, :, 0], want[page, :, 1] = rows[1], rows[4]
            assert torch.equal(x, want)
    assert r.keep.tolist() == [18, 16]
    # and the next steps start from there (the page that the first one gives back comes to the second one a call later)
    assert r.draft(_i32([3, 2]), _i32([-1, 0, 1, -1, 0]))[:3].tolist() == [18, 19, 20] and r.tok_start.tolist() == [0, 3, 3]
    r.accept(_i32([[0], [0]]), _i32([0, 1]))
    assert r.draft(_i32([3, 2]), _i32([-1, 0, 1, -1, 0])).tolist() == [18, 19, 20, 16, 17]


@pytest.mark.parametrize("mode", [cb.RANK_FIRST_OCCURRENCE, cb.RANK_VOTES, cb.RANK_MAX_SCORE])
@pytest.mark.parametrize("bound", [64, 4096, 200000])
def test_selection_over_empty_places(mode, bound):
    """Sequences of no tokens, without pages, among others: an empty set, and the others' sets as on their own."""
    B, H, G, lens = 5, 8, 2, [0, 300, 0, 20, 0] if bound > 64 else [0, 30, 0, 20, 0]
    pages = [ref.pages(n) for n in lens]
    table = np.full((B, ref.pages(bound)), -1)
    for b, n in enumerate(pages):
        table[b, :n] = sum(pages[:b]) + np.arange(n)
    k, v = (torch.randn((sum(pages), G, 16, 128), device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((B, H, 128), device=DEV).to(torch.bfloat16)
    sets = []
    for own in ([0, 1, 2, 3, 4], [1, 3]):
        params = cb.make_params(len(own), H, G, 64, 16, rank_mode=mode)
        idx, cnt = torch.full((len(own), 64), -7, dtype=torch.int32, device=DEV), torch.full((len(own),), -7, dtype=torch.int32, device=DEV)
        kv = cb.KvCache(k, v, _i32([lens[b] for b in own]), bound, _i32(table[own]))
        print("select", mode, bound, own, flush=True)
        cb.select(params, q[own].contiguous(), kv, idx, cnt, cb.alloc_workspace(params, bound))
        torch.cuda.synchronize()
        sets.append((idx.tolist(), cnt.tolist()))
    assert sets[0][1] == [0, min(lens[1], 64), 0, 20, 0] and sets[1][1] == [min(lens[1], 64), 20]
    for i, b in enumerate((1, 3)):
        assert sets[0][0][b][: sets[0][1][b]] == sets[1][0][i][: sets[1][1][i]]
    assert all(t == -7 for b in (0, 2, 4) for t in sets[0][0][b])


def test_a_sequence_ends_and_another_takes_its_place():
    """Empty places before, beside and after: through all kinds of layers, and every page comes back."""
    schedule = [cb.LAYER_FULL, cb.LAYER_SELECT, cb.LAYER_SPARSE]
    r, kept = _started([0, 50, 40], 12, 6, 40, 20, schedule)
    for step, (asked, held) in enumerate([([0, 4, 3], [0, 50, 40]), ([0, 0, 3], [0, 0, 40]), ([0, 0, 0], [0, 0, 0]), ([2, 0, 0], [30, 0, 0])]):
        if step == 1:
            r.keep[1] = 0
        if step == 2:
            r.keep[2] = 0
        if step == 3:
            slots = torch.empty(30, dtype=torch.int64, device=DEV)
            r.admit(_i32([30, 0, 0]), slots)
            kept = []
            for i in range(3):
                _, k, v = _rows(30, 8, 2, 70 + i)
                r.append(i, slots, k, v)
                kept.append((k, v))
        n = sum(asked)
        positions = r.draft(_i32(asked), _i32(sum([list(range(-1, a - 1)) for a in asked], [])))
        assert positions.tolist() == [h + j for h, a in zip(held, asked) for j in range(a)]
        q, k, v = _rows(n, 8, 2, step)
        for i, kind in enumerate(schedule):
            out = torch.full((n, 8, 128), float("nan"), dtype=torch.bfloat16, device=DEV)
            r.layer(i, q, k, v, out)
            torch.cuda.synchronize()
            at = 0
            for b, a in enumerate(asked):
                if a == 0:
                    continue
                old = kept[i] if step == 3 else [x[:50] if b == 1 else x[50:] for x in kept[i]]
                seen = torch.arange(held[b], device=DEV)
                if kind == cb.LAYER_SPARSE:
                    seen = r.idx[b, : int(r.cnt[b])].long()
                    seen = seen[seen < held[b]]
                kk, vv = (torch.cat([c[seen], x[at: at + a]]).transpose(0, 1).double() for c, x in zip(old, (k, v)))
                want, mass = ref.attention(q[at: at + a], kk, vv, len(seen), a, np.tril(np.ones((a, a), dtype=bool)), 128 ** -0.5)
                ref.assert_attention(out[at: at + a], want, mass, f"step {step} layer {i} sequence {b}")
                at += a
        r.accept(_i32([[0]] * 3), _i32([0, 0, 0]))
    r.keep.zero_()
    r.draft(_i32([0, 0, 0]), torch.empty(0, dtype=torch.int32, device=DEV))
    assert r.pool.state.tolist()[1] == 12 and sorted(r.pool.ring.tolist()) == list(range(12))
