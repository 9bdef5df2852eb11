"""The calls of beam search against their plain statements: whole numbers bit for bit, scores and attention within bounds that count the roundings."""
import math

import numpy as np
import pytest
import torch

import beam_reference as ref
from paper_2508_07101_amd import binding as cb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


# ---- selection

# A term's exponent t is rounded three times (the difference, its product with log2 e, the constant): |t| 3 * 2^-24 in all, which moves the sum by less than the mean of |t|
# over its weights times 2^-22: for a vocabulary of 2^18 tokens that is at most 18 (the entropy in bits bounds it up to a bit or two).  A term's instruction and the sums of 64 of
# them: 2^-23 and 64 * 2^-24.  2^-17 in all; the value itself is rounded to binary32.
VALUE = 2.0 ** -17


def _select(logits, scores, width, n, ended=None, end=-1, in_place=False):
    rows, vocab = logits.shape
    groups = rows // width
    out = (torch.full((groups, n), 7.0, device=DEV), _i32(np.full((groups, n), 7)), _i32(np.full((groups, n), 7)), _i32(np.full((groups, n), 7)))
    if in_place:
        out = (scores.view(groups, n), out[1], out[2], ended.view(groups, n))
    ws = torch.full((cb.beam_workspace_bytes(rows, vocab, n),), 171, dtype=torch.uint8, device=DEV)
    cb.beam_select(logits, scores, width, out[0], out[1], out[2], ws, ended, out[3], end)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in out]


def _check_select(logits, scores, width, n, ended=None, end=-1, in_place=False):
    x, s = logits.double().cpu().numpy(), scores.cpu().numpy().copy()
    over = None if ended is None else ended.cpu().numpy().copy()
    more = ref.select(x, s, over, width, 2 * n + 8, end)          # (those behind the last place as well: one of them may be as near)
    want = [best[:n] for best in more]
    got, parents, tokens, out_ended = _select(logits, scores, width, n, ended, end, in_place)
    for g, best in enumerate(want):
        for i in range(n):
            where = f"group {g} place {i}"
            if i >= len(best):
                assert (got[g, i], parents[g, i], tokens[g, i], out_ended[g, i]) == (-math.inf, -1, -1, 0), where
                continue
            v, b, t = best[i]
            assert abs(got[g, i] - v) <= VALUE + 2.0 ** -24 * abs(v), (where, got[g, i], v)
            # (candidates as near as the bound may stand either way round; of equal logits of one row the lower token comes first)
            near = [(c[1], c[2]) for c in more[g] if abs(c[0] - v) <= 2 * VALUE]
            if len(near) == 1:
                assert (parents[g, i], tokens[g, i]) == (b, t), where
            else:
                assert (parents[g, i], tokens[g, i]) in near, where
            p = int(parents[g, i])
            assert out_ended[g, i] == int((over is not None and over[g * width + p] != 0) or tokens[g, i] == end), where
        rows = list(zip(parents[g, : len(best)].tolist(), tokens[g, : len(best)].tolist()))
        assert len(set(rows)) == len(rows)
        for (p, t), (q, u) in zip(rows, rows[1:]):
            if p == q and (over is None or not over[g * width + p]):
                assert x[g * width + p, t] > x[g * width + p, u] or (x[g * width + p, t] == x[g * width + p, u] and t < u)


def _logits(rows, vocab, kind, seed, pad=0, at=0):
    """A view of wider rows; at: elements in front."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    x = (torch.randn(rows * (vocab + pad) + at, generator=gen, device=DEV) * 3).to(kind)
    x = x[at:].view(rows, vocab + pad)[:, :vocab]
    return x, -torch.rand(rows, generator=gen, device=DEV) * 5


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("groups,width,vocab,n,pad,at", [(1, 1, 1, 1, 0, 0), (3, 2, 7, 64, 0, 0), (2, 4, 257, 4, 0, 0), (1, 4, 32000, 8, 0, 0), (5, 3, 1003, 6, 0, 1), (2, 32, 5000, 64, 8, 0),
                                                         (1, 8, 70001, 16, 3, 5), (1, 1, 131072, 64, 0, 0), (40, 4, 3001, 5, 1, 3), (1, 2, 200003, 1, 0, 7)])
def test_selection(kind, groups, width, vocab, n, pad, at):
    print("select", kind, groups, width, vocab, n, flush=True)
    x, s = _logits(groups * width, vocab, kind, vocab + n, pad, at)
    _check_select(x, s, width, n)


@pytest.mark.parametrize("vocab", [40, 3000, 66000])
def test_selection_of_equal_logits(vocab):
    """Whole rows of one value, of a few values, of zeros of both signs, rows alike: the lower row, then the lower token."""
    print("equal", vocab, flush=True)
    rng = np.random.default_rng(vocab)
    x = np.zeros((16, vocab), dtype=np.float32)
    x[1] = -0.0
    x[2, ::2] = -0.0
    x[3] = -1e4
    x[4:8] = rng.integers(0, 3, (4, vocab))
    x[8:12] = x[4]
    x[12, -3:] = 5.0
    x[13] = np.sort(rng.standard_normal(vocab))                  # every token better than the one before
    x[14] = x[13, ::-1]
    x[15] = torch.finfo(torch.bfloat16).min                      # a mask of the type's lowest value everywhere
    for kind in (torch.bfloat16, torch.float32):
        _check_select(torch.tensor(x, device=DEV).to(kind), torch.zeros(16, device=DEV), 4, 12)
    _, parents, tokens, _ = _select(torch.tensor(x[4:12], device=DEV), torch.zeros(8, device=DEV), 8, 9)
    first = np.flatnonzero(x[4] == x[4].max())
    ties = [(b, t) for b in (0, 4, 5, 6, 7) for t in first]
    if len(first) == len(np.flatnonzero(x[5] == x[5].max())) or len(first) > 9:
        assert [p for p in parents[0].tolist()] == sorted(parents[0].tolist())
    assert len(ties) >= 1


@pytest.mark.parametrize("vocab", [33, 2049, 40000])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_selection_with_masks_ended_rows_and_what_is_not_finite(vocab, kind):
    print("masks", vocab, kind, flush=True)
    x, s = _logits(24, vocab, kind, vocab)
    x[0] = -math.inf                                             # proposes nothing
    x[1, 3:] = -math.inf
    x[2, vocab // 2] = math.nan
    x[3, vocab - 1] = math.inf
    x[4, : vocab - 1] = -math.inf                                # its last token is certain
    x[5] = torch.where(torch.rand(vocab, device=DEV) < 0.9, torch.finfo(kind).min, x[5])
    s[6], s[7], s[9], s[10] = -math.inf, math.nan, math.inf, -3e38
    x[8] = math.nan
    x[12:16] = -math.inf                                         # a group without a proposal
    x[16:20, 2:] = -math.inf                                     # one with fewer than it is asked for
    ended = _i32([0, 0, 0, 0, 0, 0, 1, 1, 5, 1, 0, 0, 0, 0, 0, 0, 0, 1, 0, 0, 1, 1, 1, 1])
    _check_select(x, s, 4, 10, ended, 2)
    _check_select(x, s, 8, 3, None, vocab - 1)
    _check_select(x, s, 1, 5, ended, vocab - 1)


def test_selection_in_place_is_the_next_step():
    x, s = _logits(24, 5000, torch.bfloat16, 5)
    ended = _i32(np.arange(24) % 5 == 0)
    for _ in range(3):
        _check_select(x, s, 4, 4, ended, 17, in_place=True)


def test_selection_goes_by_the_definition_far_from_zero():
    """Scores and logits of thousands: what is added is small beside them."""
    x, s = _logits(8, 9000, torch.float32, 6)
    _check_select(x + 30000.0, s - 1000.0, 4, 8)
    _check_select(x * 1000.0, s, 4, 8)


# ---- fork

def _fork_case(rng, groups, width, prompt, tail, free, columns=0, empty=0.1, samples=False):
    lens, table, used = ref.family(rng, groups, width, prompt, tail, columns, samples)
    n_pages = used + free
    order = rng.permutation(n_pages)
    table = np.where(table >= 0, order[table], -1)
    gone = rng.random(len(lens)) < empty
    ring = np.full(n_pages, -1)
    first = int(rng.integers(0, n_pages))
    ring[(first + np.arange(free)) % n_pages] = order[used:]
    return lens, table, ring, [first, free], gone


def _check_fork(width, lens, table, ring, state, parents, ended, grow, in_place=False):
    pool = cb.PagePool(_i32(table), _i32(ring), _i32(state))
    B = len(lens)
    held, over = _i32(lens), None if ended is None else _i32(ended)
    ws = torch.full((cb.fork_workspace_bytes(*table.shape),), 171, dtype=torch.uint8, device=DEV)
    slots, copies, granted = torch.full((B,), 77, dtype=torch.int64, device=DEV), _i32(np.full((B, 4), 77)), _i32(np.full(B // width, 77))
    if in_place:
        want = ref.fork(width, lens, parents, ended, grow, table, ring, state, table)
        cb.kv_fork(pool, width, held, _i32(parents), held, slots, copies, ws, over, grow, granted=granted)
        out, got_lens, got_state = pool.block_table, held, pool.state
    else:
        out, got_lens, got_state = _i32(np.full(table.shape, -7)), _i32(np.full(B, 77)), _i32([77, 77])
        want = ref.fork(width, lens, parents, ended, grow, table, ring, state, np.full(table.shape, -7))
        cb.kv_fork(pool, width, held, _i32(parents), got_lens, slots, copies, ws, over, grow, out, got_state, granted)
    torch.cuda.synchronize()
    for name, g, w in zip(("lens", "slots", "copies", "table", "ring", "state", "granted"), (got_lens, slots, copies, out, pool.ring, got_state, granted), want):
        assert np.array_equal(g.cpu().numpy(), np.asarray(w)), name
    return want


@pytest.mark.parametrize("groups,width,prompt,tail,columns", [(1, 1, 40, 20, 0), (1, 4, 100, 60, 0), (7, 3, 300, 50, 0), (64, 4, 60, 40, 300), (3, 32, 50, 200, 0), (1, 8, 9000, 300, 0), (400, 5, 30, 30, 0),
                                                              (2, 16, 5000, 4000, 600)])
@pytest.mark.parametrize("free", [0, 5, 300])
@pytest.mark.parametrize("samples", [False, True])
def test_fork(groups, width, prompt, tail, columns, free, samples):
    print("fork", groups, width, prompt, tail, free, flush=True)
    rng = np.random.default_rng(groups * 100 + width + free)
    lens, table, ring, state, gone = _fork_case(rng, groups, width, prompt, tail, free, columns, samples=samples)
    if not len(ring):
        pytest.skip("a pool without pages")
    B = groups * width
    parents = rng.integers(-1, width + 1, B)
    parents[gone] = -1
    for grow, in_place, ended in ((True, False, None), (True, True, rng.random(B) < 0.3), (False, False, None)):
        _check_fork(width, lens, table, ring, state, parents, ended, grow, in_place)
    for own in (np.arange(B) % width, np.zeros(B, dtype=np.int64), np.full(B, -1)):       # nobody moves, all descend from the first, all end
        _check_fork(width, lens, table, ring, state, own, None, True, True)


def test_fork_over_many_steps():
    rng = np.random.default_rng(9)
    width, groups = 4, 6
    lens, table, ring, state, _ = _fork_case(rng, groups, width, 100, 30, 40, columns=14)
    for step in range(25):
        print("step", step, state, flush=True)
        parents, ended = rng.integers(-1 if step % 6 == 5 else 0, width, groups * width), rng.random(groups * width) < 0.1
        lens, _, _, table, ring, state, _ = _check_fork(width, lens, table, ring, state, parents, ended, step % 4 != 1, True)
        lens = np.asarray(lens)


def test_fork_with_numbers_out_of_range():
    """Tables and lengths that mean nothing are cut or left out; what is right stays right."""
    rng = np.random.default_rng(3)
    lens, table, ring, state, _ = _fork_case(rng, 6, 4, 60, 40, 30, columns=9)
    table[2, 1], table[5, :], table[9, 3], table[13, 2] = -1, 1 << 30, len(ring), -(1 << 31)
    lens[7], lens[12], lens[20] = -5, 1 << 30, 9 * 16
    for in_place in (False, True):
        _check_fork(4, lens, table, ring, state, rng.integers(-(1 << 30), 1 << 30, 24), None, True, in_place)
        _check_fork(4, lens, table, ring, state, rng.integers(0, 4, 24), rng.integers(-2, 2, 24), True, in_place)
    _check_fork(4, lens, table, ring, [len(ring) + 3, 1 << 20], rng.integers(0, 4, 24), None, True)
    _check_fork(4, lens, table, ring, [-1, -1], rng.integers(0, 4, 24), None, True)


def test_fork_groups_beyond_the_free_pages_stay():
    """Pages for the first groups only, and a group that asks for none behind one that does not get its own."""
    width, lens = 2, np.array([16, 16, 20, 20, 16, 16, 5, 5])
    table = np.array([[0, -1], [0, -1], [1, 2], [1, 3], [4, -1], [4, -1], [5, -1], [6, -1]])
    ring = np.array([7, 8, 9] + [-1] * 7)
    want = _check_fork(width, lens, table, ring, [0, 3], np.array([0, 1] * 4), None, True)
    assert want[-1] == [1, 1, 0, 1] and want[5] == [2, 1]
    want = _check_fork(width, np.array([32, 32] * 4), np.tile([[0, 1]], (8, 1)), ring, [0, 3], np.array([0, 1] * 4), None, True)
    assert want[-1] == [0] * 4                                   # rows as long as their tables


# ---- copies

@pytest.mark.parametrize("G,layers,n", [(8, 3, 5), (1, 1, 1), (2, 41, 9), (5, 2, 300)])
def test_copies(G, layers, n):
    print("copy", G, layers, n, flush=True)
    rng = np.random.default_rng(n)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)
    n_pages = 2 * n + 3
    k, v = (torch.randn((layers, n_pages, G, 16, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    order = rng.permutation(n_pages)
    copies = np.stack([order[rng.integers(0, n, n)], order[n: 2 * n], rng.integers(-2, 20, n), rng.integers(-9, 9, n)], axis=1)
    copies[::4, 0], copies[1::5, 1] = -1, n_pages                # of no page, and to none
    want = [x.clone() for x in (k, v)]
    for f, t, m, _ in copies:
        if 0 <= f < n_pages and 0 <= t < n_pages:
            for x, w in zip((k, v), want):
                w[:, t, :, : max(0, min(m, 16))] = x[:, f, :, : max(0, min(m, 16))]
    params, one = cb.make_params(1, G, G, 1, 0), _i32([[0]])
    copy = cb.KvCopy(params, [cb.KvCache(k[i], v[i], _i32([1]), 16, one) for i in range(layers)])
    copy.run(_i32(copies))
    copy.run(_i32(copies[:0]))
    torch.cuda.synchronize()
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


# ---- lists of pages

def _check_shared(width, lens, table, n_pages, max_len):
    want = ref.shared(width, lens, table, n_pages, max_len)
    groups = len(lens) // width
    most = min(width * ref.pages(max_len), n_pages)
    s = cb.SharedPages(width, _i32(np.full((groups, most, 4), 77)), _i32(np.full((groups, 2), 77)))
    ws = torch.full((cb.pages_workspace_bytes(len(lens), max_len),), 171, dtype=torch.uint8, device=DEV)
    cb.shared_pages(_i32(table), _i32(lens), max_len, n_pages, s, ws)
    torch.cuda.synchronize()
    got, count = s.entries.cpu().numpy(), s.count.tolist()
    for g, (entries, whole) in enumerate(want):
        n = min(len(entries), most)
        assert count[g] == [n, min(whole, n)], g
        assert np.array_equal(got[g, :n].astype(np.int64) & 0xffffffff, np.asarray(entries[:n], dtype=np.int64).reshape(-1, 4) & 0xffffffff), g
        assert (got[g, n:] == 77).all()


@pytest.mark.parametrize("groups,width,prompt,tail", [(1, 1, 40, 20), (1, 4, 100, 60), (7, 3, 300, 50), (64, 4, 2000, 40), (3, 32, 50, 200), (1, 8, 9000, 300), (1, 1, 70000, 1), (2, 32, 20000, 3000), (3, 4, 40000, 900)])
@pytest.mark.parametrize("samples", [False, True])
def test_lists_of_pages(groups, width, prompt, tail, samples):
    print("pages", groups, width, prompt, tail, flush=True)
    rng = np.random.default_rng(groups + width)
    lens, table, used = ref.family(rng, groups, width, prompt, tail, samples=samples)
    n_pages = used + 5
    order = rng.permutation(n_pages)
    table = np.where(table >= 0, order[table], -1)
    _check_shared(width, lens, table, n_pages, max(1, int(lens.max())))
    lens[rng.random(len(lens)) < 0.3] = 0                         # empty rows hold nothing
    table[rng.random(table.shape) < 0.01] = -1                   # entries that name no page
    table[rng.random(table.shape) < 0.01] = n_pages
    _check_shared(width, lens, table, n_pages, max(1, int(lens.max()) - 3))


def test_lists_of_tables_that_no_search_makes():
    """A page in several columns and groups, lengths beyond the bounds: lists are cut to their room."""
    rng = np.random.default_rng(1)
    lens = np.array([100, -4, 1 << 30, 17, 0, 160, 33, 160])
    _check_shared(4, lens, rng.integers(-2, 6, (8, 10)), 5, 160)
    _check_shared(8, lens, np.zeros((8, 10), dtype=np.int64), 1, 150)
    _check_shared(2, np.zeros(8, dtype=np.int64), np.zeros((8, 10), dtype=np.int64), 9, 160)
