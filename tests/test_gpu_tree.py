"""Trees of drafted tokens on the GPU against plain statements of the calls: whole numbers and moved rows exactly, attention
within the bound that its roundings give."""
import numpy as np
import pytest
import torch

import tree_reference as ref
from paper_2508_07101_amd import binding as cb

pytestmark = pytest.mark.gpu
DEV = "cuda"
PAGE = 16


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


# ---- plan

def _run_plan(held, keep, add, max_tokens, cap, table=None, ring=None, state=None, in_place=True):
    n = len(held)
    th, tk, ta = _i32(held), _i32(keep), _i32(add)
    lens = th if in_place else torch.zeros(n, dtype=torch.int32, device=DEV)
    start, slots = torch.zeros(n + 1, dtype=torch.int32, device=DEV), torch.full((max_tokens,), 77, dtype=torch.int64, device=DEV)
    ws = cb.alloc_plan_workspace(n)
    if table is None:
        cb.kv_plan(th, tk, ta, lens, start, slots, ws, capacity=cap)
        torch.cuda.synchronize()
        return lens.tolist(), start.tolist(), slots.tolist()
    pool = cb.PagePool(_i32(table), _i32(ring), _i32(state))
    out = None if in_place else torch.zeros(2, dtype=torch.int32, device=DEV)
    cb.kv_plan(th, tk, ta, lens, start, slots, ws, pool, out)
    torch.cuda.synchronize()
    if not in_place:
        assert pool.state.tolist() == list(state) and th.tolist() == list(held)
    return lens.tolist(), start.tolist(), slots.tolist(), pool.block_table.cpu().numpy(), pool.ring.cpu().numpy(), (pool.state if in_place else out).tolist()


def _same_plan(got, want):
    for g, w in zip(got, want):
        assert np.array_equal(np.asarray(g), np.asarray(w))


@pytest.mark.parametrize("batch,most,add,spare", [(1, 50, 20, 2.0), (3, 100, 40, 1.0), (64, 700, 64, 0.5), (64, 0, 300, 1.1), (1000, 60, 9, 0.8), (1024, 30, 4, 1.0),
                                                  (1025, 30, 4, 0.4), (3000, 50, 5, 1.0)])
@pytest.mark.parametrize("seed", [1, 2])
def test_plan_of_a_paged_cache(batch, most, add, spare, seed):
    print("plan", batch, most, add, spare, seed, flush=True)
    rng = np.random.default_rng(seed * 1000 + batch)
    held = rng.integers(0, most + 1, batch)
    keep = np.where(rng.random(batch) < 0.3, 0, np.maximum(held - rng.integers(0, 40, batch), 0))
    add = np.where(rng.random(batch) < 0.2, 0, rng.integers(0, add + 1, batch))
    used = [ref.pages(int(h)) for h in held]
    max_pages = ref.pages(most + int(add.max())) + 1
    n_pages = sum(used) + max(1, int(sum(ref.pages(int(a)) for a in add) * spare))
    perm = rng.permutation(n_pages)
    table = np.full((batch, max_pages), -1)
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = perm[at: at + u]
        at += u
    free = n_pages - at
    first = int(rng.integers(0, n_pages))
    ring = np.full(n_pages, -1)
    ring[(first + np.arange(free)) % n_pages] = perm[at:]
    for max_tokens in sorted({int(add.sum()) + 5, int(add.sum()) // 2, 5000}):
        want = ref.plan(held, keep, add, max_tokens, max_pages * PAGE, table, ring, [first, free])
        for in_place in (True, False):
            _same_plan(_run_plan(held, keep, add, max_tokens, 0, table, ring, [first, free], in_place), want)


@pytest.mark.parametrize("batch,max_tokens", [(1, 7), (5, 100), (70, 9000)])
def test_plan_of_a_contiguous_cache(batch, max_tokens):
    rng = np.random.default_rng(batch)
    held, add = rng.integers(0, 200, batch), rng.integers(0, 150, batch)
    keep = np.maximum(held - rng.integers(0, 10, batch), 0)
    _same_plan(_run_plan(held, keep, add, max_tokens, 256), ref.plan(held, keep, add, max_tokens, 256))


def test_plan_cuts_values_out_of_range():
    held, keep, add = [-5, 1 << 30, 100, 40, 2 ** 31 - 1, 0], [3, 7, 200, -1, 2 ** 31 - 1, 0], [2, 2 ** 31 - 1, -8, 5, 2 ** 31 - 1, 64]
    table = np.tile(np.array([0, 99, 2, -3]), (6, 1))
    for n in (64, 5000):
        for state in ([21, 4], [-1, -3]):
            want = ref.plan(held, keep, add, n, 64, table, np.arange(16), state)
            _same_plan(_run_plan(held, keep, add, n, 0, table, np.arange(16), state), want)
        # a queue that claims more free pages than there are: where those are that come back to it is not defined
        want = ref.plan(held, keep, add, n, 64, table, np.arange(16), [0, 500])
        got = _run_plan(held, keep, add, n, 0, table, np.arange(16), [0, 500])
        assert got[:2] == want[:2] and got[5] == want[5]


def test_plan_captured_and_replayed():
    """A decode loop's plans from one graph: trees are granted, cut back and granted again, and no page is lost."""
    n, max_pages, n_pages = 5, 12, 40
    pool = cb.PagePool.empty(n, max_pages, n_pages)
    lens, keep, add = _i32([0] * n), _i32([0] * n), _i32([30, 17, 16, 1, 0])
    start, slots, ws = torch.zeros(n + 1, dtype=torch.int32, device=DEV), torch.zeros(120, dtype=torch.int64, device=DEV), cb.alloc_plan_workspace(n)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            cb.kv_plan(lens, keep, add, lens, start, slots, ws, pool)
    torch.cuda.synchronize()
    state = ([0] * n, np.full((n, max_pages), -1), np.arange(n_pages), [0, n_pages])
    rng = np.random.default_rng(3)
    for step in range(12):
        k, a = [max(0, x - int(rng.integers(0, 20))) for x in state[0]], rng.integers(0, 25, n).tolist()
        keep.copy_(_i32(k))
        add.copy_(_i32(a))
        graph.replay()
        torch.cuda.synchronize()
        want = ref.plan(state[0], k, a, 120, max_pages * PAGE, *state[1:])
        _same_plan((lens.tolist(), start.tolist(), slots.tolist(), pool.block_table.cpu().numpy(), pool.ring.cpu().numpy(), pool.state.tolist()), want)
        state = (want[0], want[3], want[4], want[5])
        held = [int(p) for b in range(n) for p in want[3][b][: ref.pages(want[0][b])]]
        free = [int(want[4][(want[5][0] + i) % n_pages]) for i in range(want[5][1])]
        assert sorted(held + free) == list(range(n_pages))


# ---- caches

def _cache(layout, B, G, cap, seed, extra_pages=2):
    """K, V and (paged) the table of caches of cap[b] positions, filled with normal values."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    table = None
    if layout == "paged":
        n = [ref.pages(c) for c in cap]
        perm = np.random.default_rng(seed).permutation(sum(n) + extra_pages)
        t = np.full((B, max(max(n), 1)), -1)
        at = 0
        for b in range(B):
            t[b, : n[b]] = perm[at: at + n[b]]
            at += n[b]
        table, shape = _i32(t), (sum(n) + extra_pages, G, PAGE, 128)
    else:
        shape = (B, max(cap), G, 128) if layout == "token_major" else (B, G, max(cap), 128)
    k, v = (torch.randn(shape, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    if layout == "token_major":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return k, v, table


def _put(x, table, b, pos, rows):
    if table is None:
        x[b, :, pos] = rows
    else:
        x[int(table[b, pos // PAGE]), :, pos % PAGE] = rows


# ---- append

@pytest.mark.parametrize("layout", ["paged", "head_major", "token_major"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("G,n", [(1, 1), (8, 3), (5, 40), (8, 513)])
def test_append(layout, dtype, G, n):
    print("append", layout, dtype, G, n, flush=True)
    rng = np.random.default_rng(n + G)
    B, cap = 3, [200, 300, 250]
    k, v, table = _cache(layout, B, G, cap, n)
    where = [(b, p) for b in range(B) for p in range(cap[b])]
    chosen = [where[i] for i in rng.permutation(len(where))[:n]]
    slots = [int(table[b, p // PAGE]) * PAGE + p % PAGE if table is not None else (b << 32) + p for b, p in chosen]
    new = torch.randn((n, 2 * G + 3, 128), device=DEV).to(dtype)           # heads of a fused projection
    new[0, 0, :4] = torch.tensor([float("inf"), float("nan"), -0.0, 65504.0], device=DEV).to(dtype)
    k_new, v_new = new[:, 3: 3 + G], new[:, 3 + G:]
    want_k, want_v = k.clone(), v.clone()
    for i, (b, p) in enumerate(chosen):
        if i % 7 == 3:                                                      # a slot that names nothing
            n_pages = k.shape[0]
            slots[i] = [-1, -(1 << 40), n_pages * PAGE, 1 << 62][i % 4] if table is not None else [-1, (B << 32), (1 << 32) + max(cap), 1 << 62][i % 4]
            continue
        _put(want_k, table, b, p, k_new[i].to(torch.bfloat16))
        _put(want_v, table, b, p, v_new[i].to(torch.bfloat16))
    params = cb.make_params(B, G, G, 1, 0)
    kv = cb.KvCache(k, v, _i32(cap), max(cap), table)
    cb.kv_append(params, kv, torch.tensor(slots, dtype=torch.int64, device=DEV), k_new, v_new)
    torch.cuda.synchronize()
    assert torch.equal(k.float().nan_to_num(7.0), want_k.float().nan_to_num(7.0)) and torch.equal(v.float().nan_to_num(7.0), want_v.float().nan_to_num(7.0))
    assert torch.equal(k.isnan(), want_k.isnan())


# ---- masks

@pytest.mark.parametrize("max_nodes", [1, 2, 31, 63, 64, 65, 128, 200, 256])
def test_masks(max_nodes):
    rng = np.random.default_rng(max_nodes)
    n = rng.integers(0, max_nodes + 1, 7)
    n[0], n[3] = max_nodes, 0
    parents = [np.array([int(rng.integers(-1, j + 2)) if rng.random() < 0.3 else j - 1 if kind else int(rng.integers(max(0, j - 9), j + 1)) - 1 for j in range(c)], dtype=np.int64)
               for kind, c in zip([1, 0, 1, 0, 1, 0, 1], n)]
    parents[0][:] = np.arange(max_nodes) - 1                                # a chain: as deep as can be
    base, words, total = rng.integers(0, 5000, 7), cb.mask_words(max_nodes), int(n.sum())
    masks = torch.full((total + 2, words), 5, dtype=torch.int64, device=DEV)
    pos = torch.full((total + 2,), 5, dtype=torch.int32, device=DEV)
    flat = np.concatenate(parents + [np.array([0, 0])])
    cb.tree_masks(_i32(base), _i32(np.concatenate([[0], np.cumsum(n)])), _i32(flat), masks, pos, max_nodes)
    again = torch.zeros_like(masks)
    cb.tree_masks(_i32(base), _i32(np.concatenate([[0], np.cumsum(n)])), _i32(flat), again, None, max_nodes)
    torch.cuda.synchronize()
    want = [ref.masks(p, words) for p in parents]
    rows = np.concatenate([w[0] for w in want])
    assert np.array_equal(masks[:total].cpu().numpy().view(np.uint64), rows) and np.array_equal(again[:total].cpu().numpy().view(np.uint64), rows)
    assert pos[:total].tolist() == [int(b) + d for b, w in zip(base, want) for d in w[1]]
    assert (masks[total:] == 5).all() and (pos[total:] == 5).all()          # rows of no sequence


# ---- attention

def _bits(n, words, rng, kind):
    if kind == "tree":
        return ref.masks([int(rng.integers(-1, j)) if j else -1 for j in range(n)], words)[0]
    rows = rng.integers(0, 1 << 63, (n, words), dtype=np.uint64) if kind == "any" else np.zeros((n, words), dtype=np.uint64)
    return rows | (rng.integers(0, 2, (n, words), dtype=np.uint64) << np.uint64(63)) if kind == "any" else rows


class _Case:
    """A batch of trees over a cache; out() runs the library, want() the reference."""

    def __init__(self, layout, H, G, before, n, seed, max_nodes=None, budget=0, kind="tree", fused=False, max_len=None):
        self.rng = rng = np.random.default_rng(seed)
        self.layout, self.H, self.G, self.before, self.n = layout, H, G, list(before), list(n)
        B = len(n)
        self.lens = [a + b for a, b in zip(before, n)]
        self.k, self.v, self.table = _cache(layout, B, G, [max(x, 1) for x in self.lens], seed)
        self.max_nodes = max_nodes or max(max(n), 1)
        self.words = cb.mask_words(self.max_nodes)
        self.total = sum(n)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed + 1)
        self.q = torch.randn((max(self.total, 1), H + (2 * G if fused else 0), 128), generator=gen, device=DEV).to(torch.bfloat16)[:, :H]
        self.bits = [_bits(c, self.words, rng, kind) for c in n]
        masks = np.concatenate(self.bits + ([np.zeros((1, self.words), dtype=np.uint64)] if self.total == 0 else []))
        self.tree = cb.Tree(_i32(np.concatenate([[0], np.cumsum(n)])), torch.from_numpy(masks.view(np.int64).copy()).to(DEV), self.max_nodes)
        self.max_len = max_len or max(max(self.lens), 1)
        self.params = cb.make_params(B, H, G, budget or 1, 0)
        self.idx = self.cnt = None
        if budget:
            self.sets = [np.sort(rng.choice(p + 1, size=min(p + 1, budget, int(rng.integers(1, budget + 1))), replace=False)) for p in before]
            self.idx, self.cnt = torch.zeros((B, budget), dtype=torch.int32, device=DEV), _i32([len(x) for x in self.sets])
            for b, x in enumerate(self.sets):
                self.idx[b, : len(x)] = _i32(x)

    def kv(self):
        if self.layout == "paged" and self.table.shape[1] * PAGE < self.max_len:
            more = torch.full((self.table.shape[0], ref.pages(self.max_len) - self.table.shape[1]), -1, dtype=torch.int32, device=DEV)
            self.table = torch.cat([self.table, more], dim=1).contiguous()
        return cb.KvCache(self.k, self.v, _i32(self.lens), self.max_len, self.table)

    def out(self, fill=7.0):
        out = torch.full((max(self.total, 1), self.H, 128), fill, dtype=torch.bfloat16, device=DEV)
        ws = cb.alloc_tree_workspace(self.params, self.max_len, max(self.total, 1), self.max_nodes)
        ws.fill_(255)                                                      # NaN wherever a piece is read that nobody wrote
        print("tree", self.layout, self.H, self.G, self.before[:4], self.n[:4], self.max_nodes, self.params.budget, flush=True)
        cb.tree_attn(self.params, self.q, self.kv(), self.tree, out, ws, self.idx, self.cnt)
        torch.cuda.synchronize()
        return out

    def want(self):
        outs, masses, at = [], [], 0
        for b, n in enumerate(self.n):
            p = self.before[b]
            seen = np.arange(p) if self.idx is None else self.sets[b][(self.sets[b] < p) & (self.sets[b] >= 0)]
            pos = torch.as_tensor(np.concatenate([seen, np.arange(p, p + n)]).astype(np.int64), device=DEV)
            if n:
                o, m = ref.attention(self.q[at: at + n], ref.cache_rows(self.k, self.table, b, pos), ref.cache_rows(self.v, self.table, b, pos), len(seen), n,
                                     ref.allowed(self.bits[b], n), 128 ** -0.5)
                outs.append(o)
                masses.append(m)
            at += n
        return torch.cat(outs), torch.cat(masses)

    def check(self, what=""):
        got = self.out()
        want, mass = self.want()
        ref.assert_attention(got, want, mass, what)
        assert torch.equal(got, self.out(3.0))                             # bit for bit, whatever was in the output and the workspace
        return got


@pytest.mark.parametrize("layout", ["paged", "head_major", "token_major"])
@pytest.mark.parametrize("budget", [0, 100])
@pytest.mark.parametrize("H,G", [(8, 8), (16, 8), (4, 1), (24, 3), (40, 5), (64, 8)])
def test_attention_over_layouts_and_groups(layout, budget, H, G):
    _Case(layout, H, G, [0, 1, 15, 300, 777], [3, 1, 0, 8, 5], 11, budget=budget, fused=H == 24).check()


@pytest.mark.parametrize("nodes", [1, 2, 4, 7, 8, 9, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200, 255, 256])
@pytest.mark.parametrize("H,G,budget", [(8, 2, 0), (16, 2, 64), (2, 2, 0)])
def test_attention_over_tree_sizes(nodes, H, G, budget):
    _Case("paged", H, G, [500, 31, 0], [nodes, max(1, nodes // 2), nodes], nodes, budget=budget).check()


@pytest.mark.parametrize("before", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1023, 1025, 2500, 9001])
@pytest.mark.parametrize("nodes", [5, 20, 70])
def test_attention_over_lengths(before, nodes):
    _Case("paged" if before % 2 else "head_major", 8, 2, [before, max(0, before - 1)], [nodes, nodes - 1], before + nodes).check()


@pytest.mark.parametrize("nodes", [3, 16, 40, 100])
def test_attention_with_any_masks(nodes):
    """Bits anywhere, above the diagonal and behind the tree's nodes as well, and rows without any."""
    for kind in ("any", "none"):
        for before in (0, 40):
            c = _Case("paged", 16, 4, [before, 0], [nodes, 2], nodes, kind=kind)
            got = c.check(kind)
            if kind == "none" and before == 0:
                assert (got == 0).all()


def test_rows_of_no_sequence_are_not_written():
    c = _Case("paged", 8, 2, [50, 60], [5, 6], 5, max_nodes=16)
    c.tree.tok_start = _i32([2, 5, 9])                                      # rows 2..4 and 5..8 of 11
    out = c.out(9.0)
    assert (out[:2] == 9).all() and (out[9:] == 9).all() and (out[2:9] != 9).any(dim=-1).all()


def test_trees_longer_than_the_bounds_are_cut():
    """Counts beyond max_nodes, beyond the cache's tokens, starts out of range: nothing out of range is touched."""
    c = _Case("head_major", 8, 2, [30, 30, 0], [6, 6, 6], 5, max_nodes=6)
    c.lens = [36, 4, 1 << 30]
    c.tree.tok_start = _i32([-3, 6, 1 << 30, -(1 << 30)])
    out = c.out(9.0)
    assert torch.isfinite(out.float()).all()


@pytest.mark.parametrize("H,G", [(8, 2), (32, 8)])
def test_rows_between_trees_beyond_the_bound_need_no_workspace(H, G):
    """A sequence that owns more rows than max_nodes: the next one's rows start behind batch * max_nodes, its pieces' partial results do not."""
    c = _Case("paged", H, G, [3000, 2500], [4, 4], 6, max_nodes=4)
    want = c.check()
    q, masks = (torch.zeros((100,) + x.shape[1:], dtype=x.dtype, device=DEV) for x in (c.q, c.tree.masks))
    for x, y in ((q, c.q), (masks, c.tree.masks)):
        x[:4], x[90:94] = y[:4], y[4:]
    out = torch.full((100, H, 128), 9.0, dtype=torch.bfloat16, device=DEV)
    need = cb.tree_workspace_bytes(c.params, c.max_len, 100, 4)
    ws = torch.full((need + 64 * H * 128 * 100,), 255, dtype=torch.uint8, device=DEV)
    cb.tree_attn(c.params, q, c.kv(), cb.Tree(_i32([0, 90, 94]), masks, 4), out, ws[:need])
    torch.cuda.synchronize()
    assert torch.equal(out[:4], want[:4]) and torch.equal(out[90:94], want[4:])
    assert (out[4:90] == 9).all() and (out[94:] == 9).all() and (ws[need:] == 255).all()


@pytest.mark.parametrize("budget", [0, 4000])
def test_long_prefixes_and_bounds_far_above_the_lengths(budget):
    for before, nodes, H in (([40000], [60], 32), ([131000], [3], 8), ([20000, 100, 7000], [17, 30, 1], 32)):
        c = _Case("paged", H, 8, before, nodes, 3, budget=budget, max_len=140000)
        c.check()


@pytest.mark.parametrize("batch,nodes,whole", [(1, 4, 768), (1, 14, 384), (2, 33, 256), (16, 36, 1536), (33, 3, 4096)])
def test_sequences_about_as_long_as_stay_whole(batch, nodes, whole):
    """The last length that is one piece, and the first that may be cut: the same bound, and a batch of which one sequence alone is that long."""
    for length in (whole, whole + 1):
        _Case("paged", 32, 8, [length - nodes] * batch, [nodes] * batch, 4).check()
        _Case("head_major", 32, 8, [length - nodes] + [40] * (batch - 1), [nodes] * batch, 4).check()


def test_many_sequences():
    rng = np.random.default_rng(8)
    _Case("paged", 32, 8, rng.integers(0, 600, 70), rng.integers(0, 20, 70), 3).check()


def test_peaked_scores_and_growing_maxima():
    """Scores that grow along the prefix, far beyond what one exponent holds, and one token above all others."""
    c = _Case("head_major", 8, 2, [3000], [20], 4)
    c.k[0, :, :3000] *= torch.linspace(0.01, 12.0, 3000, device=DEV).to(torch.bfloat16)[None, :, None]
    c.check("growing")
    c.k[0, :, 1234] = (c.q[0].float().view(2, 4, 128).sum(1) * 8).to(torch.bfloat16)
    c.check("peaked")


@pytest.mark.parametrize("layout", ["paged", "head_major"])
@pytest.mark.parametrize("nodes", [6, 20, 50])
def test_values_that_are_not_finite_reach_only_those_that_attend_to_them(layout, nodes):
    c = _Case(layout, 16, 4, [75], [nodes], 4)
    clean = c.out()
    at = nodes // 2
    seen = ref.allowed(c.bits[0], nodes)[:, at]
    for val in (float("nan"), float("inf"), -float("inf")):
        save_k, save_v = c.k.clone(), c.v.clone()
        row = c.v[0, :, 75 + at].clone() if c.table is None else c.v[int(c.table[0, (75 + at) // PAGE]), :, (75 + at) % PAGE].clone()
        row[:, 5:90:3] = val
        _put(c.v, c.table, 0, 75 + at, row)
        got = c.out()
        for j in range(nodes):
            if not seen[j]:
                assert torch.equal(got[j], clean[j]), f"{val}: node {j} does not attend to {at}"
            else:
                hit = torch.zeros(128, dtype=torch.bool, device=DEV)
                hit[5:90:3] = True
                assert torch.equal(got[j][:, ~hit], clean[j][:, ~hit])
                assert (got[j][:, hit].isnan() if val != val else got[j][:, hit] == val).all()
        c.k, c.v = save_k, save_v
        # the same in a key: nodes that do not attend to it are as before
        save_k = c.k.clone()
        _put(c.k, c.table, 0, 75 + at, torch.full((4, 128), val, dtype=torch.bfloat16, device=DEV))
        got = c.out()
        assert torch.equal(got[~seen], clean[~seen])
        c.k = save_k


def test_what_lies_behind_the_sequences_does_not_matter():
    """NaN in the pages' tails and in pages of nobody."""
    c = _Case("paged", 8, 2, [75, 20], [9, 5], 4)
    want = c.out()
    used = torch.zeros(c.k.shape[0], PAGE, dtype=torch.bool, device=DEV)
    for b, n in enumerate(c.lens):
        for p in range(n):
            used[int(c.table[b, p // PAGE]), p % PAGE] = True
    for x in (c.k, c.v):
        x.permute(0, 2, 1, 3)[~used] = float("nan")
    assert torch.equal(c.out(), want)


def test_entries_that_name_no_page_are_left_out():
    c = _Case("paged", 8, 2, [200], [7], 4)
    table = c.table.clone()
    c.table[0, 3], c.table[0, 7] = -1, 1 << 30
    got = c.out()
    keep = torch.cat([torch.arange(48, device=DEV), torch.arange(64, 112, device=DEV), torch.arange(128, 207, device=DEV)])
    want, mass = ref.attention(c.q, ref.cache_rows(c.k, table, 0, keep), ref.cache_rows(c.v, table, 0, keep), len(keep) - 7, 7, ref.allowed(c.bits[0], 7), 128 ** -0.5)
    ref.assert_attention(got, want, mass, "bad pages")


def test_list_entries_outside_the_prefix_are_left_out():
    c = _Case("paged", 8, 2, [200, 90], [7, 3], 4, budget=64)
    c.sets = [np.array([0, 5, 77, 199]), np.array([], dtype=np.int64)]
    c.idx[0, :8] = _i32([-4, 0, 5, 77, 199, 200, 206, 2 ** 31 - 1])
    c.cnt = _i32([8, -3])
    c.check("lists")
    c.cnt = _i32([8, 0])
    c.check("empty list")
    c.sets[1] = np.arange(64)
    c.idx[1] = _i32(np.arange(64))
    c.cnt = _i32([8, 1 << 30])
    c.check("long count")


def test_offsets_beyond_32_bits():
    """Sequences more than 2^32 bytes apart, and a pool of as many."""
    B, G, cap = 2, 2, 300
    sb = (1 << 31) + 4096
    base_k, base_v = (torch.empty(sb + G * cap * 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k, v = (x.as_strided((B, G, cap, 128), (sb, cap * 128, 128, 1)) for x in (base_k, base_v))
    c = _Case("head_major", 8, G, [280, 270], [9, 20], 4)
    for x, y in ((k, c.k), (v, c.v)):
        x[:, :, : y.shape[2]] = y
    want = c.out()
    c.k, c.v = k, v
    assert torch.equal(c.out(), want)
    p = _Case("paged", 8, G, [280, 270], [9, 20], 4)
    n_pages = p.k.shape[0]
    far = (1 << 31) // (G * PAGE * 128) + 3                                 # pages before these
    pk, pv = (x[: (far + n_pages) * G * PAGE * 128].view(-1, G, PAGE, 128) if x.numel() >= (far + n_pages) * G * PAGE * 128 else
              torch.empty((far + n_pages, G, PAGE, 128), dtype=torch.bfloat16, device=DEV) for x in (base_k, base_v))
    want = p.out()
    pk[far:], pv[far:] = p.k, p.v
    p.k, p.v, p.table = pk, pv, torch.where(p.table >= 0, p.table + far, p.table)
    assert torch.equal(p.out(), want)
    new = torch.randn((2, G, 128), device=DEV).to(torch.bfloat16)
    slot = (far + 1) * PAGE + 5
    cb.kv_append(p.params, p.kv(), torch.tensor([slot, -1], dtype=torch.int64, device=DEV), new, new)
    torch.cuda.synchronize()
    assert torch.equal(pk[far + 1, :, 5], new[0])


def test_another_stream_and_a_graph():
    """Captured once and replayed over growing sequences with the program's own work between; equal to eager calls."""
    c = _Case("paged", 32, 8, [3000, 500], [20, 9], 4, max_len=4000)
    c.lens = [3000, 500]
    kv = c.kv()
    out, ws = torch.zeros((c.total, 32, 128), dtype=torch.bfloat16, device=DEV), cb.alloc_tree_workspace(c.params, 4000, c.total, c.max_nodes)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            cb.tree_attn(c.params, c.q, kv, c.tree, out, ws)
    torch.cuda.synchronize()
    for lens in ([3000, 500], [2900, 400], [3020, 30], [29, 509]):
        kv.seq_lens.copy_(_i32(lens))
        graph.replay()
        torch.cuda.synchronize()
        c.lens = lens
        eager = c.out()
        assert torch.equal(out, eager)
        torch.randn(1000, device=DEV).sum().item()
    with torch.cuda.stream(s):
        other = c.out()
    assert torch.equal(other, eager)


def test_one_node_is_a_decode_step():
    """A tree of the step's token alone: what full attention and sparse attention give, up to the order of sums and the weights' rounding."""
    c = _Case("paged", 32, 8, [2000, 777], [1, 1], 4)
    ws = cb.alloc_workspace(c.params, c.max_len)
    full = torch.zeros((2, 32, 128), dtype=torch.bfloat16, device=DEV)
    cb.full_attn(c.params, c.q.contiguous(), c.kv(), full, ws)
    torch.cuda.synchronize()
    want, mass = c.want()
    ref.assert_attention(c.out(), want, mass, "tree")
    ref.assert_attention(full, want, mass, "full")


# ---- commit

@pytest.mark.parametrize("layout", ["paged", "head_major", "token_major"])
@pytest.mark.parametrize("layers,max_path", [(1, 1), (2, 5), (3, 16), (35, 17), (2, 100)])
def test_commit(layout, layers, max_path):
    print("commit", layout, layers, max_path, flush=True)
    rng = np.random.default_rng(layers + max_path)
    B, G, nodes = 4, 3, max(8, max_path + 20)
    base = [0, 13, 200, 40]
    caches = [_cache(layout, B, G, [b + nodes for b in base], 5 + i) for i in range(layers)]
    table = caches[0][2]
    path, n_path = np.zeros((B, max_path), dtype=np.int64), [max_path, max(1, max_path // 2), 0, max_path]
    for b in range(B):
        path[b] = np.sort(rng.choice(nodes, size=max_path, replace=False))
    path[3] = np.arange(max_path) + (1 if max_path > 1 else 0)              # every row is the next one's goal
    kvs = [cb.KvCache(k, v, _i32([b + nodes for b in base]), max(base) + nodes, table) for k, v, _ in caches]
    want = []
    for k, v, _ in caches:
        for x in (k, v):
            y = x.clone()
            for b in range(B):
                for i in range(n_path[b]):
                    src = base[b] + int(path[b, i])
                    _put(y, table, b, base[b] + i, x[b, :, src] if table is None else x[int(table[b, src // PAGE]), :, src % PAGE])
            want.append(y)
    keep = torch.zeros(B, dtype=torch.int32, device=DEV)
    cb.kv_commit(cb.make_params(B, G, G, 1, 0), kvs, _i32(base), _i32(path), _i32(n_path), keep)
    torch.cuda.synchronize()
    assert keep.tolist() == [b + n for b, n in zip(base, n_path)]
    for (k, v, _), i in zip(caches, range(layers)):
        assert torch.equal(k, want[2 * i]) and torch.equal(v, want[2 * i + 1])


def test_commit_leaves_out_what_is_out_of_range():
    k, v, table = _cache("paged", 2, 2, [40, 40], 3)
    kv = cb.KvCache(k, v, _i32([40, 40]), 40, table)
    before = k.clone()
    keep = torch.zeros(2, dtype=torch.int32, device=DEV)
    cb.kv_commit(cb.make_params(2, 2, 2, 1, 0), [kv], _i32([-7, 38]), _i32([[0, 1, 2], [1, 9, 1 << 30]]), _i32([3, 1 << 30]), keep)
    torch.cuda.synchronize()
    want = before.clone()
    _put(want, table, 1, 38, before[int(table[1, 2]), :, 39 % PAGE])
    assert torch.equal(k, want) and keep.tolist() == [-4, 41]
