"""Beam search's plain statements hold what they promise, and the library refuses what its calls cannot serve.  No kernel is launched by anything in this file."""
import ctypes

import numpy as np
import pytest

import beam_reference as ref
from paper_2508_07101_amd import binding as cb

FAKE = 0x10000


@pytest.mark.parametrize("width", [1, 2, 4, 7, 32])
@pytest.mark.parametrize("free", [3, 40])
def test_every_page_is_held_or_queued_once(width, free):
    """Steps of random searches: a page is in the queue, or held by rows of one group in one column; rows write to pages of their own; their tokens are their ancestors'."""
    rng = np.random.default_rng(width + free)
    groups = max(1, 8 // width)
    lens, table, used = ref.family(rng, groups, width, 60, 40, columns=12)
    n_pages = used + free
    ring = np.concatenate([np.arange(used, n_pages), np.full(used, -1)])
    state, tokens = [0, free], {}                                # (page, place) -> what is written there
    for b, n in enumerate(lens):
        for t in range(n):
            tokens.setdefault((int(table[b, t // 16]), t % 16), (int(table[b, t // 16]), t))
    story = [[tokens[int(table[b, t // 16]), t % 16] for t in range(n)] for b, n in enumerate(lens)]
    for step in range(30):
        parents, ended = rng.integers(-1 if step % 5 == 0 else 0, width, groups * width), rng.random(groups * width) < 0.2
        before = story
        lens, slots, copies, table, ring, state, granted = ref.fork(width, lens, parents, ended, step % 7 != 3, table, ring, state, table)
        for f, t, n, _ in copies:
            for i in range(n):
                tokens[t, i] = tokens[f, i]
        story = []
        for b in range(groups * width):
            g = b // width
            s = g * width + parents[b]
            story.append(list(before[b]) if not granted[g] else [] if parents[b] < 0 else list(before[s]))
            if slots[b] >= 0:
                assert slots[b] not in [x for o, x in enumerate(slots) if o != b]
                tokens[slots[b] // 16, slots[b] % 16] = (step, b)
                story[b].append((step, b))
            assert len(story[b]) == lens[b]
        held = {}
        for b in range(groups * width):
            for j in range(ref.pages(lens[b])):
                held.setdefault(int(table[b, j]), set()).add((b // width, j))
            assert [tokens[int(table[b, t // 16]), t % 16] for t in range(lens[b])] == story[b]
        queued = [int(ring[(state[0] + i) % n_pages]) for i in range(state[1])]
        assert all(len(where) == 1 for where in held.values())
        assert sorted(list(held) + queued) == list(range(n_pages))


def _beams(**kw):
    d = dict(logits=FAKE, dtype=0, stride=100, rows=8, width=4, vocab=100, n=4, end_token=-1)
    d.update(kw)
    return cb.CusaBeams(**d)


def _select(b, scores=FAKE, ended=None, out_scores=FAKE + 4096, parents=FAKE, tokens=FAKE, out_ended=None, ws=FAKE, size=1 << 30):
    return cb.load().cusa_beam_select(ctypes.byref(b), scores, ended, out_scores, parents, tokens, out_ended, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), cb.ERR_INVALID_ARG), (dict(logits=FAKE + 1), cb.ERR_INVALID_ARG), (dict(dtype=3), cb.ERR_INVALID_ARG), (dict(dtype=2, logits=FAKE + 2), cb.ERR_INVALID_ARG),
    (dict(stride=99), cb.ERR_INVALID_ARG), (dict(rows=0), cb.ERR_INVALID_ARG), (dict(rows=9), cb.ERR_INVALID_ARG), (dict(width=0), cb.ERR_INVALID_ARG),
    (dict(rows=66, width=33), cb.ERR_UNSUPPORTED), (dict(n=0), cb.ERR_INVALID_ARG), (dict(n=65), cb.ERR_UNSUPPORTED), (dict(vocab=0), cb.ERR_INVALID_ARG),
    (dict(rows=65536), cb.ERR_UNSUPPORTED), (dict(end_token=-2), cb.ERR_INVALID_ARG), (dict(end_token=100), cb.ERR_INVALID_ARG)])
def test_selections_that_cannot_be(kw, status):
    assert _select(_beams(**kw)) == status


def test_selection_arguments():
    b = _beams()
    for kw in (dict(scores=None), dict(out_scores=None), dict(parents=None), dict(tokens=None), dict(ws=None), dict(ws=FAKE + 16), dict(ended=FAKE)):
        assert _select(b, **kw) == cb.ERR_INVALID_ARG, kw
    assert _select(b, size=255) == cb.ERR_WORKSPACE_TOO_SMALL
    wider = _beams(n=8, end_token=5)                             # in place only where the outputs are the next step's rows
    assert _select(wider, out_scores=FAKE) == cb.ERR_INVALID_ARG
    assert _select(wider, ended=FAKE + 8192, out_ended=FAKE + 8192) == cb.ERR_INVALID_ARG
    assert cb.load().cusa_beam_select(None, FAKE, None, FAKE, FAKE, FAKE, None, FAKE, 1 << 30, None) == cb.ERR_INVALID_ARG
    n = ctypes.c_size_t(0)
    for args, status in (((0, 10, 4), cb.ERR_INVALID_ARG), ((4, 0, 4), cb.ERR_INVALID_ARG), ((4, 10, 65), cb.ERR_UNSUPPORTED), ((4, 10, 4), cb.OK)):
        assert cb.load().cusa_beam_workspace_bytes(*args, ctypes.byref(n)) == status
    assert n.value > 0 and n.value % 256 == 0
    assert cb.load().cusa_beam_workspace_bytes(4, 10, 4, None) == cb.ERR_INVALID_ARG


def _pool(**kw):
    d = dict(layout=cb.KV_PAGED, batch=8, capacity=0, block_table=FAKE, max_pages=10, page_size=16, n_pages=100, ring=FAKE, state=FAKE, state_out=FAKE)
    d.update(kw)
    return cb.CusaPool(**d)


def _fork(pool, width=4, held=FAKE, parents=FAKE, ended=None, table_out=FAKE, lens=FAKE + 4096, slots=FAKE, copies=FAKE, ws=FAKE, size=1 << 30):
    return cb.load().cusa_kv_fork(ctypes.byref(pool) if pool else None, width, held, parents, ended, 1, table_out, lens, slots, copies, None, ws, size, None)


def test_forks_that_cannot_be():
    assert _fork(None) == cb.ERR_INVALID_ARG
    assert _fork(_pool(layout=cb.KV_CONTIGUOUS, capacity=100)) == cb.ERR_UNSUPPORTED
    assert _fork(_pool(page_size=32)) == cb.ERR_UNSUPPORTED
    for kw in (dict(block_table=None), dict(ring=None), dict(state=None), dict(state_out=None), dict(max_pages=0), dict(n_pages=0), dict(batch=0)):
        assert _fork(_pool(**kw)) == cb.ERR_INVALID_ARG, kw
    for width, status in ((0, cb.ERR_INVALID_ARG), (3, cb.ERR_INVALID_ARG), (-4, cb.ERR_INVALID_ARG)):
        assert _fork(_pool(), width) == status
    assert _fork(_pool(batch=33), 33) == cb.ERR_UNSUPPORTED
    for kw in (dict(held=None), dict(parents=None), dict(table_out=None), dict(lens=None), dict(slots=None), dict(copies=None), dict(copies=FAKE + 4), dict(lens=FAKE),
               dict(ended=FAKE + 4096), dict(ws=None), dict(ws=FAKE + 8)):
        assert _fork(_pool(), **kw) == cb.ERR_INVALID_ARG, kw
    need = cb.fork_workspace_bytes(8, 10)
    assert need > 0 and _fork(_pool(), size=need - 1) == cb.ERR_WORKSPACE_TOO_SMALL
    assert [cb.fork_workspace_bytes(*a) for a in ((0, 10), (8, 0), (65536, 1), (65535, 1 << 20))] == [0] * 4


def _paged(**kw):
    d = dict(k=FAKE, v=FAKE, layout=cb.KV_PAGED, stride_batch=0, stride_head=0, stride_token=0, block_table=FAKE, max_pages=10, page_size=16, n_pages=100, seq_lens=FAKE, max_seq_len=160)
    d.update(kw)
    return cb.CusaKv(**d)


def test_copies_that_cannot_be():
    p, lib = cb.make_params(1, 8, 8, 1, 0), cb.load()

    def call(kv, n=1, copies=FAKE, layers=1):
        return lib.cusa_kv_copy(ctypes.byref(p), layers, ctypes.byref(kv) if kv else None, copies, n, None)

    assert call(_paged(layout=cb.KV_CONTIGUOUS, stride_token=128)) == cb.ERR_UNSUPPORTED
    assert call(_paged(page_size=8)) == cb.ERR_UNSUPPORTED
    assert call(_paged(k=None)) == cb.ERR_INVALID_ARG and call(_paged(v=FAKE + 8)) == cb.ERR_INVALID_ARG and call(_paged(n_pages=0)) == cb.ERR_INVALID_ARG
    assert call(_paged(n_pages=1 << 30)) == cb.ERR_UNSUPPORTED and call(_paged(), n=1 << 24) == cb.ERR_UNSUPPORTED
    assert call(None) == cb.ERR_INVALID_ARG and call(_paged(), layers=0) == cb.ERR_INVALID_ARG and call(_paged(), n=-1) == cb.ERR_INVALID_ARG
    assert call(_paged(), copies=None) == cb.ERR_INVALID_ARG and call(_paged(), copies=FAKE + 8) == cb.ERR_INVALID_ARG
    assert call(_paged(block_table=None, seq_lens=None, max_seq_len=0), n=0) == cb.OK    # nothing to copy, and nothing else is read
    assert lib.cusa_kv_copy(None, 1, ctypes.byref(_paged()), FAKE, 1, None) == cb.ERR_INVALID_ARG


def _list(**kw):
    d = dict(width=4, max_entries=40, entries=FAKE, count=FAKE)
    d.update(kw)
    return cb.CusaShared(**d)


BAD_LISTS = [(dict(width=0), cb.ERR_INVALID_ARG), (dict(width=3), cb.ERR_INVALID_ARG), (dict(entries=None), cb.ERR_INVALID_ARG), (dict(entries=FAKE + 8), cb.ERR_INVALID_ARG),
             (dict(count=None), cb.ERR_INVALID_ARG), (dict(max_entries=39), cb.ERR_INVALID_ARG), (dict(max_entries=0), cb.ERR_INVALID_ARG)]


def _pages_call(kv, shared, batch=8, ws=FAKE, size=1 << 30):
    return cb.load().cusa_shared_pages(ctypes.byref(kv) if kv else None, batch, ctypes.byref(shared) if shared else None, ws, size, None)


def test_lists_that_cannot_be():
    for kw, status in BAD_LISTS:
        assert _pages_call(_paged(), _list(**kw)) == status, kw
    assert _pages_call(None, _list()) == cb.ERR_INVALID_ARG and _pages_call(_paged(), None) == cb.ERR_INVALID_ARG
    for kw, status in ((dict(layout=cb.KV_CONTIGUOUS), cb.ERR_UNSUPPORTED), (dict(page_size=32), cb.ERR_UNSUPPORTED), (dict(layout=7), cb.ERR_INVALID_ARG), (dict(block_table=None), cb.ERR_INVALID_ARG),
                       (dict(seq_lens=None), cb.ERR_INVALID_ARG), (dict(max_seq_len=0), cb.ERR_INVALID_ARG), (dict(max_seq_len=161), cb.ERR_INVALID_ARG), (dict(n_pages=0), cb.ERR_INVALID_ARG),
                       (dict(n_pages=1 << 32), cb.ERR_UNSUPPORTED)):
        assert _pages_call(_paged(**kw), _list()) == status, kw
    assert _pages_call(_paged(), _list(), batch=0) == cb.ERR_INVALID_ARG
    assert _pages_call(_paged(), _list(width=33), batch=66) == cb.ERR_UNSUPPORTED
    assert _pages_call(_paged(), _list(), ws=None) == cb.ERR_INVALID_ARG and _pages_call(_paged(), _list(), ws=FAKE + 1) == cb.ERR_INVALID_ARG
    assert _pages_call(_paged(), _list(), size=cb.pages_workspace_bytes(8, 160) - 1) == cb.ERR_WORKSPACE_TOO_SMALL


def _attn(kv=None, shared=None, q=FAKE, stride=4 * 128, out=FAKE, ws=FAKE, size=1 << 40, **params):
    p = cb.make_params(**{**dict(batch=8, n_q_heads=4, n_kv_heads=2, budget=1, window=0), **params})
    return cb.load().cusa_beam_attn(ctypes.byref(p), q, stride, ctypes.byref(kv or _paged()), ctypes.byref(shared or _list()), out, ws, size, None)


def test_attention_that_cannot_be():
    for kw, status in BAD_LISTS:
        assert _attn(shared=_list(**kw)) == status, kw
    for kw, status in ((dict(q=None), cb.ERR_INVALID_ARG), (dict(q=FAKE + 8), cb.ERR_INVALID_ARG), (dict(stride=4 * 128 - 8), cb.ERR_INVALID_ARG), (dict(stride=4 * 128 + 4), cb.ERR_INVALID_ARG),
                       (dict(out=None), cb.ERR_INVALID_ARG), (dict(out=FAKE + 2), cb.ERR_INVALID_ARG), (dict(ws=None), cb.ERR_INVALID_ARG), (dict(ws=FAKE + 16), cb.ERR_INVALID_ARG),
                       (dict(size=0), cb.ERR_WORKSPACE_TOO_SMALL), (dict(n_q_heads=6), cb.ERR_UNSUPPORTED), (dict(batch=10), cb.ERR_INVALID_ARG), (dict(head_dim=64), cb.ERR_UNSUPPORTED),
                       (dict(kv=_paged(layout=cb.KV_CONTIGUOUS, stride_token=128)), cb.ERR_UNSUPPORTED), (dict(kv=_paged(seq_lens=None)), cb.ERR_INVALID_ARG),
                       (dict(kv=_paged(n_pages=1 << 30), shared=_list(max_entries=1 << 20)), cb.ERR_UNSUPPORTED), (dict(kv=_paged(page_size=1)), cb.ERR_UNSUPPORTED)):
        assert _attn(**kw) == status, kw
    p, n = cb.make_params(8, 4, 2, 1, 0), ctypes.c_size_t(0)
    lib = cb.load()
    assert lib.cusa_beam_attn_workspace_bytes(ctypes.byref(p), 160, ctypes.byref(_list()), ctypes.byref(n)) == cb.OK and n.value > 0
    assert lib.cusa_beam_attn_workspace_bytes(ctypes.byref(p), 160, None, ctypes.byref(n)) == cb.ERR_INVALID_ARG
    assert lib.cusa_beam_attn_workspace_bytes(ctypes.byref(p), 0, ctypes.byref(_list()), ctypes.byref(n)) == cb.ERR_INVALID_ARG
    assert lib.cusa_beam_attn_workspace_bytes(ctypes.byref(p), 160, ctypes.byref(_list(width=5)), ctypes.byref(n)) == cb.ERR_INVALID_ARG


def test_attention_over_long_lists():
    """Groups of up to 2^19 pages, whatever the lengths; a launch of up to 2^24 workgroups."""
    lib, n = cb.load(), ctypes.c_size_t(0)

    def need(batch, width, max_entries, max_len, H=4, G=2):
        return lib.cusa_beam_attn_workspace_bytes(ctypes.byref(cb.make_params(batch, H, G, 1, 0)), max_len, ctypes.byref(_list(width=width, max_entries=max_entries)), ctypes.byref(n))

    assert need(32, 32, 1 << 19, 1 << 20) == cb.OK and n.value > 0
    assert need(32, 32, (1 << 19) + 1, 1 << 20) == cb.ERR_UNSUPPORTED
    assert need(32, 32, 1 << 30, 1 << 18) == cb.OK and need(32, 32, 1 << 30, (1 << 18) + 1) == cb.ERR_UNSUPPORTED
    assert need(4, 4, 1 << 30, 1 << 21) == cb.OK and need(4, 4, 1 << 30, (1 << 21) + 1) == cb.ERR_UNSUPPORTED
    assert _attn(batch=65535, n_q_heads=512, n_kv_heads=512, stride=512 * 128, shared=_list(width=1, max_entries=10)) == cb.ERR_UNSUPPORTED


@pytest.mark.parametrize("rows,G", [(1, 8), (16, 8), (256, 1), (65535, 1)])
def test_workspaces_grow_with_the_lists(rows, G):
    """A piece for each 128 tokens and no more than 64: a workspace made for longer sequences serves shorter ones."""
    lib, width = cb.load(), 1
    sizes = []
    for max_len in (1, 16, 1000, 2048, 2049, 4096, 4097, 10000, 1 << 17, 1 << 20, 1 << 23):
        n = ctypes.c_size_t(0)
        p = cb.make_params(rows, 4 * G, G, 1, 0)
        assert lib.cusa_beam_attn_workspace_bytes(ctypes.byref(p), max_len, ctypes.byref(_list(width=width, max_entries=1 << 30)), ctypes.byref(n)) == cb.OK
        sizes.append(n.value)
    assert sizes == sorted(sizes) and sizes[-1] <= rows * 4 * G * 64 * 130 * 4 + rows * 4 + 1024
