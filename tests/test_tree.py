"""Trees of drafted tokens, what needs no GPU: refusals (no kernel is launched by anything in this file), workspaces, the references."""
import ctypes

import numpy as np
import pytest
import torch

import tree_reference as ref
from paper_2508_07101_amd import binding as cb

FAKE = ctypes.c_void_p(0x10000)
OTHER = ctypes.c_void_p(0x20000)


def _paged(**more):
    f = dict(k=0x1000, v=0x2000, layout=cb.KV_PAGED, stride_batch=0, stride_head=0, stride_token=0, block_table=0x4000, max_pages=256,
             page_size=16, n_pages=1000, seq_lens=0x3000, max_seq_len=4096)
    f.update(more)
    return cb.CusaKv(*f.values())


def _flat(**more):
    f = dict(k=0x1000, v=0x2000, layout=cb.KV_CONTIGUOUS, stride_batch=8 * 4096 * 128, stride_head=4096 * 128, stride_token=128, block_table=None,
             max_pages=0, page_size=0, n_pages=0, seq_lens=0x3000, max_seq_len=4096)
    f.update(more)
    return cb.CusaKv(*f.values())


def _pool(**more):
    f = dict(layout=cb.KV_PAGED, batch=4, capacity=0, block_table=0x4000, max_pages=256, page_size=16, n_pages=1000, ring=0x5000, state=0x6000,
             state_out=0x6000)
    f.update(more)
    return cb.CusaPool(*f.values())


def _plan(pool, held=FAKE, keep=FAKE, add=OTHER, max_tokens=100, lens=FAKE, tok_start=FAKE, slots=FAKE, ws=FAKE, ws_bytes=1 << 20):
    return cb.load().cusa_kv_plan(ctypes.byref(pool), held, keep, add, max_tokens, lens, tok_start, slots, ws, ws_bytes, None)


@pytest.mark.parametrize("pool,status", [
    (dict(batch=0), cb.ERR_INVALID_ARG), (dict(batch=70000), cb.ERR_UNSUPPORTED), (dict(layout=7), cb.ERR_INVALID_ARG),
    (dict(page_size=32), cb.ERR_UNSUPPORTED), (dict(block_table=None), cb.ERR_INVALID_ARG), (dict(ring=None), cb.ERR_INVALID_ARG),
    (dict(state=None), cb.ERR_INVALID_ARG), (dict(state_out=None), cb.ERR_INVALID_ARG), (dict(max_pages=0), cb.ERR_INVALID_ARG),
    (dict(n_pages=0), cb.ERR_INVALID_ARG), (dict(n_pages=1 << 31), cb.ERR_UNSUPPORTED),
    (dict(batch=60000, max_pages=60000), cb.ERR_UNSUPPORTED), (dict(layout=cb.KV_CONTIGUOUS, capacity=0), cb.ERR_INVALID_ARG)])
def test_plan_refuses_pools(pool, status):
    assert _plan(_pool(**pool)) == status


@pytest.mark.parametrize("args,status", [
    (dict(held=None), cb.ERR_INVALID_ARG), (dict(keep=None), cb.ERR_INVALID_ARG), (dict(add=None), cb.ERR_INVALID_ARG),
    (dict(lens=None), cb.ERR_INVALID_ARG), (dict(tok_start=None), cb.ERR_INVALID_ARG), (dict(slots=None), cb.ERR_INVALID_ARG),
    (dict(max_tokens=-1), cb.ERR_INVALID_ARG), (dict(ws=None), cb.ERR_INVALID_ARG), (dict(ws=ctypes.c_void_p(0x10010)), cb.ERR_INVALID_ARG),
    (dict(ws_bytes=256), cb.ERR_WORKSPACE_TOO_SMALL)])
def test_plan_refuses_arguments(args, status):
    assert _plan(_pool(), **args) == status


def _append(kv=None, rows=None, slots=FAKE, params=None):
    r = dict(k=0x7000, v=0x8000, dtype=0, n=10, stride_token=1024, stride_head=128)
    r.update(rows or {})
    p = params or cb.make_params(4, 32, 8, 1, 0)
    return cb.load().cusa_kv_append(ctypes.byref(p), ctypes.byref(kv or _paged()), slots, ctypes.byref(cb.CusaRows(*r.values())), None)


@pytest.mark.parametrize("rows,status", [
    (dict(k=None), cb.ERR_INVALID_ARG), (dict(k=0x7008), cb.ERR_INVALID_ARG), (dict(dtype=3), cb.ERR_INVALID_ARG), (dict(n=-1), cb.ERR_INVALID_ARG),
    (dict(stride_token=1028), cb.ERR_INVALID_ARG), (dict(stride_head=4), cb.ERR_INVALID_ARG), (dict(stride_token=-1024), cb.ERR_INVALID_ARG),
    (dict(dtype=2, stride_token=1026), cb.ERR_INVALID_ARG), (dict(n=0), cb.OK)])
def test_append_refuses_rows(rows, status):
    assert _append(rows=rows) == status


@pytest.mark.parametrize("kv,status", [
    (_paged(page_size=8), cb.ERR_UNSUPPORTED), (_paged(n_pages=0), cb.ERR_INVALID_ARG), (_paged(k=0x1004), cb.ERR_INVALID_ARG),
    (_flat(stride_token=64), cb.ERR_INVALID_ARG), (_flat(max_seq_len=0), cb.ERR_INVALID_ARG), (_paged(n_pages=1 << 30), cb.ERR_UNSUPPORTED),
    (_flat(layout=9), cb.ERR_INVALID_ARG)])
def test_append_refuses_caches(kv, status):
    assert _append(kv=kv) == status


def test_append_needs_slots_and_known_heads():
    assert _append(slots=None) == cb.ERR_INVALID_ARG
    assert _append(params=cb.make_params(4, 32, 8, 1, 0, head_dim=64)) == cb.ERR_UNSUPPORTED


@pytest.mark.parametrize("args,status", [
    (dict(batch=0), cb.ERR_INVALID_ARG), (dict(batch=70000), cb.ERR_UNSUPPORTED), (dict(parents=None), cb.ERR_INVALID_ARG), (dict(masks=None), cb.ERR_INVALID_ARG),
    (dict(base=None), cb.ERR_INVALID_ARG), (dict(max_nodes=0), cb.ERR_INVALID_ARG), (dict(max_nodes=257), cb.ERR_UNSUPPORTED), (dict(max_tokens=0), cb.ERR_INVALID_ARG)])
def test_masks_refuse(args, status):
    f = dict(batch=2, base=FAKE, tok_start=FAKE, parents=FAKE, max_tokens=20, max_nodes=10, masks=FAKE, positions=FAKE, stream=None)
    f.update(args)
    assert cb.load().cusa_tree_masks(*f.values()) == status


def _attn(kv=None, tree=None, params=None, q=FAKE, idx=None, cnt=None, out=FAKE, ws=FAKE, ws_bytes=1 << 34):
    t = dict(tok_start=0x9000, masks=0xa000, max_tokens=240, max_nodes=60, q_stride=32 * 128)
    t.update(tree or {})
    p = params or cb.make_params(4, 32, 8, 1024, 256)
    return cb.load().cusa_tree_attn(ctypes.byref(p), q, ctypes.byref(kv or _paged()), ctypes.byref(cb.CusaTree(*t.values())), idx, cnt, out, ws, ws_bytes, None)


@pytest.mark.parametrize("args,status", [
    (dict(q=None), cb.ERR_INVALID_ARG), (dict(q=ctypes.c_void_p(0x10008)), cb.ERR_INVALID_ARG), (dict(out=None), cb.ERR_INVALID_ARG),
    (dict(ws=None), cb.ERR_INVALID_ARG), (dict(ws=ctypes.c_void_p(0x10010)), cb.ERR_INVALID_ARG), (dict(ws_bytes=256), cb.ERR_WORKSPACE_TOO_SMALL),
    (dict(idx=FAKE), cb.ERR_INVALID_ARG), (dict(cnt=FAKE), cb.ERR_INVALID_ARG), (dict(tree=dict(tok_start=None)), cb.ERR_INVALID_ARG),
    (dict(tree=dict(masks=None)), cb.ERR_INVALID_ARG), (dict(tree=dict(max_nodes=257)), cb.ERR_UNSUPPORTED), (dict(tree=dict(max_nodes=0)), cb.ERR_INVALID_ARG),
    (dict(tree=dict(max_tokens=0)), cb.ERR_INVALID_ARG), (dict(tree=dict(q_stride=31 * 128)), cb.ERR_INVALID_ARG), (dict(tree=dict(q_stride=32 * 128 + 4)), cb.ERR_INVALID_ARG),
    (dict(kv=_paged(max_pages=10)), cb.ERR_INVALID_ARG), (dict(kv=_paged(block_table=None)), cb.ERR_INVALID_ARG), (dict(kv=_paged(seq_lens=None)), cb.ERR_INVALID_ARG),
    (dict(kv=_flat(max_seq_len=(1 << 30) + 1)), cb.ERR_UNSUPPORTED), (dict(params=cb.make_params(4, 32, 8, 1024, 2048)), cb.ERR_INVALID_ARG),
    (dict(params=cb.make_params(4, 24, 8, 1024, 256)), cb.ERR_UNSUPPORTED)])
def test_attention_refuses(args, status):
    assert _attn(**args) == status


@pytest.mark.parametrize("args,status", [
    (dict(n_layers=0), cb.ERR_INVALID_ARG), (dict(base=None), cb.ERR_INVALID_ARG), (dict(path=None), cb.ERR_INVALID_ARG), (dict(n_path=None), cb.ERR_INVALID_ARG),
    (dict(max_path=0), cb.ERR_INVALID_ARG), (dict(keep=FAKE), cb.ERR_INVALID_ARG), (dict(kv=_paged(block_table=None)), cb.ERR_INVALID_ARG),
    (dict(kv=_flat(k=None)), cb.ERR_INVALID_ARG)])
def test_commit_refuses(args, status):
    f = dict(n_layers=2, kv=_paged(), base=FAKE, path=OTHER, max_path=4, n_path=OTHER, keep=None)
    f.update(args)
    kvs = (cb.CusaKv * 2)(_paged(), f["kv"])
    p = cb.make_params(4, 32, 8, 1, 0)
    assert cb.load().cusa_kv_commit(ctypes.byref(p), f["n_layers"], kvs, f["base"], f["path"], f["max_path"], f["n_path"], f["keep"], None) == status


def test_binding_refuses_tensors_of_other_types():
    i32 = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        cb.kv_plan(i32.long(), i32, i32, i32, torch.zeros(5, dtype=torch.int32), torch.zeros(8, dtype=torch.int64), i32)
    with pytest.raises(ValueError):
        cb.tree_masks(i32[:1], i32[:2], i32, torch.zeros((4, 1), dtype=torch.int32), i32, 4)
    kv = cb.KvCache(torch.zeros((1, 8, 32, 128), dtype=torch.bfloat16), torch.zeros((1, 8, 32, 128), dtype=torch.bfloat16), i32[:1], 32)
    p = cb.make_params(1, 8, 8, 1, 0)
    for bad in (torch.zeros((2, 8, 128), dtype=torch.float64), torch.zeros((2, 4, 128)), torch.zeros((2, 8, 256))[:, :, ::2]):
        with pytest.raises(ValueError):
            cb.kv_append(p, kv, torch.zeros(2, dtype=torch.int64), bad, bad)


@pytest.mark.parametrize("H,G,B", [(32, 8, 1), (8, 8, 3), (64, 8, 1), (16, 8, 64)])
def test_a_workspace_serves_every_smaller_batch_of_tokens(H, G, B):
    p = cb.make_params(B, H, G, 2048, 512)
    for length in (1, 300, 4096, 32768):
        before = 0
        for nodes in (1, 3, 4, 5, 8, 9, 16, 17, 32, 33, 60, 64, 65, 128, 129, 200, 256):
            n = cb.tree_workspace_bytes(p, length, B * nodes, nodes)
            assert n >= before and n % 256 == 0
            before = n
    before = 0
    for length in list(range(1, 9000, 97)) + [32768, 131072]:
        n = cb.tree_workspace_bytes(p, length, B * 60, 60)
        assert n >= before
        before = n


def test_reference_plan_by_hand():
    table = np.full((3, 4), -1, dtype=np.int32)
    table[0, :2], table[1, :1] = [5, 7], [2]
    ring = np.array([9, 9, 0, 1, 3, 4, 6, 9], dtype=np.int32)          # free: 0 1 3 4 6, from entry 2 on
    # sequence 0: 20 tokens, keeps 18, adds 15 (pages 5, 7 and a new one); 1 ends; 2 starts with 33
    lens, start, slots, t, r, s = ref.plan([20, 9, 0], [18, 0, 0], [15, 0, 33], 60, 64, table, ring, [2, 5])
    assert lens == [33, 0, 33] and start == [0, 15, 15, 48]
    assert t[0].tolist() == [5, 7, 0, -1] and t[2].tolist() == [1, 3, 4, -1]
    assert slots[:3] == [7 * 16 + 2, 7 * 16 + 3, 7 * 16 + 4] and slots[14] == 0 and slots[15] == 16 and slots[47] == 4 * 16 and slots[48:] == [-1] * 12
    assert s == [6, 2] and r[6] == 6 and r[7] == 2


def test_binding_refuses_caches_of_other_shapes_and_host_memory():
    i32, p = torch.zeros(4, dtype=torch.int32), cb.make_params(2, 8, 8, 1, 0)
    rows, slots = torch.zeros((2, 8, 128), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int64)

    def cache(shape, dtype=torch.bfloat16, table=None):
        return cb.KvCache(torch.zeros(shape, dtype=dtype), torch.zeros(shape, dtype=dtype), i32, 16, table)

    for kv in (cache((2, 4, 16, 128)), cache((1, 8, 16, 128)), cache((2, 8, 16, 64)), cache((2, 8, 16, 128), torch.float16),
               cache((2, 8, 16, 128)), cache((9, 8, 16, 128), table=torch.zeros((1, 4), dtype=torch.int32))):
        with pytest.raises(ValueError):
            cb.KvCommit(p, [kv])
        with pytest.raises(ValueError):
            cb.kv_append(p, kv, slots, rows, rows)
        with pytest.raises(ValueError):
            cb.tree_attn(p, rows, kv, cb.Tree(i32, torch.zeros((2, 1), dtype=torch.int64), 2), rows, i32)
    pool = cb.PagePool.empty(2, 3, 5, "cpu")
    with pytest.raises(ValueError, match="on the GPU"):
        cb.kv_plan(i32[:2], i32[:2], i32[2:], i32[:2], i32[:3], slots, i32, pool)
    with pytest.raises(ValueError, match="on the GPU"):
        cb.tree_masks(i32, i32[:2], i32, torch.zeros((4, 1), dtype=torch.int64), None, 4)
