"""The forms of tree attention for many rows (65 to 256 of a KV head, tree_shapes.py) over all layouts, masks, values that are not finite and entries that
name nothing, against 64 bits."""
import numpy as np
import pytest
import torch

import tree_reference as ref
from test_gpu_tree import PAGE, _Case, _i32, _put
from tree_shapes import SHAPES

pytestmark = pytest.mark.gpu
DEV = "cuda"
LAYOUTS = ["paged", "head_major", "token_major"]


def _case(layout, name, seed, **more):
    s = SHAPES[name]
    return _Case(layout, s["H"], s["G"], s["before"], s["n"], seed, budget=s["budget"], **more)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("kind", ["tree", "any"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_attention(layout, name, kind):
    _case(layout, name, 21, kind=kind, fused=kind == "tree").check(f"{layout} {name} {kind}")


@pytest.mark.parametrize("name", ["steps", "lists", "two workgroups"])
def test_nodes_that_attend_to_no_node(name):
    c = _case("token_major", name, 22, kind="none")
    got = c.check(name)
    assert (got[: c.n[0]] == 0).all()                                       # the first sequence has no prefix


def _rows_of_nodes(c):
    at = 0
    for b, n in enumerate(c.n):
        yield b, n, slice(at, at + n)
        at += n


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("name", ["steps", "pieces", "lists", "long lists", "128 rows", "two workgroups of lists"])
def test_values_that_are_not_finite_reach_only_those_that_attend_to_them(layout, name):
    c = _case(layout, name, 23)
    clean = c.out()
    for val in (float("nan"), -float("inf")):
        save_k, save_v = c.k.clone(), c.v.clone()
        for b, n, _ in _rows_of_nodes(c):
            pos = c.before[b] + n // 2
            row = (c.v[b, :, pos] if c.table is None else c.v[int(c.table[b, pos // PAGE]), :, pos % PAGE]).clone()
            row[:, 5:90:3] = val
            _put(c.v, c.table, b, pos, row)
        got = c.out()
        hit = torch.zeros(128, dtype=torch.bool, device=DEV)
        hit[5:90:3] = True
        for b, n, own in _rows_of_nodes(c):
            seen = torch.as_tensor(ref.allowed(c.bits[b], n)[:, n // 2], device=DEV)
            assert torch.equal(got[own][~seen], clean[own][~seen]), f"{val}: sequence {b}"
            assert torch.equal(got[own][seen][..., ~hit], clean[own][seen][..., ~hit])
            there = got[own][seen][..., hit]
            assert (there.isnan() if val != val else there == val).all()
        c.v = save_v
        for b, n, _ in _rows_of_nodes(c):
            _put(c.k, c.table, b, c.before[b] + n // 2, torch.full((c.G, 128), val, dtype=torch.bfloat16, device=DEV))
        got = c.out()
        for b, n, own in _rows_of_nodes(c):
            seen = torch.as_tensor(ref.allowed(c.bits[b], n)[:, n // 2], device=DEV)
            assert torch.equal(got[own][~seen], clean[own][~seen]), f"{val} in a key: sequence {b}"
        c.k = save_k


@pytest.mark.parametrize("name", ["steps", "pieces", "128 rows", "two workgroups"])
def test_entries_that_name_no_page_are_left_out(name):
    """Every fifth page of the prefixes, the first one of some among them."""
    c = _case("paged", name, 24)
    table = c.table.clone()
    gone = [[p for p in range(b % 5, c.before[b] // PAGE, 5)] for b in range(len(c.n))]
    for b, pages in enumerate(gone):
        for i, p in enumerate(pages):
            c.table[b, p] = [-1, 1 << 30, c.k.shape[0]][i % 3]
    got = c.out()
    for b, n, own in _rows_of_nodes(c):
        pos = torch.as_tensor([t for t in range(c.before[b] + n) if t // PAGE not in gone[b]], device=DEV)
        want, mass = ref.attention(c.q[own], ref.cache_rows(c.k, table, b, pos), ref.cache_rows(c.v, table, b, pos), len(pos) - n, n, ref.allowed(c.bits[b], n), 128 ** -0.5)
        ref.assert_attention(got[own], want, mass, f"{name} sequence {b}")


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("name", ["lists", "long lists", "128 rows of lists", "two workgroups of lists"])
def test_list_entries_outside_the_prefix_are_left_out(layout, name):
    c = _case(layout, name, 25)
    for b in range(len(c.n)):
        entries, outside = c.sets[b].copy(), [-1, c.before[b], c.before[b] + c.n[b] - 1, 2 ** 31 - 1, -(1 << 31)]
        out = np.arange(b % 4, len(entries), 7)
        for i, e in enumerate(out):
            entries[e] = outside[i % 5]
        c.idx[b, : len(entries)] = _i32(entries)
        c.sets[b] = np.delete(entries, out)
    c.check(f"{layout} {name}")


def test_the_single_token_of_a_transposed_projection():
    """[H, 1, 128] seen as [1, H, 128]: the stride of the one token means nothing."""
    c = _Case("head_major", 8, 2, [300], [1], 26)
    want = c.out()
    c.q = c.q.reshape(8, 1, 128).transpose(0, 1)
    assert c.q.stride(0) == 128 and torch.equal(c.out(), want)
