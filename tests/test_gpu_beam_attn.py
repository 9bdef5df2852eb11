"""Attention over a group's pages against every row's own attention in 64 bits."""
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


class Case:
    def __init__(self, groups, width, H, G, prompt, tail, seed, samples=False, fused=False, lens=None, table=None, columns=0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        if lens is None:
            lens, table, used = ref.family(rng, groups, width, prompt, tail, columns, samples)
        else:
            used = int(np.max(table)) + 1
        self.n_pages = used + 3
        order = rng.permutation(self.n_pages)
        table = np.where(table >= 0, order[table], -1)
        self.width, self.H, self.G, self.lens, self.table = width, H, G, lens, table
        self.k, self.v = (torch.randn((self.n_pages, G, 16, 128), generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
        q = torch.randn((len(lens), H + 2 * G if fused else H, 128), generator=gen, device=DEV).to(torch.bfloat16)
        self.q = q[:, :H]
        self.params = cb.make_params(len(lens), H, G, 1, 0)

    def run(self, max_len=None, out=None):
        max_len = max_len or max(1, int(max(self.lens)))
        s = cb.SharedPages.empty(len(self.lens), self.width, max_len, self.n_pages)
        kv = cb.KvCache(self.k, self.v, _i32(self.lens), max_len, _i32(self.table))
        cb.shared_pages(kv.block_table, kv.seq_lens, max_len, self.n_pages, s, cb.alloc_pages_workspace(len(self.lens), max_len))
        ws = torch.full((cb.beam_attn_workspace_bytes(self.params, max_len, s),), 255, dtype=torch.uint8, device=DEV)
        out = torch.full((len(self.lens), self.H, 128), 7.0, dtype=torch.bfloat16, device=DEV) if out is None else out
        cb.beam_attn(self.params, self.q, kv, s, out, ws)
        torch.cuda.synchronize()
        return out

    def rows(self, b):
        pos = torch.arange(int(self.lens[b]), device=DEV)
        page = torch.as_tensor(self.table[b], device=DEV)[pos // 16]
        return tuple(x[page, :, pos % 16].transpose(0, 1).double() for x in (self.k, self.v))

    def check(self, out, rows=None):
        # A weight is off by 2^-15; scores (128 products) and sums of up to 2^13 terms in 32 bits move a weight by less than 2^-11 of itself; the output is rounded to bf16.
        for b in range(len(self.lens)) if rows is None else rows:
            if self.lens[b] <= 0:
                assert not out[b].any(), f"row {b} has no tokens"
                continue
            want, mass = ref.attention(self.q[b], *self.rows(b), 128 ** -0.5)
            tol = (2.0 ** -14 + 2.0 ** -11) * mass + 2.0 ** -8 * want.abs() + 1e-30
            err = (out[b].double() - want).abs()
            assert (err <= tol).all(), f"row {b} of {self.lens[b]} tokens: worst {float((err / tol).max()):.3g} of the bound"


@pytest.mark.parametrize("H,G", [(8, 8), (8, 4), (32, 8), (16, 2), (4, 1)])
@pytest.mark.parametrize("groups,width,prompt,tail", [(1, 1, 1, 0), (1, 4, 700, 90), (3, 2, 40, 3), (2, 7, 1500, 300), (1, 32, 500, 100), (5, 12, 333, 64), (1, 8, 6000, 500)])
@pytest.mark.parametrize("samples", [False, True])
def test_attention(H, G, groups, width, prompt, tail, samples):
    print("beam attn", H, G, groups, width, prompt, tail, samples, flush=True)
    c = Case(groups, width, H, G, prompt, tail, groups + width + H, samples, fused=samples)
    c.check(c.run())


@pytest.mark.parametrize("width,H,G", [(4, 32, 8), (16, 32, 8), (32, 16, 2)])
def test_attention_of_many_groups_of_any_length(width, H, G):
    print("many", width, flush=True)
    c = Case(192 // width, width, H, G, 900, 700, width, samples=True, columns=125)
    c.lens[::5] = 0
    c.lens[1] = min(c.lens[1], 1)
    c.check(c.run(max_len=2000))


def test_attention_with_heavy_tokens():
    """A few tokens outweigh all others: in the common prompt, at its end, in a row's own tokens."""
    c = Case(2, 4, 32, 8, 2000, 300, 77)
    for b in range(8):
        for pos in (0, int(c.lens[b]) // 2, int(c.lens[b]) - 1):
            c.k[c.table[b, pos // 16], :, pos % 16] = (c.q[b].float().view(8, 4, 128).sum(1)).to(torch.bfloat16)
    c.check(c.run())


@pytest.mark.parametrize("width,H,G", [(4, 16, 4), (12, 16, 4), (20, 8, 2), (32, 8, 1)])
def test_what_a_row_does_not_attend_to_does_not_reach_it(width, H, G):
    """NaN and infinities behind the rows' ends, in pages of other rows and of nobody."""
    print("foreign", width, flush=True)
    c = Case(2, width, H, G, 400, 200, width, samples=True)
    seen = torch.zeros((c.n_pages, 16), dtype=torch.int64, device=DEV)
    for b, n in enumerate(c.lens):
        pos = torch.arange(int(n), device=DEV)
        seen[torch.as_tensor(c.table[b], device=DEV)[pos // 16], pos % 16] |= 1
    for x, bad in ((c.k, math.nan), (c.v, math.inf)):
        x.copy_(torch.where((seen == 0)[:, None, :, None], torch.tensor(bad, dtype=torch.bfloat16, device=DEV), x))
    c.check(c.run())
    # rows 1 and 2 hold tokens of their own that are not finite
    for b, bad in ((1, math.nan), (2, math.inf)):
        if c.lens[b] == 0 or (c.lens[b] - 1) // 16 < ref.pages(int(min(c.lens[:width]))):
            c.lens[b] = max(c.lens[b], 1)
    fresh = [b for b in range(width) if c.lens[b] and sum(c.table[o, (c.lens[b] - 1) // 16] == c.table[b, (c.lens[b] - 1) // 16] for o in range(width) if (c.lens[o] + 15) // 16 > (c.lens[b] - 1) // 16) == 1]
    one, two = fresh[0], fresh[1]
    c.v[c.table[one, (c.lens[one] - 1) // 16], :, (c.lens[one] - 1) % 16, 5] = math.nan
    c.v[c.table[two, (c.lens[two] - 1) // 16], :, (c.lens[two] - 1) % 16, 6] = math.inf
    out = c.run()
    c.check(out, [b for b in range(2 * width) if b not in (one, two)])
    assert out[one, :, 5].isnan().all() and (out[two, :, 6] == math.inf).all()
    assert out[one, :, 6:].isfinite().all() and out[two, :, 7:].isfinite().all()


def test_a_row_whose_pages_nobody_shares():
    c = Case(1, 3, 8, 8, 0, 0, 5, lens=np.array([50, 33, 16]), table=np.array([[0, 1, 2, 3], [4, 5, 6, -1], [7, -1, -1, -1]]))
    c.check(c.run())


def test_tables_that_name_no_page():
    """Holes of a table are left out; the other tokens count."""
    c = Case(1, 4, 8, 2, 300, 100, 6)
    table = c.table.copy()
    hole = 2
    c.table[:, hole] = -1
    out = c.run()
    c.table = table
    rows = Case.rows

    def without(b):
        keep = torch.arange(int(c.lens[b]), device=DEV) // 16 != hole
        return tuple(x[:, keep] for x in rows(c, b))
    c.rows = without
    c.check(out)


def test_lists_out_of_range_do_no_harm():
    """Counts and entries that mean nothing: some output, nothing read or written elsewhere; then the right list again."""
    c = Case(2, 4, 8, 2, 300, 100, 8)
    max_len = int(c.lens.max())
    kv = cb.KvCache(c.k, c.v, _i32(c.lens), max_len, _i32(c.table))
    s = cb.SharedPages.empty(8, 4, max_len, c.n_pages)
    ws = cb.alloc_beam_attn_workspace(c.params, max_len, s)
    out = torch.zeros((9, 8, 128), dtype=torch.bfloat16, device=DEV)
    rng = np.random.default_rng(0)
    for count in ([[1 << 30, 1 << 30], [-5, 7]], [[20, -3], [9, 9]]):
        s.entries.copy_(_i32(rng.integers(-(1 << 31), 1 << 31, s.entries.shape, dtype=np.int64).astype(np.int32)))
        s.count.copy_(_i32(count))
        cb.beam_attn(c.params, c.q, kv, s, out, ws)
        torch.cuda.synchronize()
    assert not out[8].any()
    cb.shared_pages(kv.block_table, kv.seq_lens, max_len, c.n_pages, s, cb.alloc_pages_workspace(8, max_len))
    cb.beam_attn(c.params, c.q, kv, s, out, ws)
    torch.cuda.synchronize()
    c.check(out[:8])
