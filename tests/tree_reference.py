"""Plain statements of the calls for trees of drafted tokens: whole numbers in Python, attention in 64 bits."""
import numpy as np
import torch

PAGE = 16


def pages(n):
    return (n + PAGE - 1) // PAGE


def plan(held, keep, add, max_tokens, cap, table=None, ring=None, state=None):
    """lens, tok_start, slots and, for a paged cache, the table, ring and state after the call."""
    n_pages = len(ring) if ring is not None else 0
    if table is not None:
        table, ring = table.copy(), ring.copy()
        first, avail = int(state[0]), min(max(int(state[1]), 0), n_pages)
        first = first if 0 <= first < n_pages else 0
    lens, starts, slots, taken, asked, needed, pushed = [], [0], [], 0, 0, 0, []
    old_table = None if table is None else table.copy()
    for b in range(len(held)):
        h = min(max(int(held[b]), 0), cap)
        k = min(max(int(keep[b]), 0), h)
        a = max(int(add[b]), 0)
        ok = k + a <= cap
        if ok:
            asked += a
            ok = asked <= max_tokens
        if ok and table is not None:
            need = max(pages(k + a) - pages(h), 0)
            needed += need
            ok = need == 0 or needed <= avail
        n = a if ok else 0
        if table is not None:
            for p in range(pages(h), pages(k + n)):
                table[b, p] = ring[(first + taken) % n_pages]
                taken += 1
            pushed += [old_table[b, p] for p in range(pages(k + n), pages(h))]
        for pos in range(k, k + n):
            if table is None:
                slots.append((b << 32) + pos)
            else:
                page = int(table[b, pos // PAGE])
                slots.append(page * PAGE + pos % PAGE if 0 <= page < n_pages else -1)
        lens.append(k + n)
        starts.append(starts[-1] + n)
    slots += [-1] * (max_tokens - len(slots))
    if table is None:
        return lens, starts, slots
    for i, p in enumerate(pushed):
        ring[(first + avail + i) % n_pages] = p
    return lens, starts, slots, table, ring, [(first + taken) % n_pages, min(avail - taken + len(pushed), n_pages)]


def masks(parents, words):
    """Of one tree: bit rows [n][words] (uint64) and depths."""
    rows, depth = np.zeros((len(parents), words), dtype=np.uint64), []
    for j, p in enumerate(parents):
        up = 0 <= p < j
        if up:
            rows[j] = rows[p]
        rows[j, j // 64] |= np.uint64(1) << np.uint64(j % 64)
        depth.append(depth[p] + 1 if up else 0)
    return rows, depth


def allowed(bits, n):
    """Truth values [n][n] of mask rows (uint64 [n][words])."""
    return np.unpackbits(np.ascontiguousarray(bits).view(np.uint8), axis=1, bitorder="little")[:, :n].astype(bool)


def cache_rows(x, table, b, pos):
    """K or V of sequence b at positions pos, [G][len][128] in 64 bits."""
    if table is None:
        return x[b][:, pos].double()
    t = table[b].long()
    return x[t[pos // PAGE], :, pos % PAGE].transpose(0, 1).double()


def attention(q, k, v, before, n, node_bits, scale):
    """One sequence.  q [n][H][d]; k, v [G][before + n][d] in 64 bits: the looked-at prefix, then the nodes; node_bits [n][n].
    Returns the output and sum(weight * |v|), which bounds what rounded weights can do to it."""
    H, G = q.shape[1], k.shape[0]
    ok = torch.cat([torch.ones((n, before), dtype=torch.bool, device=q.device), torch.as_tensor(node_bits, device=q.device)], dim=1)
    out, mass = (torch.zeros(q.shape, dtype=torch.float64, device=q.device) for _ in range(2))
    for h in range(H):
        kv = h // (H // G)
        x = (q[:, h].double() @ k[kv].t().contiguous()) * scale
        x = x.masked_fill(~ok, float("-inf"))
        top = x.amax(-1, keepdim=True)
        w = torch.exp(x - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        total = w.sum(-1, keepdim=True)
        w = torch.where(total > 0, w / total, torch.zeros_like(w))
        out[:, h], mass[:, h] = w @ v[kv], w @ v[kv].abs()
    return out, mass


def assert_attention(got, want, mass, what):
    """A weight rounded to bf16 is off by 2^-8 of itself at most, the output by 2^-8 of itself, and sums of 128 products and of
    the weights in 32 bits move a weight by far less than 2^-10 of itself."""
    tol = (2.0 ** -8 + 2.0 ** -10) * mass + 2.0 ** -8 * want.abs() + 1e-30
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside the bound, worst {float((err / tol).max()):.3g} of it"
