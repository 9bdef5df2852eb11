"""Plain statements of the calls for beam search: whole numbers in Python, selection and attention in 64 bits."""
import math

import numpy as np
import torch

PAGE = 16


def pages(n):
    return (n + PAGE - 1) // PAGE


def select(logits, scores, ended, width, n, end):
    """Of every group [(value, row, token)], best first.  logits: float64 [rows, vocab]."""
    out = []
    for g in range(0, len(scores), width):
        found = []
        for b in range(width):
            s, x = float(scores[g + b]), logits[g + b]
            if not math.isfinite(s):
                continue
            if ended is not None and ended[g + b]:
                found.append((s, b, 0, end))
                continue
            top = x.max() if not np.isnan(x).any() else math.nan
            if not math.isfinite(top):
                continue
            v = s + ((x - top) - math.log(np.exp(x - top).sum()))
            for i, t in enumerate(np.lexsort((np.arange(len(x)), -x))[:n]):   # (a row's own go by the logits: beside a large score 64 bits may not tell them apart)
                if x[t] > -math.inf:
                    found.append((float(v[t]), b, i, int(t)))
        out.append([(v, b, t) for v, b, _, t in sorted(found, key=lambda c: (-c[0], c[1], c[2]))[:n]])
    return out


def fork(width, held, parents, ended, grow, table, ring, state, table_out):
    """lens, slots, copies, table_out, ring, state, granted."""
    B, C = table.shape
    n_pages = len(ring)
    first, avail = int(state[0]), min(max(int(state[1]), 0), n_pages)
    first = first if 0 <= first < n_pages else 0
    table_out, ring = table_out.copy(), ring.copy()
    held = [min(max(int(h), 0), C * PAGE) for h in held]
    lens, slots, copies, granted, needed, taken, freed = list(held), [-1] * B, [[-1, -1, 0, 0] for _ in range(B)], [], 0, 0, []
    for g in range(0, B, width):
        rows = range(g, g + width)
        src = {b: g + int(parents[b]) if 0 <= parents[b] < width else None for b in rows}
        kept = {b: held[src[b]] if src[b] is not None else 0 for b in rows}
        wants = {b: bool(src[b] is not None and grow and not (ended is not None and ended[b])) for b in rows}
        writers, holders = {}, {}                                # of (column, page)
        for b in rows:
            if src[b] is None:
                continue
            for j in range(pages(kept[b])):
                holders.setdefault((j, int(table[src[b], j])), []).append(b)
            if wants[b] and kept[b] % PAGE:
                writers.setdefault((kept[b] // PAGE, int(table[src[b], kept[b] // PAGE])), []).append(b)
        new = {}
        for b in rows:
            if not wants[b]:
                continue
            j = kept[b] // PAGE
            if kept[b] % PAGE == 0:
                new[b] = "fresh"
            else:
                page = int(table[src[b], j])
                if 0 <= page < n_pages and not (writers[j, page] == holders[j, page] and b == writers[j, page][0]):
                    new[b] = "copy"
        fits = all(kept[b] + wants[b] <= C * PAGE for b in rows)
        needed += len(new) if fits else 0
        ok = fits and (not new or needed <= avail)
        granted.append(int(ok))
        for b in rows:
            if not ok:
                table_out[b, : pages(held[b])] = table[b, : pages(held[b])]
                continue
            lens[b] = kept[b] + wants[b]
            if src[b] is not None:
                table_out[b, : pages(kept[b])] = table[src[b], : pages(kept[b])]
            j = kept[b] // PAGE
            if b in new:
                page = int(ring[(first + taken) % n_pages])
                taken += 1
                if new[b] == "copy":
                    copies[b] = [int(table[src[b], j]), page, kept[b] % PAGE, 0]
                table_out[b, j] = page
            if wants[b] and 0 <= table_out[b, j] < n_pages:
                slots[b] = int(table_out[b, j]) * PAGE + kept[b] % PAGE
        if ok:
            stay = {s for s in src.values() if s is not None}
            for j in range(C):
                for b in rows:
                    page = int(table[b, j])
                    if j >= pages(held[b]) or not 0 <= page < n_pages or b in stay:
                        continue
                    if not any(j < pages(held[o]) and table[o, j] == page and (o in stay or o < b) for o in rows):
                        freed.append(page)
    for i, page in enumerate(freed):
        ring[(first + avail + i) % n_pages] = page
    return lens, slots, copies, table_out, ring, [(first + taken) % n_pages, min(avail - taken + len(freed), n_pages)], granted


def shared(width, lens, table, n_pages, max_len):
    """Of every group its entries [page, column, bits, 0], and how many at the front all rows attend to as a whole."""
    out = []
    for g in range(0, len(lens), width):
        n = [min(max(int(x), 0), max_len) for x in lens[g: g + width]]
        there = [b for b in range(width) if n[b]]
        entries, whole = [], None
        for j in range(pages(max(n))):
            of = {}
            for b in there:
                if j < pages(n[b]) and 0 <= table[g + b, j] < n_pages:
                    of.setdefault(int(table[g + b, j]), []).append(b)
            for page, holders in of.items():                     # (in order of the lowest row)
                if whole is None and (holders != there or min(n[b] for b in there) < (j + 1) * PAGE):
                    whole = len(entries)
                entries.append([page, j, sum(1 << b for b in holders), 0])
        out.append((entries, len(entries) if whole is None else whole))
    return out


def attention(q, k, v, scale):
    """One row: q [H][d], k and v [G][L][d] in 64 bits.  The output and sum(weight * |v|), which bounds what inexact weights can do to it."""
    H, G = q.shape[0], k.shape[0]
    x = torch.matmul(q.double().view(G, H // G, -1), k.transpose(1, 2).contiguous()) * scale
    w = torch.softmax(x, dim=-1)
    return torch.matmul(w, v).reshape(H, -1), torch.matmul(w, v.abs()).reshape(H, -1)


def family(rng, groups, width, prompt, tail, columns=0, samples=False):
    """Lengths and a table of pages numbered as they come: rows of a group share whole pages up to where they part from the row that they descend from."""
    lens = np.zeros(groups * width, dtype=np.int64)
    rows, used = [], 0
    for g in range(groups):
        p = int(rng.integers(0, prompt + 1))
        own, t = [], int(rng.integers(0, tail + 1))
        for b in range(width):
            n = p + (int(rng.integers(0, tail + 1)) if samples else t)
            lens[g * width + b] = n
            shared_pages = 0
            if b:
                up = int(rng.integers(0, b))
                part = p if samples else int(rng.integers(p, p + t + 1))
                shared_pages = min(part, n, int(lens[g * width + up])) // PAGE
                row = own[up][:shared_pages]
            else:
                row = []
            fresh = pages(n) - len(row)
            row = row + list(range(used, used + fresh))
            used += fresh
            own.append(row)
        rows += own
    columns = max(columns, max((len(r) for r in rows), default=0) + 1)
    table = np.full((len(rows), columns), -1, dtype=np.int64)
    for b, r in enumerate(rows):
        table[b, : len(r)] = r
    return lens, table, used
