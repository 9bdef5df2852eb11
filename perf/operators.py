"""Performance cases of decoding with trees of drafted tokens: what is timed, on which inputs, and the same in plain torch.

A speculative step drafts a small tree of tokens for every sequence and checks all its nodes in one pass.  Its calls:

* ``plan``    block tables and the slot map of the new tokens, from the sequences' lengths (``binding.kv_plan``): once a
  step for the drafted nodes, and once for the prompts of requests that come in.
* ``append``  new K and V rows of one layer written at those slots (``binding.kv_append``).
* ``masks``   which nodes a node attends to, and the nodes' positions, from the trees' parents (``binding.tree_masks``).
* ``attn``    attention of all nodes over the cached prefix, or the part of it that a selection layer chose, and over
  their own branch (``binding.tree_attn``); every layer of the model, by far the most of the step's time.
* ``commit``  the accepted branch's rows moved together in all layers' caches (``binding.kv_commit``).

Sizes: those of the decode cases (1 to 64 sequences of up to 131 072 cached tokens, 8 to 64 query heads over 8 KV heads,
head-major, token-major and paged caches), trees of 1 to 256 nodes, prompts up to the cached lengths.  Caches and
queries are bf16; new rows come as bf16, fp16 or fp32.  There is no backward pass: the path only decodes.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEVICE = "cuda"
D = 128
PAGE = 16


def _lib():
    from paper_2508_07101_amd import binding
    return binding


# ---- the cases

def _attn(name, batch, heads, seq_len, nodes, **more):
    c = dict(name=name, kind="attn", batch=batch, heads=heads, kv_heads=8, seq_len=seq_len, min_len=0, nodes=nodes, min_nodes=0,
             budget=0, layout="head_major", fused=False, len_seed=1)
    c.update(more)
    return c


def listed():
    return [
        # the drafted trees of a serving batch get their pages and slots: a few pages, where latency is all
        dict(name="plan_step", kind="plan", batch=64, seq_len=32768, min_len=8192, add=64, min_add=1, drop=40, layout="paged", spare=1.5, len_seed=2),
        # the prompts of 64 new requests get theirs: 1.3 million slots
        dict(name="plan_prompts", kind="plan", batch=64, seq_len=0, min_len=0, add=32768, min_add=8192, drop=0, layout="paged", spare=1.1, len_seed=3),
        # one layer's rows of a serving batch's trees, straight from a fused projection
        dict(name="append_step", kind="append", batch=64, heads=32, kv_heads=8, seq_len=1024, add=64, min_add=1, layout="paged", dtype="bfloat16", fused=True, len_seed=2),
        # one layer's rows of eight long prompts, rotated in 32 bits
        dict(name="append_prompts", kind="append", batch=8, heads=32, kv_heads=8, seq_len=0, add=16384, min_add=16384, layout="head_major", dtype="float32", fused=False, len_seed=1),
        # a single user's tree: the smallest call there is
        dict(name="masks_single", kind="masks", batch=1, seq_len=32768, nodes=60, min_nodes=60, len_seed=1),
        # a serving batch with the widest trees
        dict(name="masks_serving", kind="masks", batch=64, seq_len=32768, nodes=256, min_nodes=30, len_seed=1),
        # a short draft over a short chat's token set: a sparse layer where latency counts
        _attn("attn_sparse_small", 1, 32, 4096, 5, min_nodes=5, budget=1024),
        # a single user far into a long trace, a full tree, a dense layer
        _attn("attn_full_single", 1, 32, 32768, 60, min_nodes=60),
        # eight long traces in step, sparse layers with the largest budget, queries from a fused projection
        _attn("attn_sparse_batch", 8, 32, 16384, 64, min_nodes=33, budget=4096, fused=True),
        # a serving batch of ragged requests and trees in pages, a dense layer: the most work of all
        _attn("attn_full_serving", 64, 32, 32768, 64, min_len=8192, min_nodes=1, layout="paged"),
        # the accepted branch of a single user's tree, all 36 layers
        dict(name="commit_single", kind="commit", batch=1, kv_heads=8, seq_len=4096, nodes=60, min_nodes=60, path=5, layers=36, layout="head_major", len_seed=1),
        # those of a serving batch, in pages, long branches
        dict(name="commit_serving", kind="commit", batch=64, kv_heads=8, seq_len=700, nodes=128, min_nodes=40, path=16, layers=32, layout="paged", len_seed=4),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    kind = rng.choice(["attn", "attn", "attn", "attn", "plan", "append", "masks", "commit"])
    batch, layout = log(1, 64), rng.choice(["head_major", "token_major", "paged", "paged"])
    seed = rng.randrange(1 << 30)
    if kind == "plan":
        if rng.random() < 0.5:
            seq = log(100, 131072)
            return dict(kind=kind, batch=batch, seq_len=seq, min_len=seq // 3, add=log(1, 256), min_add=0, drop=rng.choice([0, 7, 100]),
                        layout=layout, spare=rng.choice([0.3, 1.0, 1.5]), len_seed=seed)
        add = log(30, min(131072, 1300000 // batch))
        return dict(kind=kind, batch=batch, seq_len=0, min_len=0, add=add, min_add=add // rng.choice([1, 2, 9]), drop=0, layout=layout,
                    spare=rng.choice([0.6, 1.0, 1.2]), len_seed=seed)
    if kind == "append":
        add = log(1, min(16384, 131072 // batch))
        return dict(kind=kind, batch=batch, heads=rng.choice([8, 16, 32, 64]), kv_heads=8, seq_len=log(1, 1500), add=add, min_add=add // 2, layout=layout,
                    dtype=rng.choice(["bfloat16", "bfloat16", "float16", "float32"]), fused=rng.random() < 0.5, len_seed=seed)
    if kind == "masks":
        nodes = log(1, 256)
        return dict(kind=kind, batch=batch, seq_len=log(1, 131072), nodes=nodes, min_nodes=rng.choice([0, nodes]), len_seed=seed)
    if kind == "commit":
        batch, layers = log(1, 32), rng.randint(1, 36)
        nodes = log(2, 256)
        return dict(kind=kind, batch=batch, kv_heads=8, seq_len=log(1, 150000 // (batch * layers)) + 16, nodes=nodes, min_nodes=nodes // 2,
                    path=log(1, 32), layers=layers, layout=layout, len_seed=seed)
    heads = rng.choice([8, 16, 32, 32, 64])
    seq_len = log(1, min(131072, 1250000 // batch))
    # no more products than the serving batch: its trees' nodes times tokens, about 40 million for 32 heads
    nodes = log(1, min(256, max(1, 40000000 * 32 // (heads * batch * seq_len))))
    return dict(kind=kind, batch=batch, heads=heads, kv_heads=8, seq_len=seq_len, min_len=rng.choice([0, seq_len // 2, seq_len // 16]), nodes=nodes,
                min_nodes=rng.choice([0, nodes // 2, nodes]), budget=rng.choice([0, 0, 256, 1024, 2048, 4096]), layout=layout,
                fused=rng.random() < 0.5, len_seed=seed)


# ---- inputs

def _ragged(c, most, least, salt):
    """One number a sequence: part of the case, not of the seed."""
    rng = np.random.default_rng(c["len_seed"] * 8 + salt)
    return [int(v) for v in rng.integers(min(least, most), most + 1, size=c["batch"])]


def _lengths(c):
    return _ragged(c, c["seq_len"], c["min_len"] if c.get("min_len") else c["seq_len"], 0)


def _nodes(c):
    n = _ragged(c, c["nodes"], c["min_nodes"], 1)
    return n if sum(n) else [1] + n[1:]


def _adds(c):
    n = _ragged(c, c["add"], c["min_add"], 2)
    return n if sum(n) else [1] + n[1:]


def _gen(seed, salt):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed % (1 << 40) * 16 + salt)
    return g


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _starts(n):
    return _ints([0] + list(np.cumsum(n)))


def _parents(n_list, seed):
    """Drafted trees, level by level: the first node hangs on the last cached token, every other on one of the last level's
    better candidates."""
    rng = np.random.default_rng(seed)
    out = []
    for n in n_list:
        par = np.full(n, -1, dtype=np.int64)
        lo, hi = 0, 1                                     # the last level's nodes
        at = 1
        while at < n:
            width = min(n - at, int(rng.integers(1, 2 * (hi - lo) + 3)))
            par[at: at + width] = np.sort(lo + np.minimum((rng.random(width) ** 2 * (hi - lo)).astype(np.int64), hi - lo - 1))
            lo, hi, at = at, at + width, at + width
        out.append(par)
    return out


def _mask_words(par, words):
    """Bit i of row j: node j attends to node i, itself and its ancestors."""
    rows = np.zeros((len(par), words), dtype=np.uint64)
    for j, p in enumerate(par):
        if p >= 0:
            rows[j] = rows[p]
        rows[j, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return rows


def _cache(c, cap, gen, layers=0):
    """K and V of one layer (or of several) in the case's layout, and the block table of a paged one."""
    lead = (layers,) if layers else ()
    B, G = c["batch"], c["kv_heads"]
    table = None
    if c["layout"] == "paged":
        pages = [(n + PAGE - 1) // PAGE for n in cap]
        n_pages = max(1, sum(pages))
        perm = torch.randperm(n_pages, generator=gen, device=DEVICE).to(torch.int32).cpu()
        table = torch.zeros((B, max(1, max(pages))), dtype=torch.int32)
        at = 0
        for b, n in enumerate(pages):
            table[b, :n] = perm[at: at + n]
            at += n
        table = table.to(DEVICE)
        shape = lead + (n_pages, G, PAGE, D)
    else:
        shape = lead + ((B, max(cap), G, D) if c["layout"] == "token_major" else (B, G, max(cap), D))
    k, v = (torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.bfloat16) for _ in range(2))
    if c["layout"] == "token_major":
        k, v = k.transpose(-3, -2), v.transpose(-3, -2)
    return k, v, table


def _plan_inputs(c, seed):
    B = c["batch"]
    lens, most_add = _lengths(c), _adds(c)
    drop = [min(d, n) for d, n in zip(_ragged(c, c["drop"], 0, 3), lens)]     # rejected nodes of the step before

    def pages(n):
        return (n + PAGE - 1) // PAGE

    # room for the case's numbers; the seed takes a few tokens off everywhere
    s = {"max_tokens": sum(most_add), "capacity": max(max(n - d + a for n, d, a in zip(lens, drop, most_add)), max(lens))}
    n_pages = sum(pages(n) for n in lens)
    free = max(1, int(sum(max(0, pages(n - d + a) - pages(n)) for n, d, a in zip(lens, drop, most_add)) * c["spare"]))
    fewer = np.random.default_rng(seed).integers(0, 1000, size=B)
    add = [a - min(int(f) * max(a, 1) // 8000, a - 1) if a > 1 else a for a, f in zip(most_add, fewer)]
    lens = [n - min(int(f) % 16, n - d) for n, d, f in zip(lens, drop, fewer)]
    s.update(held=_ints(lens), keep=_ints([n - d for n, d in zip(lens, drop)]), add=_ints(add), lens=_ints([0] * B), tok_start=_ints([0] * (B + 1)),
             slots=torch.zeros(s["max_tokens"], dtype=torch.int64, device=DEVICE))
    if c["layout"] == "paged":
        used = [pages(n) for n in lens]
        n_pages += free
        free = n_pages - sum(used)
        perm = torch.randperm(n_pages, generator=_gen(seed, 0), device=DEVICE).to(torch.int32)
        max_pages = pages(s["capacity"]) + 1
        pi = torch.arange(max_pages, device=DEVICE)
        u = torch.tensor(used, device=DEVICE)
        at = (u.cumsum(0) - u)[:, None] + pi
        s["table"] = torch.where(pi < u[:, None], perm[at.clamp(max=n_pages - 1)], torch.full_like(perm[:1], -1)).contiguous()
        first = int(np.random.default_rng(seed).integers(0, n_pages))
        ring = torch.full((n_pages,), -1, dtype=torch.int32, device=DEVICE)
        ring[(first + torch.arange(free, device=DEVICE)) % n_pages] = perm[sum(used):]
        s.update(ring=ring, state=_ints([first, free]), state_out=_ints([0, 0]), n_pages=n_pages)
    return s


def _slots_of(c, lens, n, table):
    """Slots of tokens lens[b] .. lens[b] + n[b] - 1."""
    out = []
    for b in range(c["batch"]):
        pos = torch.arange(lens[b], lens[b] + n[b], device=DEVICE)
        out.append(table[b][pos // PAGE].long() * PAGE + pos % PAGE if table is not None else (b << 32) + pos)
    return torch.cat(out)


def _append_inputs(c, seed):
    gen = _gen(seed, 1)
    lens, n = _lengths(c), _adds(c)
    cap = [a + b for a, b in zip(lens, n)]
    k, v, table = _cache(c, cap, gen)
    t, G, kind = sum(n), c["kv_heads"], getattr(torch, c["dtype"])
    if c["fused"]:                                        # rows of [q | k | v]
        qkv = torch.randn((t, c["heads"] + 2 * G, D), generator=gen, device=DEVICE, dtype=torch.float32).to(kind)
        k_new, v_new = qkv[:, c["heads"]: c["heads"] + G], qkv[:, c["heads"] + G:]
    else:
        k_new, v_new = (torch.randn((t, G, D), generator=gen, device=DEVICE, dtype=torch.float32).to(kind) for _ in range(2))
    return {"k": k, "v": v, "table": table, "slots": _slots_of(c, lens, n, table), "k_new": k_new, "v_new": v_new, "lens": _ints(cap), "cap": max(cap)}


def _masks_inputs(c, seed):
    n = _nodes(c)
    par = np.concatenate(_parents(n, seed))
    words = (c["nodes"] + 63) // 64
    grown = np.random.default_rng(seed).integers(0, 1000, size=c["batch"])
    return {"base": _ints([b + int(g) for b, g in zip(_lengths(c), grown)]), "tok_start": _starts(n), "parents": _ints(par.tolist()), "max_nodes": c["nodes"],
            "masks": torch.zeros((sum(n), words), dtype=torch.int64, device=DEVICE), "positions": _ints([0] * sum(n))}


def _attn_inputs(c, seed):
    gen = _gen(seed, 2)
    B, H, G = c["batch"], c["heads"], c["kv_heads"]
    pre, n = _lengths(c), _nodes(c)
    lens = [a + b for a, b in zip(pre, n)]
    k, v, table = _cache(c, lens, gen)
    t = sum(n)
    q = torch.randn((t, H + 2 * G if c["fused"] else H, D), generator=gen, device=DEVICE, dtype=torch.bfloat16)[:, :H]
    # a few tokens that the heads attend to above all others
    rng = np.random.default_rng(seed)
    start = np.cumsum([0] + n)
    for b in range(B):
        if not n[b] or not lens[b]:
            continue
        heavy = (q[start[b]].float().view(G, -1, D).sum(1) * (2.0 / math.sqrt(H // G))).to(torch.bfloat16)
        for pos in rng.integers(0, lens[b], size=4).tolist():
            if table is not None:
                k[int(table[b, pos // PAGE]), :, pos % PAGE] = heavy
            else:
                k[b, :, pos] = heavy
    words = (c["nodes"] + 63) // 64
    masks = np.concatenate([_mask_words(p, words) for p in _parents(n, seed)])
    s = {"q": q, "k": k, "v": v, "table": table, "lens": _ints(lens), "max_len": max(lens), "tok_start": _starts(n), "max_nodes": c["nodes"],
         "masks": torch.from_numpy(masks.view(np.int64)).to(DEVICE), "n": n, "pre": pre, "idx": None, "cnt": None,
         "out": torch.zeros((t, H, D), dtype=torch.bfloat16, device=DEVICE)}
    if c["budget"]:
        # what a selection layer chose for the tree's first node: some history, a quarter of the budget as the window, which
        # ends with that node
        K = c["budget"]
        idx = torch.zeros((B, K), dtype=torch.int32, device=DEVICE)
        for b, p in enumerate(pre):
            if p + 1 <= K:
                idx[b, : p + 1] = torch.arange(p + 1, device=DEVICE, dtype=torch.int32)
                continue
            lead = p + 1 - K // 4
            hist = torch.rand(lead, generator=gen, device=DEVICE).topk(K - K // 4).indices.sort().values
            idx[b] = torch.cat([hist, torch.arange(lead, p + 1, device=DEVICE)]).to(torch.int32)
        s["idx"], s["cnt"] = idx, _ints([min(p + 1, K) for p in pre])
    return s


def _commit_inputs(c, seed):
    gen = _gen(seed, 3)
    B, n = c["batch"], _nodes(c)
    pre = _lengths(c)
    k, v, table = _cache(c, [a + b for a, b in zip(pre, n)], gen, c["layers"])
    rng = np.random.default_rng(seed)
    path = np.zeros((B, c["path"]), dtype=np.int32)
    taken = []
    for b in range(B):
        # a branch: its first nodes stand where they belong, the others anywhere behind the branch's length
        m = int(rng.integers(0, min(c["path"], n[b]) + 1))
        stay = int(rng.integers(0, m + 1))
        far = min(m - stay, n[b] - m)
        path[b, :stay] = np.arange(stay)
        path[b, stay: stay + far] = np.sort(m + rng.choice(n[b] - m, size=far, replace=False)) if far else 0
        taken.append(stay + far)
    return {"k": k, "v": v, "table": table, "base": _ints(pre), "lens": _ints([a + b for a, b in zip(pre, n)]), "max_len": max(a + b for a, b in zip(pre, n)),
            "path": torch.from_numpy(path).to(DEVICE), "n_path": _ints(taken), "keep": _ints([0] * B)}


_INPUTS = {"plan": _plan_inputs, "append": _append_inputs, "masks": _masks_inputs, "attn": _attn_inputs, "commit": _commit_inputs}


def prepare(case, seed):
    c = case
    s = _INPUTS[c["kind"]](c, seed)
    s.update(kind=c["kind"], kv_heads=c.get("kv_heads", 8), budget=c.get("budget", 0))
    if own:
        cb = _lib()
        if c["kind"] == "plan" and c["layout"] == "paged":
            s["pool"] = cb.PagePool(s["table"], s["ring"], s["state"])
        if c["kind"] == "plan":
            s["ws"] = cb.alloc_plan_workspace(c["batch"], DEVICE)
        if c["kind"] in ("append", "attn"):
            s["params"] = cb.make_params(c["batch"], c["heads"], c["kv_heads"], c.get("budget") or 1, 0)
            s["kv"] = cb.KvCache(s["k"], s["v"], s["lens"], s["cap"] if c["kind"] == "append" else s["max_len"], s["table"])
        if c["kind"] == "attn":
            s["tree"] = cb.Tree(s["tok_start"], s["masks"], s["max_nodes"])
            s["ws"] = cb.alloc_tree_workspace(s["params"], s["max_len"], s["q"].shape[0], s["max_nodes"], DEVICE)
        if c["kind"] == "commit":
            s["params"] = cb.make_params(c["batch"], c["kv_heads"], c["kv_heads"], 1, 0)
            s["commit"] = cb.KvCommit(s["params"], [cb.KvCache(s["k"][i], s["v"][i], s["lens"], s["max_len"], s["table"]) for i in range(c["layers"])])
    return s


# ---- one pass

def run(state):
    s = state
    if not own:
        return _PLAIN[s["kind"]](s)
    cb = _lib()
    if s["kind"] == "plan":
        cb.kv_plan(s["held"], s["keep"], s["add"], s["lens"], s["tok_start"], s["slots"], s["ws"], s.get("pool"), s.get("state_out"), s["capacity"])
        return _plan_outputs(s, s["lens"], s["tok_start"], s["slots"], s.get("table"), s.get("ring"), s.get("state_out"))
    if s["kind"] == "append":
        cb.kv_append(s["params"], s["kv"], s["slots"], s["k_new"], s["v_new"])
        return {"k": s["k"], "v": s["v"]}
    if s["kind"] == "masks":
        cb.tree_masks(s["base"], s["tok_start"], s["parents"], s["masks"], s["positions"], s["max_nodes"])
        return {"masks": s["masks"], "positions": s["positions"]}
    if s["kind"] == "attn":
        cb.tree_attn(s["params"], s["q"], s["kv"], s["tree"], s["out"], s["ws"], s["idx"], s["cnt"])
        return {"out": s["out"]}
    s["commit"].run(s["base"], s["path"], s["n_path"], s["keep"])
    return {"k": s["k"], "v": s["v"], "keep": s["keep"]}


def _plan_outputs(s, lens, tok_start, slots, table, ring, state_out):
    out = {"lens": lens, "tok_start": tok_start, "slots": slots}
    if table is not None:
        out.update(table=table, ring=ring, state=state_out)
    return out


def _plain_plan(s):
    paged = "table" in s
    table, n_pages = s.get("table"), s.get("n_pages", 0)
    cap = table.shape[1] * PAGE if paged else s["capacity"]
    held = s["held"].long().clamp(0, cap)
    keep = torch.minimum(s["keep"].long().clamp(min=0), held)
    a = s["add"].long().clamp(min=0)
    fits = keep + a <= cap
    ok = fits & (torch.where(fits, a, 0).cumsum(0) <= s["max_tokens"])
    h = (held + PAGE - 1) // PAGE
    if paged:
        first, avail = s["state"][0].long(), s["state"][1].long()
        need = torch.where(ok, ((keep + a + PAGE - 1) // PAGE - h).clamp(min=0), 0)
        ok = ok & ((need == 0) | (need.cumsum(0) <= avail))
    n = torch.where(ok, a, 0)
    lens = keep + n
    start = torch.cat([n.new_zeros(1), n.cumsum(0)])
    r = torch.arange(s["max_tokens"], device=n.device)
    b = torch.searchsorted(start[1:].contiguous(), r, right=True).clamp(max=len(n) - 1)
    pos = keep[b] + r - start[b]
    if not paged:
        slots = torch.where(r < start[-1], (b << 32) + pos, -1)
        return _plan_outputs(s, lens.int(), start.int(), slots, None, None, None)
    w = (lens + PAGE - 1) // PAGE
    grow, back = (w - h).clamp(min=0), (h - w).clamp(min=0)
    pi = torch.arange(table.shape[1], device=n.device)[None, :]
    pop = (first + (grow.cumsum(0) - grow)[:, None] + pi - h[:, None]) % n_pages
    new_table = torch.where((pi >= h[:, None]) & (pi < w[:, None]), s["ring"][pop], table)
    push = (first + avail + (back.cumsum(0) - back)[:, None] + pi - w[:, None]) % n_pages
    freed = (pi >= w[:, None]) & (pi < h[:, None])
    ring = torch.cat([s["ring"], s["ring"][:1]])
    ring[torch.where(freed, push, n_pages)] = table
    slots = torch.where(r < start[-1], new_table[b, (pos // PAGE).clamp(0, table.shape[1] - 1)].long() * PAGE + pos % PAGE, -1)
    state = torch.stack([(first + grow.sum()) % n_pages, avail - grow.sum() + back.sum()])
    return _plan_outputs(s, lens.int(), start.int(), slots, new_table, ring[:n_pages], state.int())


def _plain_append(s):
    if s["table"] is not None:
        page, off = s["slots"] // PAGE, s["slots"] % PAGE
        s["k"][page, :, off] = s["k_new"].to(torch.bfloat16)
        s["v"][page, :, off] = s["v_new"].to(torch.bfloat16)
    else:
        b, t = s["slots"] >> 32, s["slots"] & 0xFFFFFFFF
        s["k"][b, :, t] = s["k_new"].to(torch.bfloat16)
        s["v"][b, :, t] = s["v_new"].to(torch.bfloat16)
    return {"k": s["k"], "v": s["v"]}


def _plain_masks(s):
    """Parents to ancestors by doubling: rows of truth values, all trees side by side."""
    n, start, words = s["max_nodes"], s["tok_start"].long(), s["masks"].shape[1]
    total = s["parents"].shape[0]
    r = torch.arange(total, device=start.device)
    b = (r[:, None] >= start[1:][None, :]).sum(1)
    par = s["parents"].long()
    j = r - start[b]
    col = torch.arange(words * 64, device=start.device)
    rows = col[None, :] == j[:, None]
    up = torch.where((par >= 0) & (par < j), start[b] + par, total)   # a row of nothing stands for the prefix
    depth = torch.cat([(up < total).long(), up.new_zeros(1)])
    up = torch.cat([up, up.new_full((1,), total)])
    rows = torch.cat([rows, rows.new_zeros(1, words * 64)])
    for _ in range(max(1, (n - 1).bit_length())):
        rows = rows | rows[up]
        depth = depth + depth[up]
        up = up[up]
    bits = torch.ones(64, dtype=torch.int64, device=start.device) << torch.arange(64, device=start.device)
    masks = (rows[:total].view(total, words, 64) * bits).sum(-1)
    return {"masks": masks, "positions": (s["base"].long()[b] + depth[:total]).int()}


def _rows_of(x, table, b, pos):
    """[G][len(pos)][D] of sequence b."""
    return x[table[b][pos // PAGE].long(), :, pos % PAGE].transpose(0, 1) if table is not None else x[b][:, pos]


def _plain_attn(s):
    q, G, at = s["q"], s["kv_heads"], 0
    outs = []
    shift = torch.arange(64, device=q.device)
    for b, (p, n) in enumerate(zip(s["pre"], s["n"])):
        if not n:
            continue
        if s["idx"] is None:
            pos = torch.arange(p + n, device=q.device)
            live = pos < p
        else:
            pos = torch.cat([s["idx"][b, : min(p + 1, s["budget"])].long(), torch.arange(p, p + n, device=q.device)])
            live = pos < p
            live[-n:] = False
        kf = _rows_of(s["k"], s["table"], b, pos).float().transpose(1, 2).contiguous()
        vf = _rows_of(s["v"], s["table"], b, pos).float().contiguous()
        qf = q[at: at + n].float().view(n, G, -1, D).permute(1, 0, 2, 3).reshape(G, -1, D)
        bits = ((s["masks"][at: at + n, :, None] >> shift) & 1).view(n, -1)[:, :n].bool()
        allowed = live[None, :].repeat(n, 1)
        allowed[:, -n:] |= bits
        allowed = allowed.repeat_interleave(qf.shape[1] // n, dim=0)
        x = torch.where(allowed, torch.bmm(qf, kf) * D ** -0.5, float("-inf"))
        w = torch.exp(x - x.amax(-1, keepdim=True))
        o = torch.bmm(w, vf) / w.sum(-1, keepdim=True)
        outs.append(o.view(G, n, -1, D).permute(1, 0, 2, 3).reshape(n, -1, D))
        at += n
    return {"out": torch.cat(outs).to(torch.bfloat16)}


def _plain_commit(s):
    L, B, m = s["k"].shape[0], s["path"].shape[0], s["path"].shape[1]
    i = torch.arange(m, device=s["path"].device)
    b, i = torch.nonzero(i[None, :] < s["n_path"][:, None], as_tuple=True)
    src, dst = s["base"].long()[b] + s["path"][b, i].long(), s["base"].long()[b] + i
    for x in (s["k"], s["v"]):
        if s["table"] is not None:
            x[:, s["table"][b, dst // PAGE].long(), :, dst % PAGE] = x[:, s["table"][b, src // PAGE].long(), :, src % PAGE]
        else:
            x[:, b, :, dst] = x[:, b, :, src]
    return {"k": s["k"], "v": s["v"], "keep": s["base"] + s["n_path"]}


_PLAIN = {"plan": _plain_plan, "append": _plain_append, "masks": _plain_masks, "attn": _plain_attn, "commit": _plain_commit}


# ---- what a pass cannot do without

def work(case):
    c = case
    if c["kind"] == "plan":
        lens, add = _lengths(c), _adds(c)
        new = sum((n + a + PAGE - 1) // PAGE - (n + PAGE - 1) // PAGE for n, a in zip(lens, add)) if c["layout"] == "paged" else 0
        return {"bytes": 20 * c["batch"] + 8 * sum(add) + 8 * new, "flops": 0}   # (the seed takes a few of them off)
    if c["kind"] == "append":
        size = 4 if c["dtype"] == "float32" else 2
        return {"bytes": sum(_adds(c)) * (8 + 2 * c["kv_heads"] * D * (size + 2)), "flops": 0}
    if c["kind"] == "masks":
        return {"bytes": sum(_nodes(c)) * (8 + 8 * ((c["nodes"] + 63) // 64)) + 8 * c["batch"], "flops": 0}
    if c["kind"] == "commit":
        rows = c["batch"] * c["path"] / 2.0
        return {"bytes": rows * c["layers"] * 2 * c["kv_heads"] * D * 2 * 2 + 8 * rows, "flops": 0}
    n_bytes = n_flops = 0
    for p, n in zip(_lengths(c), _nodes(c)):
        if not n:
            continue
        seen = min(p, c["budget"]) if c["budget"] else p
        n_bytes += 2 * (seen + n) * c["kv_heads"] * D * 2 + 2 * n * c["heads"] * D * 2 + 8 * n * ((c["nodes"] + 63) // 64) + (4 * seen if c["budget"] else 0)
        n_flops += 4 * D * c["heads"] * n * (seen + min(n, 4))
    return {"bytes": n_bytes, "flops": n_flops}


# ---- the same from the definitions, in 64 bits

def exact(case, seed):
    c = case
    if c["kind"] in ("plan", "masks"):
        return None                                       # whole numbers: equal or wrong
    s = _INPUTS[c["kind"]](c, seed)
    if c["kind"] == "append":
        lens, n = _lengths(c), _adds(c)
        k, v = s["k"].double(), s["v"].double()
        at = 0
        for b in range(c["batch"]):
            for x, new in ((k, s["k_new"]), (v, s["v_new"])):
                rows = new[at: at + n[b]].double()
                if s["table"] is None:
                    x[b, :, lens[b]: lens[b] + n[b]] = rows.transpose(0, 1)
                else:
                    pos = torch.arange(lens[b], lens[b] + n[b], device=DEVICE)
                    x[s["table"][b].long()[pos // PAGE], :, pos % PAGE] = rows
            at += n[b]
        return {"k": k, "v": v}
    if c["kind"] == "commit":
        table = s["table"].tolist() if s["table"] is not None else None
        base, path, taken = s["base"].tolist(), s["path"].tolist(), s["n_path"].tolist()
        out = {"keep": None}
        for name in ("k", "v"):
            x = s[name].clone()
            for b in range(c["batch"]):
                for i in range(taken[b]):
                    f, t = base[b] + path[b][i], base[b] + i
                    if table is None:
                        x[:, b, :, t] = s[name][:, b, :, f]
                    else:
                        x[:, table[b][t // PAGE], :, t % PAGE] = s[name][:, table[b][f // PAGE], :, f % PAGE]
            out[name] = x.double()
        return out
    B, H, G = c["batch"], c["heads"], c["kv_heads"]
    start, masks = s["tok_start"].tolist(), s["masks"].cpu().numpy().view(np.uint64)
    out = torch.zeros((start[-1], H, D), dtype=torch.float64, device=DEVICE)
    for b in range(B):
        n, p = start[b + 1] - start[b], s["pre"][b]
        if not n:
            continue
        before = list(range(p)) if s["idx"] is None else [t for t in s["idx"][b, : int(s["cnt"][b])].tolist() if t < p]
        tokens = torch.tensor(before + list(range(p, p + n)), device=DEVICE)
        bits = np.unpackbits(masks[start[b]: start[b + 1]].view(np.uint8), axis=1, bitorder="little")[:, :n].astype(bool)
        away = torch.zeros((n, len(tokens)), dtype=torch.bool, device=DEVICE)
        away[:, len(before):] = torch.from_numpy(~bits).to(DEVICE)
        for g in range(G):
            kk, vv = (_rows_of(s[name][:, g: g + 1], s["table"], b, tokens)[0].double() for name in ("k", "v"))
            kt = kk.t().contiguous()
            for h in range(g * H // G, (g + 1) * H // G):
                x = (s["q"][start[b]: start[b + 1], h].double() @ kt) / math.sqrt(D)
                out[start[b]: start[b + 1], h] = torch.softmax(x.masked_fill(away, -math.inf), dim=-1) @ vv
    return {"out": out}
