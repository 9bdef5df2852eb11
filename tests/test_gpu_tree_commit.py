"""Accepted branches in more layers than a launch takes."""
import numpy as np
import pytest
import torch

from paper_2508_07101_amd import binding as cb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("layout", ["paged", "head_major"])
@pytest.mark.parametrize("layers", [39, 40, 41, 80, 83])
def test_every_layer_moves_once(layers, layout):
    """A launch takes 40 layers: the last of one and the first of the next, and keep, which the first launch writes."""
    print("commit", layout, layers, flush=True)
    B, G, tokens, base, n_path = 3, 2, 64, [5, 0, 30], [3, 0, 20]
    rng = np.random.default_rng(layers)
    path = np.zeros((B, 20), dtype=np.int64)
    for b in range(B):
        path[b, : n_path[b]] = np.sort(rng.choice(tokens - base[b], size=n_path[b], replace=False))
    table = torch.from_numpy(rng.permutation(B * 4).reshape(B, 4).astype(np.int32)).to(DEV) if layout == "paged" else None
    shape = (B * 4, G, 16, 128) if table is not None else (B, G, tokens, 128)
    kvs, want = [], []
    for _ in range(layers):
        k, v = (torch.randn(shape, device=DEV).to(torch.bfloat16) for _ in range(2))
        kvs.append(cb.KvCache(k, v, _i32([tokens] * B), tokens, table))
        for x in (k, v):
            old, new = x.clone(), x.clone()
            for b in range(B):
                for i in range(n_path[b]):
                    s, t = base[b] + int(path[b, i]), base[b] + i
                    if table is None:
                        new[b, :, t] = old[b, :, s]
                    else:
                        new[int(table[b, t // 16]), :, t % 16] = old[int(table[b, s // 16]), :, s % 16]
            want.append(new)
    keep = torch.full((B,), -1, dtype=torch.int32, device=DEV)
    cb.kv_commit(cb.make_params(B, G, G, 1, 0), kvs, _i32(base), _i32(path), _i32(n_path), keep)
    torch.cuda.synchronize()
    assert keep.tolist() == [b + n for b, n in zip(base, n_path)]
    for i, kv in enumerate(kvs):
        assert torch.equal(kv.k, want[2 * i]) and torch.equal(kv.v, want[2 * i + 1]), f"layer {i}"
