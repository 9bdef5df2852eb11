"""Groups of every kind of width, through every call: rows fill a power of two, or one more, or one less."""
import numpy as np
import pytest
import torch

import beam_reference as ref
from test_gpu_beam import _check_fork, _check_select, _check_shared, _fork_case, _i32, _logits
from test_gpu_beam_attn import Case

pytestmark = pytest.mark.gpu
DEV = "cuda"
WIDTHS = [1, 2, 3, 5, 7, 8, 9, 15, 16, 17, 20, 31, 32]


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("prompt,tail,columns", [(60, 40, 0), (3000, 200, 0), (300, 100, 1100)])
def test_fork_and_list(width, prompt, tail, columns):
    """Tables that one workgroup changes and that several do; entries of columns that some rows hold alone."""
    print("fork", width, prompt, columns, flush=True)
    rng = np.random.default_rng(width + prompt)
    for groups in (1, 5):
        for samples in (False, True):
            lens, table, ring, state, gone = _fork_case(rng, groups, width, prompt, tail, 40, columns, samples=samples)
            parents = rng.integers(-1, width, groups * width)
            parents[gone] = -1
            for own in (parents, np.sort(parents), np.full(groups * width, width - 1)):
                _check_fork(width, lens, table, ring, state, own, rng.random(groups * width) < 0.2, True, samples)
            _check_shared(width, lens, table, len(ring), max(1, int(lens.max())))
            lens[rng.random(len(lens)) < 0.4] = 0
            _check_shared(width, lens, table, len(ring), max(1, int(lens.max()) - 7))


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("vocab,n", [(900, 64), (5003, 33), (40000, 17), (70001, 1)])
def test_selection(width, vocab, n):
    print("select", width, vocab, n, flush=True)
    x, s = _logits(2 * width, vocab, torch.bfloat16, vocab + width)
    s[::3] -= 6.0                                                # (rows that the others leave nothing to)
    _check_select(x, s, width, n, _i32(np.arange(2 * width) % 7 == 6), vocab - 1)


@pytest.mark.parametrize("vocab", [64, 4096, 9001, 70000])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_selection_of_many_equal_logits(vocab, kind):
    """More than there is room for beside a wave, at the bound and above it: all alike, two values, rising and falling, a few above many."""
    rng = np.random.default_rng(vocab)
    x = np.zeros((8, vocab), dtype=np.float32)
    x[1, ::2] = 1.0
    x[2] = np.arange(vocab) / vocab
    x[3] = -x[2]
    x[4, rng.integers(0, vocab, 40)] = 2.0
    x[5] = rng.integers(0, 2, vocab)
    x[6] = -np.inf
    x[6, -1] = 3.0
    x[7] = np.where(np.arange(vocab) % 64 == 5, 4.0, -4.0)       # one lane's
    for n in (64, 63, 5):
        _check_select(torch.tensor(x, device=DEV).to(kind), torch.zeros(8, device=DEV), 8, n)
        _check_select(torch.tensor(x, device=DEV).to(kind), torch.zeros(8, device=DEV), 1, n)


@pytest.mark.parametrize("kind,at", [(torch.bfloat16, 0), (torch.bfloat16, 3), (torch.float32, 1)])
@pytest.mark.parametrize("alike", [False, True])
def test_selection_of_as_many_logits_as_there_is_room_for(kind, at, alike):
    """Rows with 370 to 410 logits that a search keeps, and the best ones at their ends, which are looked at last."""
    vocab, rows = 64 * 8 + 9, 48
    rng = np.random.default_rng(at)
    x = np.full((rows, vocab), -5.0, dtype=np.float32)
    for r in range(rows):
        low = np.r_[200:224, 456:480]                            # a lane's, whose best is the bound: 1.0
        some = np.setdiff1d(np.arange(8, vocab - 8), low)
        some = rng.permutation(some)[: 368 + r - len(low)]
        x[r, some], x[r, low] = 1.0 if alike else 1.0 + (1 + rng.permutation(len(some))) / 64.0, 1.0
        x[r, :3], x[r, -4:] = 9.0 + np.arange(3) / 8.0, 9.5 + np.arange(4) / 8.0
    flat = torch.zeros(rows * vocab + at, device=DEV).to(kind)
    logits = flat[at:].view(rows, vocab)
    logits.copy_(torch.tensor(x, device=DEV))
    for n in (64, 63):
        _check_select(logits, torch.zeros(rows, device=DEV), 1, n)


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("H,G", [(8, 8), (16, 2)])
def test_attention(width, H, G):
    """Blocks of 16 and 32 rows that are full, or one row short or over."""
    print("attn", width, H, G, flush=True)
    for samples in (False, True):
        c = Case(3, width, H, G, 300, 150, width + H, samples, fused=samples)
        c.lens[::4] = 0 if samples else c.lens[::4]
        c.check(c.run())
    c = Case(1, width, H, G, 4000, 300, width)
    c.check(c.run())
