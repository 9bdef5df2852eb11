"""Equal logits of a row: its proposals are the first tokens in order of (logit, token), exactly, whatever the values' rounding; and rows alike stand in order of row and token."""
import math

import numpy as np
import pytest
import torch

from test_gpu_beam import DEV, _i32, _logits, _select

pytestmark = pytest.mark.gpu


def _check_first(x, parents, tokens, width, ended=None):
    """Those that a row has among its group's best are the first of its own list: a row's values all come from one score and one sum, so that they fall with the logits."""
    x = x.double().cpu().numpy()
    for g in range(len(parents)):
        for b in range(width):
            got = tokens[g][parents[g] == b]
            if ended is None or not ended[g * width + b]:
                row = x[g * width + b]
                best = np.lexsort((np.arange(len(row)), -row))[: len(got)]
                assert got.tolist() == best.tolist(), (g, b)


def _tied(rows, vocab, rng):
    x = np.zeros((rows, vocab), dtype=np.float32)                # (row 0: all alike)
    x[1, ::2] = 1.0
    x[2] = rng.integers(0, 3, vocab)
    x[3, rng.integers(0, vocab, 40)] = 2.0
    x[4] = np.where(np.arange(vocab) % 64 == 5, 4.0, -4.0)       # one lane's
    x[5, vocab // 2:] = 0.5                                      # a bound that is reached late
    x[6] = np.arange(vocab) * 8 // vocab                         # eight steps up: every step's first tokens are better than all before
    x[7] = -x[6]
    x[8] = -0.0
    x[8, 1::3] = 0.0                                             # zeros of both signs are equal
    x[9] = -np.inf
    x[9, -min(vocab, 100):] = -7.0
    x[10, -3:] = x[10, :2] = 3.0                                 # at both ends
    x[11] = rng.integers(0, 2, vocab) * 0.125 + 6.0
    return x


@pytest.mark.parametrize("kind,pad,at", [(torch.bfloat16, 0, 0), (torch.bfloat16, 3, 1), (torch.float16, 1, 0), (torch.float32, 0, 0), (torch.float32, 1, 3)])
@pytest.mark.parametrize("vocab", [64, 513, 4096, 9001, 32000, 70000])
def test_of_equal_logits_of_a_row_the_lower_tokens_are_taken(vocab, kind, pad, at):
    print("ties", vocab, kind, pad, at, flush=True)
    x = _tied(12, vocab, np.random.default_rng(vocab))
    logits = torch.zeros(12 * (vocab + pad) + at, dtype=kind, device=DEV)[at:].view(12, vocab + pad)[:, :vocab]
    logits.copy_(torch.tensor(x, device=DEV))
    for n in (64, 63, 33, 32, 31, 8, 1):
        for width in (1, 12):
            _, parents, tokens, _ = _select(logits, torch.zeros(12, device=DEV), width, n)
            if width == 1:
                assert ((parents == 0).sum(1) == np.minimum(n, (x > -math.inf).sum(1))).all()
            _check_first(logits, parents, tokens, width)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_drawn_logits_of_a_row_come_in_its_order(kind):
    """Vocabularies where bf16 makes many logits equal; some rows have ended."""
    ended = np.arange(24) % 5 == 2
    for vocab, n in ((3001, 64), (50003, 40), (131072, 16)):
        x, s = _logits(24, vocab, kind, vocab)
        _, parents, tokens, _ = _select(x, s, 8, n, _i32(ended), end=3)
        _check_first(x, parents, tokens, 8, ended)


@pytest.mark.parametrize("vocab,some", [(40, 3), (3000, 5), (66000, 7)])
def test_rows_alike_stand_in_order_of_row_and_token(vocab, some):
    """Rows of one content at one alignment have one sum and so values that are equal to the last bit: of each logit, the lower row's tokens come first, then the lower token."""
    rng = np.random.default_rng(vocab)
    x = rng.integers(-3, 0, vocab).astype(np.float32)
    best, next_best = np.sort(rng.permutation(vocab)[: 2 * some].reshape(2, some))
    x[best], x[next_best] = 2.0, 1.0
    for kind in (torch.bfloat16, torch.float32):
        for width in (2, 5, 8):
            logits = torch.zeros((width, (vocab + 7) // 8 * 8), dtype=kind, device=DEV)[:, :vocab]
            logits.copy_(torch.tensor(x, device=DEV).expand(width, vocab))
            n = min(64, width * some + 2 * some + 1)             # all of the best, and the next best of two rows and one
            values, parents, tokens, _ = _select(logits, torch.full((width,), -1.5, device=DEV), width, n)
            want = [(b, t) for of in (best, next_best) for b in range(width) for t in of.tolist()][:n]
            if len(want) < n:                                    # (two rows: the rest are the third best)
                third = np.flatnonzero(x == x[x < 1.0].max()).tolist()
                want = (want + [(b, t) for b in range(width) for t in third])[:n]
            assert list(zip(parents[0].tolist(), tokens[0].tolist())) == want
            assert all(a >= b for a, b in zip(values[0], values[0][1:]))
