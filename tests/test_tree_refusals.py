"""What the tree calls' binding refuses before anything reaches the GPU: no kernel is launched by anything in this file.  The checks see stand-ins
for GPU tensors, whose memory nothing here touches."""
import pytest
import torch

from paper_2508_07101_amd import binding as cb


class _Gpu(torch.Tensor):
    """A host tensor that says it is on the GPU."""
    is_cuda = property(lambda self: True)


def _gpu(shape, dtype, strides=None):
    t = torch.zeros(shape, dtype=dtype) if strides is None else torch.zeros(sum((n - 1) * s for n, s in zip(shape, strides)) + 1, dtype=dtype).as_strided(shape, strides)
    return t.as_subclass(_Gpu)


@pytest.fixture(autouse=True)
def no_call(monkeypatch):
    """Calls that pass the checks end here."""
    class Library:
        def __getattr__(self, name):
            raise AssertionError(f"{name} was reached")
    monkeypatch.setattr(cb, "load", lambda: Library())


def _i32(*shape):
    return _gpu(shape, torch.int32)


def _cache(tokens, bound, B=2, G=4, layout="head_major"):
    shape = (B, G, tokens, 128)
    strides = None if layout == "head_major" else (tokens * G * 128, 128, G * 128, 1)
    return cb.KvCache(_gpu(shape, torch.bfloat16, strides), _gpu(shape, torch.bfloat16, strides), _i32(B), bound)


P = cb.make_params(2, 8, 4, 16, 0)


def _append(kv):
    rows = _gpu((3, 4, 128), torch.bfloat16)
    cb.kv_append(P, kv, _gpu((3,), torch.int64), rows, rows)


def _attn(kv=None, tree=None, idx=None, cnt=None, ws=None):
    q = _gpu((5, 8, 128), torch.bfloat16)
    cb.tree_attn(P, q, kv or _cache(32, 32), tree or cb.Tree(_i32(3), _gpu((5, 1), torch.int64), 40), _gpu((5, 8, 128), torch.bfloat16),
                 _gpu((1 << 20,), torch.uint8) if ws is None else ws, idx, cnt)


@pytest.mark.parametrize("layout", ["head_major", "token_major"])
@pytest.mark.parametrize("call", [_append, lambda kv: _attn(kv), lambda kv: cb.KvCommit(P, [kv])])
def test_bounds_beyond_a_contiguous_cache(call, layout):
    with pytest.raises(ValueError, match="33"):
        call(_cache(32, 33, layout=layout))


def _plan(ws):
    cb.kv_plan(_i32(2), _i32(2), _i32(2), _i32(2), _i32(3), _gpu((8,), torch.int64), ws, capacity=10)


@pytest.mark.parametrize("call", [_plan, lambda ws: _attn(ws=ws)])
@pytest.mark.parametrize("ws", [torch.zeros(1 << 20, dtype=torch.uint8), _gpu((1 << 20,), torch.int32), _gpu((1 << 20,), torch.uint8, (2,))],
                         ids=["host memory", "int32", "every second byte"])
def test_workspaces_that_are_no_bytes_on_the_gpu(call, ws):
    with pytest.raises(ValueError, match="workspace"):
        call(ws)


def _masks(masks, nodes):
    cb.tree_masks(_i32(2), _i32(3), _i32(5), masks, None, nodes)


@pytest.mark.parametrize("shape", [(5, 2), (5, 3), (5, 1, 2)])
def test_mask_rows_of_another_width(shape):
    """Trees of up to 64 nodes have rows of one word: wider rows would be read and written a word apart.  (Flat ones have no width of their own.)"""
    masks = _gpu(shape, torch.int64)
    with pytest.raises(ValueError, match="masks"):
        _masks(masks, 64)
    with pytest.raises(ValueError, match="masks"):
        _attn(tree=cb.Tree(_i32(3), masks, 64))
    for right in ((7, 1), (5,)):
        with pytest.raises(AssertionError, match="cusa_tree_masks was reached"):
            _masks(_gpu(right, torch.int64), 64)
        with pytest.raises(AssertionError, match="cusa_tree_attn was reached"):
            _attn(tree=cb.Tree(_i32(3), _gpu(right, torch.int64), 64))


@pytest.mark.parametrize("shape", [(2, 17), (2, 32), (4, 8)])
def test_lists_of_another_width(shape):
    with pytest.raises(ValueError, match="idx"):
        _attn(idx=_i32(*shape), cnt=_i32(2))
    for right in ((3, 16), (32,)):
        with pytest.raises(AssertionError, match="cusa_tree_attn was reached"):
            _attn(idx=_i32(*right), cnt=_i32(2))
