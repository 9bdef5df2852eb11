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


def _calls(monkeypatch):
    """What reaches the library: the descriptors of a call by its name."""
    seen = {}

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.setdefault(name, [getattr(a, "_obj", a) for a in args]) and 0
    monkeypatch.setattr(cb, "load", lambda: Library())
    monkeypatch.setattr(cb, "_stream", lambda: None)
    return seen


def test_strides_of_one_entry_mean_nothing(monkeypatch):
    """One token, one head, one sequence: torch may give such a dimension any stride, and calls the tensor contiguous."""
    seen = _calls(monkeypatch)
    one = cb.make_params(1, 1, 1, 16, 0)
    k, v = _gpu((1, 1, 32, 128), torch.bfloat16, (8, 24, 128, 1)), _gpu((1, 1, 32, 128), torch.bfloat16, (9, 5, 128, 1))
    kv = cb.KvCache(k, v, _i32(1), 32)
    rows, more = _gpu((1, 1, 128), torch.bfloat16, (7, 3, 1)), _gpu((1, 1, 128), torch.bfloat16, (128, 1, 1))
    cb.kv_append(one, kv, _gpu((1,), torch.int64), rows, more)
    desc, r = seen["cusa_kv_append"][1], seen["cusa_kv_append"][3]
    assert (desc.stride_batch % 8, desc.stride_head % 8, desc.stride_token) == (0, 0, 128) and (r.stride_token % 8, r.stride_head % 8) == (0, 0)
    cb.tree_attn(one, rows, kv, cb.Tree(_i32(2), _gpu((1, 1), torch.int64), 4), _gpu((1, 1, 128), torch.bfloat16), _gpu((256,), torch.uint8))
    assert seen.pop("cusa_tree_attn")[3].q_stride == 128
    # the single token of a decode step, as a transposed projection leaves it: [H, 1, 128] seen as [1, H, 128]
    cb.tree_attn(cb.make_params(1, 8, 1, 16, 0), _gpu((1, 8, 128), torch.bfloat16, (128, 128, 1)), kv, cb.Tree(_i32(2), _gpu((1, 1), torch.int64), 4),
                 _gpu((1, 8, 128), torch.bfloat16), _gpu((256,), torch.uint8))
    assert seen["cusa_tree_attn"][3].q_stride == 8 * 128
    # one position: its stride is a row's
    single = cb.KvCache(_gpu((2, 4, 1, 128), torch.bfloat16, (512, 128, 1, 1)), _gpu((2, 4, 1, 128), torch.bfloat16, (512, 128, 64, 1)), _i32(2), 1)
    cb.KvCommit(P, [single])
    rows = _gpu((3, 4, 128), torch.bfloat16)
    seen.clear()
    cb.kv_append(P, single, _gpu((3,), torch.int64), rows, rows)
    desc = seen["cusa_kv_append"][1]
    assert (desc.stride_batch, desc.stride_head, desc.stride_token) == (512, 128, 128)
    with pytest.raises(ValueError):
        cb.kv_append(P, _cache(32, 32), _gpu((3,), torch.int64), rows, _gpu((3, 4, 128), torch.bfloat16, (1024, 128, 1)))
    with pytest.raises(ValueError):
        cb.kv_append(P, cb.KvCache(_gpu((2, 4, 32, 128), torch.bfloat16), _gpu((2, 4, 32, 128), torch.bfloat16, (16384, 128, 512, 1)), _i32(2), 32),
                     _gpu((3,), torch.int64), rows, rows)
