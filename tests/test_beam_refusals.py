"""What the beam calls' binding refuses before anything reaches the GPU: no kernel is launched by anything in this file.  The checks see stand-ins
for GPU tensors, whose memory nothing here touches."""
import pytest
import torch

from paper_2508_07101_amd import binding as cb


class _Gpu(torch.Tensor):
    """A host tensor that says it is on the GPU."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


class _Other(_Gpu):
    """One on another GPU than the current one."""

    def get_device(self):
        return 1


def _gpu(shape, dtype, strides=None, kind=_Gpu):
    t = torch.zeros(shape, dtype=dtype) if strides is None else torch.zeros(sum((n - 1) * s for n, s in zip(shape, strides)) + 1, dtype=dtype).as_strided(shape, strides)
    return t.as_subclass(kind)


@pytest.fixture(autouse=True)
def calls(monkeypatch):
    """Calls that pass the checks end here: their arguments by their names."""
    seen = {}

    class Library:
        def __getattr__(self, name):
            return lambda *args: seen.__setitem__(name, [getattr(a, "_obj", a) for a in args]) or 0
    monkeypatch.setattr(cb, "load", lambda: Library())
    monkeypatch.setattr(cb, "_stream", lambda: None)
    monkeypatch.setattr(cb, "_device", lambda: 0)
    return seen


def _i32(*shape):
    return _gpu(shape, torch.int32)


WS = _gpu((1 << 20,), torch.uint8)


def _wrong(shape, dtype, width=False):
    """Stand-ins for tensors that a call that wants `shape` of this type must not take."""
    n = 1
    for x in shape:
        n *= x
    bad = {"type": _gpu(shape, torch.float64), "host": torch.zeros(shape, dtype=dtype), "other GPU": _gpu(shape, dtype, kind=_Other), "short": _gpu((n - 1,), dtype),
           "strided": _gpu((n,), dtype, (2,))}
    if width:
        bad["width"] = _gpu((n, 2 * shape[-1]), dtype)
    return bad


def _each(call, good):
    """Every argument wrong in every way, the others right."""
    call(**good)
    for name, (shape, dtype, width) in WANTS[call.__name__].items():
        for how, t in _wrong(shape, dtype, width).items():
            with pytest.raises(ValueError):
                call(**{**good, name: t})
                pytest.fail(f"{name}: {how}")


I32, I64, F32 = torch.int32, torch.int64, torch.float32
WANTS = {
    "_select": {"scores": ((6,), F32, False), "out_scores": ((2, 4), F32, False), "parents": ((2, 4), I32, True), "tokens": ((2, 4), I32, True), "ended": ((6,), I32, False), "out_ended": ((2, 4), I32, True)},
    "_fork": {"held": ((6,), I32, False), "parents": ((6,), I32, False), "lens": ((6,), I32, False), "slots": ((6,), I64, False), "copies": ((6, 4), I32, True), "ended": ((6,), I32, False),
              "table_out": ((6, 5), I32, True), "state_out": ((2,), I32, False), "granted": ((2,), I32, False)},
    "_pages": {"table": ((6, 5), I32, False), "lens": ((6,), I32, False), "entries": ((2, 9, 4), I32, False), "count": ((2, 2), I32, True)},
    "_attn": {"entries": ((2, 9, 4), I32, False), "count": ((2, 2), I32, True), "out": ((6, 8, 128), torch.bfloat16, False)},
}


def _select(logits=None, scores=None, out_scores=None, parents=None, tokens=None, ended=None, out_ended=None, ws=WS, width=3, end=1):
    cb.beam_select(_gpu((6, 50), torch.bfloat16) if logits is None else logits, _gpu((6,), F32) if scores is None else scores, width, _gpu((2, 4), F32) if out_scores is None else out_scores,
                   _i32(2, 4) if parents is None else parents, _i32(2, 4) if tokens is None else tokens, ws, ended, out_ended, end)


def test_selection(calls):
    _each(_select, dict(ended=_i32(6), out_ended=_i32(2, 4)))
    for logits in (_gpu((6, 50), torch.float64), torch.zeros((6, 50)), _gpu((6, 50), F32, kind=_Other), _gpu((300,), F32), _gpu((6, 50), F32, (1, 6)), _gpu((6, 50), F32, (40, 1)), _gpu((7, 50), F32)):
        with pytest.raises(ValueError):
            _select(logits=logits)
    for width in (0, -3, 4, 5):
        with pytest.raises(ValueError):
            _select(width=width)
    for ws in (torch.zeros(1 << 20, dtype=torch.uint8), _gpu((1 << 20,), torch.int32), _gpu((1 << 20,), torch.uint8, (2,))):
        with pytest.raises(ValueError, match="workspace"):
            _select(ws=ws)
    # a single row: torch may give it any stride; a view of wider rows keeps its own
    cb.beam_select(_gpu((1, 50), F32, (7, 1)), _gpu((1,), F32), 1, _gpu((1, 2), F32), _i32(1, 2), _i32(1, 2), WS)
    assert calls["cusa_beam_select"][0].stride == 50
    _select(logits=_gpu((6, 50), torch.float16, (64, 1)))
    d = calls["cusa_beam_select"][0]
    assert (d.stride, d.dtype, d.rows, d.width, d.vocab, d.n, d.end_token) == (64, 1, 6, 3, 50, 4, 1)


def _pool(table=None, ring=None, state=None):
    return cb.PagePool(_i32(6, 5) if table is None else table, _i32(20) if ring is None else ring, _i32(2) if state is None else state)


def _fork(pool=None, width=3, held=None, parents=None, lens=None, slots=None, copies=None, ws=WS, **more):
    cb.kv_fork(pool or _pool(), width, _i32(6) if held is None else held, _i32(6) if parents is None else parents, _i32(6) if lens is None else lens,
               _gpu((6,), I64) if slots is None else slots, _i32(6, 4) if copies is None else copies, ws, **more)


def test_fork():
    _each(_fork, dict(ended=_i32(6), table_out=_i32(6, 5), state_out=_i32(2), granted=_i32(2)))
    for pool in (_pool(table=_i32(30)), _pool(table=_i32(7, 5)), _pool(table=_gpu((6, 5), I64)), _pool(table=_gpu((6, 5), I32, (1, 6))), _pool(ring=_gpu((20,), I64)), _pool(ring=torch.zeros(20, dtype=I32)),
                 _pool(state=_i32(1)), _pool(state=_gpu((2,), I32, kind=_Other))):
        with pytest.raises(ValueError):
            _fork(pool)
    with pytest.raises(ValueError, match="workspace"):
        _fork(ws=torch.zeros(99, dtype=torch.uint8))


def _cache(**kw):
    d = dict(k=_gpu((20, 4, 16, 128), torch.bfloat16), v=_gpu((20, 4, 16, 128), torch.bfloat16), seq_lens=_i32(6), max_seq_len=80, block_table=_i32(6, 5))
    d.update(kw)
    return cb.KvCache(**d)


P = cb.make_params(6, 8, 4, 16, 0)


def test_copies(calls):
    c = cb.KvCopy(P, [_cache(), _cache()])
    c.run(_i32(0, 4))
    assert "cusa_kv_copy" not in calls                           # nothing to copy
    c.run(_i32(3, 4))
    assert calls["cusa_kv_copy"][1] == 2 and calls["cusa_kv_copy"][4] == 3
    for bad in (_i32(12), _i32(4, 3), _gpu((3, 4), I64), torch.zeros((3, 4), dtype=I32), _gpu((3, 4), I32, (8, 1)), _gpu((3, 4), I32, kind=_Other)):
        with pytest.raises(ValueError):
            c.run(bad)
    with pytest.raises(ValueError, match="paged"):
        cb.KvCopy(P, [_cache(k=_gpu((6, 4, 80, 128), torch.bfloat16), v=_gpu((6, 4, 80, 128), torch.bfloat16), block_table=None)])


def _pages(table=None, lens=None, entries=None, count=None, width=3, ws=WS):
    cb.shared_pages(_i32(6, 5) if table is None else table, _i32(6) if lens is None else lens, 80, 20,
                    cb.SharedPages(width, _i32(2, 9, 4) if entries is None else entries, _i32(2, 2) if count is None else count), ws)


def test_lists_of_pages():
    _each(_pages, {})
    for entries in (_i32(72), _i32(1, 18, 4), _i32(2, 12, 3)):
        with pytest.raises(ValueError):
            _pages(entries=entries)
    for width in (0, 4, -1):
        with pytest.raises(ValueError):
            _pages(width=width)
    with pytest.raises(ValueError, match="workspace"):
        _pages(ws=_gpu((9,), I32))


def _attn(q=None, kv=None, entries=None, count=None, out=None, ws=WS):
    cb.beam_attn(P, _gpu((6, 8, 128), torch.bfloat16) if q is None else q, kv or _cache(), cb.SharedPages(3, _i32(2, 9, 4) if entries is None else entries, _i32(2, 2) if count is None else count),
                 _gpu((6, 8, 128), torch.bfloat16) if out is None else out, ws)


def test_attention(calls):
    _each(_attn, {})
    bf16 = torch.bfloat16
    for q in (_gpu((6, 8, 128), torch.float16), _gpu((5, 8, 128), bf16), _gpu((6, 4, 128), bf16), _gpu((6, 8, 64), bf16), _gpu((6, 1024), bf16), torch.zeros((6, 8, 128), dtype=bf16),
              _gpu((6, 8, 128), bf16, kind=_Other), _gpu((6, 8, 128), bf16, (2048, 256, 1)), _gpu((6, 8, 128), bf16, (1, 768, 6))):
        with pytest.raises(ValueError):
            _attn(q=q)
    for kv in (_cache(block_table=None, k=_gpu((6, 4, 80, 128), bf16), v=_gpu((6, 4, 80, 128), bf16)), _cache(k=_gpu((20, 8, 16, 128), bf16)), _cache(seq_lens=_i32(5)), _cache(block_table=_i32(5, 5)),
               _cache(k=_gpu((20, 4, 16, 128), torch.float16)), _cache(k=_gpu((20, 4, 16, 128), bf16, kind=_Other))):
        with pytest.raises(ValueError):
            _attn(kv=kv)
    _attn(q=_gpu((6, 8, 128), bf16, (16 * 128, 128, 1)))
    assert calls["cusa_beam_attn"][2] == 16 * 128 and calls["cusa_beam_attn"][4].max_entries == 9
    # one row: whatever torch says of its stride
    one = cb.make_params(1, 8, 4, 16, 0)
    cb.beam_attn(one, _gpu((1, 8, 128), bf16, (7, 128, 1)), _cache(seq_lens=_i32(1), block_table=_i32(1, 5)), cb.SharedPages(1, _i32(1, 5, 4), _i32(1, 2)), _gpu((1, 8, 128), bf16), WS)
    assert calls["cusa_beam_attn"][2] == 8 * 128
