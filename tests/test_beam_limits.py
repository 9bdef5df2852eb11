"""Limits of the beam calls that follow from a launch's size: a workspace is sized for no call that is refused.  No kernel is launched by anything in this file."""
import ctypes

import pytest

from paper_2508_07101_amd import binding as cb

FAKE = 0x10000


def _need(rows, width, G, pages):
    """The status of the workspace's size, and of the call with lists of this many pages a group."""
    lib, n = cb.load(), ctypes.c_size_t(0)
    p = cb.make_params(rows, G, G, 1, 0)
    s = cb.CusaShared(width, pages, FAKE, FAKE)
    max_len = 16 * ((pages + width - 1) // width)
    kv = cb.CusaKv(FAKE, FAKE, cb.KV_PAGED, 0, 0, 0, FAKE, max_len // 16, 16, min(pages, 0x7fffffff // 16 // G), FAKE, max_len)
    size = lib.cusa_beam_attn_workspace_bytes(ctypes.byref(p), max_len, ctypes.byref(s), ctypes.byref(n))
    return size, n.value, lib, (ctypes.byref(p), FAKE, G * 128, ctypes.byref(kv), ctypes.byref(s), FAKE, FAKE)


@pytest.mark.parametrize("rows,width,G,pages", [(65535, 1, 8, 1 << 19), (65535, 1, 512, 10), (32768, 2, 16, 1 << 19), (65534, 2, 128, 8192 * 5)])
def test_attention_of_more_workgroups_than_a_launch_has(rows, width, G, pages):
    """2^24 workgroups: pieces times KV heads times groups, and rows of a KV head by 32.  (32767 groups of 5 pieces: 128 KV heads are 20 971 520, 64 are 10 485 440.)"""
    size, _, lib, args = _need(rows, width, G, pages)
    assert size == cb.ERR_UNSUPPORTED
    assert lib.cusa_beam_attn(*args, 1 << 62, None) == cb.ERR_UNSUPPORTED


@pytest.mark.parametrize("rows,width,G,pages", [(4, 4, 8, 1 << 19), (65535, 1, 2, 1 << 19), (65535, 1, 255, 10), (65534, 2, 64, 8192 * 5), (65534, 2, 8, 1 << 19)])
def test_attention_of_as_many_as_it_has(rows, width, G, pages):
    size, n, lib, args = _need(rows, width, G, pages)
    assert size == cb.OK and n > 0
    assert lib.cusa_beam_attn(*args, n - 1, None) == cb.ERR_WORKSPACE_TOO_SMALL


def test_forks_of_tables_with_more_columns_than_tokens_have_numbers():
    """A row has 2^31 - 1 tokens at most, in 2^27 pages: columns behind those are nobody's, and no launch has threads for them (2^30 columns would be 2^32 threads)."""
    for batch, most in ((1, 0x7fffffff), (2, 0x3fffffff), (15, 0x7fffffff // 15)):
        assert cb.fork_workspace_bytes(batch, most) == cb.fork_workspace_bytes(batch, 1 << 27) > cb.fork_workspace_bytes(batch, (1 << 27) - 256)
