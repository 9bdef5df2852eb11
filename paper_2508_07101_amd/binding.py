"""ctypes binding of libcusa's C ABI (include/cusa.h): argument marshalling only.

Every step of the path runs in the library's HIP kernels.  torch supplies device
memory (``tensor.data_ptr()``) and the stream.  If the library cannot be loaded
or built this module raises; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

from . import build as _build

LAYER_FULL, LAYER_SELECT, LAYER_SPARSE = 0, 1, 2
KV_CONTIGUOUS, KV_PAGED = 0, 1
RANK_FIRST_OCCURRENCE, RANK_VOTES, RANK_MAX_SCORE = 0, 1, 2
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE_TOO_SMALL, ERR_LAUNCH = range(5)

EXPORTS = [
    "cusa_workspace_bytes", "cusa_workspace_layout", "cusa_select", "cusa_sparse_attn",
    "cusa_select_per_head", "cusa_sparse_attn_per_head", "cusa_attention_recall", "cusa_select_layer",
    "cusa_full_attn", "cusa_decode_step", "cusa_strerror", "cusa_profile_num_kernels",
    "cusa_profile_kernel_name", "cusa_profile_enable", "cusa_profile_reset", "cusa_profile_read",
    "cusa_build_id", "cusa_probe_stream_read", "cusa_probe_traffic", "cusa_sparse_attn_noalloc", "cusa_noalloc_max_scratch_bytes",
    "cusa_kv_plan_workspace_bytes", "cusa_kv_plan", "cusa_kv_append", "cusa_tree_masks", "cusa_tree_workspace_bytes", "cusa_tree_attn",
    "cusa_kv_commit",
]


class CusaParams(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("budget", ctypes.c_int32), ("window", ctypes.c_int32),
                ("topk_per_head", ctypes.c_int32), ("n_sink", ctypes.c_int32), ("rank_mode", ctypes.c_int32),
                ("sm_scale", ctypes.c_float)]


class CusaKv(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("layout", ctypes.c_int32),
                ("stride_batch", ctypes.c_int64), ("stride_head", ctypes.c_int64),
                ("stride_token", ctypes.c_int64), ("block_table", ctypes.c_void_p),
                ("max_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int64),
                ("seq_lens", ctypes.c_void_p), ("max_seq_len", ctypes.c_int32)]


class CusaWsLayout(ctypes.Structure):
    _fields_ = [("scores_offset", ctypes.c_size_t), ("ld_scores", ctypes.c_int64),
                ("rho_head_offset", ctypes.c_size_t), ("k", ctypes.c_int32), ("total_bytes", ctypes.c_size_t),
                ("filtered_select", ctypes.c_int32), ("second_chance_offset", ctypes.c_size_t)]


class CusaPool(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("batch", ctypes.c_int32), ("capacity", ctypes.c_int32), ("block_table", ctypes.c_void_p),
                ("max_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int64), ("ring", ctypes.c_void_p),
                ("state", ctypes.c_void_p), ("state_out", ctypes.c_void_p)]


class CusaRows(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("n", ctypes.c_int32),
                ("stride_token", ctypes.c_int64), ("stride_head", ctypes.c_int64)]


class CusaTree(ctypes.Structure):
    _fields_ = [("tok_start", ctypes.c_void_p), ("masks", ctypes.c_void_p), ("max_tokens", ctypes.c_int32), ("max_nodes", ctypes.c_int32),
                ("q_stride", ctypes.c_int64)]


class CusaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


_lib = None


def lib_path() -> str:
    return _build.LIB


def built_from() -> str:
    """Build id of the library file, read from the file itself (nothing is mapped)."""
    marker = b"CUSA_BUILD_ID="
    with open(_build.LIB, "rb") as fh:
        data = fh.read()
    at = data.find(marker)
    if at < 0:
        return "none"
    return data[at + len(marker): at + len(marker) + 16].decode("ascii", "replace")


def load():
    """Load the built library.  It is built first when none exists, and rebuilt when the file found
    was compiled from other sources than those in the tree (its build id says so); if that rebuild
    is impossible the call raises rather than run kernels that do not match the sources."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB):
        _build.build_lib(force=False)
    have, want = built_from(), _build.source_id()
    if have != want:
        try:
            _build.build_lib(force=True)
        except Exception as e:
            raise RuntimeError(f"libcusa.so was built from other sources (build id {have}, tree {want}) "
                               f"and cannot be rebuilt here: {e}; run __graft_entry__.build()") from e
    lib = ctypes.CDLL(_build.LIB)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    P = ctypes.POINTER
    lib.cusa_workspace_bytes.argtypes = [P(CusaParams), i32, P(sz)]
    lib.cusa_workspace_layout.argtypes = [P(CusaParams), i32, P(CusaWsLayout)]
    lib.cusa_select.argtypes = [P(CusaParams), vp, P(CusaKv), vp, vp, vp, sz, vp]
    lib.cusa_sparse_attn.argtypes = [P(CusaParams), vp, P(CusaKv), vp, vp, vp, vp, sz, vp]
    lib.cusa_select_per_head.argtypes = [P(CusaParams), vp, P(CusaKv), vp, vp, vp, sz, vp]
    lib.cusa_sparse_attn_per_head.argtypes = [P(CusaParams), vp, P(CusaKv), vp, vp, vp, vp, sz, vp]
    lib.cusa_attention_recall.argtypes = [P(CusaParams), vp, P(CusaKv), vp, vp, i32, vp, vp, sz, vp]
    lib.cusa_select_layer.argtypes = [P(CusaParams), vp, P(CusaKv), vp, vp, vp, vp, sz, vp]
    lib.cusa_full_attn.argtypes = [P(CusaParams), vp, P(CusaKv), vp, vp, sz, vp]
    lib.cusa_decode_step.argtypes = [P(CusaParams), i32, P(i32), P(vp), P(CusaKv), P(vp), vp, vp, vp, sz, vp]
    for name in ("cusa_workspace_bytes", "cusa_workspace_layout", "cusa_select", "cusa_sparse_attn",
                 "cusa_select_per_head", "cusa_sparse_attn_per_head", "cusa_attention_recall", "cusa_select_layer",
                 "cusa_full_attn", "cusa_decode_step", "cusa_profile_read"):
        getattr(lib, name).restype = ctypes.c_int
    lib.cusa_strerror.argtypes = [ctypes.c_int]
    lib.cusa_strerror.restype = ctypes.c_char_p
    lib.cusa_profile_num_kernels.restype = i32
    lib.cusa_profile_kernel_name.argtypes = [i32]
    lib.cusa_profile_kernel_name.restype = ctypes.c_char_p
    lib.cusa_profile_enable.argtypes = [i32]
    lib.cusa_profile_reset.argtypes = []
    lib.cusa_profile_read.argtypes = [i32, P(ctypes.c_int64), P(ctypes.c_double)]
    lib.cusa_build_id.restype = ctypes.c_char_p
    lib.cusa_sparse_attn_noalloc.argtypes = [P(CusaParams), vp, P(CusaKv), vp, vp, vp, vp]
    lib.cusa_sparse_attn_noalloc.restype = ctypes.c_int
    lib.cusa_noalloc_max_scratch_bytes.argtypes = []
    lib.cusa_noalloc_max_scratch_bytes.restype = sz
    lib.cusa_kv_plan_workspace_bytes.argtypes = [i32]
    lib.cusa_kv_plan_workspace_bytes.restype = sz
    lib.cusa_kv_plan.argtypes = [P(CusaPool), vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
    lib.cusa_kv_append.argtypes = [P(CusaParams), P(CusaKv), vp, P(CusaRows), vp]
    lib.cusa_tree_masks.argtypes = [i32, vp, vp, vp, i32, i32, vp, vp, vp]
    lib.cusa_tree_workspace_bytes.argtypes = [P(CusaParams), i32, i32, i32, P(sz)]
    lib.cusa_tree_attn.argtypes = [P(CusaParams), vp, P(CusaKv), P(CusaTree), vp, vp, vp, vp, sz, vp]
    lib.cusa_kv_commit.argtypes = [P(CusaParams), i32, P(CusaKv), vp, vp, i32, vp, vp, vp]
    for name in ("cusa_kv_plan", "cusa_kv_append", "cusa_tree_masks", "cusa_tree_workspace_bytes", "cusa_tree_attn", "cusa_kv_commit"):
        getattr(lib, name).restype = ctypes.c_int
    lib.cusa_probe_stream_read.argtypes = [vp, sz, vp, vp]
    lib.cusa_probe_stream_read.restype = ctypes.c_int
    lib.cusa_probe_traffic.argtypes = [i32, vp, sz, vp, sz, vp]
    lib.cusa_probe_traffic.restype = ctypes.c_int
    _lib = lib
    return lib


def strerror(status: int) -> str:
    return load().cusa_strerror(int(status)).decode()


def _check(status: int, where: str):
    if status != OK:
        raise CusaError(status, where)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def stream_query(torch_module):
    """A function that returns the current device's current stream as a hipStream_t.  (Asked for as the raw handle: the Stream
    object that torch.cuda.current_stream() builds around it costs 2.6 us of the 11.4 a call to sparse_attn took on the host,
    more than the GPU needs for its kernels in the smallest cases.  The two names are not part of torch's public interface;
    a torch without them is asked the public way.)"""
    cuda = torch_module.cuda
    raw = getattr(torch_module._C, "_cuda_getCurrentRawStream", None)
    device = getattr(torch_module._C, "_cuda_getDevice", None)

    def public() -> int:
        return cuda.current_stream().cuda_stream

    if raw is None or device is None:
        return public
    return lambda: raw(device()) if cuda.is_initialized() else public()


_stream = stream_query(torch)


def make_params(batch, n_q_heads, n_kv_heads, budget, window, topk_per_head=0, head_dim=128,
                sm_scale=None, rank_mode=RANK_FIRST_OCCURRENCE, n_sink=0) -> CusaParams:
    if sm_scale is None:
        sm_scale = head_dim ** -0.5
    return CusaParams(batch, n_q_heads, n_kv_heads, head_dim, budget, window, topk_per_head, n_sink,
                      rank_mode, sm_scale)


@dataclass
class KvCache:
    """One layer's cache view; keeps the tensors alive and builds the C descriptor."""
    k: torch.Tensor
    v: torch.Tensor
    seq_lens: torch.Tensor                      # int32 [B] on device
    max_seq_len: int
    block_table: Optional[torch.Tensor] = None  # int32 [B, max_pages] -> paged

    def desc(self) -> CusaKv:
        if self.block_table is None:
            assert self.k.dim() == 4 and self.k.stride(3) == 1 and self.k.stride() == self.v.stride()
            sb, sh, st, _ = self.k.stride()
            return CusaKv(self.k.data_ptr(), self.v.data_ptr(), KV_CONTIGUOUS, sb, sh, st, None, 0, 0, 0,
                          self.seq_lens.data_ptr(), self.max_seq_len)
        assert self.k.is_contiguous() and self.v.is_contiguous() and self.block_table.is_contiguous()
        n_pages, _, page, _ = self.k.shape
        return CusaKv(self.k.data_ptr(), self.v.data_ptr(), KV_PAGED, 0, 0, 0, self.block_table.data_ptr(),
                      self.block_table.shape[1], page, n_pages, self.seq_lens.data_ptr(), self.max_seq_len)


def workspace_bytes(params: CusaParams, max_seq_len: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load().cusa_workspace_bytes(ctypes.byref(params), max_seq_len, ctypes.byref(n)), "cusa_workspace_bytes")
    return int(n.value)


def workspace_layout(params: CusaParams, max_seq_len: int) -> CusaWsLayout:
    lay = CusaWsLayout()
    _check(load().cusa_workspace_layout(ctypes.byref(params), max_seq_len, ctypes.byref(lay)),
           "cusa_workspace_layout")
    return lay


def alloc_workspace(params: CusaParams, max_seq_len: int, device="cuda") -> torch.Tensor:
    return torch.empty(workspace_bytes(params, max_seq_len), dtype=torch.uint8, device=device)


def select(params: CusaParams, q: torch.Tensor, kv: KvCache, idx: torch.Tensor, cnt: torch.Tensor,
           ws: torch.Tensor):
    d = kv.desc()
    _check(load().cusa_select(ctypes.byref(params), _ptr(q), ctypes.byref(d), _ptr(idx), _ptr(cnt), _ptr(ws),
                              ws.numel(), _stream()), "cusa_select")


def sparse_attn(params: CusaParams, q, kv: KvCache, idx, cnt, out, ws):
    d = kv.desc()
    _check(load().cusa_sparse_attn(ctypes.byref(params), _ptr(q), ctypes.byref(d), _ptr(idx), _ptr(cnt),
                                   _ptr(out), _ptr(ws), ws.numel(), _stream()), "cusa_sparse_attn")


def sparse_attn_noalloc(params: CusaParams, q, kv: KvCache, idx, cnt, out):
    """cusa_sparse_attn with the partials in the library's static scratch (no workspace argument)."""
    d = kv.desc()
    _check(load().cusa_sparse_attn_noalloc(ctypes.byref(params), _ptr(q), ctypes.byref(d), _ptr(idx), _ptr(cnt),
                                           _ptr(out), _stream()), "cusa_sparse_attn_noalloc")


def noalloc_max_scratch_bytes() -> int:
    return int(load().cusa_noalloc_max_scratch_bytes())


def select_per_head(params: CusaParams, q, kv: KvCache, idx_head, cnt, ws):
    """idx_head: int32 [B, H, budget]; every head keeps its own picks (head-to-head selection)."""
    d = kv.desc()
    _check(load().cusa_select_per_head(ctypes.byref(params), _ptr(q), ctypes.byref(d), _ptr(idx_head), _ptr(cnt),
                                       _ptr(ws), ws.numel(), _stream()), "cusa_select_per_head")


def sparse_attn_per_head(params: CusaParams, q, kv: KvCache, idx_head, cnt, out, ws):
    d = kv.desc()
    _check(load().cusa_sparse_attn_per_head(ctypes.byref(params), _ptr(q), ctypes.byref(d), _ptr(idx_head), _ptr(cnt),
                                            _ptr(out), _ptr(ws), ws.numel(), _stream()), "cusa_sparse_attn_per_head")


def attention_recall(params: CusaParams, q, kv: KvCache, idx, cnt, recall, ws, per_head: bool = False):
    """recall: float32 [B, H], Eq. 3 for the token set idx/cnt (idx [B, H, budget] when per_head)."""
    d = kv.desc()
    _check(load().cusa_attention_recall(ctypes.byref(params), _ptr(q), ctypes.byref(d), _ptr(idx), _ptr(cnt),
                                        1 if per_head else 0, _ptr(recall), _ptr(ws), ws.numel(), _stream()),
           "cusa_attention_recall")


def select_layer(params: CusaParams, q, kv: KvCache, out, idx, cnt, ws):
    """A selection layer in one call: full-attention output and rho from one pass over K."""
    d = kv.desc()
    _check(load().cusa_select_layer(ctypes.byref(params), _ptr(q), ctypes.byref(d), _ptr(out), _ptr(idx), _ptr(cnt),
                                    _ptr(ws), ws.numel(), _stream()), "cusa_select_layer")


def full_attn(params: CusaParams, q, kv: KvCache, out, ws):
    d = kv.desc()
    _check(load().cusa_full_attn(ctypes.byref(params), _ptr(q), ctypes.byref(d), _ptr(out), _ptr(ws),
                                 ws.numel(), _stream()), "cusa_full_attn")


class DecodeStep:
    """Marshals one decode step's per-layer pointers once, then replays cusa_decode_step."""

    def __init__(self, params: CusaParams, layer_kind: Sequence[int], q_layers: List[torch.Tensor],
                 kv_layers: List[KvCache], out_layers: List[torch.Tensor], idx, cnt, ws):
        n = len(layer_kind)
        assert len(q_layers) == len(kv_layers) == len(out_layers) == n
        self.params, self.n = params, n
        self._keep = (q_layers, kv_layers, out_layers, idx, cnt, ws)
        self.kinds = (ctypes.c_int32 * n)(*layer_kind)
        self.qs = (ctypes.c_void_p * n)(*[t.data_ptr() for t in q_layers])
        self.outs = (ctypes.c_void_p * n)(*[t.data_ptr() for t in out_layers])
        self.kvs = (CusaKv * n)(*[kv.desc() for kv in kv_layers])
        self.idx, self.cnt, self.ws = idx, cnt, ws

    def run(self):
        _check(load().cusa_decode_step(ctypes.byref(self.params), self.n, self.kinds, self.qs, self.kvs,
                                       self.outs, _ptr(self.idx), _ptr(self.cnt), _ptr(self.ws),
                                       self.ws.numel(), _stream()), "cusa_decode_step")


def decode_step(params, layer_kind, q_layers, kv_layers, out_layers, idx, cnt, ws):
    DecodeStep(params, layer_kind, q_layers, kv_layers, out_layers, idx, cnt, ws).run()


# ---- decoding with trees of drafted tokens -------------------------------------

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


@dataclass
class PagePool:
    """A paged cache's bookkeeping on the device: who holds which pages, and the queue of those that are free."""
    block_table: torch.Tensor   # int32 [B, max_pages]
    ring: torch.Tensor          # int32 [n_pages]
    state: torch.Tensor         # int32 [2]: first free entry of the ring, number of free pages

    @staticmethod
    def empty(batch: int, max_pages: int, n_pages: int, device="cuda") -> "PagePool":
        """A pool whose pages are all free."""
        return PagePool(torch.full((batch, max_pages), -1, dtype=torch.int32, device=device),
                        torch.arange(n_pages, dtype=torch.int32, device=device),
                        torch.tensor([0, n_pages], dtype=torch.int32, device=device))

    def desc(self, state_out: Optional[torch.Tensor] = None) -> CusaPool:
        assert self.block_table.is_contiguous() and self.ring.is_contiguous()
        b, max_pages = self.block_table.shape
        return CusaPool(KV_PAGED, b, 0, self.block_table.data_ptr(), max_pages, 16, self.ring.numel(), self.ring.data_ptr(),
                        self.state.data_ptr(), (self.state if state_out is None else state_out).data_ptr())


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _need_int(what: str, n: int, dtype, *tensors):
    """Every tensor holds n contiguous numbers of this type at least, on the GPU.  (A step makes these calls once a layer: the message is made when it is needed.)"""
    for t in tensors:
        if t.dtype is not dtype or t.numel() < n or not t.is_contiguous() or not t.is_cuda:
            raise ValueError(f"{what}: a tensor of {n} or more {dtype}, contiguous, on the GPU was expected, not {tuple(t.shape)} {t.dtype} on {t.device}")


def _need_rows(what: str, name: str, rows: torch.Tensor, n: int, width: int, dtype):
    """n rows of this many numbers at least (or a flat tensor of them), contiguous, on the GPU."""
    shape = rows.shape
    if rows.dtype is not dtype or rows.numel() < n * width or (len(shape) > 1 and shape[-1] != width) or not rows.is_contiguous() or not rows.is_cuda:
        raise ValueError(f"{what}: {name} of {n} or more rows of {width} {dtype}, contiguous, on the GPU was expected, not {tuple(shape)} {rows.dtype} on {rows.device}")


def _need_workspace(what: str, ws: torch.Tensor):
    if ws.dtype is not torch.uint8 or not ws.is_contiguous() or not ws.is_cuda:
        raise ValueError(f"{what}: a workspace of uint8, contiguous, on the GPU was expected, not {tuple(ws.shape)} {ws.dtype} on {ws.device}")


def _strides(t: torch.Tensor, alone):
    """A tensor's strides; those of dimensions of one entry mean nothing (torch may have anything there) and are what `alone` has."""
    return tuple(a if n == 1 else s for n, s, a in zip(t.shape, t.stride(), alone))


def _cache_desc(what: str, params: CusaParams, kv: KvCache) -> CusaKv:
    """The cache's descriptor, as KvCache.desc makes it, if it has the rows that the parameters speak of: kernels write there.  (Each of a step's calls makes
    one a layer: a tensor is asked once for each thing.)"""
    k, v, table, lens = kv.k, kv.v, kv.block_table, kv.seq_lens
    shape, batch, bf16 = k.shape, params.batch, torch.bfloat16
    if (len(shape) == 4 and v.shape == shape and shape[1] == params.n_kv_heads and shape[3] == params.head_dim and k.dtype is bf16 and v.dtype is bf16
            and k.is_cuda and v.is_cuda and lens.dtype is torch.int32 and lens.numel() >= batch and lens.is_cuda and lens.is_contiguous()):
        if table is None:
            strides, of_v = k.stride(), v.stride()
            if 1 in shape and (strides != of_v or (strides[0] | strides[1] | strides[2]) & 7 or strides[2] < params.head_dim):   # (mostly they do as they are)
                alone = (0, 0, params.head_dim, 1)
                strides, of_v = _strides(k, alone), _strides(v, alone)
            if shape[0] >= batch and strides[3] == 1 and strides == of_v and kv.max_seq_len <= shape[2]:
                return CusaKv(k.data_ptr(), v.data_ptr(), KV_CONTIGUOUS, strides[0], strides[1], strides[2], None, 0, 0, 0, lens.data_ptr(), kv.max_seq_len)
        elif (k.is_contiguous() and v.is_contiguous() and table.dim() == 2 and table.shape[0] >= batch and table.dtype is torch.int32 and table.is_cuda
                and table.is_contiguous()):
            return CusaKv(k.data_ptr(), v.data_ptr(), KV_PAGED, 0, 0, 0, table.data_ptr(), table.shape[1], shape[2], shape[0], lens.data_ptr(), kv.max_seq_len)
    raise ValueError(f"{what}: K and V are bf16 [batch or pages, {params.n_kv_heads}, tokens, {params.head_dim}] of equal strides (pages contiguous), lengths and tables int32 of "
                     f"{batch} or more sequences, contiguous, all on the GPU, max_seq_len at most the tokens of a contiguous cache; K is {tuple(shape)} {k.dtype} on {k.device}, "
                     f"max_seq_len {kv.max_seq_len}")


def kv_plan_workspace_bytes(batch: int) -> int:
    return int(load().cusa_kv_plan_workspace_bytes(batch))


def alloc_plan_workspace(batch: int, device="cuda") -> torch.Tensor:
    return torch.empty(kv_plan_workspace_bytes(batch), dtype=torch.uint8, device=device)


def kv_plan(held, keep, add, lens, tok_start, slots, ws, pool: Optional[PagePool] = None, state_out=None, capacity: int = 0):
    """Room for add[b] tokens behind the keep[b] first of the held[b] that sequence b has: block tables (pool, or a contiguous cache of
    `capacity` positions a sequence), lens, tok_start and the slots of the new rows (int64, its length bounds the batch's tokens).
    state_out: where the queue's state goes instead of back into the pool, to ask without taking."""
    n = held.numel()
    _need_int("kv_plan", n, torch.int32, held, keep, add, lens)
    _need_int("kv_plan", n + 1, torch.int32, tok_start)
    _need_int("kv_plan", 0, torch.int64, slots)
    _need_workspace("kv_plan", ws)
    if pool is None:
        d = CusaPool(KV_CONTIGUOUS, n, capacity, None, 0, 0, 0, None, None, None)
    else:
        _need(pool.block_table.shape[0] == n, "kv_plan: a row of the block table for each sequence")
        _need_int("kv_plan", 2, torch.int32, pool.state, pool.state if state_out is None else state_out)
        _need_int("kv_plan", 1, torch.int32, pool.block_table, pool.ring)
        d = pool.desc(state_out)
    _check(load().cusa_kv_plan(ctypes.byref(d), held.data_ptr(), keep.data_ptr(), add.data_ptr(), slots.numel(), lens.data_ptr(), tok_start.data_ptr(),
                               slots.data_ptr(), ws.data_ptr(), ws.numel(), _stream()), "cusa_kv_plan")


def kv_append(params: CusaParams, kv: KvCache, slots, k_new, v_new):
    """Rows k_new, v_new [n, G, 128] (bf16, fp16 or fp32; views with equal strides, as of a fused projection) to their slots in one layer's cache."""
    n, heads, d = k_new.shape
    _need(k_new.dtype in DTYPES and v_new.dtype == k_new.dtype and v_new.shape == k_new.shape and d == params.head_dim and
          heads == params.n_kv_heads, "kv_append: new rows are [n, n_kv_heads, 128] in bf16, fp16 or fp32")
    strides, of_v = k_new.stride(), v_new.stride()
    if n == 1 or heads == 1:
        strides, of_v = _strides(k_new, (0, 0, 1)), _strides(v_new, (0, 0, 1))
    _need(strides[2] == 1 and strides == of_v, "kv_append: K and V rows have the same strides, elements side by side")
    _need(k_new.is_cuda and v_new.is_cuda, "kv_append: new rows are on the GPU")
    _need_int("kv_append", n, torch.int64, slots)
    c = _cache_desc("kv_append", params, kv)
    r = CusaRows(k_new.data_ptr(), v_new.data_ptr(), DTYPES[k_new.dtype], n, strides[0], strides[1])
    _check(load().cusa_kv_append(ctypes.byref(params), ctypes.byref(c), slots.data_ptr(), ctypes.byref(r), _stream()), "cusa_kv_append")


def mask_words(max_nodes: int) -> int:
    """64-bit words of a node's mask."""
    return (max_nodes + 63) // 64


def tree_masks(base, tok_start, parents, masks, positions, max_nodes: int):
    """masks (int64 [tokens, mask_words], bit patterns) and positions (int32, or None) of trees given by their nodes' parents."""
    n = parents.numel()
    batch = tok_start.numel() - 1
    _need_int("tree_masks", batch, torch.int32, base)
    _need_int("tree_masks", 2, torch.int32, tok_start)
    _need_int("tree_masks", n, torch.int32, parents, parents if positions is None else positions)
    _need_rows("tree_masks", "masks", masks, n, mask_words(max_nodes), torch.int64)
    if n == 0:                                               # a step in which nothing was drafted
        return
    _check(load().cusa_tree_masks(batch, base.data_ptr(), tok_start.data_ptr(), parents.data_ptr(), n, max_nodes, masks.data_ptr(),
                                  _ptr(positions), _stream()), "cusa_tree_masks")


@dataclass
class Tree:
    """The drafted trees of a step, the same for all layers."""
    tok_start: torch.Tensor     # int32 [B + 1]
    masks: torch.Tensor         # int64 [tokens, mask_words(max_nodes)]
    max_nodes: int


def tree_workspace_bytes(params: CusaParams, max_seq_len: int, max_tokens: int, max_nodes: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load().cusa_tree_workspace_bytes(ctypes.byref(params), max_seq_len, max_tokens, max_nodes, ctypes.byref(n)), "cusa_tree_workspace_bytes")
    return int(n.value)


def alloc_tree_workspace(params: CusaParams, max_seq_len: int, max_tokens: int, max_nodes: int, device="cuda") -> torch.Tensor:
    return torch.empty(tree_workspace_bytes(params, max_seq_len, max_tokens, max_nodes), dtype=torch.uint8, device=device)


def tree_attn(params: CusaParams, q, kv: KvCache, tree: Tree, out, ws, idx=None, cnt=None):
    """Attention of the trees' nodes, q [tokens, H, 128] (a view of a fused projection's rows, or contiguous), over the whole prefix or
    over idx/cnt of it, and over the nodes that the masks name."""
    n, heads, d = q.shape
    strides = _strides(q, (heads * d, d, 1)) if n == 1 or heads == 1 else q.stride()
    _need(q.dtype is torch.bfloat16 and heads == params.n_q_heads and d == params.head_dim and strides[2] == 1 and strides[1] == d,
          "tree_attn: q is bf16 [tokens, n_q_heads, 128], heads side by side")
    _need(q.is_cuda and out.is_cuda, "tree_attn: q and out are on the GPU")
    _need(out.dtype == torch.bfloat16 and out.is_contiguous() and out.numel() >= n * heads * d, "tree_attn: out is bf16 [tokens, n_q_heads, 128], contiguous")
    _need_workspace("tree_attn", ws)
    _need_int("tree_attn", params.batch + 1, torch.int32, tree.tok_start)
    _need_rows("tree_attn", "masks", tree.masks, n, mask_words(tree.max_nodes), torch.int64)
    if idx is not None:
        _need_rows("tree_attn", "idx", idx, params.batch, params.budget, torch.int32)
        _need(cnt is not None, "tree_attn: idx comes with cnt")
        _need_int("tree_attn", params.batch, torch.int32, cnt)
    c = _cache_desc("tree_attn", params, kv)
    if n == 0:
        return
    t = CusaTree(tree.tok_start.data_ptr(), tree.masks.data_ptr(), n, tree.max_nodes, strides[0])
    _check(load().cusa_tree_attn(ctypes.byref(params), q.data_ptr(), ctypes.byref(c), ctypes.byref(t), _ptr(idx), _ptr(cnt), out.data_ptr(), ws.data_ptr(),
                                 ws.numel(), _stream()), "cusa_tree_attn")


class KvCommit:
    """Marshals the layers' caches once; run() moves the accepted branches' rows together in all of them."""

    def __init__(self, params: CusaParams, kv_layers: Sequence[KvCache]):
        self.params, self.n = params, len(kv_layers)
        self._keep = list(kv_layers)
        self.kvs = (CusaKv * self.n)(*[_cache_desc("kv_commit", params, kv) for kv in kv_layers])

    def run(self, base, path, n_path, keep=None):
        """Positions base[b] + path[b][i] -> base[b] + i for i < n_path[b]; keep (not base): base + n_path."""
        b = self.params.batch
        _need(path.dim() == 2 and path.shape[0] == b, "kv_commit: path is [batch, nodes]")
        _need_int("kv_commit", b, torch.int32, base, path, n_path, n_path if keep is None else keep)
        _check(load().cusa_kv_commit(ctypes.byref(self.params), self.n, self.kvs, base.data_ptr(), path.data_ptr(), path.shape[1], n_path.data_ptr(),
                                     _ptr(keep), _stream()), "cusa_kv_commit")


def kv_commit(params, kv_layers, base, path, n_path, keep=None):
    KvCommit(params, kv_layers).run(base, path, n_path, keep)


def probe_stream_read(src: torch.Tensor, sink: torch.Tensor):
    """Enqueue the streaming-read probe over the bytes of src (benchmark support)."""
    _check(load().cusa_probe_stream_read(_ptr(src), src.numel() * src.element_size(), _ptr(sink), _stream()),
           "cusa_probe_stream_read")


def probe_traffic(pattern: int, src: torch.Tensor, dst: torch.Tensor):
    """Enqueue a traffic probe (0 stream in tiles, 1 gathered rows, 2 stream + scattered writes, 3 stream + burst writes)."""
    _check(load().cusa_probe_traffic(pattern, _ptr(src), src.numel() * src.element_size(), _ptr(dst),
                                     dst.numel() * dst.element_size(), _stream()), "cusa_probe_traffic")


# ---- per-kernel timing ---------------------------------------------------------

def profile_enable(on: bool):
    load().cusa_profile_enable(1 if on else 0)


def profile_reset():
    load().cusa_profile_reset()


def profile_read() -> dict:
    lib = load()
    n = lib.cusa_profile_num_kernels()
    calls = (ctypes.c_int64 * n)()
    ms = (ctypes.c_double * n)()
    _check(lib.cusa_profile_read(n, calls, ms), "cusa_profile_read")
    return {lib.cusa_profile_kernel_name(i).decode(): {"calls": int(calls[i]), "total_ms": float(ms[i])}
            for i in range(n)}
