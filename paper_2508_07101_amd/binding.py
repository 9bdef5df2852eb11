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
    "cusa_beam_workspace_bytes", "cusa_beam_select", "cusa_kv_fork_workspace_bytes", "cusa_kv_fork", "cusa_kv_copy", "cusa_shared_pages_workspace_bytes",
    "cusa_shared_pages", "cusa_beam_attn_workspace_bytes", "cusa_beam_attn",
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


class CusaBeams(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("stride", ctypes.c_int64), ("rows", ctypes.c_int32), ("width", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("n", ctypes.c_int32), ("end_token", ctypes.c_int32)]


class CusaShared(ctypes.Structure):
    _fields_ = [("width", ctypes.c_int32), ("max_entries", ctypes.c_int32), ("entries", ctypes.c_void_p), ("count", ctypes.c_void_p)]


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
    lib.cusa_beam_workspace_bytes.argtypes = [i32, i32, i32, P(sz)]
    lib.cusa_beam_select.argtypes = [P(CusaBeams), vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.cusa_kv_fork_workspace_bytes.argtypes = [i32, i32]
    lib.cusa_kv_fork_workspace_bytes.restype = sz
    lib.cusa_kv_fork.argtypes = [P(CusaPool), i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.cusa_kv_copy.argtypes = [P(CusaParams), i32, P(CusaKv), vp, i32, vp]
    lib.cusa_shared_pages_workspace_bytes.argtypes = [i32, i32]
    lib.cusa_shared_pages_workspace_bytes.restype = sz
    lib.cusa_shared_pages.argtypes = [P(CusaKv), i32, P(CusaShared), vp, sz, vp]
    lib.cusa_beam_attn_workspace_bytes.argtypes = [P(CusaParams), i32, P(CusaShared), P(sz)]
    lib.cusa_beam_attn.argtypes = [P(CusaParams), vp, ctypes.c_int64, P(CusaKv), P(CusaShared), vp, vp, sz, vp]
    for name in ("cusa_beam_workspace_bytes", "cusa_beam_select", "cusa_kv_fork", "cusa_kv_copy", "cusa_shared_pages", "cusa_beam_attn_workspace_bytes", "cusa_beam_attn"):
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


# ---- beam search over paged caches ---------------------------------------------

def _device() -> int:
    return torch.cuda.current_device()


if hasattr(torch._C, "_cuda_getDevice"):
    _device = torch._C._cuda_getDevice                           # noqa: F811  (what current_device() asks once CUDA is up; a tenth of its time)


def _take(what: str, name: str, t: torch.Tensor, dtype, n: int, gpu: int, width: int = 0) -> int:
    """The address of a tensor that holds n contiguous numbers of this type at least (in rows of `width`, or flat), on the current GPU."""
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous() or t.get_device() != gpu or (width and t.shape[-1] != width and t.dim() > 1):
        rows = f" in rows of {width}" if width else ""
        raise ValueError(f"{what}: {name} of {n} or more {dtype}{rows}, contiguous, on the current GPU was expected, not {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _need_group(what: str, rows: int, width: int):
    if width < 1 or rows < 1 or rows % width != 0:
        raise ValueError(f"{what}: groups of {width} rows in {rows}")


def beam_workspace_bytes(rows: int, vocab: int, n: int) -> int:
    b = ctypes.c_size_t(0)
    _check(load().cusa_beam_workspace_bytes(rows, vocab, n, ctypes.byref(b)), "cusa_beam_workspace_bytes")
    return int(b.value)


def alloc_beam_workspace(rows: int, vocab: int, n: int, device="cuda") -> torch.Tensor:
    return torch.empty(beam_workspace_bytes(rows, vocab, n), dtype=torch.uint8, device=device)


def beam_select(logits, scores, width: int, out_scores, parents, tokens, ws, ended=None, out_ended=None, end_token: int = -1):
    """The best continuations of every group of `width` rows: logits [rows, vocab] (bf16, fp16 or fp32; a view of wider rows, or contiguous), scores float32 [rows];
    out_scores float32, parents, tokens and out_ended int32, [groups, n] each, best first.  ended int32 [rows]: rows that propose nothing but end_token."""
    what, gpu = "beam_select", _device()
    if logits.dim() != 2 or logits.dtype not in DTYPES or logits.get_device() != gpu:
        raise ValueError(f"{what}: logits are [rows, vocab] in bf16, fp16 or fp32, on the current GPU, not {tuple(logits.shape)} {logits.dtype} on {logits.device}")
    rows, vocab = logits.shape
    _need_group(what, rows, width)
    strides = logits.stride() if rows > 1 and vocab > 1 else _strides(logits, (vocab, 1))
    _need(strides[1] == 1 and strides[0] >= vocab, "beam_select: a row's logits stand side by side")
    groups = rows // width
    _need(out_scores.dim() == 2 and out_scores.shape[0] == groups, "beam_select: out_scores is [groups, n]")
    n = out_scores.shape[1]
    d = CusaBeams(logits.data_ptr(), DTYPES[logits.dtype], strides[0], rows, width, vocab, n, end_token)
    _check(load().cusa_beam_select(
        ctypes.byref(d), _take(what, "scores", scores, torch.float32, rows, gpu), None if ended is None else _take(what, "ended", ended, torch.int32, rows, gpu),
        _take(what, "out_scores", out_scores, torch.float32, groups * n, gpu), _take(what, "parents", parents, torch.int32, groups * n, gpu, n),
        _take(what, "tokens", tokens, torch.int32, groups * n, gpu, n), None if out_ended is None else _take(what, "out_ended", out_ended, torch.int32, groups * n, gpu, n),
        _take(what, "workspace", ws, torch.uint8, 0, gpu), ws.numel(), _stream()), "cusa_beam_select")


def fork_workspace_bytes(batch: int, max_pages: int) -> int:
    return int(load().cusa_kv_fork_workspace_bytes(batch, max_pages))


def alloc_fork_workspace(pool: PagePool) -> torch.Tensor:
    return torch.empty(fork_workspace_bytes(*pool.block_table.shape), dtype=torch.uint8, device=pool.block_table.device)


def kv_fork(pool: PagePool, width: int, held, parents, lens, slots, copies, ws, ended=None, grow: bool = True, table_out=None, state_out=None, granted=None):
    """Rows of a group take over the tokens of the rows that they descend from (parents, int32, numbers within the group; -1: none), and with `grow` each that has a parent and has
    not ended gets room for one token: lens int32 [B], slots int64 [B], copies int32 [B, 4] (from, to, tokens, 0: KvCopy makes them).
    table_out, state_out: where the new table and the queue's state go instead of back into the pool."""
    what, gpu, i32 = "kv_fork", _device(), torch.int32
    table, ring, state = pool.block_table, pool.ring, pool.state
    _need(table.dim() == 2, "kv_fork: the block table is [rows, columns]")
    n, max_pages = table.shape
    _need_group(what, n, width)
    at = _take(what, "block_table", table, i32, 1, gpu)
    at_state = _take(what, "state", state, i32, 2, gpu)
    d = CusaPool(KV_PAGED, n, 0, at, max_pages, 16, ring.numel(), _take(what, "ring", ring, i32, 1, gpu), at_state,
                 at_state if state_out is None else _take(what, "state_out", state_out, i32, 2, gpu))
    _check(load().cusa_kv_fork(
        ctypes.byref(d), width, _take(what, "held", held, i32, n, gpu), _take(what, "parents", parents, i32, n, gpu),
        None if ended is None else _take(what, "ended", ended, i32, n, gpu), 1 if grow else 0,
        at if table_out is None else _take(what, "table_out", table_out, i32, n * max_pages, gpu, max_pages), _take(what, "lens", lens, i32, n, gpu),
        _take(what, "slots", slots, torch.int64, n, gpu), _take(what, "copies", copies, i32, n * 4, gpu, 4),
        None if granted is None else _take(what, "granted", granted, i32, n // width, gpu), _take(what, "workspace", ws, torch.uint8, 0, gpu), ws.numel(), _stream()), "cusa_kv_fork")


class KvCopy:
    """Marshals the layers' caches once; run() copies pages in all of them."""

    def __init__(self, params: CusaParams, kv_layers: Sequence[KvCache]):
        self.params, self.n = params, len(kv_layers)
        self._keep = list(kv_layers)
        _need(all(kv.block_table is not None for kv in kv_layers), "kv_copy: paged caches")
        self.kvs = (CusaKv * self.n)(*[_cache_desc("kv_copy", params, kv) for kv in kv_layers])

    def run(self, copies):
        """copies int32 [n, 4]: from, to, tokens, 0."""
        _need(copies.dim() == 2, "kv_copy: copies is [n, 4]")
        n = copies.shape[0]
        if n == 0:
            return
        at = _take("kv_copy", "copies", copies, torch.int32, n * 4, _device(), 4)
        _check(load().cusa_kv_copy(ctypes.byref(self.params), self.n, self.kvs, at, n, _stream()), "cusa_kv_copy")


def kv_copy(params, kv_layers, copies):
    KvCopy(params, kv_layers).run(copies)


@dataclass
class SharedPages:
    """The pages of groups of `width` rows, each once, with the rows that hold it."""
    width: int
    entries: torch.Tensor       # int32 [groups, most, 4]: page, column, bits of the rows, 0
    count: torch.Tensor         # int32 [groups, 2]: entries, and how many at the front all rows attend to as a whole

    @staticmethod
    def empty(batch: int, width: int, max_seq_len: int, n_pages: int, device="cuda") -> "SharedPages":
        most = min(width * ((max_seq_len + 15) // 16), n_pages)
        return SharedPages(width, torch.zeros((batch // width, most, 4), dtype=torch.int32, device=device), torch.zeros((batch // width, 2), dtype=torch.int32, device=device))

    def desc(self, what: str, batch: int, gpu: int) -> CusaShared:
        e, c, width, i32 = self.entries, self.count, self.width, torch.int32
        shape, groups = e.shape, batch // width if width > 0 else 0
        # (each layer's call makes one: everything is asked once, and what is wrong only where something is)
        if (groups < 1 or groups * width != batch or len(shape) != 3 or shape[0] < groups or shape[2] != 4 or e.dtype is not i32 or c.dtype is not i32
                or c.numel() < groups * 2 or c.shape[-1] != 2 or not e.is_contiguous() or not c.is_contiguous() or e.get_device() != gpu or c.get_device() != gpu):
            _need_group(what, batch, width)
            _need(len(shape) == 3 and shape[0] >= groups and shape[2] == 4, "entries of shared pages are [groups, most, 4]")
            return CusaShared(width, shape[1], _take(what, "entries", e, i32, groups * shape[1] * 4, gpu), _take(what, "count", c, i32, groups * 2, gpu, 2))
        return CusaShared(width, shape[1], e.data_ptr(), c.data_ptr())


def pages_workspace_bytes(batch: int, max_seq_len: int) -> int:
    return int(load().cusa_shared_pages_workspace_bytes(batch, max_seq_len))


def alloc_pages_workspace(batch: int, max_seq_len: int, device="cuda") -> torch.Tensor:
    return torch.empty(pages_workspace_bytes(batch, max_seq_len), dtype=torch.uint8, device=device)


def shared_pages(block_table, lens, max_seq_len: int, n_pages: int, shared: SharedPages, ws):
    """Which pages the groups hold, from the rows' block table and lengths: once a step, for all its layers."""
    what, gpu = "shared_pages", _device()
    _need(block_table.dim() == 2, "shared_pages: block_table is [rows, columns]")
    n, columns = block_table.shape
    d = shared.desc(what, n, gpu)
    kv = CusaKv(None, None, KV_PAGED, 0, 0, 0, _take(what, "block_table", block_table, torch.int32, n * columns, gpu), columns, 16, n_pages,
                _take(what, "lens", lens, torch.int32, n, gpu), max_seq_len)
    _check(load().cusa_shared_pages(ctypes.byref(kv), n, ctypes.byref(d), _take(what, "workspace", ws, torch.uint8, 0, gpu), ws.numel(), _stream()), "cusa_shared_pages")


def beam_attn_workspace_bytes(params: CusaParams, max_seq_len: int, shared: SharedPages) -> int:
    n, d = ctypes.c_size_t(0), shared.desc("beam_attn", params.batch, shared.entries.get_device())
    _check(load().cusa_beam_attn_workspace_bytes(ctypes.byref(params), max_seq_len, ctypes.byref(d), ctypes.byref(n)), "cusa_beam_attn_workspace_bytes")
    return int(n.value)


def alloc_beam_attn_workspace(params: CusaParams, max_seq_len: int, shared: SharedPages, device="cuda") -> torch.Tensor:
    return torch.empty(beam_attn_workspace_bytes(params, max_seq_len, shared), dtype=torch.uint8, device=device)


def beam_attn(params: CusaParams, q, kv: KvCache, shared: SharedPages, out, ws):
    """Full attention of every row's token, q [B, H, 128] (a view of a fused projection's rows, or contiguous), over the pages of its group: each is read once
    for all rows that hold it.  shared: of the same tables and lengths."""
    what, gpu = "beam_attn", _device()
    shape = q.shape
    _need(len(shape) == 3, "beam_attn: q is [batch, n_q_heads, 128]")
    n, heads, d = shape
    strides = _strides(q, (heads * d, d, 1)) if n == 1 or heads == 1 else q.stride()
    if q.dtype is not torch.bfloat16 or n != params.batch or heads != params.n_q_heads or d != params.head_dim or strides[2] != 1 or strides[1] != d or q.get_device() != gpu:
        raise ValueError("beam_attn: q is bf16 [batch, n_q_heads, 128], heads side by side, on the current GPU")
    if kv.block_table is None or kv.k.get_device() != gpu:
        raise ValueError("beam_attn: a paged cache on the current GPU")
    s = shared.desc(what, n, gpu)
    c = _cache_desc(what, params, kv)
    _check(load().cusa_beam_attn(ctypes.byref(params), q.data_ptr(), strides[0], ctypes.byref(c), ctypes.byref(s), _take(what, "out", out, torch.bfloat16, n * heads * d, gpu),
                                 _take(what, "workspace", ws, torch.uint8, 0, gpu), ws.numel(), _stream()), "cusa_beam_attn")


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
