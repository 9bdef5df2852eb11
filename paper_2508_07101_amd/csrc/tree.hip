// Host side of decoding with trees of drafted tokens: argument checks and launches.  Nothing here allocates or synchronises.
#include "host.hpp"

#include <algorithm>

#include "tree_kernels.hpp"

using namespace cusa;

namespace {

constexpr int MAX_BATCH = 65535;           // a dimension of the grids
constexpr int64_t MAX_STRIDE = 1 << 26;    // elements between two tokens: some rows' offset fits 32 bits of bytes

size_t plan_ws_bytes(int batch) { return 256 + align256((size_t)batch * sizeof(PlanSeq)); }

cusa_status check_pool(const cusa_pool* p) {
    if (!p || p->batch < 1) return CUSA_ERR_INVALID_ARG;
    if (p->batch > MAX_BATCH) return CUSA_ERR_UNSUPPORTED;
    if (p->layout == CUSA_KV_CONTIGUOUS) return p->capacity < 1 ? CUSA_ERR_INVALID_ARG : CUSA_OK;
    if (p->layout != CUSA_KV_PAGED) return CUSA_ERR_INVALID_ARG;
    if (p->page_size != PAGE) return CUSA_ERR_UNSUPPORTED;
    if (!p->block_table || !p->ring || !p->state || !p->state_out || p->max_pages < 1 || p->n_pages < 1) return CUSA_ERR_INVALID_ARG;
    if (p->n_pages > 0x7fffffff || (int64_t)p->batch * p->max_pages > 0x7fffffff) return CUSA_ERR_UNSUPPORTED;
    return CUSA_OK;
}

// A cache that these kernels can address: check_kv's rules, row numbers and a token's stride that fit 31 bits.
cusa_status check_cache(const cusa_params* p, const cusa_kv* kv, bool reads_tables) {
    cusa_kv c;
    if (!kv) return CUSA_ERR_INVALID_ARG;
    c = *kv;
    if (!reads_tables) {                   // seq_lens and block_table may be missing where they are not read
        if (!c.seq_lens) c.seq_lens = reinterpret_cast<const int32_t*>(16);
        if (c.layout == CUSA_KV_PAGED && !c.block_table) c.block_table = reinterpret_cast<const int32_t*>(16);
        if (c.layout == CUSA_KV_PAGED) c.max_pages = 0x7fffffff / PAGE + 1;
    }
    const cusa_status st = check_kv(p, &c);
    if (st != CUSA_OK) return st;
    if (p->batch > MAX_BATCH || p->n_kv_heads > MAX_BATCH || kv->max_seq_len > (1 << 30)) return CUSA_ERR_UNSUPPORTED;
    if (kv->layout == CUSA_KV_CONTIGUOUS && kv->stride_token > MAX_STRIDE) return CUSA_ERR_UNSUPPORTED;
    if (kv->layout == CUSA_KV_PAGED && kv->n_pages > 0x7fffffff / PAGE / p->n_kv_heads) return CUSA_ERR_UNSUPPORTED;
    return CUSA_OK;
}

CacheArgs cache_args(const cusa_params* p, const cusa_kv* kv) {
    CacheArgs c;
    c.kv = make_view(p, kv);
    if (kv->layout != CUSA_KV_PAGED) c.kv.bt = nullptr;
    c.n_pages = (int32_t)std::min<int64_t>(kv->n_pages, 0x7fffffff);
    c.max_len = kv->max_seq_len;
    return c;
}

template <int DTYPE>
void launch_append(bool paged, dim3 grid, hipStream_t s, const AppendArgs& a) {
    if (paged) launch(KID_KV_APPEND, kv_append_kernel<DTYPE, true>, grid, APPEND_THREADS, 0, s, a);
    else launch(KID_KV_APPEND, kv_append_kernel<DTYPE, false>, grid, APPEND_THREADS, 0, s, a);
}

void launch_tree(bool paged, dim3 grid, hipStream_t s, const TreeArgs& a) {
    if (a.idx) {
        if (paged) launch(KID_TREE_ATTN, tree_attn_kernel<true, true>, grid, TREE_THREADS, 0, s, a);
        else launch(KID_TREE_ATTN, tree_attn_kernel<false, true>, grid, TREE_THREADS, 0, s, a);
    } else {
        if (paged) launch(KID_TREE_ATTN, tree_attn_kernel<true, false>, grid, TREE_THREADS, 0, s, a);
        else launch(KID_TREE_ATTN, tree_attn_kernel<false, false>, grid, TREE_THREADS, 0, s, a);
    }
}

cusa_status check_tree_sizes(int32_t max_tokens, int32_t max_nodes) {
    if (max_tokens < 1 || max_nodes < 1) return CUSA_ERR_INVALID_ARG;
    return max_nodes > TREE_MAX_NODES ? CUSA_ERR_UNSUPPORTED : CUSA_OK;
}

// Tokens of a sequence that a pass may have to look at.
int64_t tree_len(const cusa_params* p, int32_t max_seq_len, int32_t max_nodes, TreeKind kind) {
    return kind == TREE_CHOSEN ? (int64_t)p->budget + max_nodes : max_seq_len;
}

}  // namespace

extern "C" {

size_t cusa_kv_plan_workspace_bytes(int32_t batch) { return batch < 1 || batch > MAX_BATCH ? 0 : plan_ws_bytes(batch); }

cusa_status cusa_kv_plan(const cusa_pool* pool, const int32_t* held, const int32_t* keep, const int32_t* add, int32_t max_tokens,
                         int32_t* lens, int32_t* tok_start, int64_t* slots, void* ws, size_t ws_bytes, void* stream) {
    cusa_status st = check_pool(pool);
    if (st != CUSA_OK) return st;
    if (!held || !keep || !add || !lens || !tok_start || max_tokens < 0 || (max_tokens > 0 && !slots)) return CUSA_ERR_INVALID_ARG;
    if (lens == add || !ws || ((uintptr_t)ws & 255)) return CUSA_ERR_INVALID_ARG;
    if (ws_bytes < plan_ws_bytes(pool->batch)) return CUSA_ERR_WORKSPACE_TOO_SMALL;
    const bool paged = pool->layout == CUSA_KV_PAGED;
    PlanArgs a = {};
    a.held = held;
    a.keep = keep;
    a.add = add;
    a.lens = lens;
    a.tok_start = tok_start;
    a.slots = slots;
    a.table = paged ? pool->block_table : nullptr;
    a.ring = pool->ring;
    a.state = pool->state;
    a.state_out = pool->state_out;
    a.head = ws_ptr<PlanHead>(ws, 0);
    a.seq = ws_ptr<PlanSeq>(ws, 256);
    a.batch = pool->batch;
    a.max_tokens = max_tokens;
    a.max_pages = pool->max_pages;
    a.n_pages = (int32_t)pool->n_pages;
    a.cap = paged ? (int32_t)std::min<int64_t>((int64_t)pool->max_pages * PAGE, 0x7fffffff) : pool->capacity;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (max_tokens <= PLAN_ONE_LAUNCH && pool->batch <= PLAN_THREADS) {
        launch(KID_KV_PLAN, kv_plan_kernel<true>, 1, PLAN_THREADS, 0, s, a);
        return launch_status();
    }
    launch(KID_KV_PLAN, kv_plan_kernel<false>, 1, PLAN_THREADS, 0, s, a);
    if (launch_status() != CUSA_OK) return CUSA_ERR_LAUNCH;
    // enough for the tokens, and a workgroup a sequence for the pages that go back, also where no token comes
    const int64_t by_tokens = ((int64_t)max_tokens + FILL_THREADS * FILL_RUN - 1) / (FILL_THREADS * FILL_RUN);
    const int64_t wgs = std::min<int64_t>(std::max<int64_t>({by_tokens, paged ? pool->batch : 1, 1}), 2048);
    launch(KID_KV_FILL, kv_fill_kernel, dim3((unsigned)wgs), FILL_THREADS, 0, s, a);
    return launch_status();
}

cusa_status cusa_kv_append(const cusa_params* params, const cusa_kv* kv, const int64_t* slots, const cusa_rows* rows, void* stream) {
    cusa_status st = check_params(params, false);
    if (st != CUSA_OK) return st;
    if ((st = check_cache(params, kv, false)) != CUSA_OK) return st;
    if (!rows || rows->n < 0) return CUSA_ERR_INVALID_ARG;
    if (rows->n == 0) return CUSA_OK;
    if (!slots || !rows->k || !rows->v) return CUSA_ERR_INVALID_ARG;
    if (rows->dtype != CUSA_BF16 && rows->dtype != CUSA_F16 && rows->dtype != CUSA_F32) return CUSA_ERR_INVALID_ARG;
    const int align = rows->dtype == CUSA_F32 ? 4 : 8;     // elements of 16 bytes
    if (((uintptr_t)rows->k | (uintptr_t)rows->v) & 15) return CUSA_ERR_INVALID_ARG;
    if (rows->stride_token < 0 || rows->stride_head < 0 || rows->stride_token % align || rows->stride_head % align) return CUSA_ERR_INVALID_ARG;
    AppendArgs a;
    a.cache = cache_args(params, kv);
    a.slots = slots;
    a.k = rows->k;
    a.v = rows->v;
    a.st = rows->stride_token;
    a.sh = rows->stride_head;
    a.n = rows->n;
    a.batch = params->batch;
    const int64_t per_wg = APPEND_THREADS / 16 * APPEND_ROWS, wgs = ((int64_t)rows->n * 2 * params->n_kv_heads + per_wg - 1) / per_wg;
    if (wgs > 0x7fffffff) return CUSA_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)wgs);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool paged = kv->layout == CUSA_KV_PAGED;
    switch (rows->dtype) {
        case CUSA_BF16: launch_append<CUSA_BF16>(paged, grid, s, a); break;
        case CUSA_F16: launch_append<CUSA_F16>(paged, grid, s, a); break;
        default: launch_append<CUSA_F32>(paged, grid, s, a); break;
    }
    return launch_status();
}

cusa_status cusa_tree_masks(int32_t batch, const int32_t* base, const int32_t* tok_start, const int32_t* parents, int32_t max_tokens,
                            int32_t max_nodes, uint64_t* masks, int32_t* positions, void* stream) {
    if (batch < 1 || !tok_start || !parents || !masks || (positions && !base)) return CUSA_ERR_INVALID_ARG;
    const cusa_status st = check_tree_sizes(max_tokens, max_nodes);
    if (st != CUSA_OK) return st;
    if (batch > MAX_BATCH) return CUSA_ERR_UNSUPPORTED;
    const MasksArgs a = {base, tok_start, parents, masks, positions, max_tokens, max_nodes, (max_nodes + 63) / 64};
    launch(KID_TREE_MASKS, tree_masks_kernel, dim3((unsigned)batch), TREE_MAX_NODES, 0, static_cast<hipStream_t>(stream), a);
    return launch_status();
}

cusa_status cusa_tree_workspace_bytes(const cusa_params* params, int32_t max_seq_len, int32_t max_tokens, int32_t max_nodes, size_t* bytes) {
    cusa_status st = check_params(params, true);
    if (st != CUSA_OK) return st;
    if ((st = check_tree_sizes(max_tokens, max_nodes)) != CUSA_OK) return st;
    if (!bytes || max_seq_len < 1) return CUSA_ERR_INVALID_ARG;
    size_t most = 0;
    for (const TreeKind kind : {TREE_FULL, TREE_CHOSEN}) {   // of those that are served
        const int64_t len = tree_len(params, max_seq_len, max_nodes, kind);
        if (!tree_len_served(kind, len)) continue;
        most = std::max(most, tree_workspace(kind, (int)len, params->batch, params->n_q_heads, params->n_kv_heads, max_tokens, max_nodes).total);
    }
    *bytes = most;
    return CUSA_OK;
}

cusa_status cusa_tree_attn(const cusa_params* params, const void* q, const cusa_kv* kv, const cusa_tree* tree, const int32_t* idx,
                           const int32_t* cnt, void* out, void* ws, size_t ws_bytes, void* stream) {
    cusa_status st = check_params(params, true);
    if (st != CUSA_OK) return st;
    if ((st = check_cache(params, kv, true)) != CUSA_OK) return st;
    if (!tree || !tree->tok_start || !tree->masks || !q || !out || ((uintptr_t)q & 15) || ((uintptr_t)out & 15) || !idx != !cnt) return CUSA_ERR_INVALID_ARG;
    if ((st = check_tree_sizes(tree->max_tokens, tree->max_nodes)) != CUSA_OK) return st;
    if (tree->q_stride < (int64_t)params->n_q_heads * D || (tree->q_stride & 7)) return CUSA_ERR_INVALID_ARG;
    if (!ws || ((uintptr_t)ws & 255)) return CUSA_ERR_INVALID_ARG;
    const int g = params->n_q_heads / params->n_kv_heads, G = params->n_kv_heads;
    const TreeKind kind = idx ? TREE_CHOSEN : TREE_FULL;
    const int64_t len = tree_len(params, kv->max_seq_len, tree->max_nodes, kind);
    if (!tree_len_served(kind, len)) return CUSA_ERR_UNSUPPORTED;
    const TreeWs w = tree_workspace(kind, (int)len, params->batch, params->n_q_heads, G, tree->max_tokens, tree->max_nodes);
    if (ws_bytes < w.total) return CUSA_ERR_WORKSPACE_TOO_SMALL;
    const TreePlan pl = plan_tree(kind, (int)len, params->batch, G, g, tree->max_nodes);
    TreeArgs a;
    a.cache = cache_args(params, kv);
    a.q = static_cast<const uint16_t*>(q);
    a.q_stride = tree->q_stride;
    a.tok_start = tree->tok_start;
    a.idx = idx;
    a.cnt = cnt;
    a.masks = tree->masks;
    a.out = static_cast<uint16_t*>(out);
    a.part_acc = ws_ptr<float>(ws, w.acc);
    a.part_ml = ws_ptr<float>(ws, w.ml);
    a.pieces = ws_ptr<int32_t>(ws, w.pieces);
    a.scale_log2e = params->sm_scale * 1.4426950408889634f;
    a.max_tokens = tree->max_tokens;
    a.max_nodes = tree->max_nodes;
    a.words = (tree->max_nodes + 63) / 64;
    a.budget = params->budget;
    a.H = params->n_q_heads;
    a.g_shift = g == 1 ? 0 : g == 2 ? 1 : g == 4 ? 2 : 3;
    a.tile_rows = pl.rows;
    a.m_tiles = pl.m_tiles;
    a.n_splits = pl.n_splits;
    a.batch = params->batch;
    const int64_t units = ((int64_t)pl.n_splits * G * params->batch + 7) / 8 * 8 * pl.m_tiles;
    if (units > 0x7fffffff) return CUSA_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)units);
    const bool paged = kv->layout == CUSA_KV_PAGED;
    hipStream_t s = static_cast<hipStream_t>(stream);
    launch_tree(paged, grid, s, a);
    if (launch_status() != CUSA_OK) return CUSA_ERR_LAUNCH;
    if (pl.n_splits > 1) {                 // as many workgroups as have a row each, but not more than a few rounds of the chip
        const int64_t rows = ((int64_t)tree->max_nodes * params->n_q_heads + REDUCE_WAVES - 1) / REDUCE_WAVES, most = std::max(1, 8192 / params->batch);
        launch(KID_TREE_REDUCE, tree_reduce_kernel, dim3((unsigned)std::min(rows, most), params->batch), 64 * REDUCE_WAVES, 0, s, a);
    }
    return launch_status();
}

cusa_status cusa_kv_commit(const cusa_params* params, int32_t n_layers, const cusa_kv* kv_layers, const int32_t* base, const int32_t* path,
                           int32_t max_path, const int32_t* n_path, int32_t* keep, void* stream) {
    cusa_status st = check_params(params, false);
    if (st != CUSA_OK) return st;
    if (n_layers < 1 || !kv_layers || !base || !path || !n_path || max_path < 1 || keep == base || keep == n_path) return CUSA_ERR_INVALID_ARG;
    for (int i = 0; i < n_layers; ++i) {
        cusa_kv c = kv_layers[i];          // seq_lens is not read
        if (!c.seq_lens) c.seq_lens = base;
        if ((st = check_cache(params, &c, true)) != CUSA_OK) return st;
    }
    CommitArgs a = {};
    a.base = base;
    a.path = path;
    a.n_path = n_path;
    a.max_path = max_path;
    for (int i = 0; i < n_layers; i += COMMIT_LAYERS) {
        const int n = std::min(n_layers - i, COMMIT_LAYERS);
        for (int j = 0; j < n; ++j) a.layer[j] = cache_args(params, &kv_layers[i + j]);
        a.keep = i == 0 ? keep : nullptr;
        launch(KID_KV_COMMIT, kv_commit_kernel, dim3(params->n_kv_heads, params->batch, n), COMMIT_THREADS, 0, static_cast<hipStream_t>(stream), a);
        if (launch_status() != CUSA_OK) return CUSA_ERR_LAUNCH;
    }
    return CUSA_OK;
}

}  // extern "C"
