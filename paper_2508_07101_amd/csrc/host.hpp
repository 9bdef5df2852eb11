// What the host side's files share: timed launches, checks of the descriptors, small helpers.
#pragma once
#include "../../include/cusa.h"

#include <hip/hip_runtime.h>
#include <hip/hip_ext.h>

#include <algorithm>
#include <atomic>
#include <mutex>
#include <vector>

#include "cache_view.hpp"

namespace cusa {

// ------------------------------------------------------------------ profiling

enum KernelId { KID_SCORE = 0, KID_TOPK, KID_UNION, KID_ATTN_FULL, KID_ATTN_SPARSE, KID_REDUCE, KID_ATTN_SELECT, KID_ATTN_PER_HEAD, KID_RHO_PER_HEAD, KID_RANK_AGG, KID_RECALL, KID_PROBE, KID_TOPK_SLICE, KID_TOPK_MERGE, KID_PROBE_GATHER, KID_PROBE_RW_SCATTER, KID_PROBE_RW_BURST, KID_SAMPLE_THRESHOLD, KID_TOPK_FILTERED, KID_PROBE_TILES, KID_TOPK_VALUES, KID_ATTN_FILTER, KID_KV_PLAN, KID_KV_FILL, KID_KV_APPEND, KID_TREE_MASKS, KID_TREE_ATTN, KID_TREE_REDUCE, KID_KV_COMMIT, KID_BEAM_ROWS, KID_BEAM_MERGE, KID_KV_FORK, KID_FORK_TABLES, KID_FORK_PAGES, KID_KV_COPY, KID_SHARED_PAGES, KID_BEAM_ATTN, KID_BEAM_REDUCE, KID_COUNT };
inline const char* const kKernelNames[KID_COUNT] = {"score_kernel", "topk_kernel", "union_kernel",
                                             "attn_kernel<full>", "attn_kernel<sparse>", "attn_reduce_kernel",
                                             "attn_kernel<full+score>", "attn_kernel<per-head>", "per_head_rho_kernel",
                                             "rank_aggregate_kernel", "recall_kernel", "probe_stream_read_kernel", "topk_kernel<slice>",
                                             "topk_kernel<merge>", "probe_traffic_kernel<gather>", "probe_traffic_kernel<scattered writes>",
                                             "probe_traffic_kernel<burst writes>", "sample_threshold_kernel", "topk_kernel<filtered>", "probe_traffic_kernel<stream>", "topk_values_kernel", "attn_kernel<full+filter>",
                                             "kv_plan_kernel", "kv_fill_kernel", "kv_append_kernel", "tree_masks_kernel", "tree_attn_kernel", "tree_reduce_kernel", "kv_commit_kernel",
                                             "beam_rows_kernel", "beam_merge_kernel", "kv_fork_kernel", "fork_tables_kernel", "fork_pages_kernel", "kv_copy_kernel", "shared_pages_kernel",
                                             "beam_attn_kernel", "beam_reduce_kernel"};

// With the profiler on, every launch carries a start and a stop event that the runtime fills
// from the dispatch's own begin and end timestamps (hipExtLaunchKernelGGL), which is what a
// kernel trace reports: the figures exclude the gaps between kernels and the events' own cost.
struct ProfRec {
    int id;
    hipEvent_t start, stop;
};
struct Profiler {
    std::mutex mu;
    std::atomic<bool> on{false};
    std::vector<ProfRec> recs;
    std::vector<hipEvent_t> pool;
    int64_t calls[KID_COUNT] = {0};
    double ms[KID_COUNT] = {0};
};
inline Profiler g_prof;

inline hipEvent_t prof_event() {
    if (!g_prof.pool.empty()) {
        hipEvent_t e = g_prof.pool.back();
        g_prof.pool.pop_back();
        return e;
    }
    hipEvent_t e = nullptr;
    if (hipEventCreate(&e) != hipSuccess) {
        (void)hipGetLastError();
        return nullptr;
    }
    return e;
}

template <typename T>
struct same_as { using type = T; };

// Every kernel of the library is launched through here; the arguments are converted to the
// kernel's parameter types before they are packed.
template <typename... KArgs>
void launch(int kid, void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t shmem, hipStream_t s,
            typename same_as<KArgs>::type... args) {
    if (!g_prof.on.load(std::memory_order_acquire)) {
        kernel<<<grid, block, shmem, s>>>(args...);
        return;
    }
    ProfRec rec;
    rec.id = kid;
    {
        std::lock_guard<std::mutex> lk(g_prof.mu);
        rec.start = prof_event();
        rec.stop = prof_event();
        if (!rec.start || !rec.stop) {                // no events to be had: launch untimed
            if (rec.start) g_prof.pool.push_back(rec.start);
            if (rec.stop) g_prof.pool.push_back(rec.stop);
            rec.start = rec.stop = nullptr;
        }
    }
    if (!rec.start) {
        kernel<<<grid, block, shmem, s>>>(args...);
        return;
    }
    hipExtLaunchKernelGGL(kernel, grid, block, (uint32_t)shmem, s, rec.start, rec.stop, 0, args...);
    std::lock_guard<std::mutex> lk(g_prof.mu);
    g_prof.recs.push_back(rec);
}

// ------------------------------------------------------------------ validation

inline bool valid_group(int g) { return g == 1 || g == 2 || g == 4 || g == 8; }

inline int resolved_k(const cusa_params* p) { return p->topk_per_head > 0 ? p->topk_per_head : p->budget - p->window; }

inline cusa_status check_params(const cusa_params* p, bool need_budget) {
    if (!p) return CUSA_ERR_INVALID_ARG;
    if (p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1) return CUSA_ERR_INVALID_ARG;
    if (p->n_q_heads % p->n_kv_heads != 0) return CUSA_ERR_INVALID_ARG;
    if (p->head_dim != D) return CUSA_ERR_UNSUPPORTED;
    if (!valid_group(p->n_q_heads / p->n_kv_heads)) return CUSA_ERR_UNSUPPORTED;
    if (p->batch > 65535 || p->n_q_heads > 65535) return CUSA_ERR_UNSUPPORTED;
    if (!(p->sm_scale > 0.0f) || !(p->sm_scale < 1e30f)) return CUSA_ERR_INVALID_ARG;
    if (need_budget) {
        if (p->budget < 1 || p->window < 0 || p->window > p->budget) return CUSA_ERR_INVALID_ARG;
        if (p->topk_per_head < 0) return CUSA_ERR_INVALID_ARG;
        if (p->n_sink < 0 || p->n_sink > p->budget - p->window) return CUSA_ERR_INVALID_ARG;
        if (p->rank_mode != CUSA_RANK_FIRST_OCCURRENCE && p->rank_mode != CUSA_RANK_VOTES &&
            p->rank_mode != CUSA_RANK_MAX_SCORE)
            return CUSA_ERR_INVALID_ARG;
        const int k = resolved_k(p);
        if (k < p->budget - p->window - p->n_sink) return CUSA_ERR_INVALID_ARG;
        if (k > 8192) return CUSA_ERR_UNSUPPORTED;
    }
    return CUSA_OK;
}

inline cusa_status check_kv(const cusa_params* p, const cusa_kv* kv) {
    if (!kv || !kv->k || !kv->v || !kv->seq_lens) return CUSA_ERR_INVALID_ARG;
    if (kv->max_seq_len < 1) return CUSA_ERR_INVALID_ARG;
    if (((uintptr_t)kv->k | (uintptr_t)kv->v) & 15) return CUSA_ERR_INVALID_ARG;
    if (kv->layout == CUSA_KV_CONTIGUOUS) {
        if (kv->stride_token < D || (kv->stride_token & 7) || (kv->stride_head & 7) || (kv->stride_batch & 7))
            return CUSA_ERR_INVALID_ARG;
        if (kv->stride_head < 0 || kv->stride_batch < 0) return CUSA_ERR_INVALID_ARG;
    } else if (kv->layout == CUSA_KV_PAGED) {
        if (kv->page_size != PAGE) return CUSA_ERR_UNSUPPORTED;
        if (!kv->block_table || kv->n_pages < 1) return CUSA_ERR_INVALID_ARG;
        if ((int64_t)kv->max_pages * PAGE < kv->max_seq_len) return CUSA_ERR_INVALID_ARG;
    } else {
        return CUSA_ERR_INVALID_ARG;
    }
    (void)p;
    return CUSA_OK;
}

inline KvView make_view(const cusa_params* p, const cusa_kv* kv) {
    KvView v;
    v.k = static_cast<const uint16_t*>(kv->k);
    v.v = static_cast<const uint16_t*>(kv->v);
    v.sb = kv->stride_batch;
    v.sh = kv->stride_head;
    v.st = kv->stride_token;
    v.bt = kv->block_table;
    v.max_pages = kv->max_pages;
    v.G = p->n_kv_heads;
    v.seq_lens = kv->seq_lens;
    return v;
}

constexpr int MAX_BATCH = 65535;           // a dimension of the grids
constexpr int64_t MAX_STRIDE = 1 << 26;    // elements between two tokens: some rows' offset fits 32 bits of bytes

inline cusa_status check_pool(const cusa_pool* p) {
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
inline cusa_status check_cache(const cusa_params* p, const cusa_kv* kv, bool reads_tables) {
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

inline CacheArgs cache_args(const cusa_params* p, const cusa_kv* kv) {
    CacheArgs c;
    c.kv = make_view(p, kv);
    if (kv->layout != CUSA_KV_PAGED) c.kv.bt = nullptr;
    c.n_pages = (int32_t)std::min<int64_t>(kv->n_pages, 0x7fffffff);
    c.max_len = kv->max_seq_len;
    return c;
}

// ------------------------------------------------------------------ helpers

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

template <typename T>
T* ws_ptr(void* ws, size_t off) {
    return reinterpret_cast<T*>(static_cast<char*>(ws) + off);
}

inline cusa_status launch_status() { return hipGetLastError() == hipSuccess ? CUSA_OK : CUSA_ERR_LAUNCH; }

}  // namespace cusa
