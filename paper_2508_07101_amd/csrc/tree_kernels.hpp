// Device code for decoding with trees of drafted tokens.
//
//   kv_plan_kernel      which sequences get room, in one workgroup: three sums over the sequences, in order
//   kv_fill_kernel      the slots, table entries and queue entries that follow from it
//   kv_append_kernel    new rows into their slots
//   tree_masks_kernel   ancestors from parents, by doubling
//   kv_commit_kernel    an accepted branch's rows moved together, all layers
#pragma once
#include "tree_attn.hpp"

namespace cusa {

// ---------------------------------------------------------------- page plan

constexpr int PLAN_ONE_LAUNCH = 4096;      // tokens up to which the planning workgroup fills the slots itself

struct PlanSeq {                           // what filling needs of a sequence, in the workspace behind PlanHead
    int32_t keep, old_pages, pop, push;    // pop, push: its first page's place among all that are taken, given back
};
struct PlanHead {
    int32_t first, avail;                  // of the queue, before the call
};
struct PlanArgs {
    const int32_t *held, *keep, *add;
    int32_t *lens, *tok_start;
    int64_t* slots;
    int32_t* table;                        // nullptr: contiguous
    int32_t* ring;
    const int32_t* state;
    int32_t* state_out;
    PlanHead* head;
    PlanSeq* seq;
    int32_t batch, max_tokens, max_pages, n_pages, cap;
};

constexpr int FILL_RUN = 4;                              // consecutive tokens of a thread: mostly of one page
// Slots of tokens and pages from the queue, by thread `at` of `step`; pages to the queue's end.  starts, seq, lens: in LDS where they fit.
__device__ __forceinline__ void plan_fill(const PlanArgs& a, const int32_t* starts, const PlanSeq* seq, const int32_t* lens, int first, int avail, int64_t at,
                                          int64_t step, int seq_at, int seq_step, int lane, int lanes) {
    const int total = starts[a.batch];
    const bool wide = ((uintptr_t)a.slots & 15) == 0;
    for (int64_t r0 = at * FILL_RUN; r0 < a.max_tokens; r0 += step * FILL_RUN) {
        int64_t slot[FILL_RUN];
        int lo = 0, hi = a.batch - 1;                    // the last sequence that starts at or before r0
        if (r0 < total) {
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (starts[mid] <= r0) lo = mid;
                else hi = mid - 1;
            }
        }
        PlanSeq s = seq[lo];
        int32_t start = starts[lo], next = starts[lo + 1], id = -1;
        bool held = false;                               // id is the page of the token before
#pragma unroll
        for (int j = 0; j < FILL_RUN; ++j) {
            const int64_t r = r0 + j;
            slot[j] = -1;
            if (r >= total) continue;
            if (r >= next) {
                do next = starts[++lo + 1];              // (total lies behind r: one comes)
                while (r >= next);
                s = seq[lo];
                start = starts[lo];
                held = false;
            }
            const int64_t pos = s.keep + (r - start);
            if (!a.table) {
                slot[j] = ((int64_t)lo << 32) + pos;
                continue;
            }
            if (!held || (pos & (PAGE - 1)) == 0) {
                const int page = (int)(pos >> 4);
                int32_t* const entry = a.table + (int64_t)lo * a.max_pages + page;
                if (page < s.old_pages) {
                    id = *entry;
                } else {
                    uint32_t from = (uint32_t)first + (uint32_t)(s.pop + (page - s.old_pages));   // (what is granted was free: below n_pages each)
                    if (from >= (uint32_t)a.n_pages) from -= a.n_pages;
                    id = a.ring[from];
                    if ((pos & (PAGE - 1)) == 0) *entry = id;   // a new page's first token is always among the new ones
                }
                held = true;
            }
            if ((uint32_t)id < (uint32_t)a.n_pages) slot[j] = (int64_t)id * PAGE + (pos & (PAGE - 1));
        }
        if (wide && r0 + FILL_RUN <= a.max_tokens) {
            typedef int64_t i64x2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int j = 0; j < FILL_RUN; j += 2) *reinterpret_cast<i64x2*>(a.slots + r0 + j) = i64x2{slot[j], slot[j + 1]};
        } else {
#pragma unroll
            for (int j = 0; j < FILL_RUN; ++j)
                if (r0 + j < a.max_tokens) a.slots[r0 + j] = slot[j];
        }
    }
    if (!a.table) return;
    for (int b = seq_at; b < a.batch; b += seq_step) {
        const PlanSeq s = seq[b];
        const int now = pages_of(lens[b]);
        for (int i = lane; i < s.old_pages - now; i += lanes)
            a.ring[ring_at((int64_t)first + avail + s.push + i, a.n_pages)] = a.table[(int64_t)b * a.max_pages + now + i];
    }
}

// A thread for each sequence, 1024 at a time.  Latency is all: a read of the numbers, three sums, a search, a page's entry.  What the slots need of
// up to 1024 sequences stays in LDS (searched in memory, 64 sequences' 2000 slots took 10.9 us in all, so 7.1).
template <bool FILL>
__global__ __launch_bounds__(PLAN_THREADS) void kv_plan_kernel(PlanArgs a) {
    __shared__ int64_t scratch[3][2][PLAN_THREADS / 64];
    __shared__ int32_t starts[PLAN_THREADS + 1], lengths[PLAN_THREADS];
    __shared__ PlanSeq seqs[PLAN_THREADS];
    const int tid = threadIdx.x;
    int64_t asked = 0, needed = 0, granted = 0, taken = 0, returned = 0;   // of the sequences before this round's
    int first = 0, avail = 0;
    if (a.table) {
        first = a.state[0];
        avail = clampi(a.state[1], 0, a.n_pages);
        if ((uint32_t)first >= (uint32_t)a.n_pages) first = 0;
    }
    for (int base = 0; base < a.batch; base += PLAN_THREADS) {
        const int b = base + tid;
        const bool here = b < a.batch;
        const int held = here ? clampi(a.held[b], 0, a.cap) : 0;
        const int keep = here ? clampi(a.keep[b], 0, held) : 0;
        const int add = here ? max(a.add[b], 0) : 0;
        const bool fits = (int64_t)keep + add <= a.cap;
        const int waves = min((a.batch - base + 63) >> 6, PLAN_THREADS / 64);
        int64_t sum;
        const int64_t tokens = fits ? add : 0, tokens_before = asked + plan_scan(tokens, sum, scratch[0], waves);
        asked += sum;
        bool ok = fits && tokens_before + tokens <= a.max_tokens;
        const int old_pages = pages_of(held);
        if (a.table) {
            const int64_t need = ok ? max(pages_of(keep + add) - old_pages, 0) : 0, need_before = needed + plan_scan(need, sum, scratch[1], waves);
            needed += sum;
            ok = ok && (need == 0 || need_before + need <= avail);
        }
        const int n = ok ? add : 0, len = keep + n, change = a.table ? pages_of(len) - old_pages : 0;
        // tokens; pages taken and given back, 32 bits each (n_pages < 2^31)
        int64_t v[2] = {n, ((int64_t)max(-change, 0) << 32) + max(change, 0)}, both[2];
        plan_scan(v, both, scratch[2], waves);
        const int start = (int)(granted + v[0]);
        const PlanSeq s = {keep, old_pages, (int)(taken + (v[1] & 0xffffffff)), (int)(returned + (v[1] >> 32))};
        granted += both[0];
        taken += both[1] & 0xffffffff;
        returned += both[1] >> 32;
        if (here) {
            a.lens[b] = len;
            a.tok_start[b] = start;
            if (!FILL) a.seq[b] = s;
            if (FILL) {
                lengths[tid] = len;
                starts[tid] = start;
                seqs[tid] = s;
            }
        }
    }
    if (tid == 0) {
        a.tok_start[a.batch] = (int)granted;
        if (FILL) starts[a.batch] = (int)granted;
        if (a.table) {
            if (!FILL) *a.head = PlanHead{first, avail};
            a.state_out[0] = (int)ring_at((int64_t)first + taken, a.n_pages);
            a.state_out[1] = (int)min((int64_t)avail - taken + returned, (int64_t)a.n_pages);
        }
    }
    if (FILL) {                                          // (up to PLAN_THREADS sequences)
        __syncthreads();
        plan_fill(a, starts, seqs, lengths, first, avail, tid, PLAN_THREADS, tid >> 6, PLAN_THREADS / 64, tid & 63, 64);
    }
}

// The same by many workgroups, for prompts: the starts are searched in LDS, four tokens a thread share a page's entry and go out in two 16-byte stores.
// 1.3 million slots (11 MB): 7.4 us, of which 2 are the stores and 3 a launch; the planning launch before it 4.4.
constexpr int FILL_THREADS = 256;
__global__ __launch_bounds__(FILL_THREADS) void kv_fill_kernel(PlanArgs a) {
    __shared__ int32_t starts[PLAN_THREADS + 1];
    const int64_t at = (int64_t)blockIdx.x * FILL_THREADS + threadIdx.x, step = (int64_t)gridDim.x * FILL_THREADS;
    const int first = a.table ? a.head->first : 0, avail = a.table ? a.head->avail : 0;
    if (a.batch <= PLAN_THREADS) {
        for (int i = threadIdx.x; i <= a.batch; i += FILL_THREADS) starts[i] = a.tok_start[i];
        __syncthreads();
        plan_fill(a, starts, a.seq, a.lens, first, avail, at, step, blockIdx.x, gridDim.x, threadIdx.x, FILL_THREADS);
    } else {
        plan_fill(a, a.tok_start, a.seq, a.lens, first, avail, at, step, blockIdx.x, gridDim.x, threadIdx.x, FILL_THREADS);
    }
}

// ---------------------------------------------------------------- append

constexpr int APPEND_THREADS = 256;
constexpr int APPEND_ROWS = 4;             // rows of a group of 16 lanes, all under way at once

struct AppendArgs {
    CacheArgs cache;
    const int64_t* slots;
    const void *k, *v;
    int64_t st, sh;
    int32_t n, batch;
};

template <int DTYPE>                       // cusa_dtype
__device__ __forceinline__ u32x4 load_as_bf16(const void* base, int64_t at) {
    if constexpr (DTYPE == 0) {
        return *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + at);
    } else {
        float f[8];
        if constexpr (DTYPE == 1) {
            typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
            const f16x8 h = *reinterpret_cast<const f16x8*>(static_cast<const _Float16*>(base) + at);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)h[i];
        } else {
            const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + at);
            const f32x4 x = p[0], y = p[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) { f[i] = x[i]; f[4 + i] = y[i]; }
        }
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = (uint32_t)f32_to_bf16_rne(f[2 * i]) | (uint32_t)f32_to_bf16_rne(f[2 * i + 1]) << 16;
        return r;
    }
}

// A group of 16 lanes for a row of 128 elements.  Rows are numbered (token, K heads then V heads).  Bound by memory: 131 072 fp32 rows of 8 KV heads (1.6 GB read
// and written) take 304 us, 5.3 TB/s, as much as a plain copy's rate; 2388 bf16 rows from a fused projection (20 MB) 5.9 us, mostly latency.
template <int DTYPE, bool PAGED>
__global__ __launch_bounds__(APPEND_THREADS) void kv_append_kernel(AppendArgs a) {
    constexpr int PER_WG = APPEND_THREADS / 16 * APPEND_ROWS;
    const int G = a.cache.kv.G, both = 2 * G, c = threadIdx.x & 15;
    const int64_t base = (int64_t)blockIdx.x * PER_WG;
    const int token0 = (int)(base / both);                // uniform
    const int rest = (int)(base - (int64_t)token0 * both) + (threadIdx.x >> 4);
    u32x4 x[APPEND_ROWS];
    uint16_t* to[APPEND_ROWS];
#pragma unroll
    for (int i = 0; i < APPEND_ROWS; ++i) {
        const int item = rest + i * (APPEND_THREADS / 16), t = item / both, j = item - t * both;
        const int64_t token = (int64_t)token0 + t;
        to[i] = nullptr;
        if (token >= a.n) continue;
        const int64_t slot = a.slots[token];
        const int kvh = j < G ? j : j - G;
        x[i] = load_as_bf16<DTYPE>(j < G ? a.k : a.v, token * a.st + (int64_t)kvh * a.sh + c * 8);
        if (slot < 0) continue;
        int64_t off;
        if (PAGED) {
            const int64_t page = slot >> 4;
            if (page >= a.cache.n_pages) continue;
            off = ((page * G + kvh) * PAGE + (slot & (PAGE - 1))) * D;
        } else {
            const int64_t b = slot >> 32, pos = slot & 0xffffffff;
            if (b >= a.batch || pos >= a.cache.max_len) continue;
            off = cache_offset<false>(a.cache, (int)b, kvh, (int)pos);
        }
        to[i] = const_cast<uint16_t*>(j < G ? a.cache.kv.k : a.cache.kv.v) + off + c * 8;
    }
#pragma unroll
    for (int i = 0; i < APPEND_ROWS; ++i)
        if (to[i]) *reinterpret_cast<u32x4*>(to[i]) = x[i];
}

// ---------------------------------------------------------------- masks

struct MasksArgs {
    const int32_t *base, *tok_start, *parents;
    uint64_t* masks;
    int32_t* positions;
    int32_t max_tokens, max_nodes, words;
};

// One workgroup for a tree, a thread for a node.  Who stands above a node is known after as many rounds as the depth has bits: each
// round a node takes over what the node it points to knows, and points where that one points.  Latency is all: 60 nodes 3.3 us (a launch that does
// nothing takes about 3), 64 trees of up to 256 nodes 5.5.
__global__ __launch_bounds__(TREE_MAX_NODES) void tree_masks_kernel(MasksArgs a) {
    __shared__ uint64_t rows[TREE_MAX_NODES / 64][TREE_MAX_NODES];
    __shared__ int up[TREE_MAX_NODES], deep[TREE_MAX_NODES];
    const int j = threadIdx.x, b = blockIdx.x;
    int start;
    const int n = tree_span(a.tok_start, b, a.max_tokens, a.max_nodes, start);
    const int parent = j < n ? a.parents[start + j] : -1;
    int u = parent >= 0 && parent < j ? parent : -1, d = u >= 0 ? 1 : 0;
    uint64_t w[TREE_MAX_NODES / 64];
#pragma unroll
    for (int i = 0; i < TREE_MAX_NODES / 64; ++i) w[i] = (j >> 6) == i ? 1ull << (j & 63) : 0;
    while (__syncthreads_or(u >= 0)) {
#pragma unroll
        for (int i = 0; i < TREE_MAX_NODES / 64; ++i) rows[i][j] = w[i];
        up[j] = u;
        deep[j] = d;
        __syncthreads();
        if (u >= 0) {
#pragma unroll
            for (int i = 0; i < TREE_MAX_NODES / 64; ++i) w[i] |= rows[i][u];
            d += deep[u];
            u = up[u];
        }
    }
    if (j >= n) return;
    for (int i = 0; i < a.words; ++i) a.masks[(int64_t)(start + j) * a.words + i] = i == 0 ? w[0] : i == 1 ? w[1] : i == 2 ? w[2] : w[3];
    if (a.positions) a.positions[start + j] = a.base[b] + d;
}

// ---------------------------------------------------------------- commit

constexpr int COMMIT_LAYERS = 40;          // layers of a launch: their descriptors travel as arguments (4 KB at most)
constexpr int COMMIT_THREADS = 256;

struct CommitArgs {
    const int32_t *base, *path, *n_path;
    int32_t* keep;
    int32_t max_path;
    CacheArgs layer[COMMIT_LAYERS];
};
static_assert(sizeof(CommitArgs) <= 4096, "a launch's arguments");

// One workgroup for a (layer, sequence, KV head): 16 rows at a time are read, then written.  path ascends, so a row that is still to be read lies
// behind every row written so far.  Bound by memory: the branches of 64 sequences in 32 layers take 19.9 us; those of one sequence in 36 layers 3.2, latency.
__device__ __forceinline__ bool commit_row(const CacheArgs& c, bool paged, int b, int kvh, int64_t pos, int64_t& off) {
    if (pos < 0 || pos >= c.max_len) return false;
    const int row = paged ? cache_row<true>(c, b, kvh, (int)pos) : (int)pos;
    if (row < 0) return false;
    off = paged ? cache_offset<true>(c, b, kvh, row) : cache_offset<false>(c, b, kvh, row);
    return true;
}
__global__ __launch_bounds__(COMMIT_THREADS) void kv_commit_kernel(CommitArgs a) {
    const int kvh = blockIdx.x, b = blockIdx.y, c = threadIdx.x & 15;
    const CacheArgs& cache = a.layer[blockIdx.z];
    const bool paged = cache.kv.bt != nullptr;
    const int n = clampi(a.n_path[b], 0, a.max_path);
    const int64_t base = a.base[b];
    if (a.keep && blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x == 0) a.keep[b] = (int)(base + n);
    uint16_t* const k = const_cast<uint16_t*>(cache.kv.k);
    uint16_t* const v = const_cast<uint16_t*>(cache.kv.v);
    for (int i0 = 0; i0 < n; i0 += COMMIT_THREADS / 16) {
        const int i = i0 + (threadIdx.x >> 4);
        int64_t from = 0, to = 0;
        bool move = false;
        if (i < n) {
            const int p = a.path[(int64_t)b * a.max_path + i];
            move = p >= 0 && p != i && commit_row(cache, paged, b, kvh, base + p, from) && commit_row(cache, paged, b, kvh, base + i, to);
        }
        u32x4 x, y;
        if (move) {
            x = *reinterpret_cast<const u32x4*>(k + from + c * 8);
            y = *reinterpret_cast<const u32x4*>(v + from + c * 8);
        }
        __syncthreads();
        if (move) {
            *reinterpret_cast<u32x4*>(k + to + c * 8) = x;
            *reinterpret_cast<u32x4*>(v + to + c * 8) = y;
        }
    }
}

}  // namespace cusa
