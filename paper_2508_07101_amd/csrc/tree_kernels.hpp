// Device code for decoding with trees of drafted tokens.
//
//   kv_plan_kernel      which sequences get room, in one workgroup: three sums over the sequences, in order
//   kv_fill_kernel      the slots, table entries and queue entries that follow from it
//   kv_append_kernel    new rows into their slots
//   tree_masks_kernel   ancestors from parents, by doubling
//   tree_attn_kernel    attention of a tree's nodes over the prefix (or the part of it that was chosen) and their branch
//   tree_reduce_kernel  merges the pieces of a long prefix
//   kv_commit_kernel    an accepted branch's rows moved together, all layers
#pragma once
#include "cache_view.hpp"
#include "tree_plan.hpp"

namespace cusa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ int pages_of(int tokens) { return (int)(((int64_t)tokens + PAGE - 1) / PAGE); }

// ---------------------------------------------------------------- page plan

constexpr int PLAN_THREADS = 1024;
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

// Sum over the workgroup's threads before this one; total: of all.  scratch: a word for each wave, and a barrier before its next use.
__device__ __forceinline__ int64_t plan_scan(int64_t v, int64_t* scratch, int64_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    if (lane == 63) scratch[wave] = x;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < PLAN_THREADS / 64; ++w) {
        const int64_t s = scratch[w];
        if (w < wave) before += s;
        all += s;
    }
    __syncthreads();
    total = all;
    return before + x - v;
}

// Slots of tokens and pages from the queue, by thread `at` of `step`; pages to the queue's end.
__device__ __forceinline__ void plan_fill(const PlanArgs& a, int64_t at, int64_t step, int seq_at, int seq_step, int lane, int lanes) {
    const int total = a.tok_start[a.batch];
    const int first = a.table ? a.head->first : 0, avail = a.table ? a.head->avail : 0;
    for (int64_t r = at; r < a.max_tokens; r += step) {
        if (r >= total) {
            a.slots[r] = -1;
            continue;
        }
        int lo = 0, hi = a.batch - 1;                    // the last sequence that starts at or before r and is not empty: tok_start[lo] <= r < tok_start[lo + 1]
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.tok_start[mid] <= r) lo = mid;
            else hi = mid - 1;
        }
        const PlanSeq s = a.seq[lo];
        const int64_t pos = s.keep + (r - a.tok_start[lo]);
        if (!a.table) {
            a.slots[r] = ((int64_t)lo << 32) + pos;
            continue;
        }
        const int page = (int)(pos >> 4);
        int32_t* const entry = a.table + (int64_t)lo * a.max_pages + page;
        int32_t id;
        if (page < s.old_pages) {
            id = *entry;
        } else {
            id = a.ring[((int64_t)first + s.pop + (page - s.old_pages)) % a.n_pages];
            if ((pos & (PAGE - 1)) == 0) *entry = id;    // a new page's first token is always among the new ones
        }
        a.slots[r] = (uint32_t)id < (uint32_t)a.n_pages ? (int64_t)id * PAGE + (pos & (PAGE - 1)) : -1;
    }
    if (!a.table) return;
    for (int b = seq_at; b < a.batch; b += seq_step) {
        const PlanSeq s = a.seq[b];
        const int now = pages_of(a.lens[b]);
        for (int i = lane; i < s.old_pages - now; i += lanes)
            a.ring[((int64_t)first + avail + s.push + i) % a.n_pages] = a.table[(int64_t)b * a.max_pages + now + i];
    }
}

// A thread for each sequence, 1024 at a time.  Latency is all: a few dependent reads and the three sums.
template <bool FILL>
__global__ __launch_bounds__(PLAN_THREADS) void kv_plan_kernel(PlanArgs a) {
    __shared__ int64_t scratch[PLAN_THREADS / 64];
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
        int64_t sum;
        const int64_t tokens = fits ? add : 0, tokens_before = asked + plan_scan(tokens, scratch, sum);
        asked += sum;
        bool ok = fits && tokens_before + tokens <= a.max_tokens;
        const int old_pages = pages_of(held);
        if (a.table) {
            const int64_t need = ok ? max(pages_of(keep + add) - old_pages, 0) : 0, need_before = needed + plan_scan(need, scratch, sum);
            needed += sum;
            ok = ok && (need == 0 || need_before + need <= avail);
        }
        const int n = ok ? add : 0, len = keep + n;
        const int64_t start = granted + plan_scan(n, scratch, sum);
        granted += sum;
        int64_t pop = 0, push = 0;
        if (a.table) {
            const int change = pages_of(len) - old_pages;
            int64_t both;                                // taken and given back: 32 bits each (n_pages < 2^31)
            const int64_t v = ((int64_t)max(-change, 0) << 32) + max(change, 0), before = plan_scan(v, scratch, both);
            pop = taken + (before & 0xffffffff);
            push = returned + (before >> 32);
            taken += both & 0xffffffff;
            returned += both >> 32;
        }
        if (here) {
            a.lens[b] = len;
            a.tok_start[b] = (int)start;
            a.seq[b] = PlanSeq{keep, old_pages, (int)pop, (int)push};
        }
    }
    if (tid == 0) {
        a.tok_start[a.batch] = (int)granted;
        if (a.table) {
            *a.head = PlanHead{first, avail};
            a.state_out[0] = (int)(((int64_t)first + taken) % a.n_pages);
            a.state_out[1] = (int)min((int64_t)avail - taken + returned, (int64_t)a.n_pages);
        }
    }
    if (FILL) {
        __syncthreads();
        plan_fill(a, tid, PLAN_THREADS, tid >> 6, PLAN_THREADS / 64, tid & 63, 64);
    }
}

constexpr int FILL_THREADS = 256;
__global__ __launch_bounds__(FILL_THREADS) void kv_fill_kernel(PlanArgs a) {
    plan_fill(a, (int64_t)blockIdx.x * FILL_THREADS + threadIdx.x, (int64_t)gridDim.x * FILL_THREADS, blockIdx.x, gridDim.x, threadIdx.x, FILL_THREADS);
}

// ---------------------------------------------------------------- rows of a cache

struct CacheArgs {
    KvView kv;
    int32_t n_pages;                       // paged: pages of the pool
    int32_t max_len;                       // positions that may be touched
};

// The row of one position (its number in the pool, or in the sequence's own rows), or -1 for an entry that names no page.
template <bool PAGED>
__device__ __forceinline__ int cache_row(const CacheArgs& c, int b, int kvh, int pos) {
    if (!PAGED) return pos;
    const int page = c.kv.bt[(int64_t)b * c.kv.max_pages + (pos >> 4)];
    return (uint32_t)page < (uint32_t)c.n_pages ? (page * c.kv.G + kvh) * PAGE + (pos & (PAGE - 1)) : -1;
}
// Elements between the cache's start and its row: 64 bits, a cache may be longer than 32 count.
template <bool PAGED>
__device__ __forceinline__ int64_t cache_offset(const CacheArgs& c, int b, int kvh, int row) {
    return PAGED ? (int64_t)row * D : (int64_t)b * c.kv.sb + (int64_t)kvh * c.kv.sh + (int64_t)row * c.kv.st;
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

// A group of 16 lanes for a row of 128 elements.  Rows are numbered (token, K heads then V heads).
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

// The rows of sequence b in packed arrays: [start, start + n).
__device__ __forceinline__ int tree_span(const int32_t* tok_start, int b, int max_tokens, int max_nodes, int& start) {
    start = clampi(tok_start[b], 0, max_tokens);
    const int stop = clampi(tok_start[b + 1], start, max_tokens);
    return min(stop - start, max_nodes);
}

// One workgroup for a tree, a thread for a node.  Who stands above a node is known after as many rounds as the depth has bits: each
// round a node takes over what the node it points to knows, and points where that one points.
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

// ---------------------------------------------------------------- attention

struct TreeArgs {
    CacheArgs cache;
    const uint16_t* q;
    int64_t q_stride;
    const int32_t *tok_start, *idx, *cnt;
    const uint64_t* masks;
    uint16_t* out;
    float *part_acc, *part_ml;
    float scale_log2e;
    int32_t max_tokens, max_nodes, words, budget, H, g_shift, m_tiles, n_splits;
};

constexpr int TREE_WAVES = 8, TREE_THREADS = 64 * TREE_WAVES;

// What a workgroup of one sequence has to do, the same in the attention and in the merge.
struct TreeSpan {
    int start, n;          // its nodes' rows in the packed arrays
    int before, pre, all;  // P; tokens of the prefix that are looked at; the same and the nodes
    int chunk;             // tokens of a piece
};
template <bool SPARSE>
__device__ __forceinline__ TreeSpan tree_work(const TreeArgs& a, int b, int unit) {
    TreeSpan s;
    const int L = clampi(a.cache.kv.seq_lens[b], 0, a.cache.max_len);
    s.n = min(tree_span(a.tok_start, b, a.max_tokens, a.max_nodes, s.start), L);
    s.before = L - s.n;
    s.pre = SPARSE ? clampi(a.cnt[b], 0, a.budget) : s.before;
    s.all = s.pre + s.n;
    const int piece = (s.all + a.n_splits - 1) / a.n_splits;
    s.chunk = max(piece + unit - 1, TREE_MIN_PIECE) / unit * unit;
    return s;
}
constexpr int TREE_UNIT = 256;             // tokens that a workgroup's waves take at a time, at most

// Bits o .. o + 31 of a node's mask (o may be negative; bits before the first and behind the last are 0).
__device__ __forceinline__ uint32_t mask_window(const uint64_t* row, int words, int o) {
    if (o <= -32) return 0;
    if (o < 0) return (uint32_t)row[0] << -o;
    const int w = o >> 6, sh = o & 63;
    uint64_t x = w < words ? row[w] >> sh : 0;
    if (sh > 32 && w + 1 < words) x |= row[w + 1] << (64 - sh);
    return (uint32_t)x;
}

// Of the lane's value and that of its counterpart in the other half of the wave.
__device__ __forceinline__ float other_half_max(float v) {
    const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}

// 16 bytes a lane from memory to LDS at `lds` + 16 * lane, past the registers.  Not the builtin: for that, the compiler lets every later
// LDS read wait for all such loads, which leaves one tile under way at most.  Whoever uses the bytes waits for them (wait_tiles) and, where
// another wave asked for them, meets it at a barrier.
__device__ __forceinline__ void load_to_lds(const uint16_t* from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory");
}
// Until all but the newest `n` of this wave's requests of OPS each have arrived (n <= 2).
template <int OPS>
__device__ __forceinline__ void wait_tiles(int n) {
    if (n >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * OPS) : "memory");
    else if (n == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(OPS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}
__device__ __forceinline__ void wave_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

constexpr int TREE_LIST = 4096;            // entries of a workgroup's list of rows: tokens of a chosen prefix, pages of a whole one
constexpr int TREE_RING = 128 * 1024;      // bytes of LDS for token tiles
struct TreeLds {
    __attribute__((aligned(16))) unsigned char ring[TREE_RING];
    int32_t list[TREE_LIST];
    float m[TREE_ROWS], l[TREE_ROWS];      // of every row, a set for each team
    uint32_t odd[TREE_MAX_NODES / 32];     // nodes among this workgroup's tokens with a value that is not finite
};

typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

// The state of a wave's 32 rows, one to a lane and its counterpart in the other half of the wave.
struct TreeRow {
    bf16x8 q[8];           // columns 16 k + 8 half ..
    f32x16 o[4];           // columns 32 d + 8 (i / 4) + 4 half + i % 4
    float m, l;            // reference of the weights in log2 units, the half's sum of weights
};

// 32 tokens: scores, weights, and their share of the output.  S^T = K Q^T takes K's rows as they stand in the tile; a lane gets its row's scores of
// the 16 tokens 8 (i / 4) + 4 half + i % 4.  In that order they are O^T += V^T P^T's operand, with V's columns from transposing LDS reads.
// A row's reference follows its maximum only when that has grown by more than 8 (weights of up to 2^8, in 32 bits until they are rounded to bf16 relative
// to themselves): the output's 64 registers are hardly ever rescaled.
// EDGE: the row attends to the tokens `allowed` (a bit each), and not every row to those outside `common`.  Values that are not finite must not meet
// the weight 0 of a row that does not attend to them: outside `common` they are left out, and the lane's tokens with such values returned.
template <bool EDGE>
__device__ __forceinline__ uint32_t tree_step(TreeRow& r, const unsigned char* kt, const unsigned char* vt, uint32_t allowed, uint32_t common,
                                              float scale_log2e, int lane) {
    const int half = lane >> 5, col = lane & 31;
    const unsigned char* const krow = kt + col * 256;
    const int kx = (half ^ (col & 15)) << 4;                      // chunk 2 k + half of the row stands at (2 k + half) ^ (row & 15)
    f32x16 x;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.0f;
    bf16x8 kf[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) kf[k] = *reinterpret_cast<const bf16x8*>(krow + (kx ^ (k << 5)));
    __builtin_amdgcn_sched_barrier(0);                            // all reads first: left alone, the products wait for one read after the other
#pragma unroll
    for (int k = 0; k < 8; ++k) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k], r.q[k], x, 0, 0, 0);
    // 16 lanes transpose 4 tokens by 16 columns: tokens 16 k + 4 half + .. and 8 further on
    s16x8 vf[2][4];
    const int tok = 4 * half + ((lane >> 2) & 3);
    const unsigned char* const vrow = vt + tok * 256 + (lane & 1) * 8;
    const int vx = (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) << 4, vs = ((lane >> 2) & 3) << 6;
    auto values = [&](int k, int d) {
        const unsigned char* at = vrow + k * 4096 + (vx | ((d << 6) ^ vs));
        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)at);
        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 2048));
        return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    if (!EDGE) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int d = 0; d < 4; ++d) vf[k][d] = values(k, d);
    }
    if (EDGE) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (!(allowed >> (8 * (i >> 2) + 4 * half + (i & 3)) & 1)) x[i] = -INFINITY;
    }
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, x[i]);
    mx = other_half_max(mx) * scale_log2e;
    const bool raise = mx > r.m + 8.0f;
    if (__any(raise)) {
        const float to = raise ? mx : r.m, f = exp2f(r.m - to);  // a row's sums do not depend on its neighbours
        r.m = to;
        r.l *= f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) r.o[d][i] *= f;
    }
    bf16x8 p[2];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], scale_log2e, -r.m));
        sum += e;
        p[i >> 3][i & 7] = (__bf16)e;
    }
    r.l += sum;
    uint32_t odd = 0;
    const uint32_t wash = ~common >> (4 * half);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            if (EDGE) {
                u32x4 v = __builtin_bit_cast(u32x4, values(k, d));
#pragma unroll
                for (int j = 0; j < 4; ++j) {                     // two tokens a word
                    const uint32_t at = 1u << (16 * k + 2 * (j & 1) + 8 * (j >> 1));
                    if ((v[j] & 0x7f80u) == 0x7f80u && (wash & at)) {
                        odd |= at;
                        v[j] &= 0xffff0000u;
                    }
                    if ((v[j] & 0x7f800000u) == 0x7f800000u && (wash & at << 1)) {
                        odd |= at << 1;
                        v[j] &= 0xffffu;
                    }
                }
                vf[k][d] = __builtin_bit_cast(s16x8, v);
                asm volatile("" ::: "memory");                    // one operand at a time: no registers for more
            }
            r.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vf[k][d]), p[k], r.o[d], 0, 0, 0);
        }
    odd <<= 4 * half;
    return odd;
}

// A workgroup's rows against tokens [begin, end).  RG waves share a token tile and split the rows; 8 / RG such teams split the tokens and are added up in
// LDS at the end.  Two waves to a SIMD: one's softmax runs beside the other's products.  Tiles come by loads from memory straight to LDS, several of
// them under way.
template <int RG, bool PAGED, bool SPARSE>
__device__ __forceinline__ void tree_rows(const TreeArgs& a, const TreeSpan& s, TreeLds& lds, int b, int kvh, int row0, int begin, int end) {
    constexpr int TEAMS = TREE_WAVES / RG;
    constexpr int SUB = RG == 8 ? 2 : 1, TT = 32 * SUB;           // tokens of a team's tile
    constexpr int ROWS = 32 * RG;
    constexpr int TILE_BYTES = TT * 256;                          // of K, and again of V
    constexpr int STAGES = TREE_RING / (TEAMS * 2 * TILE_BYTES);  // 1, 2, 4, 4
    constexpr int AHEAD = RG == 1 ? 1 : STAGES - 1;               // tiles asked for before one is used
    constexpr int MINE = TT / RG;                                 // rows that a wave loads
    constexpr int OPS = 2 * MINE / 4;                             // its loads for a tile
    constexpr bool LIST = PAGED || SPARSE;
    static_assert(TEAMS * ROWS * D * 4 <= TREE_RING && TEAMS * ROWS <= TREE_ROWS && MINE % 4 == 0, "the teams' sums take the tiles' place");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int team = wave / RG, mine = wave % RG, half = lane >> 5, col = lane & 31;
    const int g = 1 << a.g_shift, rows = s.n << a.g_shift;
    if (tid < TREE_MAX_NODES / 32) lds.odd[tid] = 0;
    __syncthreads();

    TreeRow row;
    const int my_row = row0 + mine * 32 + col;
    const bool mine_there = my_row < rows;
    const int node = mine_there ? my_row >> a.g_shift : 0;
    {
        const uint16_t* p = a.q + (int64_t)(s.start + node) * a.q_stride + ((kvh << a.g_shift) + (my_row & (g - 1))) * D + half * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            u32x4 v = *reinterpret_cast<const u32x4*>(p + k * 16);
            if (!mine_there) v = u32x4{0, 0, 0, 0};
            row.q[k] = __builtin_bit_cast(bf16x8, v);
        }
    }
    row.m = LOWEST;
    row.l = 0.0f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) row.o[d][i] = 0.0f;
    const bool idle = row0 + mine * 32 >= rows;                   // a wave without rows loads its share and computes nothing

    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds.ring;
    const uint16_t* const kbase = a.cache.kv.k + (PAGED ? 0 : (int64_t)b * a.cache.kv.sb + (int64_t)kvh * a.cache.kv.sh);
    const uint16_t* const vbase = a.cache.kv.v + (PAGED ? 0 : (int64_t)b * a.cache.kv.sb + (int64_t)kvh * a.cache.kv.sh);
    const int64_t stride = PAGED ? D : a.cache.kv.st;
    // A lane's part of a row, in the order in which LDS holds it: K's 16-byte chunk c of row r stands at c ^ (r & 15), V's at c ^ (4 (r & 3)), so
    // that neither the rows of an operand nor the transposing reads meet in a bank.
    const int lr = lane >> 4, vchunk = (lane & 15) ^ (lr << 2), koff = ((lane & 15) ^ ((mine * MINE + lr) & 15)) << 3;
    const int64_t lane_off = (mine * MINE + lr) * stride;

    for (int c0 = begin; c0 < end;) {                             // as many tokens as the list has room for
        const int c1 = LIST ? min(end, c0 + (SPARSE ? TREE_LIST : TREE_LIST * PAGE)) : end;
        const int steps = (c1 - c0 + TT * TEAMS - 1) / (TT * TEAMS);
        bool good = true;
        if (LIST) {
            const int entries = SPARSE ? min(steps * TT * TEAMS, TREE_LIST) : (c1 - c0 + PAGE - 1) / PAGE;
            bool bad = false;
            for (int e = tid; e < entries; e += TREE_THREADS) {
                int at = -1;
                if (SPARSE) {
                    const int i = c0 + e;
                    if (i < c1) {
                        const int pos = i < s.pre ? a.idx[(int64_t)b * a.budget + i] : s.before + (i - s.pre);
                        if (i >= s.pre || (uint32_t)pos < (uint32_t)s.before) at = cache_row<PAGED>(a.cache, b, kvh, pos);
                        bad |= at < 0;
                    }
                } else {
                    at = cache_row<PAGED>(a.cache, b, kvh, c0 + e * PAGE);
                    bad |= at < 0;
                }
                lds.list[e] = at;
            }
            good = !__syncthreads_or(bad);
        }
        auto request = [&](int it) {
            const int t = c0 + (it * TEAMS + team) * TT, r0 = mine * MINE;
            const uint32_t kt = ring + ((it % STAGES) * TEAMS + team) * (2 * TILE_BYTES) + r0 * 256, vt = kt + TILE_BYTES;
#pragma unroll
            for (int n = 0; n < MINE / 4; ++n) {
                const int r = n * 4 + lr;                         // (K's chunks are turned by r0 + r: koff)
                int64_t off;
                if (SPARSE) {
                    off = (int64_t)max(lds.list[min(t - c0 + r0 + r, TREE_LIST - 1)], 0) * stride;
                } else if (PAGED) {
                    // a wave's rows of a tile share pages of 16; behind the list's last entry row 0 has to do
                    const int page = (t - c0 + r0 + n * 4) >> 4;
                    off = (int64_t)((t + r0 + n * 4 < c1 ? max(lds.list[page], 0) : 0) + ((r0 + n * 4) & (PAGE - 1)) + lr) * D;
                } else {
                    off = t + TT <= end ? (t + n * 4) * stride + lane_off : min(t + r0 + r, end - 1) * stride;
                }
                load_to_lds(kbase + off + (koff ^ ((n * 4 & 15) << 3)), kt + n * 1024);
                load_to_lds(vbase + off + (vchunk << 3), vt + n * 1024);
            }
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (i < steps) request(i);
        auto arrive = [&](int it) {                               // tile `it` is there, for the team
            wait_tiles<OPS>(min(steps - 1 - it, AHEAD - 1));
            if (RG > 1) {
                wave_barrier();
                if (it + AHEAD < steps) request(it + AHEAD);
            }
        };
        auto leave = [&](int it) {
            if (RG == 1 && it + AHEAD < steps) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the buffer's last reads
                request(it + AHEAD);
            }
        };
        auto tile_of = [&](int it) -> const unsigned char* { return lds.ring + ((it % STAGES) * TEAMS + team) * (2 * TILE_BYTES); };
        // Tiles that every row attends to as a whole, then the others.  (In one loop the two forms' registers got in each other's way.)
        const int plain = good ? max(0, min(s.pre, c1) - c0) / (TT * TEAMS) : 0;
#pragma unroll 1
        for (int it = 0; it < plain; ++it) {
            arrive(it);
            const unsigned char* const kt = tile_of(it);
            if (!idle) {
#pragma unroll 1
                for (int sub = 0; sub < SUB; ++sub) tree_step<false>(row, kt + sub * 8192, kt + TILE_BYTES + sub * 8192, 0, 0, a.scale_log2e, lane);
            }
            leave(it);
        }
#pragma unroll 1
        for (int it = plain; it < steps; ++it) {
            arrive(it);
            const unsigned char* const kt = tile_of(it);
#pragma unroll 1
            for (int sub = 0; sub < SUB; ++sub) {
                const int t = c0 + (it * TEAMS + team) * TT + 32 * sub;
                uint32_t there = t + 32 <= c1 ? 0xffffffffu : t >= c1 ? 0u : (1u << (c1 - t)) - 1;
                if (LIST && !good) {
                    const int i = t - c0 + col;
                    there = (uint32_t)__ballot(t + col < c1 && lds.list[SPARSE ? i : i >> 4] >= 0);
                }
                if (there == 0 || idle) continue;
                const int from = s.pre - t;                       // tokens of the prefix in this step
                const uint32_t prefix = from >= 32 ? 0xffffffffu : from <= 0 ? 0u : (1u << from) - 1;
                const uint32_t own = mask_window(a.masks + (int64_t)(s.start + node) * a.words, a.words, t - s.pre);
                uint32_t odd = tree_step<true>(row, kt + sub * 8192, kt + TILE_BYTES + sub * 8192, (prefix | own) & there, prefix & there, a.scale_log2e, lane);
                for (odd &= there; odd; odd &= odd - 1) {         // nodes (what is not there stays away)
                    const int i = t + __builtin_ctz(odd) - s.pre;
                    atomicOr(&lds.odd[i >> 5], 1u << (i & 31));
                }
            }
            leave(it);
        }
        c0 = c1;
        if (LIST && c0 < end) __syncthreads();                    // before the list's next entries, and the ring's first tiles
    }

    // The teams' sums, brought to a common maximum, meet in LDS and leave it row by row.
    row.l += __shfl_xor(row.l, 32);
    {
        const int r = team * ROWS + mine * 32 + col;
        if (half == 0) {
            lds.m[r] = row.m;
            lds.l[r] = row.l;
        }
    }
    __syncthreads();
    {
        const int r = mine * 32 + col;
        float top = lds.m[r];
#pragma unroll
        for (int w = 1; w < TEAMS; ++w) top = fmaxf(top, lds.m[w * ROWS + r]);
        const float f = exp2f(row.m - top);
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const int c = 8 * d + 2 * q4 + half;              // 16 bytes of the row
                *reinterpret_cast<f32x4*>(lds.ring + (team * ROWS + r) * (D * 4) + ((c ^ (r & 31)) << 4)) =
                    f32x4{row.o[d][q4 * 4] * f, row.o[d][q4 * 4 + 1] * f, row.o[d][q4 * 4 + 2] * f, row.o[d][q4 * 4 + 3] * f};
            }
    }
    __syncthreads();
    const bool whole = s.chunk >= s.all;
    bool any_odd = false;
#pragma unroll
    for (int i = 0; i < TREE_MAX_NODES / 32; ++i) any_odd |= lds.odd[i] != 0;
    for (int item = tid; item < ROWS * 32; item += TREE_THREADS) {
        const int r = item >> 5, c = item & 31, row = row0 + r;
        if (row >= rows) break;
        float top = lds.m[r];
#pragma unroll
        for (int w = 1; w < TEAMS; ++w) top = fmaxf(top, lds.m[w * ROWS + r]);
        float sum = 0.0f;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < TEAMS; ++w) {
            sum += lds.l[w * ROWS + r] * exp2f(lds.m[w * ROWS + r] - top);
            v += *reinterpret_cast<const f32x4*>(lds.ring + (w * ROWS + r) * (D * 4) + ((c ^ (r & 31)) << 4));
        }
        if (any_odd) {
            // Nodes with values that are not finite: the rows that attend to them get those values (whatever the weight: it is not 0).
            const uint64_t* mask = a.masks + (int64_t)(s.start + (row >> a.g_shift)) * a.words;
            for (int i = 0; i < s.n; ++i) {
                if (!(lds.odd[i >> 5] >> (i & 31) & 1) || !(mask[i >> 6] >> (i & 63) & 1)) continue;
                const int at = cache_row<PAGED>(a.cache, b, kvh, s.before + i);
                const u32x2 w = *reinterpret_cast<const u32x2*>(a.cache.kv.v + cache_offset<PAGED>(a.cache, b, kvh, max(at, 0)) + c * 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t x = (j & 1) ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16;
                    if ((x & 0x7f800000u) == 0x7f800000u) v[j] += __uint_as_float(x);
                }
            }
        }
        const int64_t to = (int64_t)(s.start + (row >> a.g_shift)) * a.H + (kvh << a.g_shift) + (row & (g - 1));
        if (whole) {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            const u32x2 w = {(uint32_t)f32_to_bf16_rne(v[0] * inv) | (uint32_t)f32_to_bf16_rne(v[1] * inv) << 16,
                             (uint32_t)f32_to_bf16_rne(v[2] * inv) | (uint32_t)f32_to_bf16_rne(v[3] * inv) << 16};
            *reinterpret_cast<u32x2*>(a.out + to * D + c * 4) = w;
        } else {
            const int64_t piece = to * a.n_splits + blockIdx.x;
            *reinterpret_cast<f32x4*>(a.part_acc + piece * D + c * 4) = v;
            if (c == 0) *reinterpret_cast<f32x2*>(a.part_ml + piece * 2) = f32x2{top, sum};
        }
    }
}

// Which form a workgroup takes goes by the rows that its own tree has, not by the bound: trees of a batch differ.
template <bool PAGED, bool SPARSE>
__global__ __launch_bounds__(TREE_THREADS, 2) void tree_attn_kernel(TreeArgs a) {
    __shared__ TreeLds lds;
    const int b = blockIdx.z, kvh = blockIdx.y / a.m_tiles, row0 = (blockIdx.y % a.m_tiles) * TREE_ROWS;
    const TreeSpan s = tree_work<SPARSE>(a, b, TREE_UNIT);
    const int left = (s.n << a.g_shift) - row0;
    const int begin = blockIdx.x * s.chunk;
    if (left <= 0 || begin >= s.all) return;
    const int end = min(begin + s.chunk, s.all);
    if (left <= 32) tree_rows<1, PAGED, SPARSE>(a, s, lds, b, kvh, row0, begin, end);
    else if (left <= 64) tree_rows<2, PAGED, SPARSE>(a, s, lds, b, kvh, row0, begin, end);
    else if (left <= 128) tree_rows<4, PAGED, SPARSE>(a, s, lds, b, kvh, row0, begin, end);
    else tree_rows<8, PAGED, SPARSE>(a, s, lds, b, kvh, row0, begin, end);
}

// A wave for a row: a lane for each piece's weight, then two columns a lane.
template <bool SPARSE>
__global__ __launch_bounds__(256) void tree_reduce_kernel(TreeArgs a) {
    const int lane = threadIdx.x & 63, b = blockIdx.y;
    const TreeSpan s = tree_work<SPARSE>(a, b, TREE_UNIT);
    const int r = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (s.chunk >= s.all || r >= s.n * a.H) return;
    const int pieces = (s.all + s.chunk - 1) / s.chunk;
    const int64_t row = (int64_t)s.start * a.H + r, first = row * a.n_splits;
    float m = LOWEST, l = 0.0f;
    if (lane < pieces) {
        const f32x2 ml = *reinterpret_cast<const f32x2*>(a.part_ml + (first + lane) * 2);
        m = ml[0];
        l = ml[1];
    }
    float top = m;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float w = exp2f(m - top);
    float sum = lane < pieces ? w * l : 0.0f;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    f32x2 acc = {0.0f, 0.0f};
    for (int p = 0; p < pieces; ++p) {
        const f32x2 v = *reinterpret_cast<const f32x2*>(a.part_acc + (first + p) * D + lane * 2);
        const float wp = __shfl(w, p);
        acc[0] += wp * v[0];
        acc[1] += wp * v[1];
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    *reinterpret_cast<uint32_t*>(a.out + row * D + lane * 2) = (uint32_t)f32_to_bf16_rne(acc[0] * inv) | (uint32_t)f32_to_bf16_rne(acc[1] * inv) << 16;
}

// ---------------------------------------------------------------- commit

constexpr int COMMIT_LAYERS = 32;          // layers of a launch: their descriptors travel as arguments
constexpr int COMMIT_THREADS = 256;

struct CommitArgs {
    const int32_t *base, *path, *n_path;
    int32_t* keep;
    int32_t max_path;
    CacheArgs layer[COMMIT_LAYERS];
};

// One workgroup for a (layer, sequence, KV head): 16 rows at a time are read, then written.  path ascends, so a row that is still to be read lies
// behind every row written so far.
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
