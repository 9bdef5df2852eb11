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

constexpr int TREE_THREADS = 256;

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
constexpr int TREE_UNIT = 128;             // tokens that a workgroup's waves take at a time, at most

// Bits o .. o + 31 of a node's mask (o may be negative; bits before the first and behind the last are 0).
__device__ __forceinline__ uint32_t mask_window(const uint64_t* row, int words, int o) {
    if (o <= -32) return 0;
    if (o < 0) return (uint32_t)row[0] << -o;
    const int w = o >> 6, sh = o & 63;
    uint64_t x = w < words ? row[w] >> sh : 0;
    if (sh > 32 && w + 1 < words) x |= row[w + 1] << (64 - sh);
    return (uint32_t)x;
}

__device__ __forceinline__ float other_half_max(float v) { return fmaxf(v, __shfl_xor(v, 32)); }

// A wave's 32 RT rows against 32 tokens at a time, with V_MFMA_F32_32X32X16_BF16:
//   S^T = K Q^T      operands: K's rows as they stand, Q's rows (in registers throughout); a lane gets one row's scores of 16 tokens, so that
//                    the softmax runs along registers, with one exchange between the two halves of the wave
//   O^T += V^T P^T   the scores' registers are P^T's operand as they are: 16 tokens of a product are taken in the order in which the lanes
//                    hold them.  V's columns come by transposing LDS reads.
// RG waves share a token tile and split the rows; 4 / RG such teams split the tokens and are added up in LDS at the end.
template <int RT, int RG, bool PAGED, bool SPARSE>
__global__ __launch_bounds__(TREE_THREADS, 1) void tree_attn_kernel(TreeArgs a) {
    constexpr int TEAMS = 4 / RG;
    constexpr int SUB = RG == 4 ? 2 : 1, TT = 32 * SUB;           // tokens of a team's tile
    constexpr int ROWS = 32 * RT * RG;
    constexpr int TILE_BYTES = TT * 256;                          // of K, and again of V
    constexpr int LDS_TILES = TEAMS * 2 * 2 * TILE_BYTES, LDS_OUT = TEAMS * ROWS * D * 4;
    __shared__ __attribute__((aligned(16))) unsigned char smem[LDS_TILES > LDS_OUT ? LDS_TILES : LDS_OUT];
    __shared__ float sm_m[TEAMS][ROWS], sm_l[TEAMS][ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int team = wave / RG, mine = wave % RG, half = lane >> 5, col = lane & 31;
    const int b = blockIdx.z, kvh = blockIdx.y / a.m_tiles, m_tile = blockIdx.y % a.m_tiles;
    const TreeSpan s = tree_work<SPARSE>(a, b, TREE_UNIT);
    const int g = 1 << a.g_shift, rows = s.n << a.g_shift, row0 = m_tile * ROWS;
    const int begin = blockIdx.x * s.chunk;
    if (row0 >= rows || begin >= s.all) return;
    const int end = min(begin + s.chunk, s.all);

    bf16x8 qf[RT][8];
    int node[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = row0 + (mine * RT + rt) * 32 + col;
        const bool there = r < rows;
        node[rt] = there ? r >> a.g_shift : 0;
        const uint16_t* p = a.q + (int64_t)(s.start + node[rt]) * a.q_stride + ((kvh << a.g_shift) + (r & (g - 1))) * D + half * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            u32x4 v = *reinterpret_cast<const u32x4*>(p + k * 16);
            if (!there) v = u32x4{0, 0, 0, 0};
            qf[rt][k] = __builtin_bit_cast(bf16x8, v);
        }
    }
    f32x16 o[RT][4];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        m[rt] = LOWEST;
        l[rt] = 0.0f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[rt][d][i] = 0.0f;
    }

    // Tokens [t0, t0 + TT) of the team into its buffer `st`; returns which of them are there, a bit each.
    auto tile_at = [&](int st, int which) -> unsigned char* { return smem + ((team * 2 + st) * 2 + which) * TILE_BYTES; };
    auto load = [&](int t0, int st) -> uint64_t {
        const int i = t0 + (lane & (TT - 1));
        bool ok = i < end;
        int pos = i;
        if (SPARSE) {
            pos = ok ? (i < s.pre ? a.idx[(int64_t)b * a.budget + i] : s.before + (i - s.pre)) : 0;
            ok = ok && (i >= s.pre || (uint32_t)pos < (uint32_t)s.before);
        }
        if (!ok) pos = 0;
        int row = cache_row<PAGED>(a.cache, b, kvh, pos);
        if (row < 0) ok = false;
        if (!ok) row = 0;
        const uint64_t live = __ballot(ok);
#pragma unroll
        for (int n = 0; n < TT / RG / 4; ++n) {
            const int r0 = mine * (TT / RG) + n * 4, r = r0 + (lane >> 4);
            const int64_t off = cache_offset<PAGED>(a.cache, b, kvh, __shfl(row, r));
            const int ck = (lane & 15) ^ (r & 15), cv = (lane & 15) ^ ((r & 3) << 2);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(a.cache.kv.k + off + ck * 8),
                                             (__attribute__((address_space(3))) void*)(tile_at(st, 0) + r0 * 256), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(a.cache.kv.v + off + cv * 8),
                                             (__attribute__((address_space(3))) void*)(tile_at(st, 1) + r0 * 256), 16, 0, 0);
        }
        return TT == 32 ? live & 0xffffffffull : live;
    };

    const int steps = (end - begin + TT * TEAMS - 1) / (TT * TEAMS);
    uint64_t live = load(begin + team * TT, 0);
    for (int it = 0; it < steps; ++it) {
        __builtin_amdgcn_s_waitcnt(0x0f70);                       // vmcnt(0)
        __syncthreads();
        const int t0 = begin + (it * TEAMS + team) * TT, st = it & 1;
        uint64_t next = 0;
        if (it + 1 < steps) next = load(t0 + TEAMS * TT, st ^ 1);
        const unsigned char* kt = tile_at(st, 0);
        const unsigned char* vt = tile_at(st, 1);
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) {
            const uint32_t there = (uint32_t)(live >> (32 * sub));
            if (there == 0) continue;
            const int t = t0 + 32 * sub;
            const bool edge = there != 0xffffffffu || t + 32 > s.pre;
            f32x16 x[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[rt][i] = 0.0f;
            const int kr = sub * 32 + col;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kt + kr * 256 + (((2 * k + half) ^ (kr & 15)) << 4));
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) x[rt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[rt][k], x[rt], 0, 0, 0);
            }
            uint32_t allowed[RT];
            if (edge) {
                const int from = s.pre - t;                       // tokens of the prefix in this step
                const uint32_t prefix = from >= 32 ? 0xffffffffu : from <= 0 ? 0u : (1u << from) - 1;
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const uint32_t own = mask_window(a.masks + (int64_t)(s.start + node[rt]) * a.words, a.words, t - s.pre);
                    allowed[rt] = (prefix | own) & there;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (!(allowed[rt] >> (8 * (i >> 2) + 4 * half + (i & 3)) & 1)) x[rt][i] = -INFINITY;
                }
            }
            bool raise = false;
            float mt[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float mx = x[rt][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) mx = fmaxf(mx, x[rt][i]);
                mt[rt] = other_half_max(mx) * a.scale_log2e;
                raise |= mt[rt] > m[rt] + 8.0f;
            }
            if (__any(raise)) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const float to = mt[rt] > m[rt] + 8.0f ? mt[rt] : m[rt], f = exp2f(m[rt] - to);   // a row's sums do not depend on its neighbours
                    m[rt] = to;
                    l[rt] *= f;
#pragma unroll
                    for (int d = 0; d < 4; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[rt][d][i] *= f;
                }
            }
            bf16x8 p[RT][2];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[rt][i], a.scale_log2e, -m[rt]));
                    l[rt] += e;
                    p[rt][i >> 3][i & 7] = (__bf16)e;
                }
            uint32_t odd = 0;                                     // edge: this lane's tokens with a value that is not finite
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const int tok = sub * 32 + 16 * k + 4 * half + ((lane >> 2) & 3);
                    const int chunk = (4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ (((lane >> 2) & 3) << 2);
                    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
                    const unsigned char* at = vt + tok * 256 + (chunk << 4) + (lane & 1) * 8;
                    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
                    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 8 * 256));
                    typedef short s16x8 __attribute__((ext_vector_type(8)));
                    s16x8 v = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
                    if (edge) {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if ((v[j] & 0x7f80) == 0x7f80) {
                                odd |= 1u << (16 * k + 4 * half + (j & 3) + 8 * (j >> 2));
                                v[j] = 0;
                            }
                    }
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
                        o[rt][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), p[rt][k], o[rt][d], 0, 0, 0);
                }
            if (edge && __any(odd != 0)) {
                // Values that are not finite reach the rows that attend to them, and only those: a weight of 0 would make NaN of them.
                // (They were left out above; what they give does not depend on the weight.)
                for (int tok = 0; tok < 32; ++tok) {
                    if (!__any(odd >> tok & 1)) continue;
#pragma unroll
                    for (int d = 0; d < 4; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int c = 32 * d + 8 * (i >> 2) + 4 * half + (i & 3), row = sub * 32 + tok;
                            const uint16_t w = *reinterpret_cast<const uint16_t*>(vt + row * 256 + (((c >> 3) ^ ((row & 3) << 2)) << 4) + (c & 7) * 2);
                            if ((w & 0x7f80) != 0x7f80) continue;
#pragma unroll
                            for (int rt = 0; rt < RT; ++rt)
                                if (allowed[rt] >> tok & 1) o[rt][d][i] += __uint_as_float((uint32_t)w << 16);
                        }
                }
            }
        }
        live = next;
    }

    // The teams' sums, brought to a common maximum, meet in LDS and leave it row by row.
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] += __shfl_xor(l[rt], 32);
        if (half == 0) {
            const int r = (mine * RT + rt) * 32 + col;
            sm_m[team][r] = m[rt];
            sm_l[team][r] = l[rt];
        }
    }
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = (mine * RT + rt) * 32 + col;
        float top = sm_m[0][r];
#pragma unroll
        for (int w = 1; w < TEAMS; ++w) top = fmaxf(top, sm_m[w][r]);
        const float f = exp2f(m[rt] - top);
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const int c = 8 * d + 2 * q4 + half;              // 16 bytes of the row
                *reinterpret_cast<f32x4*>(smem + (team * ROWS + r) * (D * 4) + ((c ^ (r & 31)) << 4)) =
                    f32x4{o[rt][d][q4 * 4] * f, o[rt][d][q4 * 4 + 1] * f, o[rt][d][q4 * 4 + 2] * f, o[rt][d][q4 * 4 + 3] * f};
            }
    }
    __syncthreads();
    const bool whole = s.chunk >= s.all;
    for (int item = tid; item < ROWS * 32; item += TREE_THREADS) {
        const int r = item >> 5, c = item & 31, row = row0 + r;
        if (row >= rows) break;
        float top = sm_m[0][r];
#pragma unroll
        for (int w = 1; w < TEAMS; ++w) top = fmaxf(top, sm_m[w][r]);
        float sum = 0.0f;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < TEAMS; ++w) {
            sum += sm_l[w][r] * exp2f(sm_m[w][r] - top);
            v += *reinterpret_cast<const f32x4*>(smem + (w * ROWS + r) * (D * 4) + ((c ^ (r & 31)) << 4));
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
