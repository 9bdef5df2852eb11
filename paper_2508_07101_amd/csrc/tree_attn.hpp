// Attention of several rows of queries over one sequence's tokens, or over the pages of a group of sequences.
//
//   tree_attn_kernel    attention of a tree's nodes over the prefix (or the part of it that was chosen) and their branch
//   tree_reduce_kernel  merges the pieces of a long prefix
//
// The second form of both, BEAM: instead of a tree's nodes the rows of a group, instead of a sequence's tokens the group's list of pages (cusa_shared), each with the rows that
// hold it.  The pages that all rows attend to as a whole come first and are the prefix; behind them a row attends to the tokens of the pages that it holds, up to its length.
#pragma once
#include <type_traits>

#include "plan_scan.hpp"
#include "tree_plan.hpp"

namespace cusa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- attention

// The rows of sequence b in packed arrays: [start, start + n).
__device__ __forceinline__ int tree_span(const int32_t* tok_start, int b, int max_tokens, int max_nodes, int& start) {
    start = clampi(tok_start[b], 0, max_tokens);
    const int stop = clampi(tok_start[b + 1], start, max_tokens);
    return min(stop - start, max_nodes);
}
struct TreeArgs {
    CacheArgs cache;
    const uint16_t* q;
    int64_t q_stride;
    const int32_t *tok_start, *idx, *cnt;
    const uint64_t* masks;
    uint16_t* out;
    float *part_acc, *part_ml;
    int32_t* pieces;       // of each sequence's tokens, for the merge
    float scale_log2e;
    int32_t batch, max_tokens, max_nodes, words, budget, H, g_shift, tile_rows /* 128 or 256 */, m_tiles, n_splits;
    // groups: batch of them, of max_nodes rows each
    const int32_t *entries, *count;
    int32_t max_entries;   // of a group, looked at
    int64_t entry_stride;
};

constexpr int TREE_WAVES = 8, TREE_THREADS = 64 * TREE_WAVES;
constexpr int TREE_TILE = 32;              // tokens of a tile: pieces are whole tiles

// What a workgroup of one sequence has to do, the same in the attention and in the merge.
struct TreeSpan {
    int start, n;          // its nodes' rows in the packed arrays
    int part;              // its first row among the partial results
    int before, pre, all;  // P; tokens of the prefix that are looked at; the same and the nodes
    int chunk;             // tokens of a piece
};
// The workspace has rows for max_nodes nodes of a sequence.  A sequence that owns more rows of the packed arrays has only its first max_nodes looked at:
// the next one's start there may lie behind the workspace's rows, and its partial results move up (to rows of their own: starts are apart by as much).
__device__ __forceinline__ int part_row(const TreeArgs& a, int b, int start) { return min(start, b * a.max_nodes); }
template <bool SPARSE, bool BEAM>
__device__ __forceinline__ TreeSpan tree_span(const TreeArgs& a, int b) {
    TreeSpan s;
    if constexpr (BEAM) {
        const int n = clampi(a.count[b * 2], 0, a.max_entries);
        s.n = a.max_nodes;
        s.start = s.part = b * s.n;
        s.before = 0;
        s.pre = clampi(a.count[b * 2 + 1], 0, n) * PAGE;
        s.all = n * PAGE;
        return s;
    }
    const int L = clampi(a.cache.kv.seq_lens[b], 0, a.cache.max_len);
    s.n = min(tree_span(a.tok_start, b, a.max_tokens, a.max_nodes, s.start), L);
    s.part = part_row(a, b, s.start);
    s.before = L - s.n;
    s.pre = SPARSE ? clampi(a.cnt[b], 0, a.budget) : s.before;
    s.all = s.n > 0 ? s.pre + s.n : 0;
    return s;
}
__device__ __forceinline__ int tiles_of(int tokens) { return (tokens + TREE_TILE - 1) / TREE_TILE; }
// The batch's pieces are of one length, which goes by the lengths that there are.  With the tiles T of all KV heads' sequences, W of these in number
// and at most M tiles in one, pieces of ceil(M / floor(R / W)) tiles are R at most, and so are pieces of T / (R - W) tiles (a last piece each is shorter):
// the first is exact for sequences of one length, the second close for any.  R: one to eight workgroups for each CU; more are better balanced, but
// each costs about TREE_PIECE_COST tiles besides its own (its start, and partial sums written and read).
template <bool SPARSE, bool BEAM>
__device__ __forceinline__ int tree_piece(const TreeArgs& a, const TreeSpan& own) {   // tiles; 0: no sequence is cut
    if (a.n_splits == 1) return 0;
    int total = 0, pairs = 0, most = 0, piece = 0;
    for (int i = threadIdx.x & 63; i < a.batch || (a.batch == 1 && i < 64); i += 64) {   // (of one sequence every lane has the numbers already)
        const TreeSpan o = a.batch == 1 ? own : tree_span<SPARSE, BEAM>(a, i);
        const int wgs = a.cache.kv.G * (((o.n << a.g_shift) + a.tile_rows - 1) >> __builtin_ctz(a.tile_rows)), t = tiles_of(o.all);
        total += t * wgs;
        pairs += wgs;
        most = max(most, t);
    }
    if (a.batch > 1) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            total += __shfl_xor(total, o);
            pairs += __shfl_xor(pairs, o);
            most = max(most, __shfl_xor(most, o));
        }
    }
    total = __builtin_amdgcn_readfirstlane(total);
    pairs = max(__builtin_amdgcn_readfirstlane(pairs), 1);
    most = __builtin_amdgcn_readfirstlane(most);
    // a lane for each R, of which the first eight count (the others repeat them); one sequence takes R = 1
    const int r = (threadIdx.x & (a.batch > 1 ? 7 : 0)) + 1, wgs = r * TREE_CUS;
    int cost = 0x7fffffff;
    if (wgs >= pairs) {
        piece = (most + wgs / pairs - 1) / (wgs / pairs);
        if (wgs > pairs) piece = min(piece, (total + wgs - pairs - 1) / (wgs - pairs));
        piece = max(piece, TREE_MIN_PIECE / TREE_TILE);
        cost = r * (piece + TREE_PIECE_COST);
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
        const int other_cost = __shfl_xor(cost, o), other_piece = __shfl_xor(piece, o);
        if (other_cost < cost || (other_cost == cost && other_piece > piece)) {
            cost = other_cost;
            piece = other_piece;
        }
    }
    piece = __builtin_amdgcn_readfirstlane(piece);
    return piece > 0 ? piece : most;                              // (0: more sequences than pieces would balance, which stay whole)
}
template <bool SPARSE>
__device__ __forceinline__ TreeSpan tree_work(const TreeArgs& a, int b) {
    TreeSpan s = tree_span<SPARSE, false>(a, b);
    int piece = tree_piece<SPARSE, false>(a, s);
    if (a.n_splits == 1) {
        piece = tiles_of(s.all);
    } else {
        piece = min(piece, (SPARSE ? TREE_LIST : TREE_LIST * PAGE) / TREE_TILE);   // what a workgroup's list has room for
        piece = max(piece, (tiles_of(s.all) + a.n_splits - 1) / a.n_splits);       // what the launch has pieces for
    }
    s.chunk = piece * TREE_TILE;
    return s;
}

// The same for groups: unit u of a launch is a KV head and the u / G -th of all groups' pieces, one group after the other, so that all that have work come first.  (In order of the pieces' numbers, with
// those that short groups do not have in between, workgroups waited for places while CUs of other shader engines had some: 8 samples of 8 prompts of 1024 to 2048 tokens, 488 pieces: 24 of the 256 CUs
// had three, 48 one, and the last began after 146 of 242 us.)  False: there is no such piece.  A group without tokens has one.
__device__ __forceinline__ bool group_work(const TreeArgs& a, int u, TreeSpan& s, int& b, int& kvh, int& split) {
    const int G = a.cache.kv.G, v = u / G, lane = threadIdx.x & 63;
    kvh = u - v * G;
    split = 0;
    if (a.n_splits == 1) {
        b = v;
        if (b >= a.batch) return false;
        s = tree_span<false, true>(a, b);
        s.chunk = tiles_of(s.all) * TREE_TILE;
        return true;
    }
    if (a.batch == 1) s = tree_span<false, true>(a, 0);
    const int piece = min(tree_piece<false, true>(a, s), BEAM_LIST * PAGE / TREE_TILE);   // (what a workgroup's list has room for)
    for (int i0 = 0, before = 0; i0 < a.batch; i0 += 64) {
        const int i = i0 + lane, t = i < a.batch ? tiles_of(tree_span<false, true>(a, i).all) : 0;
        const int chunk = max(piece, (t + a.n_splits - 1) / a.n_splits), n = i < a.batch ? max((t + chunk - 1) / chunk, 1) : 0;   // (what the launch has pieces for)
        int sum = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(sum, o);
            if (lane >= o) sum += y;
        }
        const uint64_t behind = __ballot(before + sum > v);
        if (behind) {
            const int at = __builtin_ctzll(behind);
            b = i0 + at;
            split = v - before - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(n, at));
            s = tree_span<false, true>(a, b);
            s.chunk = __builtin_amdgcn_readlane(chunk, at) * TREE_TILE;
            return true;
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

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
// m0 is a reserved register: the compiler keeps nothing in it.  With the streaming hint: the caches need not keep what is read once (a copy of 128 MB to LDS by 256 workgroups: 24.4 us, so 19.7).
__device__ __forceinline__ void load_to_lds(const uint16_t* from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(lds), "v"(from) : "memory");
}
// The same from a uniform address and 32 bits of offset a lane.
__device__ __forceinline__ void load_to_lds(const uint16_t* base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(offset), "s"(base) : "memory");
}
// Until all but the newest min(n, MOST) of this wave's requests of OPS loads each have arrived.
template <int OPS, int MOST>
__device__ __forceinline__ void wait_tiles(int n) {
    static_assert(OPS * MOST < 64, "the counter's range");
    if (MOST > 0 && n >= MOST) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(OPS * MOST) : "memory");
        return;
    }
    if constexpr (MOST > 1) wait_tiles<OPS, MOST - 1>(n);
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}
__device__ __forceinline__ void wave_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

constexpr int TREE_RING = 128 * 1024;      // bytes of LDS for token tiles
template <bool BEAM>
struct TreeLds {
    static constexpr int LIST = BEAM ? BEAM_LIST : TREE_LIST;
    __attribute__((aligned(16))) unsigned char ring[TREE_RING];
    int32_t list[LIST];
    float m[TREE_ROWS], l[TREE_ROWS];      // of every row, a set for each team
    uint32_t odd[(BEAM ? LIST : TREE_MAX_NODES) / 32];   // nodes (pages) among this workgroup's tokens with a value that is not finite
    int32_t first_bad;                     // entry of the list that names no row (0: a page has such a value)
    int32_t first[BEAM ? LIST : 1];        // of a group's page: its first position, and the rows that hold it
    uint32_t holders[BEAM ? LIST : 1];
};

typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

// The state of a wave's 32 rows: a lane and its counterpart in the other half of the wave have one row.
struct TreeRow {
    bf16x8 q[8];           // columns 16 k + 8 half ..
    f32x16 o[4];           // columns 32 d + 8 (i / 4) + 4 half + i % 4
    float m, l;            // reference of the weights in log2 units, the half's sum of weights
};

// S^T = K Q^T of 32 tokens: K's rows as they stand in the tile; a lane gets its row's scores of the tokens 8 (i / 4) + 4 half + i % 4.
struct TreeKeys {
    bf16x8 f[8];
};
// Where a lane reads in a tile, for the tile at LDS address 0: chunk 2 k + half of K's row `col` stands at (2 k + half) ^ (col & 15).  V's columns 32 d .. of
// the tokens 16 k .. come in the order in which the lanes hold the scores: 16 lanes transpose 4 tokens by 16 columns, tokens 16 k + 4 half + .. and
// 8 further on.
__device__ __forceinline__ uint32_t key_at(int lane, int k) { return (lane & 31) * 256 + ((((lane >> 5) ^ (lane & 15)) << 4) ^ (k << 5)); }
__device__ __forceinline__ uint32_t value_at(int lane, int d) {
    const int row4 = (lane >> 2) & 3;
    return (4 * (lane >> 5) + row4) * 256 + (lane & 1) * 8 + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) << 4) | ((d ^ row4) << 6));
}
typedef const __attribute__((address_space(3))) bf16x8* lds_bf16x8;
__device__ __forceinline__ bf16x8 read_key(uint32_t at) { return *(lds_bf16x8)(uintptr_t)at; }
__device__ __forceinline__ s16x8 read_value(uint32_t at) {
    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)at);
    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(at + 2048));
    return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ void read_keys(TreeKeys& kf, uint32_t kt, int lane) {
#pragma unroll
    for (int k = 0; k < 8; ++k) kf.f[k] = read_key(kt + key_at(lane, k));
}
__device__ __forceinline__ f32x16 score(const TreeRow& r, const TreeKeys& kf) {
    f32x16 x;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf.f[k], r.q[k], x, 0, 0, 0);
    return x;
}
struct TreeValues {
    s16x8 f[2][4];
};
__device__ __forceinline__ void read_values(TreeValues& vf, uint32_t vt, int lane) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int d = 0; d < 4; ++d) vf.f[k][d] = read_value(vt + 4096 * k + value_at(lane, d));
}
// O^T += V^T P^T: the weights are the product's operand in the order in which the lanes hold them.
// Up to 64 rows, where memory bounds the time, a weight is two bf16 numbers, f + rest, and takes two products: it is off by 2^-15 of itself at most.  (Over
// 64 sequences of 20480 tokens this costs 1 % for up to 32 rows and 2 to 5 % for 64.)  Above, where the products bound the time, it is one, off by 2^-8 at
// most, and the row's sum adds up the rounded weights: a token that outweighs the others is rounded alike in both.
struct TreeWeights {
    bf16x8 f[2];
};
struct TreeFineWeights {
    bf16x8 f[2], rest[2];
};
__device__ __forceinline__ void add_product(f32x16& o, s16x8 v, const TreeWeights& p, int k) {
    o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), p.f[k], o, 0, 0, 0);
}
__device__ __forceinline__ void add_product(f32x16& o, s16x8 v, const TreeFineWeights& p, int k) {
    o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), p.rest[k], o, 0, 0, 0);
    o = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), p.f[k], o, 0, 0, 0);
}
template <int K, typename W>
__device__ __forceinline__ void add_values(TreeRow& r, const TreeValues& vf, const W& p) {
#pragma unroll
    for (int d = 0; d < 4; ++d) add_product(r.o[d], vf.f[K][d], p, K);
}
template <typename W>
__device__ __forceinline__ void add_values(TreeRow& r, const TreeValues& vf, const W& p) {
    add_values<0>(r, vf, p);
    add_values<1>(r, vf, p);
}
// A weight 2^(scale x - m).  The instruction makes 0 of results below 2^-126, which beside a value of 2^120 are not nothing: it makes the weight's 2^64-fold.
// (With the sums below 1 to 2 % for 128 to 512 rows.)
__device__ __forceinline__ float weight(float m, float x, float scale_log2e) {
    return __builtin_amdgcn_exp2f(__builtin_fmaf(x, scale_log2e, 64.0f - m)) * 0x1p-64f;
}
// The weights' sum, in 32 bits, is of the rounded ones: two-element dot products.  These wait for the matrix pipe, so they stand where this wave has no products to
// issue beside them.  (64 sequences of 20480 tokens under 64 nodes, 256 rows: weights below 2^-126 left out and sums unrounded 1508 us; both in, dot products among the
// products 1559, behind them 1520.  Taking the weights apart again and adding them one by one: 4 to 6 % for 128 to 512 rows.)
template <int FROM, int TO>
__device__ __forceinline__ void weigh(float m, const f32x16& x, float scale_log2e, TreeWeights& p) {
#pragma unroll
    for (int i = FROM; i < TO; ++i) p.f[i >> 3][i & 7] = (__bf16)weight(m, x[i], scale_log2e);
}
__device__ __forceinline__ float add_up(const TreeWeights& p) {
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{p.f[i >> 3][i & 7], p.f[i >> 3][(i & 7) + 1]}, ones, sum, false);
    return sum;
}
__device__ __forceinline__ float weigh(float m, const f32x16& x, float scale_log2e, TreeWeights& p) {
    weigh<0, 16>(m, x, scale_log2e, p);
    return add_up(p);
}
// f: the weight cut to bf16, less one step; rest: what is missing, a step to two, rounded.  Neither is negative or, from 2^-132 on, 0, so that a value that is
// infinite stays so in both products.
__device__ __forceinline__ float weigh(float m, const f32x16& x, float scale_log2e, TreeFineWeights& p) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const float w0 = weight(m, x[i], scale_log2e), w1 = weight(m, x[i + 1], scale_log2e);
        const uint32_t cut = __builtin_amdgcn_perm(__float_as_uint(w1), __float_as_uint(w0), 0x07060302);
        const uint32_t less = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, cut), u16x2{1, 1}));
        const bf16x2 f = __builtin_bit_cast(bf16x2, less);
        p.f[i >> 3][i & 7] = f[0];
        p.f[i >> 3][(i & 7) + 1] = f[1];
        p.rest[i >> 3][i & 7] = (__bf16)(w0 - __uint_as_float(less << 16));
        p.rest[i >> 3][(i & 7) + 1] = (__bf16)(w1 - __uint_as_float(less & 0xffff0000u));
        sum += w0;
        sum += w1;
    }
    return sum;
}
// A row's reference m follows its scores only when their weights have outgrown 2^8 (they are held in 32 bits until they are rounded relative to
// themselves, so that nothing is lost up to there): the weights' sum, which is needed anyway, tells, and no maximum is taken otherwise.
// From LOWEST, any score does.  NaN scores come here at every step.
constexpr float TREE_RAISE = 256.0f;
template <typename W>
__device__ __forceinline__ void raise_and_weigh(TreeRow& r, const f32x16& x, float scale_log2e, W& p, float sum) {
    if (__any(!(sum <= TREE_RAISE))) {
        float mx = x[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, x[i]);
        mx = other_half_max(mx) * scale_log2e;
        // a row's sums do not depend on its neighbours
        const float grown = other_half_max(sum <= TREE_RAISE ? 0.0f : 1.0f), to = grown != 0.0f ? fmaxf(mx, r.m) : r.m, f = exp2f(r.m - to);
        r.m = to;
        r.l *= f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) r.o[d][i] *= f;
        sum = weigh(to, x, scale_log2e, p);
    }
    r.l += sum;
}

// One step of a run of tiles that every row attends to as a whole: this tile's weights p from its scores x, and beside them, independent of them, the
// next tile's scores y and the last tile's share of the output (weights p_last).  The tiles' buffers stand NEXT_K, LAST_V behind the lane's
// addresses: a constant of the instruction, where the loop is unrolled over the buffers.
template <int NEXT_K, int LAST_V>
__device__ __forceinline__ void tree_step(TreeRow& r, const f32x16& x, f32x16& y, TreeWeights& p, const TreeWeights& p_last, const uint32_t (&key)[8],
                                          const uint32_t (&value)[4], float scale_log2e) {
    TreeKeys kf;
    TreeValues vf;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int d = 0; d < 4; ++d) vf.f[k][d] = read_value(value[d] + LAST_V + 4096 * k);
#pragma unroll
    for (int k = 0; k < 4; ++k) kf.f[k] = read_key(key[k] + NEXT_K);
    __builtin_amdgcn_sched_barrier(0);
    weigh<0, 8>(r.m, x, scale_log2e, p);                          // (while the operands are on their way)
    __builtin_amdgcn_sched_barrier(0);
    // products and softmax in turn: in this order they issue, and neither pipe waits for the other
    add_values<0>(r, vf, p_last);
    weigh<8, 12>(r.m, x, scale_log2e, p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, 3, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 4; k < 8; ++k) kf.f[k] = read_key(key[k] + NEXT_K);   // (in the first values' registers)
    __builtin_amdgcn_sched_barrier(0);
    add_values<1>(r, vf, p_last);
    weigh<12, 16>(r.m, x, scale_log2e, p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, 3, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    y = score(r, kf);
    __builtin_amdgcn_sched_barrier(0);
    raise_and_weigh(r, x, scale_log2e, p, add_up(p));
}
// A tile that not every row attends to as a whole: scores of the tokens outside `allowed` (a bit each) weigh nothing.
__device__ __forceinline__ void mask_scores(f32x16& x, uint32_t allowed, int half) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (!(allowed >> (8 * (i >> 2) + 4 * half + (i & 3)) & 1)) x[i] = -INFINITY;
}
// Its share of the output.  Values that are not finite must not meet the weight 0 of a row that does not attend to them: those of the tokens in `wash`,
// which not every row attends to, are left out, and the lane's tokens with such values returned.
template <typename W>
__device__ __forceinline__ uint32_t add_washed(TreeRow& r, const W& p, uint32_t vt, uint32_t wash, int lane) {
    const int half = lane >> 5;
    uint32_t odd = 0;
    wash >>= 4 * half;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            u32x4 v = __builtin_bit_cast(u32x4, read_value(vt + 4096 * k + value_at(lane, d)));
#pragma unroll
            for (int j = 0; j < 4; ++j) {                         // two tokens a word
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
            asm volatile("" ::: "memory");                        // one operand at a time: no registers for more
            add_product(r.o[d], __builtin_bit_cast(s16x8, v), p, k);
        }
    return odd << (4 * half);
}
// The same for tiles that mostly hold nothing to leave out, those of pages that some rows hold: a look at all values first, two words of work for two of them, and the plain products if they are
// finite.  (8 samples of 8 prompts, 270 000 tokens of their own: value by value 196 us, so 179.)
template <typename W>
__device__ __forceinline__ uint32_t add_looked_over(TreeRow& r, const W& p, uint32_t vt, uint32_t wash, int lane) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 most = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const u32x4 v = __builtin_bit_cast(u32x4, read_value(vt + 4096 * k + value_at(lane, d)));
#pragma unroll
            for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, v[j] & 0x7fff7fffu));
        }
    if (__any(most[0] >= 0x7f80 || most[1] >= 0x7f80)) return add_washed(r, p, vt, wash, lane);
    asm volatile("" ::: "memory");                                // (read again: no registers for all values beside the search)
    TreeValues vf;
    read_values(vf, vt, lane);
    add_values(r, vf, p);
    return 0;
}

// A workgroup's rows against tokens [begin, end).  RG waves share a token tile and split the rows; 8 / RG such teams split the tokens and are added up in
// LDS at the end.  Two waves to a SIMD.  Tiles come by loads from memory straight to LDS, several of them under way.
// One pass: S^T = K Q^T, weights 2^(scale S - m) against a reference m that the row keeps, O^T += V^T P^T, divided by the weights' sum at the end.
// What bounds it goes by the rows that share a KV head's tokens (64 sequences of 20480 tokens, 32 heads over 8, paged): memory up to 128 rows (nodes times
// query heads of a KV head): 4 rows 6.5 TB/s, 32 rows 6.2, 64 rows 5.6 to 5.9, 128 rows 5.2 to 5.4 TB/s and 660 to 690 TFLOP/s; above that the matrix cores and the softmax
// beside them: 256 rows 856 to 873 TFLOP/s, 512 rows 933 (a library product of 8192^3 reaches 1210).  192 rows cost as much as 256 do on half of the SIMDs: 717.  One
// sequence of 32768 tokens, 240 rows: 50 us, of which about 29 are the tiles' arrival, 6 the way to the first tile, 5 the partial sums' way out.
template <int RG, bool PAGED, bool SPARSE, bool BEAM>
__device__ __forceinline__ void tree_rows(const TreeArgs& a, const TreeSpan& s, TreeLds<BEAM>& lds, int b, int kvh, int row0, int split, int begin, int end) {
    constexpr int TEAMS = TREE_WAVES / RG;
    constexpr int TT = TREE_TILE;                                 // tokens of a team's tile
    constexpr int ROWS = 32 * RG;
    constexpr int TILE_BYTES = TT * 256;                          // of K or V
    constexpr int STAGES = TREE_RING / 2 / (TEAMS * TILE_BYTES);  // buffers of K, and of V: as many as waves in a team
    constexpr int MINE = TT / RG;                                 // rows that a wave loads
    constexpr int OPS = 2 * MINE / 4;                             // its loads for a tile of K and one of V
    constexpr bool LIST = PAGED || SPARSE;
    static_assert(TREE_LIST % (TT * TEAMS) == 0, "a full list is whole steps");
    static_assert(TEAMS * ROWS * D * 4 <= TREE_RING && TEAMS * ROWS <= TREE_ROWS && MINE % 4 == 0, "the teams' sums take the tiles' place");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int team = wave / RG, mine = wave % RG, half = lane >> 5, col = lane & 31;
    const int g = 1 << a.g_shift, rows = s.n << a.g_shift;
    if (tid < (BEAM ? BEAM_LIST : TREE_MAX_NODES) / 32) lds.odd[tid] = 0;
    if (tid == 0) lds.first_bad = 0x7fffffff;
    __syncthreads();

    // (a group's list is asked for before q: one way to memory and back instead of two)
    const i32x4* const list = BEAM ? reinterpret_cast<const i32x4*>(a.entries) + b * a.entry_stride + begin / PAGE : nullptr;
    i32x4 entry = {0, 0, 0, 0};
    if constexpr (BEAM) entry = list[min(tid, (end - begin) / PAGE - 1)];
    TreeRow row;
    const int my_row = row0 + mine * 32 + col;
    const bool there = my_row < rows;
    const int node = there ? my_row >> a.g_shift : 0;
    {
        const uint16_t* p = a.q + (int64_t)(s.start + node) * a.q_stride + ((kvh << a.g_shift) + (my_row & (g - 1))) * D + half * 8;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            u32x4 v = *reinterpret_cast<const u32x4*>(p + k * 16);
            if (!there) v = u32x4{0, 0, 0, 0};
            row.q[k] = __builtin_bit_cast(bf16x8, v);
        }
    }
    row.m = LOWEST;
    row.l = 0.0f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) row.o[d][i] = 0.0f;
    const int row_len = BEAM ? clampi(a.cache.kv.seq_lens[s.start + node], 0, a.cache.max_len) : 0;
    const bool idle = row0 + mine * 32 >= rows;                   // a wave without rows loads its share and computes nothing

    const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds.ring;
    const uint16_t* const kbase = a.cache.kv.k + (PAGED ? 0 : (int64_t)b * a.cache.kv.sb + (int64_t)kvh * a.cache.kv.sh);
    const uint16_t* const vbase = a.cache.kv.v + (PAGED ? 0 : (int64_t)b * a.cache.kv.sb + (int64_t)kvh * a.cache.kv.sh);
    const uint32_t stride = PAGED ? D : (uint32_t)a.cache.kv.st;   // (below 2^31: the host checks)
    // A lane's part of a row, in the order in which LDS holds it: K's 16-byte chunk c of row r stands at c ^ (r & 15), V's at c ^ (4 (r & 3)), so
    // that neither the rows of an operand nor the transposing reads meet in a bank.
    const int lr = lane >> 4, vchunk = ((lane & 15) ^ (lr << 2)) << 3, kchunk = ((lane & 15) ^ ((mine * MINE + lr) & 15)) << 3;
    const uint64_t lane_off = (uint64_t)(uint32_t)(mine * MINE + lr) * stride;

    const int steps = (end - begin + TT * TEAMS - 1) / (TT * TEAMS);
    int good = end;                                               // tokens before this one are all there
    if constexpr (BEAM) {
        const int entries = (end - begin) / PAGE;
        for (int e = tid; e < entries; e += TREE_THREADS) {
            const i32x4 x = e < TREE_THREADS ? entry : list[e];
            const bool is = (uint32_t)x[0] < (uint32_t)a.cache.n_pages && x[1] >= 0;   // (all are, of a list that cusa_shared_pages made for this pool)
            lds.list[e] = is ? (x[0] * a.cache.kv.G + kvh) * PAGE : 0;
            lds.first[e] = min(x[1], 0x7fffffff / PAGE) * PAGE;
            lds.holders[e] = is ? (uint32_t)x[2] : 0;
        }
        __syncthreads();
    } else if (LIST) {
        const int entries = SPARSE ? steps * TT * TEAMS : (end - begin + PAGE - 1) / PAGE;
        constexpr int RUN = 4;                                    // entries of a thread under way at once
        for (int e0 = tid; e0 < entries; e0 += RUN * TREE_THREADS) {
            int pos[RUN], at[RUN];
#pragma unroll
            for (int j = 0; j < RUN; ++j) {
                const int e = e0 + j * TREE_THREADS, i = SPARSE ? begin + e : begin + e * PAGE;
                pos[j] = SPARSE ? s.before + (i - s.pre) : i;
                if (e >= entries || i >= end) pos[j] = -1;
                else if (SPARSE && i < s.pre) pos[j] = a.idx[(int64_t)b * a.budget + i];
            }
#pragma unroll
            for (int j = 0; j < RUN; ++j) {
                const int i = begin + e0 + j * TREE_THREADS;
                at[j] = -1;
                if (pos[j] >= 0 && (!SPARSE || i >= s.pre || pos[j] < s.before)) at[j] = cache_row<PAGED>(a.cache, b, kvh, pos[j]);
            }
#pragma unroll
            for (int j = 0; j < RUN; ++j) {
                const int e = e0 + j * TREE_THREADS;
                if (e >= entries) continue;
                if (at[j] < 0 && (SPARSE ? begin + e : begin + e * PAGE) < end) atomicMin(&lds.first_bad, e);
                lds.list[e] = at[j];
            }
        }
        __syncthreads();
        const int bad = __builtin_amdgcn_readfirstlane(lds.first_bad);
        if (bad != 0x7fffffff) good = begin + (SPARSE ? bad : bad * PAGE);   // (a list that ends with the tree's first node has one in its last tile)
    }
    auto k_at = [&](int it) { return ((it % STAGES) * TEAMS + team) * TILE_BYTES; };
    auto v_at = [&](int it) { return TREE_RING / 2 + ((it % STAGES) * TEAMS + team) * TILE_BYTES; };
    auto request = [&](int it, bool values) {
        const int t = begin + (it * TEAMS + team) * TT, r0 = mine * MINE;
        const uint32_t to = ring + (values ? v_at(it) : k_at(it)) + r0 * 256;
        int chunk = values ? vchunk : kchunk;
        asm volatile("" : "+v"(chunk));                           // else every row's address parts are kept in registers all along
#pragma unroll
        for (int n = 0; n < MINE / 4; ++n) {
            const int r = n * 4 + lr;                             // (K's chunks are turned by r0 + r: kchunk)
            int64_t off;
            if (SPARSE) {
                off = (int64_t)((uint64_t)(uint32_t)max(lds.list[t - begin + r0 + r], 0) * stride);
            } else if (PAGED) {
                // a wave's rows of a tile share pages of 16; behind the list's last entry row 0 has to do
                const int page = (t - begin + r0 + n * 4) >> 4;
                off = (int64_t)((t + r0 + n * 4 < end ? max(lds.list[page], 0) : 0) + ((r0 + n * 4) & (PAGE - 1)) + lr) * D;
            } else {
                off = (int64_t)(t + TT <= end ? (uint64_t)(uint32_t)(t + n * 4) * stride + lane_off : (uint64_t)(uint32_t)min(t + r0 + r, end - 1) * stride);
            }
            load_to_lds((values ? vbase : kbase) + off + (values ? chunk : chunk ^ ((n * 4 & 15) << 3)), to + n * 1024);
        }
    };
    // Which tokens of tile `it` are there, and which of them this wave's rows attend to (`common`: all of them).
    auto attended = [&](int it, uint32_t& there, uint32_t& common) -> uint32_t {
        const int t = begin + (it * TEAMS + team) * TT;
        there = t + 32 <= end ? 0xffffffffu : t >= end ? 0u : (1u << (end - t)) - 1;
        if constexpr (BEAM) {
            const int in_front = s.pre - t;                       // tokens of pages that all rows attend to as a whole
            common = in_front >= 32 ? 0xffffffffu : in_front >= 16 ? 0xffffu : 0u;
            common &= there;
            uint32_t own = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int e = min((t - begin) / PAGE + j, BEAM_LIST - 1);
                const int n = clampi(row_len - lds.first[e], 0, PAGE);
                if (lds.holders[e] >> (node & 31) & 1) own |= ((1u << n) - 1) << (16 * j);
            }
            return (common | own) & there;
        }
        if (LIST && t + 32 > good) there = (uint32_t)__ballot(t + col < end && lds.list[SPARSE ? t - begin + col : (t - begin + col) >> 4] >= 0);
        const int from = s.pre - t;                               // tokens of the prefix in this step
        const uint32_t prefix = from >= 32 ? 0xffffffffu : from <= 0 ? 0u : (1u << from) - 1;
        common = prefix & there;
        return (prefix | mask_window(a.masks + (int64_t)(s.start + node) * a.words, a.words, t - s.pre)) & there;
    };
    auto note_odd = [&](int it, uint32_t odd) {                   // nodes with values that were left out
        const int t = begin + (it * TEAMS + team) * TT;
        for (; odd; odd &= odd - 1) {
            const int i = BEAM ? (t - begin + __builtin_ctz(odd)) / PAGE : t + __builtin_ctz(odd) - s.pre;
            atomicOr(&lds.odd[i >> 5], 1u << (i & 31));
            if (BEAM) lds.first_bad = 0;
        }
    };
    const int plain = max(0, min(s.pre, good) - begin) / (TT * TEAMS);   // tiles that every row attends to as a whole: the first ones
    if constexpr (RG < 4) {
        // Few rows: the products are short, and what counts is that tiles keep coming.  A tile is a step.  A wave on its own asks for the next when it
        // has read one, while seven others are elsewhere; a team of two has a second buffer for it.
        auto request_tile = [&](int n) {
            if (n < steps) {
                request(n, false);
                request(n, true);
            }
        };
        auto arrive = [&](int it) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (RG > 1) {
                wave_barrier();
                request_tile(it + 1);
            }
        };
        auto leave = [&](int it) {
            if (RG == 1) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the buffers' last reads
                request_tile(it + 1);
            }
        };
        request_tile(0);
        int it = 0;
        // (Two loops: in one, the two forms' registers get in each other's way.)
#pragma unroll 1
        for (; it < plain; ++it) {
            arrive(it);
            if (!idle) {
                TreeKeys kf;
                TreeValues vf;
                TreeFineWeights p;
                read_keys(kf, ring + k_at(it), lane);
                f32x16 x = score(row, kf);
                read_values(vf, ring + v_at(it), lane);
                const float sum = weigh(row.m, x, a.scale_log2e, p);
                raise_and_weigh(row, x, a.scale_log2e, p, sum);
                add_values(row, vf, p);
            }
            leave(it);
        }
#pragma unroll 1
        for (; it < steps; ++it) {
            arrive(it);
            uint32_t there, common;
            const uint32_t allowed = attended(it, there, common);
            if (!idle && there != 0 && (!BEAM || __any(allowed != 0))) {   // (of a page that none of a wave's rows hold it only loads its share)
                TreeKeys kf;
                TreeFineWeights p;
                read_keys(kf, ring + k_at(it), lane);
                f32x16 x = score(row, kf);
                mask_scores(x, allowed, half);
                const float sum = weigh(row.m, x, a.scale_log2e, p);
                raise_and_weigh(row, x, a.scale_log2e, p, sum);
                if constexpr (BEAM) note_odd(it, add_looked_over(row, p, ring + v_at(it), ~common, lane) & there);
                else note_odd(it, add_washed(row, p, ring + v_at(it), ~common, lane) & there);
            }
            leave(it);
        }
    } else {
        // Step `it` takes tile it's weights, the next tile's scores and the last tile's share of the output: it needs K of tile it + 1 and V of tile
        // it - 1.  After the first two K, V of tile n and K of tile n + 2 are asked for together, as pair n, for step n + 1; a block of half
        // the buffers at a time: while the team works on one, the next is under way.  The waves meet once a block only: in between, one of a SIMD's two
        // is ahead, at its softmax while the other has the products.  (Meeting at every step, both wait for the same pipe: 2030 cycles a step of 256 rows,
        // of which the products are 1024.)
        constexpr int BLOCK = STAGES / 2;
        auto request_pair = [&](int n) {
            if (n < steps) request(n, true);
            if (n + 2 < steps) request(n + 2, false);
        };
        const int full = (good - begin) / (TT * TEAMS);           // whole tiles
        uint32_t part_k[MINE / 4], part_v[MINE / 4];              // the lane's part of a row's address
#pragma unroll
        for (int i = 0; i < MINE / 4; ++i) {
            const uint32_t at = SPARSE ? 0 : ((PAGED ? (mine * MINE) & (PAGE - 1) : 0) + i * 4 + lr) * stride;
            part_k[i] = (at + (kchunk ^ ((i * 4 & 15) << 3))) * 2;
            part_v[i] = (at + vchunk) * 2;
        }
        // Pairs n .. n + BLOCK - 1.  Whole tiles of a whole prefix: the rows of a wave's part are one after the other, in a page or in the sequence, and a
        // uniform address serves.  Of a chosen prefix each lane has its own; the list's entries come all at once.
        constexpr int GROUPS = MINE / 4;
        auto request_block = [&](int n) {
            if (n + BLOCK + 2 > full) {
#pragma unroll
                for (int j = 0; j < BLOCK; ++j) request_pair(n + j);
                return;
            }
            const int t = (n * TEAMS + team) * TT + mine * MINE;  // the wave's first row of tile n
            int entry[BLOCK + 2][SPARSE ? GROUPS : 1];
            if (LIST) {
#pragma unroll
                for (int j = 0; j < BLOCK + 2; ++j)
#pragma unroll
                    for (int i = 0; i < (SPARSE ? GROUPS : 1); ++i)
                        entry[j][i] = lds.list[SPARSE ? t + j * (TEAMS * TT) + i * 4 + lr : (t + j * (TEAMS * TT)) >> 4];
            }
            auto row_at = [&](int j) {                            // the first of the wave's rows of tile n + j, in elements
                if (PAGED) return (int64_t)__builtin_amdgcn_readfirstlane(entry[j][0]) * D;
                return (int64_t)((uint64_t)(uint32_t)(begin + t + j * (TEAMS * TT)) * stride);
            };
#pragma unroll
            for (int j = 0; j < BLOCK; ++j) {
                const uint32_t kt = ring + k_at(n + j + 2) + mine * MINE * 256, vt = ring + v_at(n + j) + mine * MINE * 256;
                if constexpr (SPARSE) {
#pragma unroll
                    for (int i = 0; i < GROUPS; ++i) {
                        load_to_lds(vbase + (uint64_t)(uint32_t)entry[j][i] * stride + part_v[i] / 2, vt + i * 1024);
                        load_to_lds(kbase + (uint64_t)(uint32_t)entry[j + 2][i] * stride + part_k[i] / 2, kt + i * 1024);
                    }
                } else {
                    const uint16_t *v = vbase + row_at(j), *k = kbase + row_at(j + 2);
#pragma unroll
                    for (int i = 0; i < GROUPS; ++i) {
                        load_to_lds(v, part_v[i], vt + i * 1024);
                        load_to_lds(k, part_k[i], kt + i * 1024);
                    }
                }
            }
        };
        // Before the first step of a block (it - 1 a multiple of BLOCK): its pairs have arrived, for the whole team, and what the last block read is free.
        auto begin_block = [&](int it) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            wave_barrier();
            request_block(it - 1 + BLOCK);
        };
        request(0, false);
        if (steps > 1) request(1, false);
#pragma unroll
        for (int n = 0; n < BLOCK; ++n) request_pair(n);
        wait_tiles<OPS, BLOCK>(steps - 2);                        // (pairs without K do not count as under way)
        wave_barrier();
        f32x16 x;
        TreeWeights p;
        uint32_t there = 0xffffffffu, common = 0xffffffffu;       // of the tile that p belongs to
        bool live = true;                                         // some row of the wave attends to it (of a group's pages, mostly few do)
        int it = 0;
        if (!idle) {
            TreeKeys kf;
            read_keys(kf, ring + k_at(0), lane);
            x = score(row, kf);
        }
        // One step, by dynamic addresses: the first, those of a broken block, and where rows attend to parts of a tile.
        auto any_step = [&]() {
            if (it > 0) {
                if (common == 0xffffffffu) {
                    TreeValues vf;
                    read_values(vf, ring + v_at(it - 1), lane);
                    add_values(row, vf, p);
                } else if constexpr (BEAM) {
                    if (live) note_odd(it - 1, add_looked_over(row, p, ring + v_at(it - 1), ~common, lane) & there);
                } else if (there != 0) {
                    note_odd(it - 1, add_washed(row, p, ring + v_at(it - 1), ~common, lane) & there);
                }
            }
            if (it >= steps) return;
            there = common = 0xffffffffu;
            if constexpr (BEAM) {
                live = true;
                if (it >= plain) {
                    const uint32_t allowed = attended(it, there, common);
                    live = __any(allowed != 0);
                    if (live) mask_scores(x, allowed, half);
                }
                if (live) {
                    const float sum = weigh(row.m, x, a.scale_log2e, p);
                    raise_and_weigh(row, x, a.scale_log2e, p, sum);
                }
            } else {
                if (it >= plain) mask_scores(x, attended(it, there, common), half);
                const float sum = weigh(row.m, x, a.scale_log2e, p);
                raise_and_weigh(row, x, a.scale_log2e, p, sum);
            }
            if (it + 1 < steps) {
                TreeKeys kf;
                read_keys(kf, ring + k_at(it + 1), lane);
                x = score(row, kf);
            }
        };
        if (!idle) any_step();
        it = 1;
        {
            // Blocks, unrolled: the buffers' places are constants of the instructions then, and two steps' registers change places.
            static_assert(BLOCK == 2 || BLOCK == 4, "the loop's steps");
            uint32_t key[8], value[4];
#pragma unroll
            for (int k = 0; k < 8; ++k) key[k] = ring + k_at(0) + key_at(lane, k);
#pragma unroll
            for (int d = 0; d < 4; ++d) value[d] = ring + v_at(0) + value_at(lane, d);
            constexpr int NEXT = TEAMS * TILE_BYTES;              // bytes from one buffer of a team to the next
            f32x16 y;
            TreeWeights p2;
            // The buffers' two halves take turns: K goes over to the other in the middle of a block (it is two tiles ahead), V between blocks.
            int k_other = BLOCK * NEXT, v_other = BLOCK * NEXT;
            auto step = [&](auto place) {                         // it = 1 + place, mod BLOCK
                constexpr int J = decltype(place)::value;
                if (J == 0) begin_block(it);
                if (J + 2 == BLOCK) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) key[k] += k_other;
                    k_other = -k_other;
                }
                constexpr int K = (J + 2) % BLOCK * NEXT, V = J * NEXT;
                if (!idle) {
                    if (J & 1) tree_step<K, V>(row, y, x, p, p2, key, value, a.scale_log2e);
                    else tree_step<K, V>(row, x, y, p2, p, key, value, a.scale_log2e);
                }
                if (J + 1 == BLOCK) {
#pragma unroll
                    for (int d = 0; d < 4; ++d) value[d] += v_other;
                    v_other = -v_other;
                }
                ++it;
            };
            const int until = min(plain, steps - 1);              // (a step makes the next tile's scores)
            auto swap = [&]() {                                   // after an odd number of steps
                x = y;
                p = p2;
            };
#pragma unroll 1
            while (it < until) {
                step(std::integral_constant<int, 0>());
                if (it >= until) {
                    swap();
                    break;
                }
                step(std::integral_constant<int, 1>());
                if constexpr (BLOCK == 4) {
                    if (it >= until) break;
                    step(std::integral_constant<int, 2>());
                    if (it >= until) {
                        swap();
                        break;
                    }
                    step(std::integral_constant<int, 3>());
                }
            }
        }
#pragma unroll 1
        for (; it <= steps; ++it) {                               // (the last: only the last tile's share)
            if ((it - 1) % BLOCK == 0) begin_block(it);
            if (!idle) any_step();
        }
    }

    // The teams' sums, brought to a common maximum, meet in LDS and leave it row by row.
    row.l += __shfl_xor(row.l, 32);
    if (half == 0) {
        const int r = team * ROWS + mine * 32 + col;
        lds.m[r] = row.m;
        lds.l[r] = row.l;
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
    if constexpr (BEAM) {
        any_odd = lds.first_bad == 0;
    } else {
#pragma unroll
        for (int i = 0; i < TREE_MAX_NODES / 32; ++i) any_odd |= lds.odd[i] != 0;
    }
    // (four items of a thread at a time: their reads are under way together)
    constexpr int ITEMS = ROWS * 32 / TREE_THREADS, RUN = ITEMS < 4 ? ITEMS : 4;
    static_assert(ITEMS % RUN == 0, "whole runs");
    const int c = tid & 31;
#pragma unroll 1
    for (int i0 = 0; i0 < ITEMS; i0 += RUN) {
        if (row0 + i0 * (TREE_THREADS / 32) >= rows) break;
        float top[RUN], sum[RUN];
        f32x4 v[RUN];
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            const int r = (i0 + i) * (TREE_THREADS / 32) + (tid >> 5);
            top[i] = lds.m[r];
            sum[i] = lds.l[r];
            v[i] = *reinterpret_cast<const f32x4*>(lds.ring + r * (D * 4) + ((c ^ (r & 31)) << 4));
            if constexpr (TEAMS > 1) {
                const float own = top[i];
#pragma unroll
                for (int w = 1; w < TEAMS; ++w) top[i] = fmaxf(top[i], lds.m[w * ROWS + r]);
                sum[i] *= exp2f(own - top[i]);
#pragma unroll
                for (int w = 1; w < TEAMS; ++w) {
                    sum[i] += lds.l[w * ROWS + r] * exp2f(lds.m[w * ROWS + r] - top[i]);
                    v[i] += *reinterpret_cast<const f32x4*>(lds.ring + (w * ROWS + r) * (D * 4) + ((c ^ (r & 31)) << 4));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            const int row = row0 + (i0 + i) * (TREE_THREADS / 32) + (tid >> 5);
            if (row >= rows) break;
            if constexpr (BEAM) {
                const int of = s.start + (row >> a.g_shift), len = a.cache.kv.seq_lens[of];
                if (any_odd) {                                    // (as below, for the tokens of pages)
                    for (int e = 0; e < (end - begin) / PAGE; ++e) {
                        if (!(lds.odd[e >> 5] >> (e & 31) & 1) || !(lds.holders[e] >> (of - s.start) & 1)) continue;
                        for (int j = 0; j < min(min(len, a.cache.max_len) - lds.first[e], PAGE); ++j) {
                            const u32x2 w = *reinterpret_cast<const u32x2*>(a.cache.kv.v + (int64_t)(lds.list[e] + j) * D + c * 4);
#pragma unroll
                            for (int n = 0; n < 4; ++n) {
                                const uint32_t x = (n & 1) ? w[n >> 1] & 0xffff0000u : w[n >> 1] << 16;
                                if ((x & 0x7f800000u) == 0x7f800000u) v[i][n] += __uint_as_float(x);
                            }
                        }
                    }
                }
                if (len <= 0) {                                   // a row without tokens
                    top[i] = LOWEST;
                    sum[i] = 0.0f;
                    v[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                }
            } else if (any_odd) {
                // Nodes with values that are not finite: the rows that attend to them get those values (whatever the weight: it is not 0).
                const uint64_t* mask = a.masks + (int64_t)(s.start + (row >> a.g_shift)) * a.words;
                for (int n = 0; n < s.n; ++n) {
                    if (!(lds.odd[n >> 5] >> (n & 31) & 1) || !(mask[n >> 6] >> (n & 63) & 1)) continue;
                    const int at = cache_row<PAGED>(a.cache, b, kvh, s.before + n);
                    const u32x2 w = *reinterpret_cast<const u32x2*>(a.cache.kv.v + cache_offset<PAGED>(a.cache, b, kvh, max(at, 0)) + c * 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t x = (j & 1) ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16;
                        if ((x & 0x7f800000u) == 0x7f800000u) v[i][j] += __uint_as_float(x);
                    }
                }
            }
            const int head = (kvh << a.g_shift) + (row & (g - 1));
            if (whole) {
                const int64_t to = (int64_t)(s.start + (row >> a.g_shift)) * a.H + head;
                const float inv = sum[i] == 0.0f ? 0.0f : 1.0f / sum[i];
                const u32x2 w = {(uint32_t)f32_to_bf16_rne(v[i][0] * inv) | (uint32_t)f32_to_bf16_rne(v[i][1] * inv) << 16,
                                 (uint32_t)f32_to_bf16_rne(v[i][2] * inv) | (uint32_t)f32_to_bf16_rne(v[i][3] * inv) << 16};
                *reinterpret_cast<u32x2*>(a.out + to * D + c * 4) = w;
            } else {
                const int64_t piece = ((int64_t)(s.part + (row >> a.g_shift)) * a.H + head) * a.n_splits + split;
                *reinterpret_cast<f32x4*>(a.part_acc + piece * D + c * 4) = v[i];
                if (c == 0) *reinterpret_cast<f32x2*>(a.part_ml + piece * 2) = f32x2{top[i], sum[i]};
            }
        }
    }
}

// Which form a workgroup takes goes by the rows that its own tree has, not by the bound: trees of a batch differ.
template <bool PAGED, bool SPARSE, bool BEAM = false>
__global__ __launch_bounds__(TREE_THREADS, 2) void tree_attn_kernel(TreeArgs a) {
    __shared__ TreeLds<BEAM> lds;
    // Workgroups go to the 8 XCDs in turn: those that share a KV head's tokens come 8 apart, to the same L2.  First pieces first: behind them come
    // those that short sequences do not have.
    const uint32_t turn = blockIdx.x >> 3, m_tile = turn % (uint32_t)a.m_tiles, unit = turn / (uint32_t)a.m_tiles * 8 + (blockIdx.x & 7);
    if constexpr (BEAM) {
        TreeSpan s;
        int b, kvh, split;
        if (!group_work(a, (int)unit, s, b, kvh, split)) return;
        const int row0 = m_tile * a.tile_rows, left = min((s.n << a.g_shift) - row0, a.tile_rows), begin = split * s.chunk, end = min(begin + s.chunk, s.all);
        if (left <= 0) return;
        if (s.all == 0) {                                         // a group without tokens
            for (int i = threadIdx.x; i < (left << 5); i += TREE_THREADS) {
                const int row = row0 + (i >> 5);
                const int64_t to = (int64_t)(s.start + (row >> a.g_shift)) * a.H + (kvh << a.g_shift) + (row & ((1 << a.g_shift) - 1));
                *reinterpret_cast<u32x2*>(a.out + to * D + (i & 31) * 4) = u32x2{0, 0};
            }
        }
        if (a.n_splits > 1 && split == 0 && kvh == 0 && m_tile == 0 && threadIdx.x == 0) a.pieces[b] = s.all ? (s.all + s.chunk - 1) / s.chunk : 0;
        if (begin >= end) return;
        if (left <= 32) tree_rows<1, PAGED, SPARSE, BEAM>(a, s, lds, b, kvh, row0, split, begin, end);
        else if (left <= 64) tree_rows<2, PAGED, SPARSE, BEAM>(a, s, lds, b, kvh, row0, split, begin, end);
        else if (left <= 128) tree_rows<4, PAGED, SPARSE, BEAM>(a, s, lds, b, kvh, row0, split, begin, end);
        else tree_rows<8, PAGED, SPARSE, BEAM>(a, s, lds, b, kvh, row0, split, begin, end);
    } else {
        const uint32_t G = a.cache.kv.G, pairs = G * (uint32_t)a.batch, pair = unit % pairs;
        const int split = unit / pairs, b = pair / G, kvh = pair - b * G, row0 = m_tile * a.tile_rows;
        if (split >= a.n_splits) return;
        const TreeSpan s = tree_work<SPARSE>(a, b);
        const int left = min((s.n << a.g_shift) - row0, a.tile_rows), begin = split * s.chunk;
        if (left <= 0 || begin >= s.all) return;
        // (a piece has no more tokens or pages than the list has room for: plan_tree)
        const int end = min(begin + s.chunk, s.all);
        if (a.n_splits > 1 && split == 0 && kvh == 0 && m_tile == 0 && threadIdx.x == 0) a.pieces[b] = (s.all + s.chunk - 1) / s.chunk;
        if (left <= 32) tree_rows<1, PAGED, SPARSE, BEAM>(a, s, lds, b, kvh, row0, split, begin, end);
        else if (left <= 64) tree_rows<2, PAGED, SPARSE, BEAM>(a, s, lds, b, kvh, row0, split, begin, end);
        else if (left <= 128) tree_rows<4, PAGED, SPARSE, BEAM>(a, s, lds, b, kvh, row0, split, begin, end);
        else tree_rows<8, PAGED, SPARSE, BEAM>(a, s, lds, b, kvh, row0, split, begin, end);
    }
}

// A wave for a row: a lane for each piece's weight, then two columns a lane.  Bound by the partial sums' way back from memory: 31 MB of one sequence (1920 rows in 32
// pieces) take 6.0 us, 5.2 TB/s.
constexpr int REDUCE_WAVES = 4;
template <bool BEAM = false>
__global__ __launch_bounds__(64 * REDUCE_WAVES) void tree_reduce_kernel(TreeArgs a) {
    const int lane = threadIdx.x & 63, b = blockIdx.y;
    int start, n;
    if constexpr (BEAM) {
        start = b * a.max_nodes;
        n = a.max_nodes;
    } else {
        n = min(tree_span(a.tok_start, b, a.max_tokens, a.max_nodes, start), clampi(a.cache.kv.seq_lens[b], 0, a.cache.max_len));
    }
    if (n == 0) return;                                           // (without a node, nobody has written how many pieces there are)
    const int pieces = a.pieces[b];
    if (pieces <= 1) return;
    for (int r = blockIdx.x * REDUCE_WAVES + (threadIdx.x >> 6); r < n * a.H; r += gridDim.x * REDUCE_WAVES) {
        const int64_t row = (int64_t)start * a.H + r, first = ((int64_t)part_row(a, b, start) * a.H + r) * a.n_splits;
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
        // (a sum that is infinite stays so whatever its piece weighs: the weight is not 0, also where 32 bits hold nothing of it)
        auto add = [&](float wp, f32x2 v) {
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[j] += __builtin_isfinite(v[j]) ? wp * v[j] : v[j];
        };
        const float* part = a.part_acc + first * D + lane * 2;
        int p = 0;
        for (; p + 8 <= pieces; p += 8) {                         // eight at a time under way
            f32x2 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const f32x2*>(part + (p + i) * D);
#pragma unroll
            for (int i = 0; i < 8; ++i) add(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), p + i)), v[i]);
        }
        for (; p < pieces; ++p) {
            const f32x2 v = *reinterpret_cast<const f32x2*>(part + p * D);
            add(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), p)), v);
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        *reinterpret_cast<uint32_t*>(a.out + row * D + lane * 2) = (uint32_t)f32_to_bf16_rne(acc[0] * inv) | (uint32_t)f32_to_bf16_rne(acc[1] * inv) << 16;
    }
}

}  // namespace cusa
