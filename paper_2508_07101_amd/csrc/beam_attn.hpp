// Attention over a group's pages: each is read once for all rows of the group that hold it.
#pragma once
#include "attn_parts.hpp"
#include "beam_plan.hpp"
#include "plan_scan.hpp"

namespace cusa {

constexpr int BEAM_ATTN_WAVES = 4, BEAM_ATTN_THREADS = 64 * BEAM_ATTN_WAVES;
constexpr int BEAM_TILE = 32;              // tokens of a tile, two pages: pieces are whole tiles
constexpr int BEAM_TILE_BYTES = BEAM_TILE * 256;

struct BeamAttnArgs {
    CacheArgs cache;
    const uint16_t* q;
    int64_t q_stride;
    const int32_t *entries, *count;
    int64_t entry_stride;                  // entries of a group's list, and of these the ones that are looked at
    int32_t max_entries;
    uint16_t* out;
    float *part_acc, *part_ml;
    int32_t* pieces;                       // of each group's pages, for the merge
    float scale_log2e;
    int32_t groups, width, H, g_shift, blocks, n_splits;
};

struct BeamSpan {
    int b, kvh, split;                     // the group, the KV head, the piece
    int pre, all;                          // tokens of pages that every row attends to as a whole (the first ones), of all pages
    int chunk;                             // tokens of a piece
};
__device__ __forceinline__ int tiles_of_group(const BeamAttnArgs& a, int b) { return (clampi(a.count[b * 2], 0, a.max_entries) + 1) / 2; }

// The pieces are of one length, which goes by the lists that there are.  With the tiles T of all workgroups' rows and KV heads, W of these in number and at most M tiles in one, pieces of
// ceil(M / floor(R / W)) tiles are R at most, and so are pieces of T / (R - W) tiles (a last piece each is shorter): the first is exact for lists of one length, the second close for any.
// R: one to eight workgroups for each CU; more are better balanced, but each costs about BEAM_PIECE_COST tiles besides its own (its start, and partial sums written and read).  0: more groups than
// pieces would balance, which stay whole.
__device__ __forceinline__ int group_piece(const BeamAttnArgs& a) {
    const int lane = threadIdx.x & 63;
    int total = 0, most = 0;
    for (int i = lane; i < a.groups; i += 64) {
        const int t = tiles_of_group(a, i);
        total += t;
        most = max(most, t);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        total += __shfl_xor(total, o);
        most = max(most, __shfl_xor(most, o));
    }
    const int of_group = a.cache.kv.G * a.blocks, pairs = of_group * a.groups, r = (lane & 7) + 1, wgs = r * BEAM_CUS;   // a lane for each R (the others repeat them)
    int cost = 0x7fffffff, piece = 0;
    if (wgs >= pairs) {
        piece = (most + wgs / pairs - 1) / (wgs / pairs);
        if (wgs > pairs) piece = min(piece, (int)(((int64_t)total * of_group + wgs - pairs - 1) / (wgs - pairs)));
        piece = max(piece, BEAM_MIN_PIECE / BEAM_TILE);
        cost = r * (piece + BEAM_PIECE_COST);
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
    return piece > 0 ? piece : __builtin_amdgcn_readfirstlane(most);
}
// Unit u of a launch is a KV head and the u / G -th of all groups' pieces, one group after the other, so that all that have work come first.  (In order of the pieces' numbers, with
// those that short groups do not have in between, workgroups waited for places while CUs of other shader engines had some: 8 samples of 8 prompts of 1024 to 2048 tokens, 488 pieces: 24 of the 256 CUs
// had three, 48 one, and the last began after 146 of 242 us; so 195.)  False: there is no such piece.  A group without tokens has one.
__device__ __forceinline__ bool group_work(const BeamAttnArgs& a, int u, BeamSpan& s) {
    const int G = a.cache.kv.G, v = u / G, lane = threadIdx.x & 63;
    s.kvh = u - v * G;
    s.b = a.n_splits == 1 ? v : a.groups;
    s.split = 0;
    int tiles = 0;                                         // of a piece
    if (a.n_splits > 1) {
        const int piece = min(group_piece(a), BEAM_LIST / 2);   // (LDS has bits for BEAM_LIST pages)
        for (int i0 = 0, before = 0; i0 < a.groups; i0 += 64) {
            const int i = i0 + lane, t = i < a.groups ? tiles_of_group(a, i) : 0;
            const int chunk = max(piece, (t + a.n_splits - 1) / a.n_splits), n = i < a.groups ? max((t + chunk - 1) / chunk, 1) : 0;   // (what the launch has pieces for)
            int sum = n;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int y = __shfl_up(sum, o);
                if (lane >= o) sum += y;
            }
            const uint64_t behind = __ballot(before + sum > v);
            if (behind) {
                const int at = __builtin_ctzll(behind);
                s.b = i0 + at;
                s.split = v - before - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(n, at));
                tiles = __builtin_amdgcn_readlane(chunk, at);
                break;
            }
            before += __builtin_amdgcn_readlane(sum, 63);
        }
    }
    if (s.b >= a.groups) return false;
    const int n = clampi(a.count[s.b * 2], 0, a.max_entries);
    s.all = n * PAGE;
    s.pre = clampi(a.count[s.b * 2 + 1], 0, n) * PAGE;
    s.chunk = a.n_splits > 1 ? tiles * BEAM_TILE : (n + 1) / 2 * BEAM_TILE;
    return true;
}

template <int NB>                          // blocks of 16 rows
struct BeamAttnLds {
    __attribute__((aligned(16))) unsigned char v[BEAM_ATTN_WAVES * 2 * BEAM_TILE_BYTES];   // V of a wave's tile, and of the next one; the waves' sums at the end
    float m[BEAM_ATTN_WAVES * 16 * NB], l[BEAM_ATTN_WAVES * 16 * NB];
    uint32_t odd[BEAM_LIST / 32];          // pages with a value that is not finite and that not all rows attend to
    int32_t any_odd;
};
static_assert(BEAM_LIST / 32 == BEAM_ATTN_THREADS, "a thread clears a word");
static_assert(BEAM_ATTN_THREADS == 256, "beam_units_served counts a launch's threads");

// A tile: two pages of the list, uniform.
struct BeamTile {
    int64_t at[2];                         // elements in front of the KV head's rows
    int32_t first[2];                      // position of the page's first token
    uint32_t holders[2];
};
__device__ __forceinline__ BeamTile beam_tile(const BeamAttnArgs& a, const int32_t* list, int e, int n, int kvh) {
    typedef const __attribute__((address_space(4))) i32x4* uniform_entry;   // (no kernel of the launch writes the list)
    BeamTile t;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const i32x4 x = *(uniform_entry)(uintptr_t)(list + (int64_t)min(e + j, n - 1) * 4);
        const bool is = (uint32_t)x[0] < (uint32_t)a.cache.n_pages && x[1] >= 0 && e + j < n;   // (the second page of a list's last tile may be missing)
        t.at[j] = ((int64_t)(is ? x[0] : 0) * a.cache.kv.G + kvh) * PAGE * D;
        t.first[j] = clampi(x[1], 0, 0x7fffffff / PAGE) * PAGE;
        t.holders[j] = is ? (uint32_t)x[2] : 0;
    }
    return t;
}

__device__ __forceinline__ float of_row_max(float v) {      // over the four lanes of a row
    const auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return other_half_max(fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1])));
}

// Rows are columns of the products, so that a lane has one row's numbers (n = lane % 16, q = lane / 16):
//   S^T = K Q^T by V_MFMA_F32_16X16X32_BF16: lane (n, q) gets the scores of the tokens 4 q .. 4 q + 3 of either page;
//   O^T += V^T P^T: the same lanes hold these tokens' weights, which is the operand's order if V's tokens are taken in it: transposing LDS reads of tokens 4 q .. of either page.
// Weights are two bf16 numbers each, as in tree_rows for few rows.  The reference m follows the maximum when that is 2^8 above it.
// K goes to registers, V to LDS, both for the next tile as soon as this one's scores are there; eight waves on a CU have 128 KB under way.  Waves meet at the end alone.
// Bound by memory: 64 groups of 4 beams, prompts of 8192 to 32768 tokens, 32 query heads on 8: 5.7 GB of pages in 922 us, 6.2 TB/s (a plain read 836 us); 8 groups of 8 samples, 2048 tokens and up to 8192
// of their own: 175 us (162), and up to 220 within the first ten milliseconds after the GPU was idle.  A short search, 4 beams of 4096 tokens: 9 us and 4 for the merge (2.7), a chain of waits: list, pages, sums.
// Rows beyond 32 are other workgroups', which read the pages again, mostly from their XCD's L2: 4 groups of 32 samples 118 us (one workgroup for all rows that share a KV head, the tiles in LDS: 162), 8 groups of
// 32 beams of 2048 to 4096 tokens 67 (61), of 64 query heads 111 (105); the blocks one after the other in a workgroup 139, 252 and 222.
// K past the caches 1003 us for the 965 of then; one buffer for V and three workgroups on a CU: as long; eight waves on one workgroup's pages 908 for 926, but 180 for 175 and 28 for 24 on 64 groups of 500 tokens.
template <int NB>
__device__ __forceinline__ void beam_rows(const BeamAttnArgs& a, const BeamSpan& s, BeamAttnLds<NB>& lds, int row0) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, q4 = lane >> 4;
    const int g = 1 << a.g_shift, rows = min((a.width << a.g_shift) - row0, 16 * NB), beam0 = s.b * a.width, begin = s.split * s.chunk;
    u32x4 qv[NB][4];
    int len[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int row = row0 + min(i * 16 + n, rows - 1), beam = beam0 + (row >> a.g_shift);
        const uint16_t* const p = a.q + (int64_t)beam * a.q_stride + ((s.kvh << a.g_shift) + (row & (g - 1))) * D + q4 * 8;
#pragma unroll
        for (int k = 0; k < 4; ++k) qv[i][k] = *reinterpret_cast<const u32x4*>(p + k * 32);
        len[i] = a.cache.kv.seq_lens[beam];
    }
    lds.odd[tid] = 0;
    if (tid == 0) lds.any_odd = 0;
    __syncthreads();                                       // (odd is clear before anyone marks a page)
    const int entries = (min(begin + s.chunk, s.all) - begin) / PAGE, tiles = (entries + 1) >> 1;
    const int plain = clampi(s.pre - begin, 0, entries * PAGE) / BEAM_TILE;   // tiles that every row attends to as a whole: the first ones
    const int32_t* const list = a.entries + (s.b * a.entry_stride + begin / PAGE) * 4;

    bf16x8 qf[NB][4];
    f32x4 o[NB][8];
    float m[NB], l[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const bool there = i * 16 + n < rows;
#pragma unroll
        for (int k = 0; k < 4; ++k) qf[i][k] = __builtin_bit_cast(bf16x8, there ? qv[i][k] : u32x4{0, 0, 0, 0});
#pragma unroll
        for (int d = 0; d < 8; ++d) o[i][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        m[i] = LOWEST;
        l[i] = 0.0f;
        len[i] = there ? clampi(len[i], 0, a.cache.max_len) : 0;
    }
    const uint32_t vlds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds.v + wave * (2 * BEAM_TILE_BYTES);
    // A lane's part of K's operand; of V's rows as LDS holds them: 16-byte chunk c of token t stands at c ^ 4 (t % 4), so that the transposing reads of 16 lanes meet in no bank.
    const int k_part = n * D + q4 * 8, v_part = q4 * D + ((n ^ (q4 << 2)) << 3);
    const uint32_t v_read = (4 * q4 + ((lane >> 2) & 3)) * 256 + (((lane & 3) >> 1) << 4) + (lane & 1) * 8;
    u32x4 k[2][4];
    auto request = [&](const BeamTile& t, int buffer) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint16_t* const kp = a.cache.kv.k + t.at[j];
#pragma unroll
            for (int i = 0; i < 4; ++i) k[j][i] = *reinterpret_cast<const u32x4*>(kp + k_part + i * 32);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) load_to_lds(a.cache.kv.v + t.at[j], (uint32_t)(v_part + i * 4 * D) * 2, vlds + buffer * BEAM_TILE_BYTES + j * (PAGE * 256) + i * 1024);
    };
    // The first tile from t on that one of this workgroup's rows attends to.
    const uint32_t here = (uint32_t)((1ull << (((row0 + rows - 1) >> a.g_shift) + 1)) - (1ull << (row0 >> a.g_shift)));
    auto find = [&](int t, BeamTile& tile) {
        for (; t < tiles; t += BEAM_ATTN_WAVES) {
            tile = beam_tile(a, list, t * 2, entries, s.kvh);
            if ((tile.holders[0] | tile.holders[1]) & here) break;
        }
        return t;
    };
    BeamTile now, next;
    int t = find(wave, now), buffer = 0;
    if (t < tiles) request(now, 0);
#pragma unroll 1
    for (int t_next; t < tiles; t = t_next, buffer ^= 1) {
        t_next = find(t + BEAM_ATTN_WAVES, next);
        const bool more = t_next < tiles;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // K in registers, V in LDS
        f32x4 x[NB][2];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                x[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < 4; ++c) x[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[j][c]), qf[i][c], x[i][j], 0, 0, 0);
            }
        if (more) request(next, buffer ^ 1);
        const bool whole = t < plain;
        bf16x8 fine[NB], rest[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            if (!whole) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t held = now.holders[j] >> (((row0 + i * 16 + n) >> a.g_shift) & 31) & 1;
                    const int left = held ? len[i] - now.first[j] : 0;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (4 * q4 + c >= left) x[i][j][c] = -INFINITY;
                }
            }
            float top = fmaxf(fmaxf(fmaxf(x[i][0][0], x[i][0][1]), fmaxf(x[i][0][2], x[i][0][3])), fmaxf(fmaxf(x[i][1][0], x[i][1][1]), fmaxf(x[i][1][2], x[i][1][3])));
            top = of_row_max(top) * a.scale_log2e;
            if (__any(top > m[i] + 8.0f)) {
                const float to = top > m[i] + 8.0f ? top : m[i], f = exp2f(m[i] - to);
                m[i] = to;
                l[i] *= f;
#pragma unroll
                for (int d = 0; d < 8; ++d) o[i][d] *= f;
            }
            typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int c = 0; c < 8; c += 2) {               // (f: cut to bf16, less one step; the rest a step to two, rounded: neither is negative or, from 2^-132 on, 0, so that an infinite value stays so in both products)
                const float w0 = weight(m[i], x[i][c >> 2][c & 3], a.scale_log2e), w1 = weight(m[i], x[i][c >> 2][(c & 3) + 1], a.scale_log2e);
                const uint32_t cut = __builtin_amdgcn_perm(__float_as_uint(w1), __float_as_uint(w0), 0x07060302);
                const uint32_t less = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, cut), u16x2{1, 1}));
                const bf16x2 f = __builtin_bit_cast(bf16x2, less);
                fine[i][c] = f[0];
                fine[i][c + 1] = f[1];
                rest[i][c] = (__bf16)(w0 - __uint_as_float(less << 16));
                rest[i][c + 1] = (__bf16)(w1 - __uint_as_float(less & 0xffff0000u));
                l[i] += w0;
                l[i] += w1;
            }
        }
        u32x4 v[8];
        const uint32_t from = vlds + buffer * BEAM_TILE_BYTES + v_read, turn = ((lane >> 2) & 3) << 6;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const uint32_t at = from + ((((d >> 1) << 6) ^ turn) | (d & 1) << 5);
            const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)at);
            const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(at + PAGE * 256));
            v[d] = __builtin_bit_cast(u32x4, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        if (!whole) {                                      // a weight of 0 must not meet a value that is not finite
            typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
            u16x2 most[2] = {{0, 0}, {0, 0}};
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int c = 0; c < 4; ++c) most[c >> 1] = __builtin_elementwise_max(most[c >> 1], __builtin_bit_cast(u16x2, v[d][c] & 0x7fff7fffu));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (!__any(most[j][0] >= 0x7f80 || most[j][1] >= 0x7f80)) continue;
#pragma unroll
                for (int d = 0; d < 8; ++d)
#pragma unroll
                    for (int c = 2 * j; c < 2 * j + 2; ++c) {
                        if ((v[d][c] & 0x7f80u) == 0x7f80u) v[d][c] &= 0xffff0000u;
                        if ((v[d][c] & 0x7f800000u) == 0x7f800000u) v[d][c] &= 0xffffu;
                    }
                if (lane == 0) {
                    atomicOr(&lds.odd[(2 * t + j) >> 5], 1u << ((2 * t + j) & 31));
                    lds.any_odd = 1;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int d = 0; d < 8; ++d) {
                o[i][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[d]), rest[i], o[i][d], 0, 0, 0);
                o[i][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[d]), fine[i], o[i][d], 0, 0, 0);
            }
        now = next;
    }

    // The waves' sums, brought to a common maximum, meet in LDS and leave it row by row.
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        float sum = l[i];
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (q4 == 0) {
            lds.m[(wave * NB + i) * 16 + n] = m[i];
            lds.l[(wave * NB + i) * 16 + n] = sum;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int r = i * 16 + n;
        float top = lds.m[r];
#pragma unroll
        for (int w = 1; w < BEAM_ATTN_WAVES; ++w) top = fmaxf(top, lds.m[w * 16 * NB + r]);
        const float f = exp2f(m[i] - top);
#pragma unroll
        for (int d = 0; d < 8; ++d)                        // columns 16 d + 4 q ..
            *reinterpret_cast<f32x4*>(lds.v + (wave * 16 * NB + r) * (D * 4) + (((4 * d + q4) ^ n) << 4)) = f32x4{o[i][d][0] * f, o[i][d][1] * f, o[i][d][2] * f, o[i][d][3] * f};
    }
    __syncthreads();
    const bool some_odd = lds.any_odd != 0;
    const int c = tid & 31;
#pragma unroll 1
    for (int r = tid >> 5; r < rows; r += BEAM_ATTN_WAVES * 2) {
        float top = lds.m[r], sum = 0.0f;
#pragma unroll
        for (int w = 1; w < BEAM_ATTN_WAVES; ++w) top = fmaxf(top, lds.m[w * 16 * NB + r]);
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < BEAM_ATTN_WAVES; ++w) {
            sum += lds.l[w * 16 * NB + r] * exp2f(lds.m[w * 16 * NB + r] - top);
            v += *reinterpret_cast<const f32x4*>(lds.v + (w * 16 * NB + r) * (D * 4) + ((c ^ (r & 15)) << 4));
        }
        const int of = (row0 + r) >> a.g_shift, length = clampi(a.cache.kv.seq_lens[beam0 + of], 0, a.cache.max_len);
        if (some_odd) {
            // Pages with values that are not finite: the rows that attend to them get those values (whatever the weight: it is not 0).
            for (int e = 0; e < entries; ++e) {
                if (!(lds.odd[e >> 5] >> (e & 31) & 1)) continue;
                const BeamTile t = beam_tile(a, list, e, entries, s.kvh);
                if (!(t.holders[0] >> of & 1)) continue;
                for (int j = 0; j < min(length - t.first[0], PAGE); ++j) {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(a.cache.kv.v + t.at[0] + j * D + c * 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t y = (i & 1) ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16;
                        if ((y & 0x7f800000u) == 0x7f800000u) v[i] += __uint_as_float(y);
                    }
                }
            }
        }
        if (length == 0) {                                 // a row without tokens
            top = LOWEST;
            sum = 0.0f;
            v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const int64_t to = (int64_t)(beam0 + of) * a.H + (s.kvh << a.g_shift) + ((row0 + r) & (g - 1));
        if (s.chunk >= s.all) {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            const u32x2 w = {(uint32_t)f32_to_bf16_rne(v[0] * inv) | (uint32_t)f32_to_bf16_rne(v[1] * inv) << 16, (uint32_t)f32_to_bf16_rne(v[2] * inv) | (uint32_t)f32_to_bf16_rne(v[3] * inv) << 16};
            *reinterpret_cast<u32x2*>(a.out + to * D + c * 4) = w;
        } else {
            const int64_t piece = to * a.n_splits + s.split;
            *reinterpret_cast<f32x4*>(a.part_acc + piece * D + c * 4) = v;
            if (c == 0) *reinterpret_cast<f32x2*>(a.part_ml + piece * 2) = f32x2{top, sum};
        }
    }
}

template <int NB>
__global__ __launch_bounds__(BEAM_ATTN_THREADS, 2) void beam_attn_kernel(BeamAttnArgs a) {
    __shared__ BeamAttnLds<NB> lds;
    // Blocks of rows that share a KV head's pages: workgroups go to the 8 XCDs in turn, and theirs come 8 apart, to the same L2.
    const uint32_t turn = blockIdx.x >> 3, block = turn % (uint32_t)a.blocks, unit = turn / (uint32_t)a.blocks * 8 + (blockIdx.x & 7);
    BeamSpan s;
    if (!group_work(a, (int)unit, s)) return;
    const int row0 = block * (16 * NB), rows = min((a.width << a.g_shift) - row0, 16 * NB);
    if (a.n_splits > 1 && s.split == 0 && s.kvh == 0 && block == 0 && threadIdx.x == 0) a.pieces[s.b] = s.all ? (s.all + s.chunk - 1) / s.chunk : 0;
    if (s.all > 0) {
        beam_rows<NB>(a, s, lds, row0);
        return;
    }
    for (int i = threadIdx.x; i < rows * (D / 4); i += BEAM_ATTN_THREADS) {   // a group without tokens
        const int row = row0 + (i >> 5);
        *reinterpret_cast<u32x2*>(a.out + ((int64_t)(s.b * a.width + (row >> a.g_shift)) * a.H + (s.kvh << a.g_shift) + (row & ((1 << a.g_shift) - 1))) * D + (i & 31) * 4) = u32x2{0, 0};
    }
}

// A wave for a row: a lane for each piece's weight, then two columns a lane, eight pieces asked for at once, and the last ones by four.
constexpr int BEAM_REDUCE_WAVES = 4;
__global__ __launch_bounds__(64 * BEAM_REDUCE_WAVES) void beam_reduce_kernel(BeamAttnArgs a) {
    const int b = blockIdx.y, pieces = a.pieces[b], lane = threadIdx.x & 63;
    if (pieces <= 1) return;
    for (int r = blockIdx.x * BEAM_REDUCE_WAVES + (threadIdx.x >> 6); r < a.width * a.H; r += gridDim.x * BEAM_REDUCE_WAVES) {
        const int64_t row = (int64_t)b * a.width * a.H + r, first = row * a.n_splits;
        const float* const part = a.part_acc + first * D + lane * 2;
        const f32x2 ml = lane < pieces ? *reinterpret_cast<const f32x2*>(a.part_ml + (first + lane) * 2) : f32x2{LOWEST, 0.0f};
        float top = ml[0];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
        const float w = exp2f(ml[0] - top);
        float sum = lane < pieces ? w * ml[1] : 0.0f;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
        f32x2 acc = {0.0f, 0.0f};
        auto add = [&](int p, f32x2 v, bool is) {          // (a sum that is infinite stays so whatever its piece weighs)
            const float wp = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), p));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float x = __builtin_isfinite(v[j]) ? wp * v[j] : v[j];
                acc[j] += is ? x : 0.0f;
            }
        };
        int p = 0;
        for (; p + 8 <= pieces; p += 8) {
            f32x2 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const f32x2*>(part + (p + i) * D);
#pragma unroll
            for (int i = 0; i < 8; ++i) add(p + i, v[i], true);
        }
        for (; p < pieces; p += 4) {
            f32x2 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const f32x2*>(part + min(p + i, pieces - 1) * D);
#pragma unroll
            for (int i = 0; i < 4; ++i) add(min(p + i, pieces - 1), v[i], p + i < pieces);
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        *reinterpret_cast<uint32_t*>(a.out + row * D + lane * 2) = (uint32_t)f32_to_bf16_rne(acc[0] * inv) | (uint32_t)f32_to_bf16_rne(acc[1] * inv) << 16;
    }
}

}  // namespace cusa
