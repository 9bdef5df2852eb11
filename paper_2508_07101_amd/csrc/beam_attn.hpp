// Attention over a group's pages where a KV head has few queries: up to 16 or 32 rows (row of the group, query head).
//
// What it does for more of them, tree_attn_kernel's form for groups, needs 160 KB of LDS and eight waves that meet; here a workgroup is four waves that go their own ways until their sums
// come together, two or more of them share a CU, and nothing but V passes through LDS.
#pragma once
#include "tree_attn.hpp"

namespace cusa {

constexpr int FEW_WAVES = 4, FEW_THREADS = 64 * FEW_WAVES;

template <int NB>                          // blocks of 16 rows
struct FewLds {
    __attribute__((aligned(16))) unsigned char v[FEW_WAVES][2][TREE_TILE * 256];   // V of a tile, and of the next one; the waves' sums at the end
    float m[FEW_WAVES][16 * NB], l[FEW_WAVES][16 * NB];
    uint32_t odd[BEAM_LIST / 32];          // pages with a value that is not finite and that not all rows attend to
    int32_t any_odd;
};

// A tile: two pages of the list, uniform.
struct FewTile {
    int64_t at[2];                         // elements in front of the KV head's rows
    int32_t first[2];                      // position of the page's first token
    uint32_t holders[2];
};
__device__ __forceinline__ FewTile few_tile(const TreeArgs& a, const int32_t* list, int e, int n, int kvh) {
    typedef const __attribute__((address_space(4))) i32x4* uniform_entry;   // (no kernel of the launch writes the list)
    FewTile t;
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
// K goes to registers, V to LDS, both for the next tile as soon as this one's scores are there; eight waves on a CU have 128 KB under way.
template <int NB>
__global__ __launch_bounds__(FEW_THREADS, 2) void beam_attn_kernel(TreeArgs a) {
    __shared__ FewLds<NB> lds;
    // Workgroups go to the 8 XCDs in turn: those of one KV head's pages come 8 apart, to the same L2.
    const uint32_t turn = blockIdx.x >> 3, block = turn % (uint32_t)a.m_tiles, unit = turn / (uint32_t)a.m_tiles * 8 + (blockIdx.x & 7);
    TreeSpan s;
    int b, kvh, split;
    if (!group_work(a, (int)unit, s, b, kvh, split)) return;
    const int row0 = block * (16 * NB);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, q4 = lane >> 4;
    const int g = 1 << a.g_shift, all_rows = a.max_nodes << a.g_shift, rows = min(all_rows - row0, 16 * NB), beam0 = b * a.max_nodes;
    u32x4 qv[NB][4];
    int len[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int row = row0 + min(i * 16 + n, rows - 1), beam = beam0 + (row >> a.g_shift);
        const uint16_t* const p = a.q + (int64_t)beam * a.q_stride + ((kvh << a.g_shift) + (row & (g - 1))) * D + q4 * 8;
#pragma unroll
        for (int k = 0; k < 4; ++k) qv[i][k] = *reinterpret_cast<const u32x4*>(p + k * 32);
        len[i] = a.cache.kv.seq_lens[beam];
    }
    if (tid < BEAM_LIST / 32) lds.odd[tid] = 0;
    if (tid == 0) lds.any_odd = 0;
    if (s.all == 0) {                        // a group without tokens
        for (int i = tid; i < rows * (D / 4); i += FEW_THREADS) {
            const int row = row0 + (i >> 5);
            *reinterpret_cast<u32x2*>(a.out + ((int64_t)(beam0 + (row >> a.g_shift)) * a.H + (kvh << a.g_shift) + (row & (g - 1))) * D + (i & 31) * 4) = u32x2{0, 0};
        }
        if (a.n_splits > 1 && kvh == 0 && block == 0 && tid == 0) a.pieces[b] = 0;
        return;
    }
    const int begin = split * s.chunk;
    __syncthreads();                                       // (odd is clear before anyone marks a page)
    if (a.n_splits > 1 && split == 0 && kvh == 0 && block == 0 && tid == 0) a.pieces[b] = (s.all + s.chunk - 1) / s.chunk;
    const int entries = (min(begin + s.chunk, s.all) - begin) / PAGE, tiles = (entries + 1) >> 1;
    const int plain = clampi(s.pre - begin, 0, entries * PAGE) / TREE_TILE;   // tiles that every row attends to as a whole: the first ones
    const int32_t* const list = a.entries + (b * a.entry_stride + begin / PAGE) * 4;

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
    const uint32_t vlds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)&lds.v[wave][0][0];
    // A lane's part of K's operand; of V's rows as LDS holds them: 16-byte chunk c of token t stands at c ^ 4 (t % 4), so that the transposing reads of 16 lanes meet in no bank.
    const int k_part = n * D + q4 * 8, v_part = q4 * D + ((n ^ (q4 << 2)) << 3);
    const uint32_t v_read = (4 * q4 + ((lane >> 2) & 3)) * 256 + (((lane & 3) >> 1) << 4) + (lane & 1) * 8;
    u32x4 k[2][4];
    auto request = [&](const FewTile& t, int buffer) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint16_t* const kp = a.cache.kv.k + t.at[j];
#pragma unroll
            for (int i = 0; i < 4; ++i) k[j][i] = *reinterpret_cast<const u32x4*>(kp + k_part + i * 32);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) load_to_lds(a.cache.kv.v + t.at[j], (uint32_t)(v_part + i * 4 * D) * 2, vlds + buffer * (TREE_TILE * 256) + j * (PAGE * 256) + i * 1024);
    };
    // The first tile from t on that one of this workgroup's rows attends to.
    const uint32_t here = (uint32_t)((1ull << (((row0 + rows - 1) >> a.g_shift) + 1)) - (1ull << (row0 >> a.g_shift)));
    auto find = [&](int t, FewTile& tile) {
        for (; t < tiles; t += FEW_WAVES) {
            tile = few_tile(a, list, t * 2, entries, kvh);
            if ((tile.holders[0] | tile.holders[1]) & here) break;
        }
        return t;
    };
    FewTile now, next;
    int t = find(wave, now), buffer = 0;
    if (t < tiles) request(now, 0);
#pragma unroll 1
    for (int t_next; t < tiles; t = t_next, buffer ^= 1) {
        t_next = find(t + FEW_WAVES, next);
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
            for (int c = 0; c < 8; c += 2) {               // (as weigh for TreeFineWeights)
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
        const uint32_t from = vlds + buffer * (TREE_TILE * 256) + v_read, turn = ((lane >> 2) & 3) << 6;
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
            lds.m[wave][i * 16 + n] = m[i];
            lds.l[wave][i * 16 + n] = sum;
        }
    }
    __syncthreads();
    unsigned char* const sums = &lds.v[0][0][0];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const int r = i * 16 + n;
        float top = lds.m[0][r];
#pragma unroll
        for (int w = 1; w < FEW_WAVES; ++w) top = fmaxf(top, lds.m[w][r]);
        const float f = exp2f(m[i] - top);
#pragma unroll
        for (int d = 0; d < 8; ++d)                        // columns 16 d + 4 q ..
            *reinterpret_cast<f32x4*>(sums + (wave * 16 * NB + r) * (D * 4) + (((4 * d + q4) ^ n) << 4)) = f32x4{o[i][d][0] * f, o[i][d][1] * f, o[i][d][2] * f, o[i][d][3] * f};
    }
    __syncthreads();
    const bool any_odd = lds.any_odd != 0;
    const int c = tid & 31;
#pragma unroll 1
    for (int r = tid >> 5; r < rows; r += FEW_THREADS / 32) {
        float top = lds.m[0][r], sum = 0.0f;
#pragma unroll
        for (int w = 1; w < FEW_WAVES; ++w) top = fmaxf(top, lds.m[w][r]);
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < FEW_WAVES; ++w) {
            sum += lds.l[w][r] * exp2f(lds.m[w][r] - top);
            v += *reinterpret_cast<const f32x4*>(sums + (w * 16 * NB + r) * (D * 4) + ((c ^ (r & 15)) << 4));
        }
        const int of = (row0 + r) >> a.g_shift, length = clampi(a.cache.kv.seq_lens[beam0 + of], 0, a.cache.max_len);
        if (any_odd) {
            // Pages with values that are not finite: the rows that attend to them get those values (whatever the weight: it is not 0).
            for (int e = 0; e < entries; ++e) {
                if (!(lds.odd[e >> 5] >> (e & 31) & 1)) continue;
                const FewTile t = few_tile(a, list, e, entries, kvh);
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
        const int64_t to = (int64_t)(beam0 + of) * a.H + (kvh << a.g_shift) + ((row0 + r) & (g - 1));
        if (s.chunk >= s.all) {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            const u32x2 w = {(uint32_t)f32_to_bf16_rne(v[0] * inv) | (uint32_t)f32_to_bf16_rne(v[1] * inv) << 16, (uint32_t)f32_to_bf16_rne(v[2] * inv) | (uint32_t)f32_to_bf16_rne(v[3] * inv) << 16};
            *reinterpret_cast<u32x2*>(a.out + to * D + c * 4) = w;
        } else {
            const int64_t piece = to * a.n_splits + split;
            *reinterpret_cast<f32x4*>(a.part_acc + piece * D + c * 4) = v;
            if (c == 0) *reinterpret_cast<f32x2*>(a.part_ml + piece * 2) = f32x2{top, sum};
        }
    }
}

}  // namespace cusa
