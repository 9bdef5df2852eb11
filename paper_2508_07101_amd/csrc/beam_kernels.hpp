// Device code for beam search over paged caches: groups of rows that share pages.  (Attention over a group's pages: beam_attn.hpp.)
//
//   beam_rows_kernel     the best tokens of each row and the sum of its weights
//   beam_merge_kernel    the best of a group's rows
//   kv_fork_kernel       which groups get their pages, who writes where, in one workgroup
//   fork_tables_kernel   block tables by parents, and the pages that nobody holds any more
//   fork_pages_kernel    these to the queue's end
//   kv_copy_kernel       pages copied in all layers
//   shared_pages_kernel  each page of a group once, with the rows that hold it
#pragma once
#include "plan_scan.hpp"

namespace cusa {

constexpr int BEAM_WIDTH = 32;             // rows of a group: a bit each
constexpr int BEAM_MOST = 64;              // continuations of a group: a lane each

// ---------------------------------------------------------------- selection

struct BeamArgs {
    const void* logits;
    int64_t stride;
    const float* scores;
    const int32_t* ended;
    float* out_scores;
    int32_t *parents, *tokens, *out_ended;
    float* top;                            // [rows][parts]: the largest logit
    double* sum;                           // [rows][parts]: weights relative to it
    uint64_t* best;                        // [rows][parts][n]: keys, best first; 0: none
    int32_t rows, width, vocab, n, end_token, parts, part_len /* in 16 bytes */;
};

// Larger is better: the logit's order above, of equal ones the lower token.  0 is no token's key.
__device__ __forceinline__ uint64_t beam_key(float x, uint32_t token) {
    const uint32_t u = __float_as_uint(x + 0.0f);          // (-0 counts as 0)
    return (uint64_t)((int32_t)u < 0 ? ~u : u | 0x80000000u) << 32 | (0xffffffffu - token);
}
__device__ __forceinline__ float key_logit(uint64_t key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float((int32_t)u < 0 ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ uint32_t key_token(uint64_t key) { return 0xffffffffu - (uint32_t)key; }

// The value of the lane whose number differs in bit `stride`, without LDS.
__device__ __forceinline__ uint32_t lane_xor(uint32_t v, int stride) {
    const int x = (int)v;
    switch (stride) {                                      // (a constant wherever it is called)
        case 1: return __builtin_amdgcn_mov_dpp(x, 0xb1, 0xf, 0xf, true);              // within four lanes: 1 0 3 2
        case 2: return __builtin_amdgcn_mov_dpp(x, 0x4e, 0xf, 0xf, true);              // 2 3 0 1
        case 4: return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true);   // eight lanes turned, then four
        case 8: return __builtin_amdgcn_mov_dpp(x, 0x128, 0xf, 0xf, true);             // sixteen lanes rotated by eight
        case 16: {
            const auto w = __builtin_amdgcn_permlane16_swap(v, v, false, false);
            return (threadIdx.x & 16) ? w[0] : w[1];
        }
        default: {
            const auto w = __builtin_amdgcn_permlane32_swap(v, v, false, false);
            return (threadIdx.x & 32) ? w[0] : w[1];
        }
    }
}
__device__ __forceinline__ uint64_t lane_xor(uint64_t v, int stride) {
    return (uint64_t)lane_xor((uint32_t)(v >> 32), stride) << 32 | lane_xor((uint32_t)v, stride);
}
__device__ __forceinline__ int lane_xor(int v, int stride) { return (int)lane_xor((uint32_t)v, stride); }
__device__ __forceinline__ float lane_xor(float v, int stride) { return __uint_as_float(lane_xor(__float_as_uint(v), stride)); }
__device__ __forceinline__ double lane_xor(double v, int stride) { return __builtin_bit_cast(double, lane_xor(__builtin_bit_cast(uint64_t, v), stride)); }

// Lanes with a bit in a number of lanes, as a mask.
constexpr uint64_t lanes_with(int bit) {
    uint64_t m = 0;
    for (int i = 0; i < 64; ++i)
        if (i & bit) m |= 1ull << i;
    return m;
}
// Keeps the larger value in the lanes of `larger`, the smaller in the others.
template <typename T>
__device__ __forceinline__ T exchange(T v, int stride, uint64_t larger) {
    const T o = lane_xor(v, stride);
    return (o > v) == (bool)__builtin_amdgcn_inverse_ballot_w64(larger) ? o : v;
}
// The wave's 64 values in order over the lanes, by a bitonic network.
template <bool FALLING, typename T>
__device__ __forceinline__ T sort_lanes(T v) {
#pragma unroll
    for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
        for (int stride = size >> 1; stride > 0; stride >>= 1)
            v = exchange(v, stride, (lanes_with(stride) ^ (size < 64 ? lanes_with(size) : 0)) ^ (FALLING ? ~0ull : 0));
    return v;
}
// The 64 largest of a falling and a rising list, in falling order.
__device__ __forceinline__ uint64_t merge_lanes(uint64_t list, uint64_t rising) {
    uint64_t v = list > rising ? list : rising;
#pragma unroll
    for (int stride = 32; stride > 0; stride >>= 1) v = exchange(v, stride, ~lanes_with(stride));
    return v;
}
template <typename T, typename F>
__device__ __forceinline__ T over_lanes(T v, F f) {
#pragma unroll
    for (int stride = 1; stride < 64; stride <<= 1) v = f(v, lane_xor(v, stride));
    return v;
}
__device__ __forceinline__ uint64_t lane_key(uint64_t k, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, lane);
}
// The smallest number above x (x below +infinity).
__device__ __forceinline__ float above(float x) {
    const int32_t u = __float_as_int(x + 0.0f);
    return __int_as_float(u >= 0 ? u + 1 : u - 1);
}
__device__ __forceinline__ int lanes_before(uint64_t who) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0)); }

template <int DTYPE>                       // cusa_dtype
struct Logits {
    static constexpr int SIZE = DTYPE == 2 ? 4 : 2, PER = 16 / SIZE;
    static constexpr uint32_t NONE = DTYPE == 0 ? 0xff80ff80u : DTYPE == 1 ? 0xfc00fc00u : 0xff800000u;   // -infinity
    static __device__ __forceinline__ float at(const u32x4& x, int k) {
        if constexpr (DTYPE == 0) return __uint_as_float((k & 1) ? x[k >> 1] & 0xffff0000u : x[k >> 1] << 16);
        else if constexpr (DTYPE == 1) return (float)__builtin_bit_cast(_Float16, (uint16_t)((k & 1) ? x[k >> 1] >> 16 : x[k >> 1] & 0xffffu));
        else return __uint_as_float(x[k]);
    }
    static __device__ __forceinline__ float one(const void* p, int64_t i) {
        if constexpr (DTYPE == 0) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
        else if constexpr (DTYPE == 1) return (float)static_cast<const _Float16*>(p)[i];
        else return static_cast<const float*>(p)[i];
    }
};

constexpr int BEAM_WAVES = 4, BOUND_BY_LANES = 32;
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ void lds_of_wave() {            // what the wave's other lanes wrote to LDS is there
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The best 64 of a wave's keys, one in every lane, in falling order; keys are gathered in LDS until they are enough for a sort.
constexpr int FOUND = 400, FOUND_ENDS = 16;               // of these for what stands at a row's ends: a search leaves them free
struct Best {
    uint64_t* found;
    uint64_t list = 0;
    int n = 0;                                             // gathered: uniform
    __device__ __forceinline__ explicit Best(uint64_t* lds) : found(lds) {}
    __device__ __forceinline__ void flush() {
        const int lane = threadIdx.x & 63;
        lds_of_wave();
#pragma unroll 1
        for (int i = 0; i < n; i += 64) list = merge_lanes(list, sort_lanes<false>(i + lane < n ? found[i + lane] : (uint64_t)0));
        lds_of_wave();
        n = 0;
    }
    // The keys of the lanes in `who`; those that there is no room for are counted all the same.
    __device__ __forceinline__ void add(bool hit, uint64_t who, uint64_t key) {
        const int at = n + lanes_before(who);
        if (hit && at < FOUND) found[at] = key;
        n += __popcll(who);
    }
};

// A wave for a part of a row.  One pass: the largest logit and the sum of weights relative to it, a pair in every lane; the best tokens, one in every lane,
// in falling order.  R loads of 16 bytes a lane are looked at in a step.  Of the step's logits only those above a bound matter that n logits reach; where many lanes have such
// ones, their maxima are sorted: the n-th largest of them is the next bound, and leaves few; for more than BOUND_BY_LANES places that of all loads' maxima, found bit by bit.  (64 places, where the lanes' least maximum leaves
// hundreds: 256 rows of 32000 logits 28 us, so 13; 4 rows of 128000 21 and 9.5; 32 places 8.4 and 9.6 for 32 rows of 128000.)  Those few are gathered in LDS, and when there are enough sorted 64 at a time and merged.
// A weight is 2^((x - ref) log2 e): the difference first, so that rows that differ by a constant have the same sums, whatever the constant.  A lane's ref is a logit of its own
// that follows the largest when that is 8 above it.  So an exponent is 12 above 0 at most, and below 0 by as much as the row's entropy in bits and one or two more in the weighted mean: its three
// roundings (difference, product, constant) move the sum by less than 2^-17 of itself, or 2^-16.5 with 2^31 tokens.
// 512 rows of 131072 logits, 134 MB: bf16 30 to 33 us, 4.1 to 4.5 TB/s (a plain read 19.6 us), fp16 1 us more; 256 rows in fp32 29; with one bf16 row in 20 ended, which is not read, 29.  A wave asks for a step's logits, waits and
// computes in turn, four waves to a SIMD: vector instructions are under way for 79 % of the CUs' busy time, and waves wait for 46 % of theirs.  Which of the two it is bound by is open: without the search for
// the best those 29 are 25; weights by one multiply-add, an instruction less for each logit, take as long; the next step's logits asked for ahead into registers cost a wave to a SIMD (39 us; by four
// loads 36), and past the registers they have not been tried.  The list sorted after each step instead of a running bound 2 us longer; a bound from maxima over groups of lanes instead of the sort as long, and
// with nine logits in ten masked 26 us for 17, for the keys that it lets through.
template <int DTYPE, int R>
__global__ __launch_bounds__(64 * BEAM_WAVES) void beam_rows_kernel(BeamArgs a) {
    typedef Logits<DTYPE> X;
    constexpr int PER = X::PER;
    __shared__ uint64_t found_of[BEAM_WAVES][FOUND];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Best best(found_of[wave]);
    const int unit = blockIdx.x * BEAM_WAVES + wave, row = unit / a.parts, part = unit - row * a.parts;
    if (row >= a.rows) return;
    if ((a.ended && a.ended[row] != 0) || !__builtin_isfinite(a.scores[row])) return;   // (nobody asks for its tokens)
    const char* const base = static_cast<const char*>(a.logits) + (int64_t)row * a.stride * X::SIZE;
    const int head = min((int)((16 - ((uintptr_t)base & 15)) & 15) / X::SIZE, a.vocab);   // logits before the first 16 bytes that are aligned
    const int whole = (a.vocab - head) / PER, tail = a.vocab - head - whole * PER;
    const u32x4* const body = reinterpret_cast<const u32x4*>(base + head * X::SIZE);
    static_assert(2 * (PER - 1) <= FOUND_ENDS, "logits at the ends");
    const int begin = min(part * a.part_len, whole), end = min(begin + a.part_len, whole);
    constexpr int HALF = R < 4 ? R : 4;
    const u32x4 none = {X::NONE, X::NONE, X::NONE, X::NONE};

    float ref = -INFINITY, top = -INFINITY, seen = -INFINITY;   // seen: there are n logits or more that are not below it
    double sum = 0.0;
    auto follow = [&](float largest) {
        top = fmaxf(top, largest);
        if (__any(largest > ref + 8.0f)) {                // (the first logit above -infinity is)
            const float to = largest > ref + 8.0f ? largest : ref;
            if (ref > -INFINITY) sum *= (double)__builtin_amdgcn_exp2f((ref - to) * LOG2E);   // (before that, the sum is 0, or NaN)
            ref = to;
        }
    };
    auto weight = [&](float x) { return __builtin_amdgcn_exp2f((x - (ref > -INFINITY ? ref : 0.0f)) * LOG2E); };
    auto search = [&](int v0) {
        u32x4 x[R];
        if (v0 + 64 * R <= end) {
#pragma unroll
            for (int r = 0; r < R; ++r) x[r] = __builtin_nontemporal_load(body + v0 + r * 64 + lane);
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int v = v0 + r * 64 + lane;
                x[r] = __builtin_nontemporal_load(body + min(v, end - 1));
                if (v >= end) x[r] = none;
            }
        }
        float most[R], largest = -INFINITY;
#pragma unroll
        for (int r0 = 0; r0 < R; r0 += HALF) {                // (as many at a time as there are registers for)
            float some = -INFINITY;
#pragma unroll
            for (int r = r0; r < r0 + HALF; ++r) {
                most[r] = X::at(x[r], 0);
#pragma unroll
                for (int k = 1; k < PER; ++k) most[r] = fmaxf(most[r], X::at(x[r], k));
                some = fmaxf(some, most[r]);
            }
            largest = fmaxf(largest, some);
            follow(some);
            float half = 0.0f;
#pragma unroll
            for (int r = r0; r < r0 + HALF; ++r) {
                float w[PER];
#pragma unroll
                for (int k = 0; k < PER; ++k) w[k] = weight(X::at(x[r], k));
#pragma unroll
                for (int o = PER / 2; o > 0; o >>= 1)
#pragma unroll
                    for (int k = 0; k < o; ++k) w[k] += w[k + o];
                half += w[0];
            }
            sum += (double)half;
#pragma unroll
            for (int r = r0; r < r0 + HALF; ++r) asm volatile("" : "+v"(x[r]));   // (what is taken apart is not kept for the search below, which mostly looks at none of it)
        }
        // The tokens that may be among the n best.  (Tokens of later steps are larger: of equal logits those that are there already come first.)
        float least = above(seen);
        const int lanes = __popcll(__ballot(largest >= least));
        if (lanes == 0) return;
        const bool bound = lanes >= min(2 * a.n, 64);      // (fewer are not worth a sort)
        if (bound && a.n <= BOUND_BY_LANES) {
            seen = least = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sort_lanes<true>(largest)), a.n - 1));   // (not below the old one: n lanes are)
        } else if (bound) {                                // the n-th largest of the loads' maxima, to 16 bits, bit by bit
            uint32_t of[R], t = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const uint32_t u = __float_as_uint(most[r]);
                of[r] = ((int32_t)u < 0 ? ~u : u | 0x80000000u) >> 16;
            }
#pragma unroll 1
            for (uint32_t bit = 0x8000; bit; bit >>= 1) {
                int count = 0;
#pragma unroll
                for (int r = 0; r < R; ++r) count += __popcll(__ballot(of[r] >= (t | bit)));
                if (count >= a.n) t |= bit;
            }
            const float by = __uint_as_float((t & 0x8000) ? (t ^ 0x8000) << 16 : ~(t << 16));   // the smallest with these 16 bits
            seen = least = fmaxf(least, by);
        }
        const int before = best.n;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!__any(most[r] >= least)) continue;
            const uint32_t token = head + (v0 + r * 64 + lane) * PER;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const float y = X::at(x[r], k);
                const bool hit = y >= least;
                if (const uint64_t who = __ballot(hit)) best.add(hit, who, beam_key(y, token + k));
            }
        }
        if (best.n > FOUND - FOUND_ENDS) {                // more than there is room for: those above the bound 64 at a time, and of those that are equal to it the first n
            best.n = before;
            if (best.n > 0) best.flush();
#pragma unroll 1
            for (int r = 0; r < R; ++r) {
                const int v = v0 + r * 64 + lane;
                const u32x4 z = v < end ? body[v] : none;
#pragma unroll 1
                for (int k = 0; k < PER; ++k) {
                    const float y = X::at(z, k);
                    const uint64_t now = lane_key(best.list, a.n - 1);
                    const bool hit = (bound ? y > least : y >= least) && (!now || y >= key_logit(now));
                    if (const uint64_t who = __ballot(hit)) best.add(hit, who, beam_key(y, head + v * PER + k));
                    if (best.n > FOUND - 64) best.flush();
                }
            }
            if (best.n > 0) best.flush();
            int left = bound ? a.n : 0;
#pragma unroll 1
            for (int r = 0; r < R && left > 0; ++r) {
                const int v = v0 + r * 64 + lane;
                const u32x4 z = v < end ? body[v] : none;
                int at = 0, total = 0;
#pragma unroll
                for (int k = 0; k < PER; ++k) {
                    const uint64_t who = __ballot(X::at(z, k) == least);
                    at += lanes_before(who);
                    total += __popcll(who);
                }
#pragma unroll
                for (int k = 0; k < PER; ++k) {
                    if (X::at(z, k) != least) continue;
                    if (at < left) best.found[best.n + at] = beam_key(least, head + v * PER + k);
                    ++at;
                }
                best.n += min(total, left);
                left -= total;
            }
        }
    };
#pragma unroll 1
    for (int v0 = begin;; v0 += 64 * R) {
        if (v0 < end) search(v0);
        const bool ends = v0 + 64 * R >= end;
        if (ends && part == 0 && head + tail > 0) {        // what is not 16 aligned bytes: PER - 1 logits at either end at most
            const int i = lane < head ? lane : lane >= 32 && lane - 32 < tail ? a.vocab - tail + lane - 32 : -1;
            const float y = i >= 0 ? X::one(base, i) : -INFINITY;
            follow(y);
            sum += (double)weight(y);
            const bool hit = y > -INFINITY;
            best.add(hit, __ballot(hit), beam_key(y, i));
        }
        if (best.n >= 64 || ends) {
            best.flush();
            const uint64_t last = lane_key(best.list, a.n - 1);
            if (last) seen = fmaxf(seen, key_logit(last));
        }
        if (ends) break;
    }
    const float all = over_lanes(top, [](float x, float y) { return fmaxf(x, y); });
    const double total = over_lanes(ref == all || ref == -INFINITY ? sum : sum * (double)__builtin_amdgcn_exp2f((ref - all) * LOG2E), [](double x, double y) { return x + y; });
    if (lane < a.n) a.best[(int64_t)unit * a.n + lane] = best.list;
    if (lane == 0) {
        a.top[unit] = all;
        a.sum[unit] = total;                               // (NaN with a NaN among the logits)
    }
}

// A wave's list of candidates of a group, a lane for each, best first: worth more, of equal ones the lower number (row, place in the row's list).
struct Candidate {
    double v;
    int32_t i;
    __device__ __forceinline__ bool before(const Candidate& o) const { return v > o.v || (v == o.v && i < o.i); }
};
// The best 64 of a list and of one in reverse order.
__device__ __forceinline__ Candidate merge_candidates(Candidate c, const Candidate& rising) {
    if (rising.before(c)) c = rising;
#pragma unroll
    for (int stride = 32; stride > 0; stride >>= 1) {
        const Candidate o = {lane_xor(c.v, stride), lane_xor(c.i, stride)};
        if (o.before(c) == (bool)__builtin_amdgcn_inverse_ballot_w64(~lanes_with(stride))) c = o;
    }
    return c;
}

// A workgroup for a group, a wave for each of its rows at a time: the parts' sums and lists together, the tokens' worth in 64 bits.  Of the parts' q-th best, the m-th largest
// bounds the row's best m q from below.  With m near half of the parts and m q >= n few of the lists' keys are left.  Then the rows' lists are merged, two at a time.
// Bound by its chain of sorts and of code that runs once, a copy of which is fetched first: 64 groups of 8 rows for 8 places 6 us, 8 groups of 32 rows for 64 places 24 (each candidate counting those in
// front of it: 145).  4 rows of 32000 logits: 6 us here and 6 in beam_rows_kernel, of which a launch and the way to memory and back are most.
constexpr int MERGE_WAVES = 16;
__global__ __launch_bounds__(64 * MERGE_WAVES) void beam_merge_kernel(BeamArgs a) {
    __shared__ uint64_t found_of[MERGE_WAVES][FOUND];
    __shared__ Candidate list_of[MERGE_WAVES][64];
    __shared__ int32_t token[BEAM_WIDTH * BEAM_MOST], over[BEAM_WIDTH];
    const int group = blockIdx.x, row0 = group * a.width, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Candidate c = {-INFINITY, 0x7fffffff};
    for (int b = wave; b < a.width; b += MERGE_WAVES) {
        const int row = row0 + b;
        const float s = a.scores[row];
        const bool ended = a.ended && a.ended[row] != 0, counts = __builtin_isfinite(s);
        double v = -INFINITY;
        int t = -1;
        if (counts && ended) {
            if (lane == 0) {
                v = s;
                t = a.end_token;
            }
        } else if (counts) {
            const bool mine = lane < a.parts;
            const int64_t unit = (int64_t)row * a.parts;
            const uint64_t* const keys = a.best + unit * a.n;
            const int all = a.parts * a.n;
            const bool few = all <= 64;                    // (a row of one part among them)
            constexpr int RUN = 4;                         // loads under way at once
            uint64_t k[RUN];
            auto request = [&](int j0) {                   // a lane for each list, which is in order: what is above the bound stands in front
#pragma unroll
                for (int j = 0; j < RUN; ++j) k[j] = mine && j0 + j < a.n ? keys[(int64_t)lane * a.n + j0 + j] : 0;
            };
            const float own = mine ? a.top[unit + lane] : -INFINITY;
            double sum = mine ? a.sum[unit + lane] : 0.0;
            const int q = max(1, (2 * a.n + a.parts - 1) / a.parts);
            const uint64_t some = few ? lane < all ? keys[lane] : 0 : mine ? keys[(int64_t)lane * a.n + (q - 1)] : 0;   // (two parts or more: q <= n)
            if (!few) request(0);
            const float top = over_lanes(own, [](float x, float y) { return fmaxf(x, y); });
            if (own != top) sum *= (double)__builtin_amdgcn_exp2f((own - top) * LOG2E);   // (a part without logits above -infinity: 0, or NaN)
            sum = over_lanes(sum, [](double x, double y) { return x + y; });
            Best best(found_of[wave]);
            const uint64_t sorted = a.parts == 1 ? some : sort_lanes<true>(some);   // (one part's are in order)
            if (few) {
                best.list = sorted;
            } else {
                const uint64_t least = lane_key(sorted, (a.n + q - 1) / q - 1);
                for (int j0 = 0;;) {                       // (code that runs once waits for itself: few copies of the sorts)
                    uint64_t key = 0;
#pragma unroll 1
                    for (int j = 0; j < RUN; ++j) {
                        key = k[0];
#pragma unroll
                        for (int i = 1; i < RUN; ++i) k[i - 1] = k[i];
                        const bool hit = key != 0 && key >= least;
                        best.add(hit, __ballot(hit), key);
                    }
                    j0 += RUN;
                    const bool more = j0 < a.n && __any(key != 0 && key >= least);
                    if (more) request(j0);
                    if (!more || best.n > FOUND - 64 * RUN) best.flush();
                    if (!more) break;
                }
            }
            if (top < INFINITY && sum > 0.0 && lane < a.n && best.list) {
                v = (double)s + (((double)key_logit(best.list) - (double)top) - log(sum));
                t = key_token(best.list);
            }
        }
        if (lane < a.n) token[b * a.n + lane] = t;
        if (lane == 0) over[b] = ended;
        const int i = lane < a.n ? b * a.n + lane : 0x7fffffff;
        c = b == wave ? Candidate{v, i} : merge_candidates(c, {__shfl(v, 63 - lane), __shfl(i, 63 - lane)});
    }
    const int lists = min(a.width, MERGE_WAVES);
    for (int step = 1; step < lists; step <<= 1) {
        if ((wave & (2 * step - 1)) == step) list_of[wave][lane] = c;
        __syncthreads();
        if ((wave & (2 * step - 1)) == 0 && wave + step < lists) c = merge_candidates(c, list_of[wave + step][63 - lane]);
    }
    lds_of_wave();
    if (wave != 0 || lane >= a.n) return;
    const bool is = c.v > -INFINITY;
    const int b = is ? c.i / a.n : -1, t = is ? token[c.i] : -1;
    const int64_t to = (int64_t)group * a.n + lane;
    a.out_scores[to] = (float)c.v;
    a.parents[to] = b;
    a.tokens[to] = t;
    if (a.out_ended) a.out_ended[to] = is && (over[b] || t == a.end_token);
}

// Which of a column's rows hold this page; column: LDS, theirs side by side.
template <int ROWS>
__device__ __forceinline__ uint32_t holders_of(const int32_t* column, int32_t page) {
    constexpr int RUN = ROWS < 4 ? ROWS : 4;               // to a read
    typedef int32_t entries __attribute__((ext_vector_type(RUN)));
    uint32_t holders = 0;
#pragma unroll
    for (int o = 0; o < ROWS; o += RUN) {
        const entries x = *reinterpret_cast<const entries*>(column + o);
#pragma unroll
        for (int k = 0; k < RUN; ++k) holders |= x[k] == page ? 1u << (o + k) : 0u;
    }
    return holders;
}

// ---------------------------------------------------------------- fork

struct ForkRow {                           // what the tables need of a row, in the workspace
    int32_t src, had;                      // the row of its group whose entries it takes (-1: none), and how many
    int32_t old;                           // entries that it had itself
    int32_t col, page;                     // a new page, and where (-1: none)
};
struct ForkHead {
    int32_t first, avail, taken;           // of the queue, before the call; new pages
};
struct ForkArgs {
    const int32_t *held, *parents, *ended, *table;
    int32_t *table_out, *lens, *ring;
    int64_t* slots;
    int32_t *copies, *granted;
    const int32_t* state;
    int32_t* state_out;
    ForkHead* head;
    ForkRow* rows;
    int32_t *counts, *freed;               // of each (group, cols columns): how many pages go back, and which
    int32_t batch, width, max_pages, n_pages, cap, grow, cols, chunks;
};

// A column of a group: what the rows hold there goes from `table` to `table_out`, all of it read before any is written, so that the tables may be changed in place.  Returns the
// rows whose entry names a page that nobody holds any more (of several, the first).  entry: a column in LDS, PLAN_THREADS entries from row to row.
__device__ __forceinline__ uint32_t fork_column(const ForkArgs& a, const ForkRow* rows, int row0, int col, int32_t* entry) {
    const int32_t* const from = a.table + (int64_t)row0 * a.max_pages + col;
    int32_t* const to = a.table_out + (int64_t)row0 * a.max_pages + col;
    uint32_t alive = 0;                                    // rows that somebody descends from
#pragma unroll 4
    for (int b = 0; b < a.width; ++b) {
        entry[b * PLAN_THREADS] = col < rows[b].old ? from[(int64_t)b * a.max_pages] : -1;
        if (rows[b].src >= 0) alive |= 1u << rows[b].src;
    }
    for (int b = 0; b < a.width; ++b) {
        const ForkRow& r = rows[b];
        if (col == r.col) to[(int64_t)b * a.max_pages] = r.page;
        else if (r.src >= 0 && col < r.had) to[(int64_t)b * a.max_pages] = entry[r.src * PLAN_THREADS];
    }
    uint32_t gone = 0;
    for (uint32_t ends = ~alive & (a.width < 32 ? (1u << a.width) - 1 : 0xffffffffu); ends; ends &= ends - 1) {
        const int b = __builtin_ctz(ends);
        const int32_t e = entry[b * PLAN_THREADS];
        if ((uint32_t)e >= (uint32_t)a.n_pages) continue;
        bool last = true;                                  // nobody who stays holds it, and no row before this one did
        for (int o = 0; o < a.width; ++o) last &= !(entry[o * PLAN_THREADS] == e && ((alive >> o & 1) || o < b));
        if (last) gone |= 1u << b;
    }
    return gone;
}
__device__ __forceinline__ int fork_most(const ForkRow& r) { return max(r.old, max(r.had, r.col + 1)); }

// A thread for each row, as many whole groups at a time as 1024 hold.  Latency is all: the numbers, the parent's length, the open page's entry, two sums, a page of the queue: 6.2 us for one group,
// 6.6 for 64 of 4 rows, 9.1 for 8 of 32 (a row's numbers one word after the other, each asked for only if the one before called for it: 16).
// ALL: the workgroup changes the tables as well, a thread for a column of a group, and gives the pages back; for few rows, whose launches would take longer.
constexpr int FORK_ALL_WIDTH = 8;          // rows of a group that it has LDS for
template <bool ALL>
__global__ __launch_bounds__(PLAN_THREADS) void kv_fork_kernel(ForkArgs a) {
    __shared__ int64_t scratch[3][2][PLAN_THREADS / 64];
    __shared__ i32x4 s_open[PLAN_THREADS];                 // of a row: whose tokens it takes, in how many pages, the page that it is to write into (-1: none with tokens), and its column
    __shared__ int32_t s_need[PLAN_THREADS], s_most;
    __shared__ ForkRow s_rows[ALL ? PLAN_THREADS : 1];
    __shared__ int32_t s_entry[ALL ? FORK_ALL_WIDTH : 1][PLAN_THREADS];
    const int tid = threadIdx.x, round = PLAN_THREADS / a.width * a.width, mate0 = tid - tid % a.width;
    int first = a.state[0];
    const int avail = clampi(a.state[1], 0, a.n_pages);
    if ((uint32_t)first >= (uint32_t)a.n_pages) first = 0;
    if (ALL && tid == 0) s_most = 0;
    int64_t needed = 0, taken = 0;                         // of the groups before this round's
    for (int base = 0; base < a.batch; base += round) {
        const int b = base + tid, waves = min((min(a.batch - base, round) + 63) >> 6, PLAN_THREADS / 64);
        const bool here = tid < round && b < a.batch;
        const int parent = here ? a.parents[b] : -1;
        const bool valid = parent >= 0 && parent < a.width;
        const int src = valid ? base + mate0 + parent : -1;
        const int kept = valid ? clampi(a.held[src], 0, a.cap) : 0, held = here ? clampi(a.held[b], 0, a.cap) : 0;
        const bool wants = valid && a.grow && !(a.ended && a.ended[b] != 0), fits = !wants || kept < a.cap;
        const int off = kept & (PAGE - 1), col = kept / PAGE;
        int page = -1;                                     // that the new token goes to, where it holds tokens
        if (wants && off) page = a.table[(int64_t)src * a.max_pages + col];
        const bool open = (uint32_t)page < (uint32_t)a.n_pages;
        s_open[tid] = i32x4{src, pages_of(kept), open ? page : -1, col};
        __syncthreads();
        bool copy = false;
        if (open) {
            int holders = 0, writers = 0;
            bool lowest = true;
#pragma unroll 4
            for (int t = mate0; t < mate0 + a.width; ++t) {
                const i32x4 r = s_open[t];
                const bool there = r[0] >= 0 && r[1] > col, here_too = r[3] == col, writes = there && here_too && r[2] == page;
                writers += writes;
                holders += writes;
                lowest &= !(writes && t < tid);
                // (who writes elsewhere in this column holds another page there)
                if (there && !(here_too && r[2] >= 0)) holders += a.table[(int64_t)r[0] * a.max_pages + col] == page;
            }
            copy = !(lowest && holders == writers);
        }
        const bool need = wants && (off == 0 || copy);
        s_need[tid] = (need ? 1 : 0) | (fits ? 0 : 2);
        __syncthreads();
        int of_group = 0;
        bool group_fits = true;
        if (here) {
            for (int t = mate0; t < mate0 + a.width; ++t) {
                of_group += s_need[t] & 1;
                group_fits &= !(s_need[t] & 2);
            }
        }
        int64_t sum;
        const bool leads = here && tid == mate0;
        const int64_t v = leads && group_fits ? of_group : 0, before = plan_scan(v, sum, scratch[0], waves);
        const bool ok = here && group_fits && (of_group == 0 || needed + before + v <= avail);   // (before: for all but the first row, with their own group's)
        needed += sum;
        const bool takes = ok && need;
        const int64_t pop = taken + plan_scan(takes ? 1 : 0, sum, scratch[1], waves);
        taken += sum;
        if (here) {
            const int id = takes ? a.ring[ring_at(first + pop, a.n_pages)] : -1;
            const int to = takes ? id : page;
            a.lens[b] = ok ? kept + (wants ? 1 : 0) : held;
            a.slots[b] = ok && wants && (uint32_t)to < (uint32_t)a.n_pages ? (int64_t)to * PAGE + off : -1;
            *reinterpret_cast<i32x4*>(a.copies + (int64_t)b * 4) = ok && copy ? i32x4{page, id, off, 0} : i32x4{-1, -1, 0, 0};
            if (a.granted && leads) a.granted[b / a.width] = ok;
            const ForkRow r = ok ? ForkRow{valid ? parent : -1, pages_of(kept), pages_of(held), takes ? col : -1, id} : ForkRow{tid - mate0, pages_of(held), pages_of(held), -1, -1};
            if (ALL) {
                s_rows[tid] = r;                           // (one round: batch <= 1024)
                atomicMax(&s_most, fork_most(r));
            } else {
                a.rows[b] = r;
            }
        }
        __syncthreads();
    }
    int64_t pushed = 0;
    if constexpr (ALL) {
        const int cols = s_most, all = a.batch / a.width * cols;
        int which = 2;                                     // (plan_scan's words: not those of the call before)
        for (int i0 = 0; i0 < all; i0 += PLAN_THREADS, which = which == 2 ? 0 : 2) {
            const int i = i0 + tid, group = i < all ? i / cols : 0, row0 = group * a.width;
            uint32_t gone = i < all ? fork_column(a, s_rows + row0, row0, i - group * cols, &s_entry[0][tid]) : 0;
            int64_t sum, at = (int64_t)first + avail + pushed + plan_scan(__popc(gone), sum, scratch[which], PLAN_THREADS / 64);
            for (; gone; gone &= gone - 1) a.ring[ring_at(at++, a.n_pages)] = s_entry[__builtin_ctz(gone)][tid];
            pushed += sum;
        }
    }
    if (tid == 0) {
        a.state_out[0] = (int)ring_at((int64_t)first + taken, a.n_pages);
        if (ALL) a.state_out[1] = (int)min((int64_t)avail - taken + pushed, (int64_t)a.n_pages);
        else *a.head = ForkHead{first, avail, (int)taken};
    }
}

// A workgroup for PLAN_THREADS / ROWS columns of a group, a thread for a row's entry in a column, rows side by side (ROWS: the width, or the next power of two).  A column's rows are one wave's, which
// reads all before it writes any.  64 groups of 4 rows, 2080 columns: 4.5 us; 8 groups of 32 beams: 6.5 (a thread for a column, which goes over its rows: 6.3 and 38).
template <int ROWS>
__global__ __launch_bounds__(PLAN_THREADS) void fork_tables_kernel(ForkArgs a) {
    constexpr int WAVES = PLAN_THREADS / 64, COLS = PLAN_THREADS / ROWS;
    __shared__ __attribute__((aligned(16))) int32_t entry[WAVES][64];
    __shared__ int32_t sums[WAVES];
    const int tid = threadIdx.x, group = blockIdx.y, row0 = group * a.width, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = lane & (ROWS - 1);
    const ForkRow r = b < a.width ? a.rows[row0 + b] : ForkRow{-1, 0, 0, -1, -1};
    const int most = over_lanes(fork_most(r), [](int x, int y) { return max(x, y); });
    const uint32_t alive = over_lanes(r.src >= 0 ? 1u << r.src : 0u, [](uint32_t x, uint32_t y) { return x | y; });   // rows that somebody descends from
    const int64_t chunk = (int64_t)group * a.chunks + blockIdx.x;
    if ((int)blockIdx.x * COLS >= most) {
        if (tid == 0) a.counts[chunk] = 0;
        return;
    }
    const int col = blockIdx.x * COLS + tid / ROWS, mates = lane & ~(ROWS - 1);
    const int64_t at_table = (int64_t)(row0 + b) * a.max_pages + col;
    const int32_t e = col < r.old ? a.table[at_table] : -1;
    entry[wave][lane] = e;
    lds_of_wave();
    const uint32_t holders = holders_of<ROWS>(&entry[wave][mates], e);
    const int32_t taken = entry[wave][mates + max(r.src, 0)];
    if (col == r.col) a.table_out[at_table] = r.page;
    else if (r.src >= 0 && col < r.had) a.table_out[at_table] = taken;
    // Pages that nobody who stays holds go back, each once.
    const bool gone = !(alive >> b & 1) && (uint32_t)e < (uint32_t)a.n_pages && (holders & (alive | ((1u << b) - 1))) == 0;
    const uint64_t who = __ballot(gone);
    if (lane == 0) sums[wave] = __popcll(who);
    __syncthreads();
    int at = lanes_before(who), total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) at += sums[w];
        total += sums[w];
    }
    if (gone) a.freed[chunk * COLS * a.width + at] = e;
    if (tid == 0) a.counts[chunk] = total;
}

// The pages that go back, in order: a thread for each, which looks up its list among 1024.  4 to 6.5 us, a launch's own time and two ways to memory.
__global__ __launch_bounds__(PLAN_THREADS) void fork_pages_kernel(ForkArgs a) {
    __shared__ int64_t scratch[2][2][PLAN_THREADS / 64];
    __shared__ int32_t start[PLAN_THREADS];
    const int tid = threadIdx.x, chunks = a.batch / a.width * a.chunks;
    const ForkHead h = *a.head;
    int64_t pushed = 0;
    int which = 0;
    for (int base = 0; base < chunks; base += PLAN_THREADS, which ^= 1) {
        int64_t sum;
        start[tid] = (int)plan_scan(base + tid < chunks ? a.counts[base + tid] : 0, sum, scratch[which], PLAN_THREADS / 64);
        __syncthreads();
        for (int i = tid; i < (int)sum; i += PLAN_THREADS) {
            int lo = 0;                                    // the last list that starts at or before i
#pragma unroll
            for (int step = PLAN_THREADS / 2; step > 0; step >>= 1)
                if (start[lo + step] <= i) lo += step;
            a.ring[ring_at((int64_t)h.first + h.avail + pushed + i, a.n_pages)] = a.freed[(int64_t)(base + lo) * a.cols * a.width + (i - start[lo])];
        }
        pushed += sum;
        __syncthreads();
    }
    if (tid == 0) a.state_out[1] = (int)min((int64_t)h.avail - h.taken + pushed, (int64_t)a.n_pages);
}

// ---------------------------------------------------------------- copy

constexpr int COPY_LAYERS = 40;            // layers of a launch: their descriptors travel as arguments (4 KB at most)
constexpr int COPY_THREADS = 256, COPY_MOST = (1 << 24) - 1;   // copies of a launch: 2^32 threads are too many

struct CopyLayer {
    uint16_t *k, *v;
    int32_t n_pages;
};
struct CopyArgs {
    const int32_t* copies;
    int32_t G;
    CopyLayer layer[COPY_LAYERS];
};
static_assert(sizeof(CopyArgs) <= 4096, "a launch's arguments");

// A workgroup for a copy in a layer: 16 lanes a row of 256 bytes, eight rows of theirs under way.  Bound by memory: 256 pages of 1 to 15 tokens, a quarter of them none, 8 KV heads, 32 layers, 441 MB read and
// written: 98 and 109 us for two caches in turn, 4.3 TB/s (a plain copy of a large tensor 5.08); stores that the caches keep 109 on average for these 103.7.  One cache again and again, of whose pages the last-level
// cache then still has some: 78 us, with stores that the caches keep 109; four rows under way 80 us, sixteen 98.  Four pages of 36 layers: 5 us, a launch's own time.
__global__ __launch_bounds__(COPY_THREADS) void kv_copy_kernel(CopyArgs a) {
    const CopyLayer& l = a.layer[blockIdx.y];
    const i32x4 copy = *reinterpret_cast<const i32x4*>(a.copies + (int64_t)blockIdx.x * 4);
    const int from = copy[0], to = copy[1], n = min(copy[2], PAGE);
    if ((uint32_t)from >= (uint32_t)l.n_pages || (uint32_t)to >= (uint32_t)l.n_pages || from == to || n <= 0) return;
    const int64_t page = (int64_t)a.G * PAGE * D;
    const int rows = a.G * n, c = (threadIdx.x & 15) * 8;  // of K, and of V
    const uint32_t over_n = (65536 + n - 1) / n;           // r / n = r over_n >> 16 for r < 4096 (r times what over_n is too large by stays below 65536 / n)
    constexpr int RUN = 8, STEP = COPY_THREADS / 16;
    for (int r0 = threadIdx.x >> 4; r0 < 2 * rows; r0 += RUN * STEP) {
        u32x4 x[RUN];
        int64_t at[RUN];
        uint16_t* pool[RUN];
#pragma unroll
        for (int j = 0; j < RUN; ++j) {
            const int r = r0 + j * STEP, row = r < rows ? r : r - rows;
            if (r >= 2 * rows) continue;
            const int head = rows <= 4096 ? (int)(row * over_n >> 16) : row / n;
            pool[j] = r < rows ? l.k : l.v;
            at[j] = (int64_t)(head * PAGE + row - head * n) * D + c;
            x[j] = *reinterpret_cast<const u32x4*>(pool[j] + from * page + at[j]);
        }
#pragma unroll
        for (int j = 0; j < RUN; ++j)
            if (r0 + j * STEP < 2 * rows) __builtin_nontemporal_store(x[j], reinterpret_cast<u32x4*>(pool[j] + to * page + at[j]));
    }
}

// ---------------------------------------------------------------- pages of groups

struct SharedArgs {
    const int32_t *table, *lens;
    int32_t *entries, *count;
    int32_t batch, width, max_pages, n_pages, max_len, max_entries;
};
constexpr int SHARED_THREADS = 1024, SHARED_STEPS = 4;

// A workgroup for a group; a thread for a row's entry in a column, rows side by side (ROWS: the width, or the next power of two), which is the list's order.  Each compares its page with those of
// the column's other rows; SHARED_STEPS entries a thread between two barriers.  Bound by the steps' latency, each waiting for the table's entries and the list's stores: 4.4 us for one group of 4 rows
// and 300 columns, 9 for 64 groups and 2080 columns, 51 for 8 groups of 32 and 2080 (a thread for a column, which goes over its rows: 5.7, 13, 170; 15 groups of 16 rows and 7 columns 28, so 5).
template <int ROWS>
__global__ __launch_bounds__(SHARED_THREADS) void shared_pages_kernel(SharedArgs a) {
    constexpr int WAVES = SHARED_THREADS / 64, COLS = SHARED_THREADS / ROWS;
    static_assert(WAVES * SHARED_STEPS == 64, "a lane for each of the waves' sums");
    __shared__ __attribute__((aligned(16))) int32_t entry[WAVES][SHARED_STEPS][64];
    __shared__ int32_t len[BEAM_WIDTH], sums[2][SHARED_STEPS * WAVES], broken;
    const int tid = threadIdx.x, group = blockIdx.x, row0 = group * a.width, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = lane & (ROWS - 1);
    if (tid < BEAM_WIDTH) len[tid] = tid < a.width ? clampi(a.lens[row0 + tid], 0, a.max_len) : 0;
    if (tid == 0) broken = 0x7fffffff;                     // the first entry that some row does not attend to as a whole
    __syncthreads();
    const uint64_t with = __ballot(lane < BEAM_WIDTH && len[lane & (BEAM_WIDTH - 1)] > 0);
    const uint32_t everyone = (uint32_t)with;
    const int own = len[lane & (BEAM_WIDTH - 1)], mine = b < a.width ? pages_of(len[b]) : 0;
    const int most = over_lanes(own, [](int x, int y) { return max(x, y); }), least = over_lanes(own > 0 ? own : 0x7fffffff, [](int x, int y) { return min(x, y); });
    const int32_t* const table = a.table + (int64_t)(row0 + min(b, a.width - 1)) * a.max_pages;
    i32x4* const list = reinterpret_cast<i32x4*>(a.entries) + (int64_t)group * a.max_entries;
    const int columns = pages_of(most);
    int64_t found = 0;
    int32_t next[SHARED_STEPS];
    auto request = [&](int c0) {
#pragma unroll
        for (int j = 0; j < SHARED_STEPS; ++j) {
            const int col = c0 + j * COLS + tid / ROWS;
            next[j] = col < mine ? table[col] : -1;
        }
    };
    request(0);
    for (int c0 = 0, which = 0; c0 < columns; c0 += SHARED_STEPS * COLS, which ^= 1) {
        int32_t e[SHARED_STEPS];
#pragma unroll
        for (int j = 0; j < SHARED_STEPS; ++j) {
            e[j] = (uint32_t)next[j] < (uint32_t)a.n_pages ? next[j] : -1;
            entry[wave][j][lane] = e[j];
        }
        request(c0 + SHARED_STEPS * COLS);
        lds_of_wave();
        uint32_t holders[SHARED_STEPS];
        uint64_t leads[SHARED_STEPS];
#pragma unroll
        for (int j = 0; j < SHARED_STEPS; ++j) {
            const int mates = lane & ~(ROWS - 1);
            const uint64_t there = __ballot(e[j] >= 0);
            if (there == 0) holders[j] = 0;
            else if (__all(e[j] < 0 || e[j] == entry[wave][j][mates])) holders[j] = (uint32_t)(there >> mates) & (uint32_t)((1ull << ROWS) - 1);   // (a common prompt's)
            else holders[j] = holders_of<ROWS>(&entry[wave][j][mates], e[j]);
            leads[j] = __ballot(e[j] >= 0 && (holders[j] & ((1u << b) - 1)) == 0);
            if (lane == 0) sums[which][j * WAVES + wave] = __popcll(leads[j]);
        }
        __syncthreads();                                   // (entry is the wave's own; sums of the step after the next wait for this one's readers at the next barrier)
        int x = sums[which][lane];
        const int own_sum = x;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(x, o);
            if (lane >= o) x += y;
        }
#pragma unroll
        for (int j = 0; j < SHARED_STEPS; ++j) {
            const int64_t at = found + __shfl(x - own_sum, j * WAVES + wave) + lanes_before(leads[j]);
            const int col = c0 + j * COLS + tid / ROWS;
            const bool is = leads[j] >> lane & 1;
            if (is && at < a.max_entries) list[at] = i32x4{e[j], col, (int)holders[j], 0};
            const uint64_t bad = __ballot(is && (holders[j] != everyone || (int64_t)(col + 1) * PAGE > least));
            if (bad && lane == __builtin_ctzll(bad)) atomicMin(&broken, (int)min(at, (int64_t)0x7fffffff));
        }
        found += __builtin_amdgcn_readlane(x, 63);
    }
    __syncthreads();
    if (tid == 0) {
        const int n = (int)min(found, (int64_t)a.max_entries);
        a.count[group * 2] = n;
        a.count[group * 2 + 1] = min(n, broken);
    }
}

}  // namespace cusa
