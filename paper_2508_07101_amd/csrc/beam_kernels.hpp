// Device code for beam search over paged caches: groups of rows that share pages.  (Attention over a group's pages is a form of tree_attn_kernel.)
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
    double* ln_sum;                        // [rows]: logarithm of the sum of weights; NaN: the row proposes nothing
    float* top;                            // [rows]: the largest logit
    uint64_t* best;                        // [rows][n]: keys, best first; 0: none
    int32_t rows, width, vocab, n, end_token;
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

template <int DTYPE>                       // cusa_dtype
__device__ __forceinline__ float load_logit(const void* p, int64_t at) {
    if constexpr (DTYPE == 0) return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16);
    else if constexpr (DTYPE == 1) return (float)static_cast<const _Float16*>(p)[at];
    else return static_cast<const float*>(p)[at];
}

constexpr int BEAM_THREADS = 256;

// A workgroup for a row: the largest logit, the sum of weights, then the best tokens one after the other, each in a pass of its own.
template <int DTYPE>
__global__ __launch_bounds__(BEAM_THREADS) void beam_rows_kernel(BeamArgs a) {
    __shared__ uint64_t key[BEAM_THREADS / 64];
    __shared__ double part[BEAM_THREADS / 64];
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t at = (int64_t)row * a.stride;
    auto largest = [&](uint64_t k) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) k = max(k, (uint64_t)__shfl_xor((unsigned long long)k, o));
        __syncthreads();
        if (lane == 0) key[wave] = k;
        __syncthreads();
        return max(max(key[0], key[1]), max(key[2], key[3]));
    };
    uint64_t mine = 0;
    for (int t = tid; t < a.vocab; t += BEAM_THREADS) {
        const float x = load_logit<DTYPE>(a.logits, at + t);
        if (x > -INFINITY) mine = max(mine, beam_key(x, t));
    }
    uint64_t next = largest(mine);
    const float top = next ? key_logit(next) : -INFINITY;
    double sum = 0.0;
    for (int t = tid; t < a.vocab; t += BEAM_THREADS) sum += (double)exp2f((load_logit<DTYPE>(a.logits, at + t) - top) * 1.4426950408889634f);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = part[0] + part[1] + part[2] + part[3];
    if (tid == 0) {
        a.top[row] = top;
        a.ln_sum[row] = log(sum);                          // (NaN of a NaN, of an infinity less itself, of nothing)
    }
    for (int i = 0; i < a.n; ++i) {
        if (tid == 0) a.best[(int64_t)row * a.n + i] = next;
        mine = 0;
        for (int t = tid; t < a.vocab; t += BEAM_THREADS) {
            const float x = load_logit<DTYPE>(a.logits, at + t);
            if (!(x > -INFINITY)) continue;
            const uint64_t k = beam_key(x, t);
            if (k < next) mine = max(mine, k);
        }
        next = largest(mine);
    }
}

// A workgroup for a group: a thread for every candidate of its rows at a time, and the best of all that are left, n times.
__global__ __launch_bounds__(BEAM_THREADS) void beam_merge_kernel(BeamArgs a) {
    __shared__ double value[BEAM_WIDTH * BEAM_MOST];
    __shared__ int32_t token[BEAM_WIDTH * BEAM_MOST], over[BEAM_WIDTH];
    const int group = blockIdx.x, row0 = group * a.width, all = a.width * a.n;
    for (int i = threadIdx.x; i < all; i += BEAM_THREADS) {
        const int r = row0 + i / a.n, j = i % a.n;
        const float s = a.scores[r];
        const bool ended = a.ended && a.ended[r] != 0;
        double v = -INFINITY;
        int t = -1;
        if (__builtin_isfinite(s)) {
            if (ended) {
                if (j == 0) {
                    v = s;
                    t = a.end_token;
                }
            } else if (const uint64_t k = a.best[(int64_t)r * a.n + j]; k && !__builtin_isnan(a.ln_sum[r])) {
                v = (double)s + (((double)key_logit(k) - a.top[r]) - a.ln_sum[r]);
                t = key_token(k);
            }
        }
        value[i] = v;
        token[i] = t;
        if (j == 0) over[i / a.n] = ended;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < all; i += BEAM_THREADS) {
        const double v = value[i];
        if (!(v > -INFINITY)) continue;
        int rank = 0;                                      // candidates that come before this one
        for (int j = 0; j < all; ++j) rank += value[j] > v || (value[j] == v && j < i);   // (a row's own come in order: beside a large score 64 bits may not tell them apart)
        if (rank >= a.n) continue;
        const int64_t to = (int64_t)group * a.n + rank;
        a.out_scores[to] = (float)v;
        a.parents[to] = i / a.n;
        a.tokens[to] = token[i];
        if (a.out_ended) a.out_ended[to] = over[i / a.n] || token[i] == a.end_token;
    }
    int there = 0;
    for (int j = 0; j < all; ++j) there += value[j] > -INFINITY;
    for (int i = there + threadIdx.x; i < a.n; i += BEAM_THREADS) {
        const int64_t to = (int64_t)group * a.n + i;
        a.out_scores[to] = -INFINITY;
        a.parents[to] = a.tokens[to] = -1;
        if (a.out_ended) a.out_ended[to] = 0;
    }
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
    int32_t *counts, *freed;               // of each (group, FORK_COLS columns): how many pages go back, and which
    int32_t batch, width, max_pages, n_pages, cap, grow, chunks;
};
constexpr int FORK_COLS = 256;

// A thread for each row, as many whole groups at a time as 1024 hold.
__global__ __launch_bounds__(PLAN_THREADS) void kv_fork_kernel(ForkArgs a) {
    __shared__ int64_t scratch[2][2][PLAN_THREADS / 64];
    __shared__ int32_t s_src[PLAN_THREADS], s_had[PLAN_THREADS], s_page[PLAN_THREADS], s_col[PLAN_THREADS], s_need[PLAN_THREADS];
    const int tid = threadIdx.x, round = PLAN_THREADS / a.width * a.width, mate0 = tid - tid % a.width;
    int first = a.state[0];
    const int avail = clampi(a.state[1], 0, a.n_pages);
    if ((uint32_t)first >= (uint32_t)a.n_pages) first = 0;
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
        s_src[tid] = src;
        s_had[tid] = pages_of(kept);
        s_page[tid] = open ? page : -1;
        s_col[tid] = col;
        __syncthreads();
        bool copy = false;
        if (open) {
            int holders = 0, writers = 0;
            bool lowest = true;
            for (int t = mate0; t < mate0 + a.width; ++t) {
                if (s_src[t] < 0 || s_had[t] <= col) continue;
                const bool writes = s_col[t] == col && s_page[t] == page;
                writers += writes;
                holders += writes || a.table[(int64_t)s_src[t] * a.max_pages + col] == page;
                if (writes && t < tid) lowest = false;
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
            a.rows[b] = ok ? ForkRow{parent < 0 || parent >= a.width ? -1 : parent, pages_of(kept), pages_of(held), takes ? col : -1, id}
                           : ForkRow{tid - mate0, pages_of(held), pages_of(held), -1, -1};
        }
        __syncthreads();
    }
    if (tid == 0) {
        *a.head = ForkHead{first, avail, (int)taken};
        a.state_out[0] = (int)ring_at((int64_t)first + taken, a.n_pages);
    }
}

// A thread for a column of a group: it reads the column of all rows before it writes any, so that the tables may be changed in place.
__global__ __launch_bounds__(FORK_COLS) void fork_tables_kernel(ForkArgs a) {
    __shared__ int32_t entry[BEAM_WIDTH][FORK_COLS];
    __shared__ ForkRow rows[BEAM_WIDTH];
    __shared__ int32_t sums[FORK_COLS / 64];
    const int tid = threadIdx.x, group = blockIdx.y, row0 = group * a.width, col = blockIdx.x * FORK_COLS + tid, lane = tid & 63, wave = tid >> 6;
    if (tid < a.width) rows[tid] = a.rows[row0 + tid];
    __syncthreads();
    uint32_t alive = 0;                                    // rows that somebody descends from
    int most = 0;
    for (int b = 0; b < a.width; ++b) {
        if (rows[b].src >= 0) alive |= 1u << rows[b].src;
        most = max(most, max(rows[b].old, max(rows[b].had, rows[b].col + 1)));
    }
    const int64_t chunk = (int64_t)group * a.chunks + blockIdx.x;
    if ((int)blockIdx.x * FORK_COLS >= most) {
        if (tid == 0) a.counts[chunk] = 0;
        return;
    }
    const int32_t* const from = a.table + (int64_t)row0 * a.max_pages + col;
    for (int b = 0; b < a.width; ++b) entry[b][tid] = col < rows[b].old ? from[(int64_t)b * a.max_pages] : -1;
    int32_t* const to = a.table_out + (int64_t)row0 * a.max_pages + col;
    for (int b = 0; b < a.width; ++b) {
        const ForkRow& r = rows[b];
        if (col == r.col) to[(int64_t)b * a.max_pages] = r.page;
        else if (r.src >= 0 && col < r.had) to[(int64_t)b * a.max_pages] = entry[r.src][tid];
    }
    uint32_t gone = 0;
    for (int b = 0; b < a.width; ++b) {
        const int32_t e = entry[b][tid];
        if ((alive >> b & 1) || (uint32_t)e >= (uint32_t)a.n_pages) continue;
        bool last = true;                                  // nobody who stays holds it, and no row before this one did
        for (int o = 0; o < a.width; ++o) last &= !(entry[o][tid] == e && ((alive >> o & 1) || o < b));
        if (last) gone |= 1u << b;
    }
    const int n = __popc(gone);
    int x = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    int at = x - n, total = 0;
#pragma unroll
    for (int w = 0; w < FORK_COLS / 64; ++w) {
        if (w < wave) at += sums[w];
        total += sums[w];
    }
    int32_t* const list = a.freed + chunk * FORK_COLS * a.width;
    for (; gone; gone &= gone - 1) list[at++] = entry[__builtin_ctz(gone)][tid];
    if (tid == 0) a.counts[chunk] = total;
}

__global__ __launch_bounds__(PLAN_THREADS) void fork_pages_kernel(ForkArgs a) {
    __shared__ int64_t scratch[2][2][PLAN_THREADS / 64], start[PLAN_THREADS];
    __shared__ int32_t number[PLAN_THREADS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, chunks = a.batch / a.width * a.chunks;
    const ForkHead h = *a.head;
    int64_t pushed = 0;
    int which = 0;
    for (int base = 0; base < chunks; base += PLAN_THREADS, which ^= 1) {
        const int n = base + tid < chunks ? a.counts[base + tid] : 0;
        int64_t sum;
        const int64_t before = pushed + plan_scan(n, sum, scratch[which], PLAN_THREADS / 64);
        start[tid] = before;
        number[tid] = n;
        __syncthreads();
        if (sum) {
            for (int i = wave; i < PLAN_THREADS; i += PLAN_THREADS / 64) {
                const int32_t* const list = a.freed + (int64_t)(base + i) * FORK_COLS * a.width;
                for (int j = lane; j < number[i]; j += 64) a.ring[ring_at((int64_t)h.first + h.avail + start[i] + j, a.n_pages)] = list[j];
            }
        }
        pushed += sum;
        __syncthreads();
    }
    if (tid == 0) a.state_out[1] = (int)min((int64_t)h.avail - h.taken + pushed, (int64_t)a.n_pages);
}

// ---------------------------------------------------------------- copy

constexpr int COPY_LAYERS = 40;            // layers of a launch: their descriptors travel as arguments (4 KB at most)
constexpr int COPY_THREADS = 256;

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

// A workgroup for a copy in a layer: 16 lanes a row of 256 bytes.
__global__ __launch_bounds__(COPY_THREADS) void kv_copy_kernel(CopyArgs a) {
    const CopyLayer& l = a.layer[blockIdx.y];
    const int32_t* const c = a.copies + (int64_t)blockIdx.x * 4;
    const int from = c[0], to = c[1], n = min(c[2], PAGE);
    if ((uint32_t)from >= (uint32_t)l.n_pages || (uint32_t)to >= (uint32_t)l.n_pages || from == to) return;
    const int64_t page = (int64_t)a.G * PAGE * D;
    for (int i = threadIdx.x; i < 2 * a.G * PAGE * 16; i += COPY_THREADS) {
        const int row = i >> 4, token = row & (PAGE - 1);
        if (token >= n) continue;
        uint16_t* const pool = row < a.G * PAGE ? l.k : l.v;
        const int64_t at = (int64_t)(row < a.G * PAGE ? row : row - a.G * PAGE) * D + (i & 15) * 8;
        *reinterpret_cast<u32x4*>(pool + to * page + at) = *reinterpret_cast<const u32x4*>(pool + from * page + at);
    }
}

// ---------------------------------------------------------------- pages of groups

struct SharedArgs {
    const int32_t *table, *lens;
    int32_t *entries, *count;
    int32_t batch, width, max_pages, n_pages, max_len, max_entries;
};
constexpr int SHARED_COLS = 256;

// A workgroup for a group, a thread for a column.
__global__ __launch_bounds__(SHARED_COLS) void shared_pages_kernel(SharedArgs a) {
    __shared__ int32_t entry[BEAM_WIDTH][SHARED_COLS], len[BEAM_WIDTH], sums[SHARED_COLS / 64], broken;
    const int tid = threadIdx.x, group = blockIdx.x, row0 = group * a.width, lane = tid & 63, wave = tid >> 6;
    if (tid < a.width) len[tid] = clampi(a.lens[row0 + tid], 0, a.max_len);
    if (tid == 0) broken = 0x7fffffff;                     // the first entry that some row does not attend to as a whole
    __syncthreads();
    uint32_t everyone = 0;
    int least = 0x7fffffff, most = 0;
    for (int b = 0; b < a.width; ++b) {
        if (len[b] == 0) continue;
        everyone |= 1u << b;
        least = min(least, len[b]);
        most = max(most, len[b]);
    }
    i32x4* const list = reinterpret_cast<i32x4*>(a.entries) + (int64_t)group * a.max_entries;
    int64_t found = 0;
    for (int c0 = 0; c0 < pages_of(most); c0 += SHARED_COLS) {
        const int col = c0 + tid;
        for (int b = 0; b < a.width; ++b) {
            const int32_t e = col < pages_of(len[b]) ? a.table[(int64_t)(row0 + b) * a.max_pages + col] : -1;
            entry[b][tid] = (uint32_t)e < (uint32_t)a.n_pages ? e : -1;
        }
        uint32_t leads = 0;
        for (int b = 0; b < a.width; ++b) {
            const int32_t e = entry[b][tid];
            bool first = e >= 0;
            for (int o = 0; o < b; ++o) first &= entry[o][tid] != e;
            if (first) leads |= 1u << b;
        }
        const int n = __popc(leads);
        int x = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(x, o);
            if (lane >= o) x += y;
        }
        if (lane == 63) sums[wave] = x;
        __syncthreads();
        int64_t at = found + x - n;
        for (int w = 0; w < SHARED_COLS / 64; ++w) {
            if (w < wave) at += sums[w];
            found += sums[w];
        }
        for (; leads; leads &= leads - 1, ++at) {
            const int32_t e = entry[__builtin_ctz(leads)][tid];
            uint32_t holders = 0;
            for (int b = 0; b < a.width; ++b)
                if (entry[b][tid] == e) holders |= 1u << b;
            if (at < a.max_entries) list[at] = i32x4{e, col, (int)holders, 0};
            if (holders != everyone || (int64_t)(col + 1) * PAGE > least) atomicMin(&broken, (int)min(at, (int64_t)0x7fffffff));
        }
        __syncthreads();
    }
    if (tid == 0) {
        const int n = (int)min(found, (int64_t)a.max_entries);
        a.count[group * 2] = n;
        a.count[group * 2 + 1] = min(n, broken);
    }
}

}  // namespace cusa
