// What the kernels that plan pages share: sums over a workgroup in order, places of the queue.
#pragma once
#include "cache_view.hpp"

namespace cusa {

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ int pages_of(int tokens) { return (int)(((int64_t)tokens + PAGE - 1) / PAGE); }

constexpr int PLAN_THREADS = 1024;

// Sums over the workgroup's threads before this one, of two values at once; total: of all.  Only the first `waves` waves hold values.  scratch: two words
// for each wave, not in use by the call before.
__device__ __forceinline__ void plan_scan(int64_t (&v)[2], int64_t (&total)[2], int64_t (*scratch)[PLAN_THREADS / 64], int waves) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t x[2] = {v[0], v[1]};
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y0 = __shfl_up(x[0], o), y1 = __shfl_up(x[1], o);
        if (lane >= o) {
            x[0] += y0;
            x[1] += y1;
        }
    }
    if (lane == 63) {
        scratch[0][wave] = x[0];
        scratch[1][wave] = x[1];
    }
    __syncthreads();
    int64_t before[2] = {0, 0}, all[2] = {0, 0};
#pragma unroll 1
    for (int w = 0; w < waves; ++w) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (w == wave) before[i] = all[i];
            all[i] += scratch[i][w];
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[i] = (wave < waves ? before[i] : all[i]) + x[i] - v[i];
        total[i] = all[i];
    }
}
__device__ __forceinline__ int64_t plan_scan(int64_t v, int64_t& total, int64_t (*scratch)[PLAN_THREADS / 64], int waves) {
    int64_t x[2] = {v, 0}, t[2];
    plan_scan(x, t, scratch, waves);                     // (what is not used is not computed)
    total = t[0];
    return x[0];
}
// A place of the queue, which has n entries, from a number that is mostly below 2 n (the division of 64 bits is long).
__device__ __forceinline__ int64_t ring_at(int64_t x, int64_t n) {
    if (x >= n) x -= n;
    if (x >= n) x %= n;
    return x;
}

}  // namespace cusa
