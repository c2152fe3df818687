// Device helpers shared by the kernels that hold a row in the registers of NT threads (norm.hip,
// residual_fwd.h, residual_bwd.h): sums over a row.
#pragma once

#include "train_util.h"

namespace mfac {
namespace {

// Sum over the NT threads that hold a row. red: two sets of NT / 64 words in
// turn, so that one barrier a sum is enough.
template <int NT>
__device__ __forceinline__ float row_sum(float v, float* red, int& turn) {
    v = wave_sum(v);
    if constexpr (NT == 64) return v;
    constexpr int NW = NT / 64;
    float* r = red + turn * NW;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) s += r[i];
    return s;
}
// The same for two sums at once.
template <int NT>
__device__ __forceinline__ void row_sum2(float& a, float& b, float* red, int& turn) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (NT == 64) return;
    constexpr int NW = NT / 64;
    float* r = red + turn * 2 * NW;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) {
        r[threadIdx.x >> 6] = a;
        r[NW + (threadIdx.x >> 6)] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        a += r[i];
        b += r[NW + i];
    }
}

constexpr int norm_block(int nt) { return nt == 64 ? 256 : nt; }

}  // namespace
}  // namespace mfac
