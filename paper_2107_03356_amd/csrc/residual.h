// Shared by the kernels of what lies between two blocks (residual_fwd.h, residual_bwd.h): which norms there are,
// parameters, the ends of rows, the threads that a row takes.
#pragma once

#include <algorithm>

#include "drop.h"
#include "internal.h"
#include "row_util.h"
#include "train.h"

namespace mfac {

template <typename T>
hipError_t residual_fwd(int wt, const Residual& g, hipStream_t st);
template <typename T>
hipError_t residual_bwd(int wt, const Residual& g, const ResidualBwd& b, hipStream_t st);

namespace {

enum : int { POST_NORM = 1, PRE_NORM = 2, LAYER_NORM = 4 };   // as MFAC_NORM_*

template <int N>
using constant = std::integral_constant<int, N>;

// f(constant of the norms); what kind they are matters only where there is one.
template <typename F>
void by_norms(int norms, F f) {
    switch (norms) {
        case 1: return f(constant<1>());
        case 2: return f(constant<2>());
        case 3: return f(constant<3>());
        case 5: return f(constant<5>());
        case 6: return f(constant<6>());
        case 7: return f(constant<7>());
        default: return f(constant<0>());
    }
}

// f(constant of the threads that hold a row, eight values each). Two chunks of eight a thread take twice the registers, and
// 16384 columns by 1024 threads would spill up to 900 bytes a lane: wider rows than these have kernels of their own.
constexpr int64_t HELD_COLS = 8192;
template <typename F>
void by_threads(int64_t cols, F f) {
    if (cols <= 512) f(constant<64>());
    else if (cols <= 1024) f(constant<128>());
    else if (cols <= 2048) f(constant<256>());
    else if (cols <= 4096) f(constant<512>());
    else f(constant<1024>());
}

__device__ __forceinline__ f8 fill8(float v) { return f8{v, v, v, v, v, v, v, v}; }
__device__ __forceinline__ void zero_past(f8& v, int64_t c, int64_t cols) {
    if (c + 8 > cols)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i >= cols) v[i] = 0.f;
}
// Columns c .. c + 7 of a parameter, or `absent` where there is none.
__device__ __forceinline__ f8 load_param(const void* p, int wt, int64_t c, int64_t cols, float absent) {
    return p ? load8_dt(p, wt, 0, c, cols) : fill8(absent);
}

}  // namespace
}  // namespace mfac
