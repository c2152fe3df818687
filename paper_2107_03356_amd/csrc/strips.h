// The pieces of work of the elementwise kernels (pack8.hip, dropout.hip, gated.hip): rows narrower than a
// wave's 512 columns share it.
#pragma once

#include <algorithm>

#include "internal.h"
#include "train_util.h"

namespace mfac {
namespace {

// log2 of the lanes that a row takes in a wave.
int lanes_log2(int64_t cols) {
    int l = 2;
    while (l < 6 && (int64_t(8) << l) < cols) ++l;
    return l;
}

// A wave's pieces of work: 64 >> ll rows by 8 << ll columns.
struct Strips {
    int64_t rows, cols, nstrips, npieces;
    int ll;
};
Strips strips_of(int64_t rows, int64_t cols) {
    Strips s{rows, cols, 0, 0, lanes_log2(cols)};
    s.nstrips = ceil_div(cols, int64_t(8) << s.ll);
    s.npieces = s.nstrips * ceil_div(rows, int64_t(64) >> s.ll);
    return s;
}
unsigned strip_grid(const Strips& s) { return (unsigned)std::min<int64_t>(ceil_div(s.npieces, 4), 4096); }

template <typename F>
__device__ __forceinline__ void for_strips(const Strips& s, F f) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lr = lane >> s.ll, lc = lane & ((1 << s.ll) - 1);
    for (int64_t u = (int64_t)blockIdx.x * 4 + wave; u < s.npieces; u += (int64_t)gridDim.x * 4) {
        const int64_t rb = u / s.nstrips, sb = u - rb * s.nstrips;
        f(rb * (64 >> s.ll) + lr, (sb << (s.ll + 3)) + lc * 8);
    }
}

}  // namespace
}  // namespace mfac
