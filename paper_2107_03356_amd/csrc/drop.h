// Dropout's mask on the device (dropout.hip, residual_fwd.h, residual_bwd.h): formed from a counter where it is
// used, forward and backward, and never stored.
//
// Philox 4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): ten rounds of
// two 32 x 32 bit products turn a counter of four words into four words. One block serves eight
// neighbouring values, 16 bits each: with the 20 products, which the vector units do at a quarter of their rate, four
// values a block would take longer than the memory's traffic of 16-bit values. A value is kept where its 16 bits are
// at least T = round(65536 p), so the probability is a multiple of 2^-16 and the factor 65536 / (65536 - T) is that of
// the probability that is meant by it: the expectation is exact.
#pragma once

#include "train_util.h"

namespace mfac {
namespace {

struct DropKey {
    unsigned k0, k1, c2, c3;   // seed, offset
};
// at: seed and offset in device memory, so that a captured graph takes what they hold when it is replayed.
__device__ __forceinline__ DropKey drop_key(const Drop& d) {
    const uint64_t seed = (uint64_t)d.at[0], offset = (uint64_t)d.at[1];
    return {(unsigned)seed, (unsigned)(seed >> 32), (unsigned)offset, (unsigned)(offset >> 32)};
}

// Columns 8 group .. + 7 of a row: kept values times d.scale, others 0 (an infinity or a NaN too). `beside`: values that become
// 0 with them, unscaled.
__device__ __forceinline__ f8 drop8(const Drop& d, const DropKey& k, unsigned row, unsigned group, f8 v, f8* beside = nullptr) {
    unsigned c0 = group, c1 = row, c2 = k.c2, c3 = k.c3, k0 = k.k0, k1 = k.k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (unsigned)(b >> 32) ^ c1 ^ k0;
        c1 = (unsigned)b;
        c2 = (unsigned)(a >> 32) ^ c3 ^ k1;
        c3 = (unsigned)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const unsigned w[4] = {c0, c1, c2, c3};
    f8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool keep = (i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu) >= d.threshold;
        r[i] = keep ? v[i] * d.scale : 0.f;
        if (beside) (*beside)[i] = keep ? (*beside)[i] : 0.f;
    }
    return r;
}

}  // namespace
}  // namespace mfac
