// Shared by the kernels of what lies between two blocks (residual_fwd.h, residual_bwd.h): which norms there are, the
// threads that a row takes, rows of any length eight values at a time, parameters.
#pragma once

#include <algorithm>

#include "drop.h"
#include "internal.h"
#include "row_util.h"
#include "train.h"

namespace mfac {

int64_t residual_bwd_grid(int dt, int norms, int64_t rows, int64_t cols);   // work-groups, each with its column sums
template <typename T>
hipError_t residual_fwd(int wt, const Residual& g, hipStream_t st);
template <typename T>
hipError_t residual_bwd(int wt, const Residual& g, const ResidualBwd& b, hipStream_t st);

namespace {

enum : int { POST_NORM = 1, PRE_NORM = 2, LAYER_NORM = 4 };   // as MFAC_NORM_*
enum : int { NOTHING_BETWEEN = 8 };   // backward, with PRE_NORM alone: no gate, no dropout

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
        case PRE_NORM | NOTHING_BETWEEN: return f(constant<PRE_NORM | NOTHING_BETWEEN>());
        case PRE_NORM | LAYER_NORM | NOTHING_BETWEEN: return f(constant<PRE_NORM | LAYER_NORM | NOTHING_BETWEEN>());
        default: return f(constant<0>());
    }
}

// Wider rows, whose values would be past the registers, have kernels of their own, which rows of fewer than eight values run
// through as well.
inline bool in_registers(int64_t cols) { return cols >= 8 && cols <= 8192; }
// Chunks of eight values that a thread of the backward pass has (see by_threads_bwd).
constexpr int residual_chunks(bool fp32, bool one) { return fp32 || one ? 1 : 2; }
// The first row of this thread's wave, as a scalar: addresses of rows are then scalars too.
template <int NT>
__device__ __forceinline__ int64_t first_row() {
    constexpr int RPB = norm_block(NT) / NT;
    if constexpr (RPB == 1) return blockIdx.x;
    return (int64_t)blockIdx.x * RPB + __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
}

__device__ __forceinline__ f8 fill8(float v) { return f8{v, v, v, v, v, v, v, v}; }
__device__ __forceinline__ void zero_past(f8& v, int64_t c, int64_t cols) {
    if (c + 8 > cols)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i >= cols) v[i] = 0.f;
}

// Eight neighbouring values of a row as loaded, where a row has at least eight: the thread at the row's end loads the last eight
// and moves what is its own to the front, zeros behind it, which takes no branch and no address of its own for each value.
struct Place {
    unsigned at;  // of the load
    int shift;    // values in it that are another thread's, 8: all
    bool ragged;  // some thread of the wave has one to seven of them
    bool past;    // some thread has eight
};
__device__ __forceinline__ Place place_of(int c, int64_t cols) {
    const int at = min(c, (int)cols - 8), shift = min(c - at, 8);
    return {(unsigned)at, shift, __any(shift % 8 != 0) != 0, __any(shift == 8) != 0};
}
template <int N>
struct Words {
    typedef unsigned type __attribute__((ext_vector_type(N)));
};
// N words, `by` words (0 to N) towards the front.
template <int N>
__device__ __forceinline__ typename Words<N>::type move_words(typename Words<N>::type w, int by) {
#pragma unroll
    for (int step = N; step > 0; step /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = by & step ? (i + step < N ? w[i + step] : 0u) : w[i];
    return w;
}
template <typename T>
struct Row8 {
    static constexpr int N = 2 * sizeof(T);
    typename Words<N>::type w;
    __device__ __forceinline__ void load(const T* __restrict__ row, const Place& p) {
        const typename VecOf<T, 8>::plain v = *reinterpret_cast<const typename VecOf<T, 8>::type*>(row + p.at);
        w = __builtin_bit_cast(typename Words<N>::type, v);
    }
    // of an 8-bit copy: q, and the group's byte in the third word
    __device__ __forceinline__ void load_copy(const int8_t* __restrict__ q, const uint8_t* __restrict__ s, int c,
                                              const Place& p) {
        const Bytes8 b = *reinterpret_cast<const Bytes8*>(q + p.at);
        w[0] = b.lo;
        w[1] = b.hi;
        w[2] = s[min((unsigned)c, p.at + 7) >> 5];   // a thread past the end reads the last
    }
    // The values. Moved here and not where they are loaded, which would wait for them there.
    __device__ __forceinline__ f8 get(const Place& p) const {
        typename Words<N>::type m = w;
        if (p.ragged) {
            if constexpr (sizeof(T) == 4) {
                m = move_words<N>(m, p.shift);
            } else {
                m = move_words<N>(m, p.shift / 2);
                if (p.shift & 1)
#pragma unroll
                    for (int i = 0; i < N; ++i) m[i] = __builtin_amdgcn_alignbit(i + 1 < N ? m[i + 1] : 0u, m[i], 16);
            }
        } else if (p.past) {
#pragma unroll
            for (int i = 0; i < N; ++i) m[i] = p.shift ? 0u : m[i];
        }
        return __builtin_convertvector(__builtin_bit_cast(typename VecOf<T, 8>::plain, m), f8);
    }
    __device__ __forceinline__ f8 get_copy(const Place& p) const {
        uint64_t v = (uint64_t)w[1] << 32 | w[0];
        if (p.ragged || p.past) v = p.shift < 8 ? v >> (8 * p.shift) : 0;
        return RawPacked8{{(unsigned)v, (unsigned)(v >> 32)}, w[2]}.get();
    }
};

// Columns c .. c + 7 of a parameter of type wt, T or fp32, or `absent` where there is none.
template <typename T>
__device__ __forceinline__ f8 load_param(const void* p, int wt, const Place& at, float absent) {
    if (!p) return fill8(absent);
    if (wt == DT_F32) {
        Row8<float> v;
        v.load((const float*)p, at);
        return v.get(at);
    }
    Row8<T> v;
    v.load((const T*)p, at);
    return v.get(at);
}
__device__ __forceinline__ f8 load_param(const void* p, int wt, int64_t c, int64_t cols, float absent) {
    return p ? load8_dt(p, wt, 0, c, cols) : fill8(absent);
}

}  // namespace
}  // namespace mfac
