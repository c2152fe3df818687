// 8-bit copies of activations, and the activation's part of the backward pass:
//
//   q = rint(x 2^-e), e by groups of 32 columns; x ~ q 2^e
//   dz = dy act'(z), a = act(z), db = sum over rows of dz
//
// A lane holds eight neighbouring columns, so four lanes hold a group and find its
// largest magnitude with two exchanges. Rows narrower than a wave's 512 columns
// share it: LPR lanes to a row, the power of two from 4 to 64 that covers
// the row. All of it is elementwise and bound by HBM: bf16 8192 x 8192 into the copy 36 us launch
// after launch (5.6 TB/s) and 41 after a pass that leaves its output in the caches (4.9), back 35
// and 32, dz and db from an 8-bit z 66 with gelu_tanh (5.1) and 78 with gelu, whose arithmetic it waits for.
#include <algorithm>

#include "internal.h"
#include "train.h"
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

template <typename T>
__global__ __launch_bounds__(256) void k_pack8(Strips s, const T* __restrict__ x, int64_t ldx, Packed p,
                                               int64_t ngroups) {
    for_strips(s, [&](int64_t row, int64_t c) {
        const bool in = row < s.rows;   // the exchanges below need every lane of the wave
        f8 v = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (in) v = load8(x + row * ldx, c, s.cols);
        pack_group(p.q + row * p.ldq, p.s + row * ngroups, in ? c : s.cols, s.cols, v);
    });
}

template <typename T>
__global__ __launch_bounds__(256) void k_unpack8(Strips s, Packed p, int64_t ngroups, T* __restrict__ y, int64_t ldy) {
    for_strips(s, [&](int64_t row, int64_t c) {
        if (row >= s.rows || c >= s.cols) return;
        f8 v = load_packed8(p.q + row * p.ldq, p.s + row * ngroups, c, s.cols);
        if constexpr (sizeof(T) == 2 && !std::is_same_v<T, bf16>)
#pragma unroll
            for (int i = 0; i < 8; ++i)   // a NaN stays one
                v[i] = v[i] > 65504.f ? 65504.f : v[i] < -65504.f ? -65504.f : v[i];
        store8(y + row * ldy, c, s.cols, v);
    });
}

template <typename T>
__global__ __launch_bounds__(256) void k_zero_matrix(Strips s, T* __restrict__ y, int64_t ldy) {
    for_strips(s, [&](int64_t row, int64_t c) {
        if (row < s.rows && c < s.cols) store8(y + row * ldy, c, s.cols, f8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f});
    });
}

// ---------------------------------------------------------------- activation, backward
template <typename T>
__device__ __forceinline__ void load_z(Raw8<T>& v, const T* z, int64_t ldz, Packed, int64_t, int64_t r, int64_t c,
                                       int64_t cols) {
    v.load(z + r * ldz, c, cols);
}
template <typename T>
__device__ __forceinline__ void load_z(RawPacked8& v, const T*, int64_t, Packed p, int64_t ngroups, int64_t r, int64_t c,
                                       int64_t cols) {
    v.load(p.q + r * p.ldq, p.s + r * ngroups, c, cols);
}

// dz is rounded to the operands' type, which is what the products on the matrix cores take:
// in bf16 dx and dW are then 2.1e-3 to 2.6e-3 from 64 bits (relative, 2-norm) against 1.7e-3
// for their own rounding alone. Two bf16 parts of dz would keep that and double both
// products. db is summed before the rounding.
// Work-group (strip blockIdx.x, part blockIdx.y): its rows part, part + nparts, ... of
// the strip's columns, by wave and sub-row; the column sums in registers, joined
// over the waves and sub-rows at the end.
template <typename T, int ZP>   // z: 0 none, 1 of type T, 2 an 8-bit copy
__global__ __launch_bounds__(256) void k_act_bwd(Strips s, int act, const T* dy, int64_t lddy, const T* z, int64_t ldz,
                                                 Packed p, int64_t ngroups, T* dz, int64_t lddz, T* a, int64_t lda,
                                                 float* part) {
    __shared__ float sums[256 * 8];
    const int lane = threadIdx.x & 63, rpw = 64 >> s.ll;
    const int lc = lane & ((1 << s.ll) - 1);
    const int64_t c = ((int64_t)blockIdx.x << (s.ll + 3)) + lc * 8;
    const int64_t sub = (int64_t)(threadIdx.x >> 6) * rpw + (lane >> s.ll), nsub = 4 * rpw;
    f8 sum = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    with_act(ZP ? act : 0, [&](auto tag) {
        constexpr int ACT = decltype(tag)::value;
        if (c >= s.cols) return;
        const int64_t step = gridDim.y * nsub;
        int64_t row = blockIdx.y * nsub + sub;
        // the next row is on its way while this one is worked on
        Raw8<T> d_next;
        std::conditional_t<ZP == 2, RawPacked8, Raw8<T>> z_next;
        auto load = [&](int64_t r) {
            d_next.load(dy + r * lddy, c, s.cols);
            if constexpr (ACT != 0) load_z(z_next, z, ldz, p, ngroups, r, c, s.cols);
        };
        if (row < s.rows) load(row);
        for (; row < s.rows; row += step) {
            f8 d = d_next.get(), v{};
            if constexpr (ACT != 0) v = z_next.get();
            if (row + step < s.rows) load(row + step);
            if constexpr (ACT != 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float av;
                    d[i] *= act_slope<ACT>(v[i], &av);
                    v[i] = av;
                }
                if (a) store8(a + row * lda, c, s.cols, v);
            }
            sum += d;
            if (dz) store8(dz + row * lddz, c, s.cols, d);
        }
    });
    if (!part) return;
    *reinterpret_cast<f8*>(&sums[threadIdx.x * 8]) = sum;
    __syncthreads();
    if (threadIdx.x < (1u << s.ll)) {
        for (int r = 1; r < nsub; ++r) sum += *reinterpret_cast<const f8*>(&sums[((r << s.ll) + lc) * 8]);
        store8(part + (int64_t)blockIdx.y * s.cols, c, s.cols, sum);
    }
}

// ---------------------------------------------------------------- joining column sums
// A work-group holds 64 columns; its 16 waves take every 16th part each, and their
// sums are joined in order. blockIdx.y: the first or the second of two outputs.
template <typename TO>
__global__ __launch_bounds__(1024) void k_column_sums(const float* __restrict__ part, int64_t nparts, int64_t stride,
                                                      int64_t cols, TO* out_a, TO* out_b) {
    __shared__ float s[16][64];
    TO* out = blockIdx.y ? out_b : out_a;
    if (!out) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float v = 0.f;
    if (c < cols) {
        const float* p = part + blockIdx.y * cols + c;
#pragma unroll 8
        for (int64_t i = wave; i < nparts; i += 16) v += p[i * stride];
    }
    s[wave][lane] = v;
    __syncthreads();
    if (wave == 0 && c < cols) {
#pragma unroll
        for (int w = 1; w < 16; ++w) v += s[w][lane];
        out[c] = (TO)v;
    }
}

template <typename F>
hipError_t by_type(int dt, F f) {
    if (dt == DT_F32) return f((float*)nullptr);
    if (dt == DT_BF16) return f((bf16*)nullptr);
    return f((f16*)nullptr);
}

}  // namespace

hipError_t launch_pack8(int dt, int64_t rows, int64_t cols, const void* x, int64_t ldx, Packed p, hipStream_t st) {
    const Strips s = strips_of(rows, cols);
    return by_type(dt, [&](auto* t) {
        using T = std::remove_reference_t<decltype(*t)>;
        k_pack8<T><<<strip_grid(s), 256, 0, st>>>(s, (const T*)x, ldx, p, ceil_div(cols, 32));
        return hipGetLastError();
    });
}

hipError_t launch_unpack8(int dt, int64_t rows, int64_t cols, Packed p, void* y, int64_t ldy, hipStream_t st) {
    const Strips s = strips_of(rows, cols);
    return by_type(dt, [&](auto* t) {
        using T = std::remove_reference_t<decltype(*t)>;
        k_unpack8<T><<<strip_grid(s), 256, 0, st>>>(s, p, ceil_div(cols, 32), (T*)y, ldy);
        return hipGetLastError();
    });
}

hipError_t launch_zero_matrix(int dt, int64_t rows, int64_t cols, void* y, int64_t ldy, hipStream_t st) {
    const Strips s = strips_of(rows, cols);
    return by_type(dt, [&](auto* t) {
        using T = std::remove_reference_t<decltype(*t)>;
        k_zero_matrix<T><<<strip_grid(s), 256, 0, st>>>(s, (T*)y, ldy);
        return hipGetLastError();
    });
}

// Parts: as many as give about 2048 work-groups, at most one for each row that a work-group has at a time; one for
// up to eight rows to each of them, whose sums are then db without a launch that joins parts.
int64_t act_bwd_parts(int64_t rows, int64_t cols) {
    const Strips s = strips_of(rows, cols);
    const int64_t nsub = 4 * (64 >> s.ll);
    if (rows <= 8 * nsub) return 1;
    return std::min(ceil_div(rows, nsub), ceil_div(2048, s.nstrips));
}

hipError_t launch_act_bwd(int dt, int act, int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* z,
                          int64_t ldz, Packed p, void* dz, int64_t lddz, void* a, int64_t lda, float* db, float* part,
                          hipStream_t st) {
    const Strips s = strips_of(rows, cols);
    const int64_t ng = ceil_div(cols, 32), nparts = rows > 0 ? act_bwd_parts(rows, cols) : 0;
    if (!db) part = nullptr;
    else if (nparts == 1) part = db;
    if (rows > 0) {
        const dim3 grid((unsigned)s.nstrips, (unsigned)nparts);
        const hipError_t e = by_type(dt, [&](auto* t) {
            using T = std::remove_reference_t<decltype(*t)>;
#define LAUNCH(ZP)                                                                                            \
    k_act_bwd<T, ZP><<<grid, 256, 0, st>>>(s, act, (const T*)dy, lddy, (const T*)z, ldz, p, ng, (T*)dz, lddz, \
                                           (T*)a, lda, part)
            if (act == 0) LAUNCH(0);
            else if (p.q) LAUNCH(2);
            else LAUNCH(1);
#undef LAUNCH
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    return db && nparts != 1 ? launch_column_sums(part, nparts, cols, cols, DT_F32, db, nullptr, st) : hipSuccess;
}

hipError_t launch_column_sums(const float* part, int64_t nparts, int64_t stride, int64_t cols, int out_dt, void* out_a,
                              void* out_b, hipStream_t st) {
    return by_type(out_dt, [&](auto* t) {
        using T = std::remove_reference_t<decltype(*t)>;
        k_column_sums<T><<<dim3((unsigned)ceil_div(cols, 64), out_b ? 2 : 1), 1024, 0, st>>>(part, nparts, stride, cols,
                                                                                           (T*)out_a, (T*)out_b);
        return hipGetLastError();
    });
}

}  // namespace mfac
