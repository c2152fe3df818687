// The gate's part of a gated layer's backward pass, for z = [zg zu] (tensors or 8-bit copies):
//
//   dz_g = da zu act'(zg), dz_u = da act(zg), a = act(zg) zu, db = column sums of dz
//
// Elementwise, with the column sums as in the activation's backward pass (pack8.hip): work-group (strip blockIdx.x, part
// blockIdx.y) goes over its rows of the strip's columns, sums in registers, joined over its waves and sub-rows at the end.
#include "internal.h"
#include "strips.h"
#include "train.h"

namespace mfac {
namespace {

template <typename T, typename TA, bool PACKED>
__global__ __launch_bounds__(256) void k_gated_act_bwd(Strips s, const TA* da, int64_t ldda, Epilogue e, float* part) {
    __shared__ __attribute__((aligned(32))) float sums[2][256 * 8];
    const int lane = threadIdx.x & 63, rpw = 64 >> s.ll;
    const int lc = lane & ((1 << s.ll) - 1);
    const int64_t c = ((int64_t)blockIdx.x << (s.ll + 3)) + lc * 8, ngroups = (s.cols + 31) / 32;
    const int64_t sub = (int64_t)(threadIdx.x >> 6) * rpw + (lane >> s.ll), nsub = 4 * rpw;
    f8 sum_g = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, sum_u = sum_g;
    if (c < s.cols) {
        const int64_t step = gridDim.y * nsub;
        int64_t row = blockIdx.y * nsub + sub;
        // the next row is on its way while this one is worked on
        Raw8<TA> next{};   // without da (a alone is formed) zeros
        std::conditional_t<PACKED, RawPacked8, Raw8<T>> zg, zu;
        auto load = [&](int64_t r) {
            if (da) next.load(da + r * ldda, c, s.cols);
            if constexpr (PACKED) {
                zg.load(e.p.q + r * e.p.ldq, e.p.s + r * ngroups, c, s.cols);
                zu.load(e.p2.q + r * e.p2.ldq, e.p2.s + r * ngroups, c, s.cols);
            } else {
                zg.load((const T*)e.z + r * e.ldz, c, s.cols);
                zu.load((const T*)e.z2 + r * e.ldz, c, s.cols);
            }
        };
        if (row < s.rows) load(row);
        for (; row < s.rows; row += step) {
            f8 d[1] = {next.get()}, a[1] = {zg.get()}, u[1] = {zu.get()};
            if (row + step < s.rows) load(row + step);
            gate_slopes(e.act, a, u, d);
            sum_g += d[0];
            sum_u += u[0];
            store_dz<T>(e, s.cols, row, c, d[0], u[0], a[0]);
        }
    }
    if (!part) return;
    *reinterpret_cast<f8*>(&sums[0][threadIdx.x * 8]) = sum_g;
    *reinterpret_cast<f8*>(&sums[1][threadIdx.x * 8]) = sum_u;
    __syncthreads();
    if (threadIdx.x < (2u << s.ll)) {   // the first lanes the gate's columns, the others the other half's
        const int half = threadIdx.x >> s.ll, at = threadIdx.x & ((1 << s.ll) - 1);
        const int64_t col = ((int64_t)blockIdx.x << (s.ll + 3)) + at * 8;
        f8 v = *reinterpret_cast<const f8*>(&sums[half][at * 8]);
        for (int r = 1; r < nsub; ++r) v += *reinterpret_cast<const f8*>(&sums[half][((r << s.ll) + at) * 8]);
        store8(part + ((int64_t)blockIdx.y * 2 + half) * s.cols, col, s.cols, v);
    }
}

// The largest finite magnitude of four matrices: work-group (i, j) goes over its pieces of the j-th. With the factors 11 us for
// 1537 rows, 520 to 1365; for 8192 rows, 2048 to 8192, 70 of the pass's 2450 (the pre-activations are read once more; of
// copies their bytes s alone, 15 to 40).
struct Range {
    Magnitudes of[4];
    Strips s[4];
};
__global__ __launch_bounds__(256) void k_magnitudes(Range r, float* part) {
    __shared__ unsigned red[4];
    const Magnitudes& m = r.of[blockIdx.y];
    unsigned most = 0;
    if (m.p)
        for_strips(r.s[blockIdx.y], [&](int64_t row, int64_t c) {
            if (row >= m.rows || c >= m.cols) return;
            if (m.dt < 0) {   // 127 times the power of a group
                const uint8_t* s = (const uint8_t*)m.p + row * m.ld;
                for (int64_t i = c; i < min(c + 8, m.cols); ++i)
                    if (s[i] != 255) most = max(most, __float_as_uint(127.f * unpack_scale(min((unsigned)s[i], 247u))));
                return;
            }
            const f8 v = m.dt == DT_F32 ? load8((const float*)m.p + row * m.ld, c, m.cols) : load8((const f16*)m.p + row * m.ld, c, m.cols);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, abs_bits(v[i]) < 0x7f800000u ? abs_bits(v[i]) : 0u);
        });
#pragma unroll
    for (int step = 1; step < 64; step *= 2) most = max(most, (unsigned)__shfl_xor((int)most, step));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x == 0)
        part[blockIdx.y * RANGE_WGS + blockIdx.x] = __uint_as_float(max(max(red[0], red[1]), max(red[2], red[3])));
}
// The factors, 2^-k by which bounds of dz and a come below 2^15: |da| <= sums max|dy| max|w| (or is given), act's slope is
// at most 1.13 and |act(z)| at most |z|. k is 0 for values of ordinary size. The two parts of a value are within 2^(k - 36)
// of it (or 2^-22 of itself): the bound is below 2^(k + 15), so a value has all of its digits unless it is 2^29 times
// smaller than the bound, which with normally distributed dy, W and z is 10^3 to 10^4 times dz's usual size.
__global__ __launch_bounds__(RANGE_WGS) void k_range_factors(float* range, float sums) {
    __shared__ float red[4][RANGE_WGS / 64];
    for (int j = 0; j < 4; ++j) {
        float v = range[4 + j * RANGE_WGS + threadIdx.x];
#pragma unroll
        for (int step = 1; step < 64; step *= 2) v = fmaxf(v, __shfl_xor(v, step));
        if ((threadIdx.x & 63) == 0) red[j][threadIdx.x >> 6] = v;
    }
    __syncthreads();
    if (threadIdx.x >= 2) return;
    double m[4] = {0., 0., 0., 0.};
    for (int j = 0; j < 4; ++j)
        for (int i = 0; i < RANGE_WGS / 64; ++i) m[j] = fmax(m[j], (double)red[j][i]);
    const double bound = threadIdx.x ? m[2] * m[3] : m[0] * (sums > 0.f ? sums * m[1] : 1.) * 1.13 * fmax(m[2], m[3]);
    const int exponent = (int)(__double_as_longlong(bound) >> 52) - 1022;   // bound < 2^exponent
    const unsigned k = (unsigned)max(0, min(exponent - 15, 126));
    range[threadIdx.x] = __uint_as_float((127u - k) << 23);
    range[2 + threadIdx.x] = __uint_as_float((127u + k) << 23);
}

}  // namespace

hipError_t launch_gate_range(const Magnitudes& d, const Magnitudes& w, int64_t sums, int64_t rows, int64_t hidden, const Epilogue& e,
                             hipStream_t st) {
    const int64_t groups = ceil_div(hidden, 32);
    auto pre = [&](const void* z, const Packed& p) {
        return p.q ? Magnitudes{p.s, groups, rows, groups, -1} : Magnitudes{z, e.ldz, rows, hidden, DT_F16};
    };
    Range r{{e.out ? d : Magnitudes{}, e.out ? w : Magnitudes{}, pre(e.z, e.p), pre(e.z2, e.p2)}, {}};
    for (int j = 0; j < 4; ++j)
        if (r.of[j].p) r.s[j] = strips_of(r.of[j].rows, r.of[j].cols);
    k_magnitudes<<<dim3(RANGE_WGS, 4), 256, 0, st>>>(r, e.range + 4);
    k_range_factors<<<1, RANGE_WGS, 0, st>>>(e.range, w.p ? (float)sums : 0.f);
    return hipGetLastError();
}

// As many as give about 2048 work-groups; one for up to eight rows to each of a work-group's, whose sums are then db without
// a launch that joins parts.
int64_t gated_bwd_parts(int64_t rows, int64_t hidden) { return act_bwd_parts(rows, hidden); }

hipError_t launch_gated_act_bwd(int dt, int da_dt, int64_t rows, int64_t hidden, const void* da, int64_t ldda,
                                const Epilogue& e, float* db, float* part, hipStream_t st) {
    if (e.range && rows > 0) {
        const hipError_t err = launch_gate_range({da, ldda, rows, hidden, da_dt}, {}, 0, rows, hidden, e, st);
        if (err != hipSuccess) return err;
    }
    const Strips s = strips_of(rows, hidden);
    const int64_t nparts = rows > 0 ? gated_bwd_parts(rows, hidden) : 0;
    if (!db) part = nullptr;
    else if (nparts == 1) part = db;
    if (rows > 0) {
        auto run = [&](auto* t, auto* ta) {
            using T = std::remove_reference_t<decltype(*t)>;
            using TA = std::remove_reference_t<decltype(*ta)>;
            const dim3 grid((unsigned)s.nstrips, (unsigned)nparts);
            if (e.p.q) k_gated_act_bwd<T, TA, true><<<grid, 256, 0, st>>>(s, (const TA*)da, ldda, e, part);
            else k_gated_act_bwd<T, TA, false><<<grid, 256, 0, st>>>(s, (const TA*)da, ldda, e, part);
            return hipGetLastError();
        };
        float* f = nullptr;
        bf16* b = nullptr;
        f16* h = nullptr;
        const hipError_t err = dt == DT_F32    ? run(f, f)
                               : dt == DT_BF16 ? (da_dt == DT_F32 ? run(b, f) : run(b, b))
                                               : (da_dt == DT_F32 ? run(h, f) : run(h, h));
        if (err != hipSuccess) return err;
    }
    return db && nparts != 1 ? launch_column_sums(part, nparts, 2 * hidden, 2 * hidden, DT_F32, db, nullptr, st) : hipSuccess;
}

}  // namespace mfac
