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
        Raw8<TA> next;
        std::conditional_t<PACKED, RawPacked8, Raw8<T>> zg, zu;
        auto load = [&](int64_t r) {
            next.load(da + r * ldda, c, s.cols);
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

}  // namespace

// As many as give about 2048 work-groups; one for up to eight rows to each of a work-group's, whose sums are then db without
// a launch that joins parts.
int64_t gated_bwd_parts(int64_t rows, int64_t hidden) { return act_bwd_parts(rows, hidden); }

hipError_t launch_gated_act_bwd(int dt, int da_dt, int64_t rows, int64_t hidden, const void* da, int64_t ldda,
                                const Epilogue& e, float* db, float* part, hipStream_t st) {
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
