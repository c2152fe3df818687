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

template <typename T>
struct GatedArgs {
    const T* da;
    int64_t ldda;
    const T *zg, *zu;
    int64_t ldz;
    Packed pg, pu;
    T* dz;   // rows x 2 hidden
    int64_t lddz;
    T* a;
    int64_t lda;
    float* part;   // [parts][2 hidden]
    int64_t ngroups;
    int act;
};

template <typename T, bool PACKED>
__global__ __launch_bounds__(256) void k_gated_act_bwd(Strips s, GatedArgs<T> g) {
    __shared__ __attribute__((aligned(32))) float sums[2][256 * 8];
    const int lane = threadIdx.x & 63, rpw = 64 >> s.ll;
    const int lc = lane & ((1 << s.ll) - 1);
    const int64_t c = ((int64_t)blockIdx.x << (s.ll + 3)) + lc * 8;
    const int64_t sub = (int64_t)(threadIdx.x >> 6) * rpw + (lane >> s.ll), nsub = 4 * rpw;
    f8 sum_g = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, sum_u = sum_g;
    if (c < s.cols) {
        const int64_t step = gridDim.y * nsub;
        int64_t row = blockIdx.y * nsub + sub;
        // the next row is on its way while this one is worked on
        Raw8<T> da;
        std::conditional_t<PACKED, RawPacked8, Raw8<T>> zg, zu;
        auto load = [&](int64_t r) {
            da.load(g.da + r * g.ldda, c, s.cols);
            if constexpr (PACKED) {
                zg.load(g.pg.q + r * g.pg.ldq, g.pg.s + r * g.ngroups, c, s.cols);
                zu.load(g.pu.q + r * g.pu.ldq, g.pu.s + r * g.ngroups, c, s.cols);
            } else {
                zg.load(g.zg + r * g.ldz, c, s.cols);
                zu.load(g.zu + r * g.ldz, c, s.cols);
            }
        };
        if (row < s.rows) load(row);
        for (; row < s.rows; row += step) {
            f8 d[1] = {da.get()}, a[1] = {zg.get()}, u[1] = {zu.get()};
            if (row + step < s.rows) load(row + step);
            gate_slopes(g.act, a, u, d);
            sum_g += d[0];
            sum_u += u[0];
            store8(g.dz + row * g.lddz, c, s.cols, d[0]);
            store8(g.dz + row * g.lddz + s.cols, c, s.cols, u[0]);
            if (g.a) store8(g.a + row * g.lda, c, s.cols, a[0]);
        }
    }
    if (!g.part) return;
    *reinterpret_cast<f8*>(&sums[0][threadIdx.x * 8]) = sum_g;
    *reinterpret_cast<f8*>(&sums[1][threadIdx.x * 8]) = sum_u;
    __syncthreads();
    if (threadIdx.x < (2u << s.ll)) {   // the first lanes the gate's columns, the others the other half's
        const int half = threadIdx.x >> s.ll, at = threadIdx.x & ((1 << s.ll) - 1);
        const int64_t col = ((int64_t)blockIdx.x << (s.ll + 3)) + at * 8;
        f8 v = *reinterpret_cast<const f8*>(&sums[half][at * 8]);
        for (int r = 1; r < nsub; ++r) v += *reinterpret_cast<const f8*>(&sums[half][((r << s.ll) + at) * 8]);
        store8(g.part + ((int64_t)blockIdx.y * 2 + half) * s.cols, col, s.cols, v);
    }
}

}  // namespace

// As many as give about 2048 work-groups; one for up to eight rows to each of a work-group's, whose sums are then db without
// a launch that joins parts.
int64_t gated_bwd_parts(int64_t rows, int64_t hidden) { return act_bwd_parts(rows, hidden); }

hipError_t launch_gated_act_bwd(int dt, int act, int64_t rows, int64_t hidden, const void* da, int64_t ldda,
                                const void* zg, const void* zu, int64_t ldz, Packed pg, Packed pu, void* dz, int64_t lddz,
                                void* a, int64_t lda, float* db, float* part, hipStream_t st) {
    const Strips s = strips_of(rows, hidden);
    const int64_t nparts = rows > 0 ? gated_bwd_parts(rows, hidden) : 0;
    if (!db) part = nullptr;
    else if (nparts == 1) part = db;
    if (rows > 0) {
        auto run = [&](auto* t) {
            using T = std::remove_reference_t<decltype(*t)>;
            const GatedArgs<T> g{(const T*)da, ldda, (const T*)zg, (const T*)zu, ldz, pg, pu, (T*)dz, lddz,
                                 (T*)a, lda, part, ceil_div(hidden, 32), act};
            const dim3 grid((unsigned)s.nstrips, (unsigned)nparts);
            if (pg.q) k_gated_act_bwd<T, true><<<grid, 256, 0, st>>>(s, g);
            else k_gated_act_bwd<T, false><<<grid, 256, 0, st>>>(s, g);
            return hipGetLastError();
        };
        const hipError_t e = dt == DT_F32 ? run((float*)nullptr) : dt == DT_BF16 ? run((bf16*)nullptr) : run((f16*)nullptr);
        if (e != hipSuccess) return e;
    }
    return db && nparts != 1 ? launch_column_sums(part, nparts, 2 * hidden, 2 * hidden, DT_F32, db, nullptr, st) : hipSuccess;
}

}  // namespace mfac
