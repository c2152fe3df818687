// Dispatch by type of what lies between two blocks (residual_fwd.h, residual_bwd.h), and the end of its parameters'
// gradients.
#include "residual.h"

namespace mfac {

extern template hipError_t residual_fwd<float>(int, const Residual&, hipStream_t);
extern template hipError_t residual_fwd<bf16>(int, const Residual&, hipStream_t);
extern template hipError_t residual_fwd<f16>(int, const Residual&, hipStream_t);
extern template hipError_t residual_bwd<float>(int, const Residual&, const ResidualBwd&, hipStream_t);
extern template hipError_t residual_bwd<bf16>(int, const Residual&, const ResidualBwd&, hipStream_t);
extern template hipError_t residual_bwd<f16>(int, const Residual&, const ResidualBwd&, hipStream_t);

namespace {

// Joins the work-groups' column sums in order, a work-group to 64 columns, its 16 waves every 16th part each. blockIdx.y 0:
// the pre norm's gradients; 1: those behind the post norm, from P and Q.
template <typename TW>
__global__ __launch_bounds__(1024) void k_residual_params(const float* __restrict__ part, int64_t nparts, int sums,
                                                          int64_t cols, bool post, const TW* w1, const TW* b1,
                                                          const TW* gate, TW* dw1, TW* db1, TW* dgate, TW* dw2, TW* db2) {
    __shared__ float of[2][16][64];
    const int which = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float p = 0.f, q = 0.f;
    if (c < cols) {
        const float* at = part + which * cols + c;
#pragma unroll 8
        for (int64_t i = wave; i < nparts; i += 16) {
            p += at[i * sums * cols];
            if (sums > 2) q += at[(i * sums + 2) * cols];
        }
    }
    of[0][wave][lane] = p;
    of[1][wave][lane] = q;
    __syncthreads();
    if (wave != 0 || c >= cols) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) {
        p += of[0][i][lane];
        q += of[1][i][lane];
    }
    if (which == 0) {
        if (dw2) dw2[c] = (TW)p;
        if (db2) db2[c] = (TW)q;
        return;
    }
    if (!post) {
        if (dgate) dgate[c] = (TW)p;
        return;
    }
    const float by = gate ? (float)gate[c] : 1.f;
    if (dw1) dw1[c] = (TW)(by * p);
    if (db1) db1[c] = (TW)(by * q);
    if (dgate) dgate[c] = (TW)((w1 ? (float)w1[c] : 1.f) * p + (b1 ? (float)b1[c] : 0.f) * q);
}

template <typename TW>
void params(const Residual& g, const ResidualBwd& b, hipStream_t st) {
    const bool post = g.norms & POST_NORM;
    k_residual_params<TW><<<dim3((unsigned)ceil_div(g.cols, 64), 2), 1024, 0, st>>>(
        b.part, g.rows > 0 ? residual_bwd_parts(g.rows, g.cols) : 0, residual_sums(g.norms), g.cols, post,
        (const TW*)(post ? g.w1 : nullptr), (const TW*)(post ? g.b1 : nullptr), (const TW*)g.gate, (TW*)b.dw1, (TW*)b.db1,
        (TW*)b.dgate, (TW*)b.dw2, (TW*)b.db2);
}

}  // namespace

// Work-groups of the backward pass, each with its column sums: two waves to a SIMD; four for narrow rows, whose sums are small.
int64_t residual_bwd_parts(int64_t rows, int64_t cols) {
    const int64_t per = cols <= 512 ? 4 : 1;
    const int64_t grid = cols > 4096 ? 256 : cols > 2048 ? 512 : 1024;
    return std::min(ceil_div(rows, per), grid);
}
// dw_pre and P; for layer norms db_pre and Q too.
int residual_sums(int norms) { return norms & LAYER_NORM ? 4 : 2; }

hipError_t launch_residual(int dt, int wt, const Residual& g, hipStream_t st) {
    if (dt == DT_F32) return residual_fwd<float>(wt, g, st);
    return dt == DT_BF16 ? residual_fwd<bf16>(wt, g, st) : residual_fwd<f16>(wt, g, st);
}

hipError_t launch_residual_bwd(int dt, int wt, const Residual& g, const ResidualBwd& b, hipStream_t st) {
    ResidualBwd k = b;
    if (!(b.dw1 || b.db1 || b.dw2 || b.db2 || b.dgate)) k.part = nullptr;
    if (g.rows > 0) {
        const hipError_t e = dt == DT_F32    ? residual_bwd<float>(wt, g, k, st)
                             : dt == DT_BF16 ? residual_bwd<bf16>(wt, g, k, st)
                                             : residual_bwd<f16>(wt, g, k, st);
        if (e != hipSuccess) return e;
    }
    if (!(b.dw1 || b.db1 || b.dw2 || b.db2 || b.dgate)) return hipSuccess;
    if (wt == DT_F32) params<float>(g, k, st);
    else if (wt == DT_BF16) params<bf16>(g, k, st);
    else params<f16>(g, k, st);
    return hipGetLastError();
}

}  // namespace mfac
