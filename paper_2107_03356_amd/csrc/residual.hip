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

// Joins the work-groups' column sums in order. A work-group has 16 columns, its 64 groups of 16 threads every 64th part each:
// with 64 columns to one, as where only one sum a column is joined, 1000 columns of 1024 parts took 23 us, what
// 32 CUs can read. blockIdx.y 0: the pre norm's gradients; 1: those behind the post norm, from P and Q.
template <typename TW>
__global__ __launch_bounds__(1024) void k_residual_params(const float* __restrict__ part, int64_t nparts, int sums,
                                                          int64_t cols, bool post, const TW* w1, const TW* b1,
                                                          const TW* gate, TW* dw1, TW* db1, TW* dgate, TW* dw2, TW* db2) {
    __shared__ float of[2][64][17];
    const int which = blockIdx.y, lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * 16 + lane;
    float p = 0.f, q = 0.f;
    if (c < cols) {
        const float* at = part + which * cols + c;
#pragma unroll 8
        for (int64_t i = group; i < nparts; i += 64) {
            p += at[i * sums * cols];
            if (sums > 2) q += at[(i * sums + 2) * cols];
        }
    }
    of[0][group][lane] = p;
    of[1][group][lane] = q;
    __syncthreads();
    if (threadIdx.x >= 16 || c >= cols) return;
#pragma unroll
    for (int i = 1; i < 64; ++i) {
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
void params(int dt, const Residual& g, const ResidualBwd& b, hipStream_t st) {
    const bool post = g.norms & POST_NORM;
    k_residual_params<TW><<<dim3((unsigned)ceil_div(g.cols, 16), 2), 1024, 0, st>>>(
        b.part, g.rows > 0 ? residual_bwd_grid(dt, g.norms, g.rows, g.cols) : 0, residual_sums(g.norms), g.cols, post,
        (const TW*)(post ? g.w1 : nullptr), (const TW*)(post ? g.b1 : nullptr), (const TW*)g.gate, (TW*)b.dw1, (TW*)b.db1,
        (TW*)b.dgate, (TW*)b.dw2, (TW*)b.db2);
}

}  // namespace

// Work-groups of the backward pass, each with its column sums: as many as are on the card at once, eight waves to a CU (sixteen where
// a row's inputs are few or the threads' chunks small), and each at least four turns, since its sums are written and read again.
int64_t residual_bwd_grid(int dt, int norms, int64_t rows, int64_t cols) {
    const bool fp32 = dt == DT_F32, post = norms & POST_NORM;
    const int64_t c = residual_chunks(fp32, norms & LAYER_NORM || !post);
    const int64_t threads = !in_registers(cols) ? 1024 : cols <= 512 ? 64 : cols > 4096 ? 512 : round_up(cols, 512 * c) / 8 / c;
    const int64_t waves = threads == 64 ? 4 : threads / 64, per = threads == 64 ? 4 : 1;
    const int64_t most = 256 * std::max(int64_t(1), (!post || (!fp32 && c == 1) ? 16 : 8) / waves);
    return std::max(int64_t(1), std::min(ceil_div(ceil_div(rows, per), 4), most));
}
// A layer norm by itself, or before the skip connection's gradient, is layer norm (norm.hip), whose kernels hold nothing of
// what may lie between: bf16 8192 x 4096 24 us forward, 48 backward with ds; the kernels here take 35 and 63, and 495 where
// those take 120 at 4096 x 16384.
bool layer_norm_alone(const Residual& g) {
    return g.norms == (PRE_NORM | LAYER_NORM) && !g.gate && !g.gates && !g.drop.threshold;
}
// Room for either: its parts have two sums.
int64_t residual_bwd_parts(int dt, int norms, int64_t rows, int64_t cols) {
    const int64_t grid = residual_bwd_grid(dt, norms, rows, cols);
    return norms == (PRE_NORM | LAYER_NORM) ? std::max(grid, ceil_div(norm_bwd_parts(rows, cols), 2)) : grid;
}
// dw_pre and P; for layer norms db_pre and Q too.
int residual_sums(int norms) { return norms & LAYER_NORM ? 4 : 2; }

hipError_t launch_residual(int dt, int wt, const Residual& g, hipStream_t st) {
    if (layer_norm_alone(g) && !g.r && !g.s)
        return launch_layer_norm(dt, wt, g.rows, g.cols, g.y, g.ldy, g.w2, g.b2, g.eps, g.h, g.ldh, g.mean2, g.rstd2, g.p, st);
    if (dt == DT_F32) return residual_fwd<float>(wt, g, st);
    return dt == DT_BF16 ? residual_fwd<bf16>(wt, g, st) : residual_fwd<f16>(wt, g, st);
}

hipError_t launch_residual_bwd(int dt, int wt, const Residual& g, const ResidualBwd& b, hipStream_t st) {
    if (layer_norm_alone(g) && !g.y && b.dy && !b.dr)
        return launch_layer_norm_bwd(dt, wt, g.rows, g.cols, b.dh, b.lddh, g.s, g.lds, g.mean2, g.rstd2, g.p, g.w2, b.ds, b.ldds, b.dy,
                                     b.lddy, b.dw2, b.db2, b.part, st);
    ResidualBwd k = b;
    if (!(b.dw1 || b.db1 || b.dw2 || b.db2 || b.dgate)) k.part = nullptr;
    if (g.rows > 0) {
        const hipError_t e = dt == DT_F32    ? residual_bwd<float>(wt, g, k, st)
                             : dt == DT_BF16 ? residual_bwd<bf16>(wt, g, k, st)
                                             : residual_bwd<f16>(wt, g, k, st);
        if (e != hipSuccess) return e;
    }
    if (!(b.dw1 || b.db1 || b.dw2 || b.db2 || b.dgate)) return hipSuccess;
    if (wt == DT_F32) params<float>(dt, g, k, st);
    else if (wt == DT_BF16) params<bf16>(dt, g, k, st);
    else params<f16>(dt, g, k, st);
    return hipGetLastError();
}

}  // namespace mfac
