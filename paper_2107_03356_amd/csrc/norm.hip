// Layer norm over the rows of a matrix, forward and backward.
//
//   mean, rstd = 1 / sqrt(mean((x - mean)^2) + eps), xhat = (x - mean) rstd, y = xhat w + b
//   h = dy w, dx = rstd (h - mean(h) - xhat mean(h xhat)) + add
//   dw = sum over rows of dy xhat, db = sum over rows of dy
//
// A row lives in the registers of the threads that hold it (NT of them, NCH
// chunks of eight neighbouring values each), so every input is read once; the
// variance is taken around the mean that was just formed, not as a difference of
// two large sums. Work-groups go over the rows with a stride and keep w, b and
// the column sums of dw and db in registers; the next row is loaded before the
// current one is reduced. Both passes are bound by HBM (a large copy reaches 4.9 TB/s here):
// forward, bf16 16384 x 4096, 48 us (5.6 TB/s), with the 8-bit copy 67 (5.1); backward 82 us
// (4.9 TB/s), from the copy and with the skip connection's gradient 92 (5.1). Without the next
// row loaded ahead that last one took 190 us. One token is one launch, 2.8 us.
#include <algorithm>

#include "internal.h"
#include "train.h"
#include "train_util.h"

namespace mfac {
namespace {

template <typename T, typename TW>
struct NormArgs {
    const T* x;
    int64_t ldx;
    const TW *w, *b;
    T* y;
    int64_t ldy;
    float *mean, *rstd;
    Packed p;
    int64_t rows, cols, ngroups;  // ngroups: groups per row of the copy
    float eps, inv_cols, ncols;   // the mean by division, so that a row of equal values has a mean of exactly that
};

// Sum over the NT threads that hold a row. red: two sets of NT / 64 words in
// turn, so that one barrier a sum is enough.
template <int NT>
__device__ __forceinline__ float row_sum(float v, float* red, int& turn) {
    v = wave_sum(v);
    if constexpr (NT == 64) return v;
    constexpr int NW = NT / 64;
    float* r = red + turn * NW;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) s += r[i];
    return s;
}
// The same for two sums at once.
template <int NT>
__device__ __forceinline__ void row_sum2(float& a, float& b, float* red, int& turn) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (NT == 64) return;
    constexpr int NW = NT / 64;
    float* r = red + turn * 2 * NW;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) {
        r[threadIdx.x >> 6] = a;
        r[NW + (threadIdx.x >> 6)] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        a += r[i];
        b += r[NW + i];
    }
}

constexpr int norm_block(int nt) { return nt == 64 ? 256 : nt; }

template <typename T, typename TW, int NT, int NCH>
__global__ __launch_bounds__(norm_block(NT)) void k_norm_fwd(NormArgs<T, TW> g) {
    constexpr int RPB = norm_block(NT) / NT;
    __shared__ float red[2 * (NT / 64)];
    int turn = 0;
    const int t = threadIdx.x % NT;
    f8 w[NCH], b[NCH];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int64_t c = (int64_t)(j * NT + t) * 8;
        w[j] = b[j] = f8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (g.w) w[j] = load8(g.w, c, g.cols);
        else w[j] += 1.f;
        if (g.b) b[j] = load8(g.b, c, g.cols);
    }
    const int64_t step = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / NT;
    Raw8<T> next[NCH];
    if (row < g.rows)
#pragma unroll
        for (int j = 0; j < NCH; ++j) next[j].load(g.x + row * g.ldx, (int64_t)(j * NT + t) * 8, g.cols);
    for (; row < g.rows; row += step) {
        f8 x[NCH];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            x[j] = next[j].get();
            sum += sum8(x[j]);
        }
        if (row + step < g.rows)
#pragma unroll
            for (int j = 0; j < NCH; ++j) next[j].load(g.x + (row + step) * g.ldx, (int64_t)(j * NT + t) * 8, g.cols);
        const float mean = row_sum<NT>(sum, red, turn) / g.ncols;
        float sq = 0.f;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int64_t c = (int64_t)(j * NT + t) * 8;
            x[j] -= mean;
            if (c + 8 > g.cols)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i >= g.cols) x[j][i] = 0.f;
            sq += sum8(x[j] * x[j]);
        }
        const float var = row_sum<NT>(sq, red, turn) * g.inv_cols;
        const float rstd = 1.f / sqrtf(var + g.eps);
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int64_t c = (int64_t)(j * NT + t) * 8;
            x[j] *= rstd;
            if (g.p.q) pack_group(g.p.q + row * g.p.ldq, g.p.s + row * g.ngroups, c, g.cols, x[j]);
            store8(g.y + row * g.ldy, c, g.cols, x[j] * w[j] + b[j]);
        }
        if (t == 0) {
            if (g.mean) g.mean[row] = mean;
            if (g.rstd) g.rstd[row] = rstd;
        }
    }
}

// Rows longer than the registers hold: one work-group a row, which is read three
// times (the second and third time from the caches).
template <typename T, typename TW>
__global__ __launch_bounds__(1024) void k_norm_fwd_long(NormArgs<T, TW> g) {
    constexpr int NT = 1024;
    __shared__ float red[2 * (NT / 64)];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
        const T* xr = g.x + row * g.ldx;
        float sum = 0.f;
        for (int64_t c = threadIdx.x * 8; c < g.cols; c += NT * 8) sum += sum8(load8(xr, c, g.cols));
        const float mean = row_sum<NT>(sum, red, turn) / g.ncols;
        float sq = 0.f;
        for (int64_t c = threadIdx.x * 8; c < g.cols; c += NT * 8) {
            f8 x = load8(xr, c, g.cols) - mean;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i >= g.cols) x[i] = 0.f;
            sq += sum8(x * x);
        }
        const float rstd = 1.f / sqrtf(row_sum<NT>(sq, red, turn) * g.inv_cols + g.eps);
        // whole groups of four lanes go around together
        for (int64_t c = threadIdx.x * 8; c < ((g.cols + 31) & ~int64_t(31)); c += NT * 8) {
            f8 x = (load8(xr, c, g.cols) - mean) * rstd;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i >= g.cols) x[i] = 0.f;
            if (g.p.q) pack_group(g.p.q + row * g.p.ldq, g.p.s + row * g.ngroups, c, g.cols, x);
            if (g.w) x *= load8(g.w, c, g.cols);
            if (g.b) x += load8(g.b, c, g.cols);
            store8(g.y + row * g.ldy, c, g.cols, x);
        }
        if (threadIdx.x == 0) {
            if (g.mean) g.mean[row] = mean;
            if (g.rstd) g.rstd[row] = rstd;
        }
    }
}

// ---------------------------------------------------------------- backward
template <typename T, typename TW>
struct NormBwdArgs {
    const T* dy;
    int64_t lddy;
    const T* x;
    int64_t ldx;
    const float *mean, *rstd;
    Packed p;
    const TW* w;
    const T* add;
    int64_t ldadd;
    T* dx;
    int64_t lddx;
    float* part;  // [part][2][cols]: dw, db
    int64_t rows, cols, ngroups;
    float inv_cols;
};

template <typename T, typename TW>
__device__ __forceinline__ f8 load_xhat(const NormBwdArgs<T, TW>& g, int64_t row, int64_t c, float mean, float rstd) {
    if (g.p.q) return load_packed8(g.p.q + row * g.p.ldq, g.p.s + row * g.ngroups, c, g.cols);
    f8 x = (load8(g.x + row * g.ldx, c, g.cols) - mean) * rstd;
    if (c + 8 > g.cols)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i >= g.cols) x[i] = 0.f;
    return x;
}

// What a row's pass takes, loaded while the row before it is worked on.
template <typename T, typename TW, int NT, int NCH, bool PACKED>
struct NormBwdRow {
    static constexpr bool ADD = NT < 1024;   // add too; without room for it it is loaded when it is used
    Raw8<T> dy[NCH], add[NCH];
    std::conditional_t<PACKED, RawPacked8, Raw8<T>> x[NCH];
    float mean, rstd;
    __device__ __forceinline__ void load(const NormBwdArgs<T, TW>& g, int64_t row, int t) {
        rstd = g.rstd[row];
        if constexpr (!PACKED) mean = g.mean[row];
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int64_t c = (int64_t)(j * NT + t) * 8;
            dy[j].load(g.dy + row * g.lddy, c, g.cols);
            if constexpr (PACKED) x[j].load(g.p.q + row * g.p.ldq, g.p.s + row * g.ngroups, c, g.cols);
            else x[j].load(g.x + row * g.ldx, c, g.cols);
            if (ADD && g.add) add[j].load(g.add + row * g.ldadd, c, g.cols);
        }
    }
};

template <typename T, typename TW, int NT, int NCH, bool PACKED>
__global__ __launch_bounds__(norm_block(NT)) void k_norm_bwd(NormBwdArgs<T, TW> g) {
    constexpr int RPB = norm_block(NT) / NT;
    __shared__ float red[4 * (NT / 64)];
    __shared__ float cols_of[RPB > 1 ? 2 * NCH : 1][RPB > 1 ? RPB * NT * 8 : 1];
    int turn = 0;
    const int t = threadIdx.x % NT;
    // 1024 threads have 128 registers each: no room for the next row, nor for w
    constexpr bool AHEAD = NT < 1024;
    f8 w[NCH], sw[NCH], sb[NCH];
    auto load_w = [&]() {
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            w[j] = f8{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
            if (g.w) w[j] = load8(g.w, (int64_t)(j * NT + t) * 8, g.cols);
        }
    };
    if (AHEAD) load_w();
#pragma unroll
    for (int j = 0; j < NCH; ++j) sw[j] = sb[j] = f8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int64_t step = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / NT;
    NormBwdRow<T, TW, NT, NCH, PACKED> next;
    if (AHEAD && row < g.rows) next.load(g, row, t);
    for (; row < g.rows; row += step) {
        if (!AHEAD) {
            next.load(g, row, t);
            load_w();
        }
        const auto now = next;
        if (AHEAD && row + step < g.rows) next.load(g, row + step, t);
        f8 h[NCH], xh[NCH];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            h[j] = now.dy[j].get();
            xh[j] = now.x[j].get();
            if constexpr (!PACKED) {
                const int64_t c = (int64_t)(j * NT + t) * 8;
                xh[j] = (xh[j] - now.mean) * now.rstd;
                if (c + 8 > g.cols)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + i >= g.cols) xh[j][i] = 0.f;
            }
            sb[j] += h[j];
            sw[j] += h[j] * xh[j];
            h[j] *= w[j];
            s1 += sum8(h[j]);
            s2 += sum8(h[j] * xh[j]);
        }
        row_sum2<NT>(s1, s2, red, turn);
        s1 *= g.inv_cols;
        s2 *= g.inv_cols;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            f8 d = (h[j] - s1 - xh[j] * s2) * now.rstd;
            if (AHEAD) {
                if (g.add) d += now.add[j].get();
            } else if (g.add) {
                d += load8(g.add + row * g.ldadd, (int64_t)(j * NT + t) * 8, g.cols);
            }
            store8(g.dx + row * g.lddx, (int64_t)(j * NT + t) * 8, g.cols, d);
        }
    }
    if (!g.part) return;
    // the column sums of this work-group's rows, joined over its waves where each has rows of
    // its own: a wave to each of the 2 NCH arrays
    float* out = g.part + (int64_t)blockIdx.x * 2 * g.cols;
    if constexpr (RPB > 1) {
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int j = 0; j < NCH; ++j) *reinterpret_cast<f8*>(&cols_of[v * NCH + j][threadIdx.x * 8]) = v ? sb[j] : sw[j];
        __syncthreads();
        const int a = threadIdx.x / NT;
        if (a >= 2 * NCH) return;
        f8 s = *reinterpret_cast<const f8*>(&cols_of[a][t * 8]);
#pragma unroll
        for (int r = 1; r < RPB; ++r) s += *reinterpret_cast<const f8*>(&cols_of[a][(r * NT + t) * 8]);
        store8(out + a / NCH * g.cols, (int64_t)(a % NCH * NT + t) * 8, g.cols, s);
    } else {
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            store8(out, (int64_t)(j * NT + t) * 8, g.cols, sw[j]);
            store8(out + g.cols, (int64_t)(j * NT + t) * 8, g.cols, sb[j]);
        }
    }
}

// Longer rows: two sweeps over each for dx. The column sums are a sweep of their own
// (k_norm_bwd_cols).
template <typename T, typename TW>
__global__ __launch_bounds__(1024) void k_norm_bwd_long(NormBwdArgs<T, TW> g) {
    constexpr int NT = 1024;
    __shared__ float red[4 * (NT / 64)];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
        const float rstd = g.rstd[row], mean = g.mean ? g.mean[row] : 0.f;
        float s1 = 0.f, s2 = 0.f;
        for (int64_t c = threadIdx.x * 8; c < g.cols; c += NT * 8) {
            f8 h = load8(g.dy + row * g.lddy, c, g.cols);
            if (g.w) h *= load8(g.w, c, g.cols);
            s1 += sum8(h);
            s2 += sum8(h * load_xhat(g, row, c, mean, rstd));
        }
        row_sum2<NT>(s1, s2, red, turn);
        s1 *= g.inv_cols;
        s2 *= g.inv_cols;
        for (int64_t c = threadIdx.x * 8; c < g.cols; c += NT * 8) {
            f8 h = load8(g.dy + row * g.lddy, c, g.cols);
            if (g.w) h *= load8(g.w, c, g.cols);
            f8 d = (h - s1 - load_xhat(g, row, c, mean, rstd) * s2) * rstd;
            if (g.add) d += load8(g.add + row * g.ldadd, c, g.cols);
            store8(g.dx + row * g.lddx, c, g.cols, d);
        }
    }
}
// Column sums of the rows blockIdx.y, blockIdx.y + gridDim.y, ...; a thread holds eight columns.
template <typename T, typename TW>
__global__ __launch_bounds__(256) void k_norm_bwd_cols(NormBwdArgs<T, TW> g) {
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (c >= g.cols) return;
    f8 sw = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, sb = sw;
    for (int64_t row = blockIdx.y; row < g.rows; row += gridDim.y) {
        const f8 d = load8(g.dy + row * g.lddy, c, g.cols);
        sb += d;
        sw += d * load_xhat(g, row, c, g.mean ? g.mean[row] : 0.f, g.rstd[row]);
    }
    float* out = g.part + (int64_t)blockIdx.y * 2 * g.cols;
    store8(out, c, g.cols, sw);
    store8(out + g.cols, c, g.cols, sb);
}

constexpr int64_t NORM_MAX_COLS = 16384;   // 1024 threads of two chunks
constexpr int64_t NORM_FWD_GRID = 2048, NORM_LONG_PARTS = 64;

int64_t rows_per_block(int64_t cols) { return cols <= 1024 ? 4 : 1; }

// k: the kernel by threads and chunks a row; one wave a row up to 1024 columns,
// then as few waves as hold it with two chunks a thread.
#define NORM_SHAPES(LAUNCH)                 \
    if (cols <= 512) LAUNCH(64, 1)          \
    else if (cols <= 1024) LAUNCH(64, 2)    \
    else if (cols <= 2048) LAUNCH(128, 2)   \
    else if (cols <= 4096) LAUNCH(256, 2)   \
    else if (cols <= 8192) LAUNCH(512, 2)   \
    else LAUNCH(1024, 2)

template <typename T, typename TW>
hipError_t norm_fwd(int64_t rows, int64_t cols, const void* x, int64_t ldx, const void* w, const void* b, float eps,
                    void* y, int64_t ldy, float* mean, float* rstd, Packed p, hipStream_t st) {
    NormArgs<T, TW> g{(const T*)x, ldx, (const TW*)w, (const TW*)b, (T*)y, ldy, mean, rstd, p, rows, cols,
                      ceil_div(cols, 32), eps, 1.f / (float)cols, (float)cols};
    if (cols > NORM_MAX_COLS) {
        k_norm_fwd_long<T, TW><<<(unsigned)std::min<int64_t>(rows, 1024), 1024, 0, st>>>(g);
        return hipGetLastError();
    }
    const int64_t grid = std::min(ceil_div(rows, rows_per_block(cols)), NORM_FWD_GRID);
#define LAUNCH(NT, NCH) k_norm_fwd<T, TW, NT, NCH><<<(unsigned)grid, norm_block(NT), 0, st>>>(g);
    NORM_SHAPES(LAUNCH)
#undef LAUNCH
    return hipGetLastError();
}

template <typename T, typename TW>
hipError_t norm_bwd(int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                    const float* mean, const float* rstd, Packed p, const void* w, const void* add, int64_t ldadd,
                    void* dx, int64_t lddx, float* part, hipStream_t st) {
    NormBwdArgs<T, TW> g{(const T*)dy, lddy, (const T*)x, ldx, mean, rstd, p, (const TW*)w, (const T*)add, ldadd,
                         (T*)dx, lddx, part, rows, cols, ceil_div(cols, 32), 1.f / (float)cols};
    if (cols > NORM_MAX_COLS) {
        if (part)   // before dx is written, which may be dy
            k_norm_bwd_cols<T, TW><<<dim3((unsigned)ceil_div(cols, 2048), (unsigned)norm_bwd_parts(rows, cols)), 256, 0,
                                     st>>>(g);
        k_norm_bwd_long<T, TW><<<(unsigned)std::min<int64_t>(rows, 1024), 1024, 0, st>>>(g);
        return hipGetLastError();
    }
    const int64_t grid = norm_bwd_parts(rows, cols);
#define LAUNCH(NT, NCH) k_norm_bwd<T, TW, NT, NCH, true><<<(unsigned)grid, norm_block(NT), 0, st>>>(g);
    if (p.q) {
        NORM_SHAPES(LAUNCH)
        return hipGetLastError();
    }
#undef LAUNCH
#define LAUNCH(NT, NCH) k_norm_bwd<T, TW, NT, NCH, false><<<(unsigned)grid, norm_block(NT), 0, st>>>(g);
    NORM_SHAPES(LAUNCH)
#undef LAUNCH
    return hipGetLastError();
}

template <typename F>
hipError_t by_types(int dt, int wt, F f) {
    if (dt == DT_F32) return f((float*)nullptr, (float*)nullptr);
    if (dt == DT_BF16) return wt == DT_F32 ? f((bf16*)nullptr, (float*)nullptr) : f((bf16*)nullptr, (bf16*)nullptr);
    return wt == DT_F32 ? f((f16*)nullptr, (float*)nullptr) : f((f16*)nullptr, (f16*)nullptr);
}

}  // namespace

// Partial column sums that the backward pass writes, one a work-group: as many as keep 8 waves
// on a CU, since they are written and read again (at 16384 x 4096 in bf16 7% of the traffic).
int64_t norm_bwd_parts(int64_t rows, int64_t cols) {
    if (cols > NORM_MAX_COLS) return std::min(rows, NORM_LONG_PARTS);
    const int64_t grid = cols <= 1024 ? 512 : cols <= 2048 ? 1024 : cols <= 4096 ? 512 : 256;
    return std::min(ceil_div(rows, rows_per_block(cols)), grid);
}

hipError_t launch_layer_norm(int dt, int wt, int64_t rows, int64_t cols, const void* x, int64_t ldx, const void* w,
                             const void* b, float eps, void* y, int64_t ldy, float* mean, float* rstd, Packed p,
                             hipStream_t st) {
    return by_types(dt, wt, [&](auto* t, auto* tw) {
        return norm_fwd<std::remove_reference_t<decltype(*t)>, std::remove_reference_t<decltype(*tw)>>(
            rows, cols, x, ldx, w, b, eps, y, ldy, mean, rstd, p, st);
    });
}

hipError_t launch_layer_norm_bwd(int dt, int wt, int64_t rows, int64_t cols, const void* dy, int64_t lddy,
                                 const void* x, int64_t ldx, const float* mean, const float* rstd, Packed p,
                                 const void* w, const void* add, int64_t ldadd, void* dx, int64_t lddx, void* dw,
                                 void* db, float* part, hipStream_t st) {
    if (!dw && !db) part = nullptr;
    hipError_t e = hipSuccess;
    if (rows > 0) {
        e = by_types(dt, wt, [&](auto* t, auto* tw) {
            return norm_bwd<std::remove_reference_t<decltype(*t)>, std::remove_reference_t<decltype(*tw)>>(
                rows, cols, dy, lddy, x, ldx, mean, rstd, p, w, add, ldadd, dx, lddx, part, st);
        });
    }
    if (e != hipSuccess || (!dw && !db)) return e;
    return launch_column_sums(part, rows > 0 ? norm_bwd_parts(rows, cols) : 0, 2 * cols, cols, wt, dw, db, st);
}

}  // namespace mfac
