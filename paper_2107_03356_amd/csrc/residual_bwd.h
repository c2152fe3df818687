// The gradients of what lies between two blocks (residual_fwd.h). With d the gradient of s,
//
//   d  = ds + N_pre'(dh)          N'(g) = rstd (g w - mean(g w) - xhat mean(g w xhat)), without the first mean for rms norm
//   dr = scale d                  t = drop(d), times the gate where it is one for each element
//   dy = N_post'(t gate)          with a gate for each channel
//   dw_pre = sum dh xhat2, db_pre = sum dh, and from P = sum t xhat1, Q = sum t (over rows):
//   dw_post = gate P, db_post = gate Q, dgate = w_post P + b_post Q   (without N_post: dgate = P, xhat1 = y)
//
// so that two sums a column serve the three gradients behind N_post. One pass over the rows, which live in registers as in
// the forward pass; the column sums of a work-group's rows are kept in registers and joined at the end, in a fixed order
// (k_residual_params in residual.hip).
#pragma once

#include "residual.h"

namespace mfac {
namespace {

// s or the 8-bit copy of its xhat, as loaded.
template <typename T>
struct RawStream {
    Raw8<T> s;
    RawPacked8 q;
    __device__ __forceinline__ void load(const Residual& g, int64_t row, int64_t c, int64_t ngroups) {
        if (g.p.q) q.load(g.p.q + row * g.p.ldq, g.p.s + row * ngroups, c, g.cols);
        else s.load((const T*)g.s + row * g.lds, c, g.cols);
    }
};

__device__ __forceinline__ f8 xhat_of(f8 x, float mean, float rstd, int64_t c, int64_t cols) {
    x = (x - mean) * rstd;
    zero_past(x, c, cols);
    return x;
}

// The two means of a norm's backward pass; rms norm has the second only.
template <int NT, bool LAYER>
__device__ __forceinline__ void row_means(float& a, float& b, float inv_cols, float* red, int& turn) {
    if constexpr (LAYER) {
        row_sum2<NT>(a, b, red, turn);
        a *= inv_cols;
    } else {
        b = row_sum<NT>(b, red, turn);
        a = 0.f;
    }
    b *= inv_cols;
}

template <typename T, int NT, int NORMS>
__global__ __launch_bounds__(norm_block(NT)) void k_residual_bwd(Residual g, ResidualBwd b, int wt) {
    constexpr int RPB = norm_block(NT) / NT;
    constexpr bool POST = NORMS & POST_NORM, PRE = NORMS & PRE_NORM, LAYER = NORMS & LAYER_NORM;
    constexpr int SUMS = LAYER ? 4 : 2;
    __shared__ float red[4 * (NT / 64)];
    __shared__ __attribute__((aligned(32))) float cols_of[RPB > 1 ? SUMS : 1][RPB > 1 ? RPB * NT * 8 : 1];
    int turn = 0;
    const int t = threadIdx.x % NT;
    const int64_t c = t * 8, cols = g.cols, ngroups = (cols + 31) / 32;
    const int64_t step = (int64_t)gridDim.x * RPB;
    const float inv_cols = 1.f / (float)cols;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / NT;
    Raw8<T> dh, ds, y, gate;
    RawStream<T> s;
    float mean1 = 0.f, rstd1 = 0.f, mean2 = 0.f, rstd2 = 0.f;
    auto load = [&](int64_t at) {
        if constexpr (PRE) {
            dh.load((const T*)b.dh + at * b.lddh, c, cols);
            s.load(g, at, c, ngroups);
            rstd2 = g.rstd2[at];
            if (LAYER && !g.p.q) mean2 = g.mean2[at];
        }
        if (b.ds) ds.load((const T*)b.ds + at * b.ldds, c, cols);
        if (g.y) y.load((const T*)g.y + at * g.ldy, c, cols);
        if constexpr (POST) {
            rstd1 = g.rstd1[at];
            if (LAYER) mean1 = g.mean1[at];
        }
        if (g.gates) gate.load((const T*)g.gates + at * g.ldgates, c, cols);
    };
    if (row < g.rows) load(row);
    f8 w2 = fill8(0.f), w1 = load_param(POST ? g.w1 : nullptr, wt, c, cols, 1.f);
    if constexpr (PRE) w2 = load_param(g.w2, wt, c, cols, 1.f);
    if (g.gate) w1 *= load8_dt(g.gate, wt, 0, c, cols);
    DropKey key{};
    if (g.drop.threshold) key = drop_key(g.drop);
    f8 sum[SUMS];   // dw_pre, P, db_pre, Q
#pragma unroll
    for (int i = 0; i < SUMS; ++i) sum[i] = fill8(0.f);
    for (; row < g.rows; row += step) {
        f8 d = fill8(0.f), h = d, xh2 = d, xh1 = d, by = d;
        if (b.ds) d = ds.get();
        if constexpr (PRE) {
            h = dh.get();
            xh2 = g.p.q ? s.q.get() : xhat_of(s.s.get(), mean2, rstd2, c, cols);
        }
        if (g.y) xh1 = y.get();
        if constexpr (POST) xh1 = xhat_of(xh1, mean1, rstd1, c, cols);
        if (g.gates) by = gate.get();
        const float r1 = rstd1, r2 = rstd2;
        if (row + step < g.rows) load(row + step);
        if constexpr (PRE) {
            sum[0] += h * xh2;
            if constexpr (LAYER) sum[2] += h;
            h *= w2;
            float m1 = sum8(h), m2 = sum8(h * xh2);
            row_means<NT, LAYER>(m1, m2, inv_cols, red, turn);
            d += (h - m1 - xh2 * m2) * r2;
            if constexpr (LAYER) zero_past(d, c, cols);   // m1 is everywhere
        }
        if (b.dr) store8((T*)b.dr + row * b.lddr, c, cols, g.scale * d);
        if (g.drop.threshold) d = drop8(g.drop, key, (unsigned)row, (unsigned)(c >> 3), d);
        if (g.gates) {   // there is no gate for each channel: w1 is N_post's
            if (b.dgates) {
                f8 n = xh1;
                if constexpr (POST) n *= w1;
                if constexpr (POST && LAYER) n += load_param(g.b1, wt, c, cols, 0.f);
                store8((T*)b.dgates + row * b.lddgates, c, cols, d * n);
            }
            d *= by;
        }
        sum[1] += d * xh1;
        if constexpr (LAYER) sum[3] += d;
        d *= w1;
        if constexpr (POST) {
            float m1 = sum8(d), m2 = sum8(d * xh1);
            row_means<NT, LAYER>(m1, m2, inv_cols, red, turn);
            d = (d - m1 - xh1 * m2) * r1;
        }
        if (b.dy) store8((T*)b.dy + row * b.lddy, c, cols, d);
    }
    if (!b.part) return;
    float* out = b.part + (int64_t)blockIdx.x * SUMS * cols;
    if constexpr (RPB > 1) {   // joined over the waves, each of which has rows of its own
#pragma unroll
        for (int i = 0; i < SUMS; ++i) *reinterpret_cast<f8*>(&cols_of[i][threadIdx.x * 8]) = sum[i];
        __syncthreads();
        const int i = threadIdx.x / NT;   // a wave to each sum
        if (i >= SUMS) return;
        f8 v = *reinterpret_cast<const f8*>(&cols_of[i][t * 8]);
#pragma unroll
        for (int r = 1; r < RPB; ++r) v += *reinterpret_cast<const f8*>(&cols_of[i][(r * NT + t) * 8]);
        store8(out + i * cols, c, cols, v);
    } else {
#pragma unroll
        for (int i = 0; i < SUMS; ++i) store8(out + i * cols, c, cols, sum[i]);
    }
}

// Wider rows: a work-group of 1024 threads a row, d in LDS in fp32, the inputs read again from the caches where they are needed
// twice, the column sums in this work-group's part of the workspace. A thread reads only what it wrote.
template <typename T, int NORMS>
__global__ __launch_bounds__(1024) void k_residual_bwd_wide(Residual g, ResidualBwd b, int wt) {
    constexpr int NT = 1024;
    constexpr bool POST = NORMS & POST_NORM, PRE = NORMS & PRE_NORM, LAYER = NORMS & LAYER_NORM;
    constexpr int SUMS = LAYER ? 4 : 2;
    extern __shared__ __attribute__((aligned(32))) float held[];
    __shared__ float red[4 * (NT / 64)];
    int turn = 0;
    const int64_t cols = g.cols, ngroups = (cols + 31) / 32;
    const float inv_cols = 1.f / (float)cols;
    DropKey key{};
    if (g.drop.threshold) key = drop_key(g.drop);
    float* out = b.part ? b.part + (int64_t)blockIdx.x * SUMS * cols : nullptr;
    bool first = true;
    auto each = [&](auto f) {
        for (int64_t c = threadIdx.x * 8; c < cols; c += NT * 8) f(c, *reinterpret_cast<f8*>(held + c));
    };
    auto add = [&](int i, int64_t c, f8 v) {
        if (!out) return;
        float* p = out + i * cols;
        store8(p, c, cols, first ? v : load8(p, c, cols) + v);
    };
    for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
        float mean1 = 0.f, rstd1 = 0.f, mean2 = 0.f, rstd2 = 0.f, m1 = 0.f, m2 = 0.f, n1 = 0.f, n2 = 0.f;
        if constexpr (PRE) {
            rstd2 = g.rstd2[row];
            if (LAYER && !g.p.q) mean2 = g.mean2[row];
        }
        if constexpr (POST) {
            rstd1 = g.rstd1[row];
            if (LAYER) mean1 = g.mean1[row];
        }
        auto xhat2 = [&](int64_t c) {
            if (g.p.q) return load_packed8(g.p.q + row * g.p.ldq, g.p.s + row * ngroups, c, cols);
            return xhat_of(load8((const T*)g.s + row * g.lds, c, cols), mean2, rstd2, c, cols);
        };
        auto xhat1 = [&](int64_t c) {
            if (!g.y) return fill8(0.f);
            const f8 y = load8((const T*)g.y + row * g.ldy, c, cols);
            return POST ? xhat_of(y, mean1, rstd1, c, cols) : y;
        };
        if constexpr (PRE) {
            each([&](int64_t c, f8&) {
                f8 h = load8((const T*)b.dh + row * b.lddh, c, cols);
                const f8 xh = xhat2(c);
                add(0, c, h * xh);
                if constexpr (LAYER) add(2, c, h);
                h *= load_param(g.w2, wt, c, cols, 1.f);
                m1 += sum8(h);
                m2 += sum8(h * xh);
            });
            row_means<NT, LAYER>(m1, m2, inv_cols, red, turn);
        }
        each([&](int64_t c, f8& held_d) {
            f8 d = fill8(0.f);
            if (b.ds) d = load8((const T*)b.ds + row * b.ldds, c, cols);
            if constexpr (PRE) {
                const f8 h = load8((const T*)b.dh + row * b.lddh, c, cols) * load_param(g.w2, wt, c, cols, 1.f);
                d += (h - m1 - xhat2(c) * m2) * rstd2;
                zero_past(d, c, cols);
            }
            const f8 xh = xhat1(c);
            if (b.dr) store8((T*)b.dr + row * b.lddr, c, cols, g.scale * d);
            if (g.drop.threshold) d = drop8(g.drop, key, (unsigned)row, (unsigned)(c >> 3), d);
            if (g.gates) {
                const f8 by = load8((const T*)g.gates + row * g.ldgates, c, cols);
                if (b.dgates) {
                    f8 n = xh;
                    if constexpr (POST) n *= load_param(g.w1, wt, c, cols, 1.f);
                    if constexpr (POST && LAYER) n += load_param(g.b1, wt, c, cols, 0.f);
                    store8((T*)b.dgates + row * b.lddgates, c, cols, d * n);
                }
                d *= by;
            }
            add(1, c, d * xh);
            if constexpr (LAYER) add(3, c, d);
            if (g.gate) d *= load8_dt(g.gate, wt, 0, c, cols);
            if constexpr (POST) {
                d *= load_param(g.w1, wt, c, cols, 1.f);
                zero_past(d, c, cols);
                n1 += sum8(d);
                n2 += sum8(d * xh);
                held_d = d;
            } else if (b.dy) {
                store8((T*)b.dy + row * b.lddy, c, cols, d);
            }
        });
        if constexpr (POST) {
            row_means<NT, LAYER>(n1, n2, inv_cols, red, turn);
            if (b.dy)
                each([&](int64_t c, f8& d) {
                    store8((T*)b.dy + row * b.lddy, c, cols, (d - n1 - xhat1(c) * n2) * rstd1);
                });
        }
        first = false;
    }
}

}  // namespace

template <typename T>
hipError_t residual_bwd(int wt, const Residual& g, const ResidualBwd& b, hipStream_t st) {
    const unsigned grid = (unsigned)residual_bwd_parts(g.rows, g.cols);
    by_norms(g.norms, [&](auto norms) {
        constexpr int NORMS = decltype(norms)::value;
        if (g.cols > HELD_COLS) {
            k_residual_bwd_wide<T, NORMS><<<grid, 1024, (size_t)round_up(g.cols, 8) * 4, st>>>(g, b, wt);
            return;
        }
        by_threads(g.cols, [&](auto nt) {
            constexpr int NT = decltype(nt)::value;
            k_residual_bwd<T, NT, NORMS><<<grid, norm_block(NT), 0, st>>>(g, b, wt);
        });
    });
    return hipGetLastError();
}

}  // namespace mfac
