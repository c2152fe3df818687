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
// (k_residual_params in residual.hip). The memory's rate bounds it: bf16 16384 x 4096 with both rms norms, a gate for each
// channel and dropout takes 166 us (4.8 TB/s of dh, ds, y, s, dy and dr) and 9 for the join; rms norm alone with ds 112
// (5.9 TB/s). Layer norms, whose sums leave fewer waves, reach 4.8 TB/s there, and 2.9 at 8192 x 8192 (276 us).
#pragma once

#include "residual.h"

namespace mfac {
namespace {

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

template <typename T, int NT, int NCH, bool AHEAD, int NORMS>
__global__ __launch_bounds__(norm_block(NT), 2) void k_residual_bwd(Residual g, ResidualBwd b, int wt) {
    constexpr int RPB = norm_block(NT) / NT;
    constexpr bool POST = NORMS & POST_NORM, PRE = NORMS & PRE_NORM, LAYER = NORMS & LAYER_NORM;
    constexpr bool BETWEEN = !(NORMS & NOTHING_BETWEEN);
    constexpr int SUMS = LAYER ? 4 : 2;   // without anything between, those behind N_post are not formed
    __shared__ float red[4 * (NT / 64)];
    __shared__ __attribute__((aligned(32))) float cols_of[RPB > 1 ? SUMS : 1][RPB > 1 ? RPB * NT * NCH * 8 : 1];
    int turn = 0;
    const int t = threadIdx.x % NT;
    const int64_t cols = g.cols, ngroups = (cols + 31) / 32;
    const int64_t step = (int64_t)gridDim.x * RPB;
    const float inv_cols = 1.f / (float)cols;
    int64_t row = first_row<NT>();
    Place at[NCH];
#pragma unroll
    for (int j = 0; j < NCH; ++j) at[j] = place_of((j * NT + t) * 8, cols);
    // AHEAD: the next row is on its way while one is worked on
    Row8<T> dh[NCH], ds[NCH], y[NCH], gate[NCH], s[NCH];   // s, or the 8-bit copy of its xhat
    float mean1 = 0.f, rstd1 = 0.f, mean2 = 0.f, rstd2 = 0.f;
    auto load = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            if constexpr (PRE) {
                dh[j].load((const T*)b.dh + row * b.lddh, at[j]);
                if (g.p.q) s[j].load_copy(g.p.q + row * g.p.ldq, g.p.s + row * ngroups, (j * NT + t) * 8, at[j]);
                else s[j].load((const T*)g.s + row * g.lds, at[j]);
            }
            if (b.ds) ds[j].load((const T*)b.ds + row * b.ldds, at[j]);
            if (BETWEEN && g.y) y[j].load((const T*)g.y + row * g.ldy, at[j]);
            if (BETWEEN && g.gates) gate[j].load((const T*)g.gates + row * g.ldgates, at[j]);
        }
        if constexpr (PRE) {
            rstd2 = g.rstd2[row];
            if (LAYER && !g.p.q) mean2 = g.mean2[row];
        }
        if constexpr (POST) {
            rstd1 = g.rstd1[row];
            if (LAYER) mean1 = g.mean1[row];
        }
    };
    if (AHEAD && row < g.rows) load(row);
    f8 w1[NCH], w2[PRE ? NCH : 1], sum[SUMS][NCH];   // dw_pre, P, db_pre, Q
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        if constexpr (BETWEEN) w1[j] = load_param<T>(g.gate, wt, at[j], 1.f) * load_param<T>(POST ? g.w1 : nullptr, wt, at[j], 1.f);
        if constexpr (PRE) w2[j] = load_param<T>(g.w2, wt, at[j], 1.f);
#pragma unroll
        for (int i = 0; i < SUMS; ++i) sum[i][j] = fill8(0.f);   // of what is between: stays 0 without it
    }
    DropKey key{};
    if (BETWEEN && g.drop.threshold) key = drop_key(g.drop);
    for (; row < g.rows; row += step) {
        if (!AHEAD) load(row);
        Row8<T> dh_now[NCH], ds_now[NCH], y_now[NCH], gate_now[NCH], s_now[NCH];   // made fp32 where they are used
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            dh_now[j] = dh[j];
            ds_now[j] = ds[j];
            y_now[j] = y[j];
            gate_now[j] = gate[j];
            s_now[j] = s[j];
        }
        const float r1 = rstd1, r2 = rstd2, mu1 = mean1, mu2 = mean2;
        if (AHEAD && row + step < g.rows) load(row + step);
        f8 d[NCH], xh[NCH];
        if constexpr (PRE) {
            float m1 = 0.f, m2 = 0.f;
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int c = (j * NT + t) * 8;
                f8 h = dh_now[j].get(at[j]);
                xh[j] = g.p.q ? s_now[j].get_copy(at[j]) : xhat_of(s_now[j].get(at[j]), mu2, r2, c, cols);
                sum[0][j] += h * xh[j];
                if constexpr (LAYER) sum[2][j] += h;
                h *= w2[j];
                m1 += sum8(h);
                m2 += sum8(h * xh[j]);
                d[j] = h;
                __builtin_amdgcn_sched_barrier(0);
            }
            row_means<NT, LAYER>(m1, m2, inv_cols, red, turn);
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                d[j] = (d[j] - m1 - xh[j] * m2) * r2;
                if constexpr (LAYER) zero_past(d[j], (j * NT + t) * 8, cols);   // m1 is everywhere
                if (b.ds) d[j] += ds_now[j].get(at[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < NCH; ++j) d[j] = ds_now[j].get(at[j]);   // there is one without N_pre
        }
        float n1 = 0.f, n2 = 0.f;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int c = (j * NT + t) * 8;
            if (b.dr) store8((T*)b.dr + row * b.lddr, c, cols, g.scale * d[j]);
            if constexpr (!BETWEEN) continue;
            xh[j] = fill8(0.f);
            if (g.y) xh[j] = y_now[j].get(at[j]);
            if constexpr (POST) xh[j] = xhat_of(xh[j], mu1, r1, c, cols);
            // y where it was dropped took no part: a NaN there must not come into dgate through 0 times it
            if (g.drop.threshold) d[j] = drop8(g.drop, key, (unsigned)row, (unsigned)(c >> 3), d[j], POST ? nullptr : &xh[j]);
            if (g.gates) {   // there is no gate for each channel: w1 is N_post's
                if (b.dgates) {
                    f8 n = xh[j];
                    if constexpr (POST) n *= w1[j];
                    if constexpr (POST && LAYER) n += load_param<T>(g.b1, wt, at[j], 0.f);
                    store8((T*)b.dgates + row * b.lddgates, c, cols, d[j] * n);
                }
                d[j] *= gate_now[j].get(at[j]);
            }
            sum[1][j] += d[j] * xh[j];
            if constexpr (LAYER) sum[3][j] += d[j];
            d[j] *= w1[j];
            n1 += sum8(d[j]);
            n2 += sum8(d[j] * xh[j]);
            __builtin_amdgcn_sched_barrier(0);   // one chunk's mask after the other's: together they take 20 registers more
        }
        if constexpr (POST) row_means<NT, LAYER>(n1, n2, inv_cols, red, turn);
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            if constexpr (POST) d[j] = (d[j] - n1 - xh[j] * n2) * r1;
            if (b.dy) store8((T*)b.dy + row * b.lddy, (j * NT + t) * 8, cols, d[j]);
        }
    }
    if (!b.part) return;
    float* out = b.part + (int64_t)blockIdx.x * SUMS * cols;
    if constexpr (RPB > 1) {   // joined over the waves, each of which has rows of its own
#pragma unroll
        for (int i = 0; i < SUMS; ++i)
#pragma unroll
            for (int j = 0; j < NCH; ++j)
                *reinterpret_cast<f8*>(&cols_of[i][((threadIdx.x / NT * NCH + j) * NT + t) * 8]) = sum[i][j];
        __syncthreads();
        const int i = threadIdx.x / NT;   // a wave to each sum
        if (i >= SUMS) return;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            f8 v = *reinterpret_cast<const f8*>(&cols_of[i][(j * NT + t) * 8]);
#pragma unroll
            for (int r = 1; r < RPB; ++r) v += *reinterpret_cast<const f8*>(&cols_of[i][((r * NCH + j) * NT + t) * 8]);
            store8(out + i * cols, (j * NT + t) * 8, cols, v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < SUMS; ++i)
#pragma unroll
            for (int j = 0; j < NCH; ++j) store8(out + i * cols, (j * NT + t) * 8, cols, sum[i][j]);
    }
}

// Wider rows: a work-group of 1024 threads a row, d in LDS in fp32, the inputs read again from the caches where they are needed
// twice, the column sums in this work-group's part of the workspace. A thread reads only what it wrote. bf16 4096 x 16384 with
// everything on takes 370 us with rms norms, 538 with layer norms (2.2 and 1.5 TB/s).
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
            f8 xh = xhat1(c);
            if (b.dr) store8((T*)b.dr + row * b.lddr, c, cols, g.scale * d);
            if (g.drop.threshold) d = drop8(g.drop, key, (unsigned)row, (unsigned)(c >> 3), d, POST ? nullptr : &xh);
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

// f(threads that hold a row, chunks of eight values that each has, whether a row is loaded ahead), as constants. A row ahead,
// its column sums and weights are most of the registers: 16-bit rows with rms norms take two chunks a thread (248
// registers, two waves to a SIMD); with layer norms, whose sums are twice as many, one (16384 x 4096 202 us, 347 with what two
// would spill), and without anything between too, whose inputs are few, for the sake of more waves (92 us against 108). Above
// 4096 columns fp32 rows and those of layer norms would need 1024 threads, which have 128 registers each: 512 with two chunks
// and no row ahead.
template <typename T, bool ONE, typename F>
void by_threads_bwd(int64_t cols, F f) {
    constexpr int C = residual_chunks(sizeof(T) == 4, ONE);
    if (cols <= 512) f(constant<64>(), constant<1>(), std::true_type());
    else if (cols <= 1024) f(constant<128 / C>(), constant<C>(), std::true_type());
    else if (cols <= 2048) f(constant<256 / C>(), constant<C>(), std::true_type());
    else if (cols <= 4096) f(constant<512 / C>(), constant<C>(), std::true_type());
    else f(constant<512>(), constant<2>(), std::bool_constant<C == 2>());
}

}  // namespace

template <typename T>
hipError_t residual_bwd(int wt, const Residual& g, const ResidualBwd& b, hipStream_t st) {
    constexpr int DT = sizeof(T) == 4 ? DT_F32 : DT_BF16;
    const unsigned grid = (unsigned)residual_bwd_grid(DT, g.norms, g.rows, g.cols);
    const bool between = g.norms & POST_NORM || g.y || g.gate || g.gates || g.drop.threshold;
    const int norms = between || !in_registers(g.cols) ? g.norms : g.norms | NOTHING_BETWEEN;
    by_norms(norms, [&](auto tag) {
        constexpr int NORMS = decltype(tag)::value;
        // fp32 with layer norms, 4096 x 8192: 342 us as a wider row, 469 with what 512 threads would spill
        constexpr bool SPILLS = sizeof(T) == 4 && NORMS & LAYER_NORM && !(NORMS & NOTHING_BETWEEN);
        if (!in_registers(g.cols) || (SPILLS && g.cols > 4096)) {
            if constexpr (!(NORMS & NOTHING_BETWEEN))
                k_residual_bwd_wide<T, NORMS><<<grid, 1024, (size_t)round_up(g.cols, 8) * 4, st>>>(g, b, wt);
            return;
        }
        by_threads_bwd<T, (NORMS & (LAYER_NORM | NOTHING_BETWEEN)) != 0>(g.cols, [&](auto nt, auto nch, auto ahead) {
            constexpr int NT = decltype(nt)::value;
            constexpr bool AHEAD = decltype(ahead)::value;
            if constexpr (AHEAD || !SPILLS)
                k_residual_bwd<T, NT, decltype(nch)::value, AHEAD, NORMS><<<grid, norm_block(NT), 0, st>>>(g, b, wt);
        });
    });
    return hipGetLastError();
}

}  // namespace mfac
