// What lies between two blocks of a network with a residual stream, in one pass over its rows:
//
//   n = N_post(y)              norm after a block (or n = y)
//   s = scale r + gate drop(n) the stream; gate: a value for each channel or for each element, or 1
//   h = N_pre(s)               norm before the next block
//
// N is rms norm, x / sqrt(mean(x^2) + eps) w, or layer norm, (x - mean) / sqrt(mean((x - mean)^2) + eps) w + b.
//
// A row lives in the registers of NT threads (NCH chunks of eight neighbouring values each), so every input is read once and s
// is not read again for h, which is formed from s before its rounding. A gate for each channel is folded into N_post's weight
// and bias: gate drop(xhat w + b) = drop(xhat (gate w) + gate b). The memory's rate bounds it: bf16 8192 x 4096 with both rms
// norms, a gate for each channel and dropout 54 us (5.0 TB/s of y, r, s and h; a copy of 4 GiB reaches 4.8), fp32 8192 x
// 4096 100 us (5.4 TB/s); layer norms, which take two sums a norm one after another, 4.4 at bf16 32768 x 1024. One token
// is 3 us.
#pragma once

#include "residual.h"

namespace mfac {
namespace {

// The row's mean (0 for rms norm) and 1 / sqrt(variance + eps) of values v, which become xhat; zeros past the end. The mean is
// that of an fp32 sum, at most some 40 units of 2^-24 of the mean magnitude off. Where a row's values lie closer together than
// that, xhat is what the mean's error leaves of them: values that are all 1000, with eps 1e-6, up to 0.08 instead of 0 (values
// whose sum is exact, as bf16 ones, 0). Summing what the mean leaves beside the squares, to take it off as well, took 10%
// longer (bf16 8192 x 4096 64.7 us, not 57.0; fp32 4096 x 8192 180, not 108).
template <int NT, int NCH, bool LAYER>
__device__ __forceinline__ void normalise(f8 (&v)[NCH], const Residual& g, int t, float* red, int& turn, float& mean,
                                          float& rstd) {
    mean = 0.f;
    float sum = 0.f;
    if constexpr (LAYER) {
#pragma unroll
        for (int j = 0; j < NCH; ++j) sum += sum8(v[j]);
        mean = row_sum<NT>(sum, red, turn) / (float)g.cols;   // by division: exact for equal values whose sum is
        sum = 0.f;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            v[j] -= mean;
            zero_past(v[j], (j * NT + t) * 8, g.cols);
        }
    }
#pragma unroll
    for (int j = 0; j < NCH; ++j) sum += sum8(v[j] * v[j]);
    rstd = 1.f / sqrtf(row_sum<NT>(sum, red, turn) / (float)g.cols + g.eps);
#pragma unroll
    for (int j = 0; j < NCH; ++j) v[j] *= rstd;
}

template <typename T, int NT, int NCH, int NORMS>
__global__ __launch_bounds__(norm_block(NT)) void k_residual_fwd(Residual g, int wt) {
    constexpr int RPB = norm_block(NT) / NT;
    constexpr bool POST = NORMS & POST_NORM, PRE = NORMS & PRE_NORM, LAYER = NORMS & LAYER_NORM;
    __shared__ float red[2 * (NT / 64)];
    int turn = 0;
    const int t = threadIdx.x % NT;
    const int64_t step = (int64_t)gridDim.x * RPB, ngroups = (g.cols + 31) / 32;
    int64_t row = first_row<NT>();
    Place at[NCH];
#pragma unroll
    for (int j = 0; j < NCH; ++j) at[j] = place_of((j * NT + t) * 8, g.cols);
    // the next row is on its way while one is worked on
    Row8<T> y[NCH], r[NCH], gate[NCH];
    auto load = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            y[j].load((const T*)g.y + row * g.ldy, at[j]);
            if (g.r) r[j].load((const T*)g.r + row * g.ldr, at[j]);
            if (g.gates) gate[j].load((const T*)g.gates + row * g.ldgates, at[j]);
        }
    };
    if (row < g.rows) load(row);
    f8 w1[NCH], b1[POST && LAYER ? NCH : 1], w2[PRE ? NCH : 1], b2[PRE && LAYER ? NCH : 1];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const f8 by = load_param<T>(g.gate, wt, at[j], 1.f);
        w1[j] = by * load_param<T>(POST ? g.w1 : nullptr, wt, at[j], 1.f);
        if constexpr (POST && LAYER) b1[j] = by * load_param<T>(g.b1, wt, at[j], 0.f);
        if constexpr (PRE) w2[j] = load_param<T>(g.w2, wt, at[j], 1.f);
        if constexpr (PRE && LAYER) b2[j] = load_param<T>(g.b2, wt, at[j], 0.f);
    }
    DropKey key{};
    if (g.drop.threshold) key = drop_key(g.drop);
    for (; row < g.rows; row += step) {
        f8 v[NCH];
        Row8<T> r_now[NCH], gate_now[NCH];   // made fp32 where they are used
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            v[j] = y[j].get(at[j]);
            r_now[j] = r[j];
            gate_now[j] = gate[j];
        }
        if (row + step < g.rows) load(row + step);
        float mean1, rstd1, mean2, rstd2;
        if constexpr (POST) normalise<NT, NCH, LAYER>(v, g, t, red, turn, mean1, rstd1);
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int c = (j * NT + t) * 8;
            v[j] *= w1[j];
            if constexpr (POST && LAYER) v[j] += b1[j];
            if (g.drop.threshold) v[j] = drop8(g.drop, key, (unsigned)row, (unsigned)(c >> 3), v[j]);
            if (g.gates) v[j] *= gate_now[j].get(at[j]);
            if (g.r) v[j] += g.scale * r_now[j].get(at[j]);
            if (g.s) store8((T*)g.s + row * g.lds, c, g.cols, v[j]);
        }
        if constexpr (PRE) {
            normalise<NT, NCH, LAYER>(v, g, t, red, turn, mean2, rstd2);
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int c = (j * NT + t) * 8;
                if (g.p.q) pack_group(g.p.q + row * g.p.ldq, g.p.s + row * ngroups, c, g.cols, v[j]);
                v[j] *= w2[j];
                if constexpr (LAYER) v[j] += b2[j];
                store8((T*)g.h + row * g.ldh, c, g.cols, v[j]);
            }
        }
        if (t == 0) {
            if (POST && g.mean1) g.mean1[row] = mean1;
            if (POST && g.rstd1) g.rstd1[row] = rstd1;
            if (PRE && g.mean2) g.mean2[row] = mean2;
            if (PRE && g.rstd2) g.rstd2[row] = rstd2;
        }
    }
}

// Wider rows: a work-group of 1024 threads a row, held in LDS in fp32. A thread reads only what it wrote. bf16 4096 x 16384 with
// everything on takes 161 us with rms norms (3.3 TB/s), 201 with layer norms: one work-group to a CU, whose turns wait for
// their row.
template <typename T, int NORMS>
__global__ __launch_bounds__(1024) void k_residual_fwd_wide(Residual g, int wt) {
    constexpr int NT = 1024;
    constexpr bool POST = NORMS & POST_NORM, PRE = NORMS & PRE_NORM, LAYER = NORMS & LAYER_NORM;
    extern __shared__ __attribute__((aligned(32))) float held[];
    __shared__ float red[2 * (NT / 64)];
    int turn = 0;
    const int64_t ngroups = (g.cols + 31) / 32, cols = g.cols, end = (cols + 31) & ~int64_t(31);   // whole groups of four lanes
    DropKey key{};
    if (g.drop.threshold) key = drop_key(g.drop);
    auto each = [&](auto f) {
        for (int64_t c = threadIdx.x * 8; c < end; c += NT * 8) f(c, *reinterpret_cast<f8*>(held + c));
    };
    auto statistics = [&](float& mean, float& rstd) {
        mean = 0.f;
        float sum = 0.f;
        if constexpr (LAYER) {
            each([&](int64_t, f8& v) { sum += sum8(v); });
            mean = row_sum<NT>(sum, red, turn) / (float)cols;
            sum = 0.f;
        }
        each([&](int64_t c, f8& v) {
            if constexpr (LAYER) {
                v -= mean;
                zero_past(v, c, cols);
            }
            sum += sum8(v * v);
        });
        rstd = 1.f / sqrtf(row_sum<NT>(sum, red, turn) / (float)cols + g.eps);
    };
    for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
        float mean1, rstd1 = 1.f, mean2, rstd2;
        each([&](int64_t c, f8& v) { v = load8((const T*)g.y + row * g.ldy, c, cols); });
        if constexpr (POST) statistics(mean1, rstd1);
        each([&](int64_t c, f8& held_v) {
            f8 v = held_v * rstd1;
            if constexpr (POST) v *= load_param(g.w1, wt, c, cols, 1.f);
            if constexpr (POST && LAYER) v += load_param(g.b1, wt, c, cols, 0.f);
            if (g.gate) v *= load8_dt(g.gate, wt, 0, c, cols);
            if (g.drop.threshold) v = drop8(g.drop, key, (unsigned)row, (unsigned)(c >> 3), v);
            if (g.gates) v *= load8((const T*)g.gates + row * g.ldgates, c, cols);
            if (g.r) v += g.scale * load8((const T*)g.r + row * g.ldr, c, cols);
            zero_past(v, c, cols);
            if (g.s) store8((T*)g.s + row * g.lds, c, cols, v);
            held_v = v;
        });
        if constexpr (PRE) {
            statistics(mean2, rstd2);
            each([&](int64_t c, f8& held_v) {
                f8 v = held_v * rstd2;
                if (g.p.q) pack_group(g.p.q + row * g.p.ldq, g.p.s + row * ngroups, c, cols, v);
                v *= load_param(g.w2, wt, c, cols, 1.f);
                if constexpr (LAYER) v += load_param(g.b2, wt, c, cols, 0.f);
                store8((T*)g.h + row * g.ldh, c, cols, v);
            });
        }
        if (threadIdx.x == 0) {
            if (POST && g.mean1) g.mean1[row] = mean1;
            if (POST && g.rstd1) g.rstd1[row] = rstd1;
            if (PRE && g.mean2) g.mean2[row] = mean2;
            if (PRE && g.rstd2) g.rstd2[row] = rstd2;
        }
    }
}

// f(constant of the threads that hold a row, constant of the chunks of eight values that each has): 32 bytes of each input a
// thread, so that eight waves to a CU keep enough of them on their way.
template <typename T, typename F>
void by_threads(int64_t cols, F f) {
    constexpr int C = sizeof(T) == 2 ? 2 : 1;
    if (cols <= 512) f(constant<64>(), constant<1>());
    else if (cols <= 1024) f(constant<128 / C>(), constant<C>());
    else if (cols <= 2048) f(constant<256 / C>(), constant<C>());
    else if (cols <= 4096) f(constant<512 / C>(), constant<C>());
    else f(constant<1024 / C>(), constant<C>());
}

}  // namespace

template <typename T>
hipError_t residual_fwd(int wt, const Residual& g, hipStream_t st) {
    by_norms(g.norms, [&](auto norms) {
        constexpr int NORMS = decltype(norms)::value;
        if (!in_registers(g.cols)) {
            const size_t lds = (size_t)round_up(g.cols, 32) * 4;
            k_residual_fwd_wide<T, NORMS><<<(unsigned)std::min<int64_t>(g.rows, 1024), 1024, lds, st>>>(g, wt);
            return;
        }
        by_threads<T>(g.cols, [&](auto nt, auto nch) {
            constexpr int NT = decltype(nt)::value;
            // as many work-groups as are on the card at once, eight waves to a CU (sixteen of the narrowest rows): bf16 8192 x
            // 4096 with everything on 53.6 us with 512, 57.6 with 2048, whose last turn leaves a third of the card idle
            constexpr int WAVES = 256 / (decltype(nch)::value * 8 * (int)sizeof(T)), BLOCK = norm_block(NT) / 64;
            const int64_t most = 256 * std::max(1, WAVES / BLOCK);
            const unsigned grid = (unsigned)std::min(ceil_div(g.rows, norm_block(NT) / NT), most);
            k_residual_fwd<T, NT, decltype(nch)::value, NORMS><<<grid, norm_block(NT), 0, st>>>(g, wt);
        });
    });
    return hipGetLastError();
}

}  // namespace mfac
