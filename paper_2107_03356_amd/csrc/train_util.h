// Device helpers shared by the training operators (norm.hip, pack8.hip,
// linear.hip): eight values at a time in and out of fp32, bf16 and fp16 rows,
// 8-bit copies, activations and sums over a wave.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "train.h"

namespace mfac {
namespace {

typedef float f8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16;
typedef __bf16 bf16;

// Vectors with the alignment of their element: global accesses need no more, so
// rows of any leading dimension take 128-bit accesses.
template <typename T, int N>
struct VecOf {
    typedef T plain __attribute__((ext_vector_type(N)));
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// Values of other lanes of a row of 16, without a trip through LDS.
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E;               // quad_perm
constexpr int DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;    // lane i of 8, of 16: 7 - i, 15 - i
template <int CTRL>
__device__ __forceinline__ unsigned dpp(unsigned v) {
    return (unsigned)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}

// Elements c .. c + 7 of a row of `cols`; zeros past its end.
template <typename T>
__device__ __forceinline__ f8 load8(const T* __restrict__ row, int64_t c, int64_t cols) {
    if (c + 8 <= cols) {
        const typename VecOf<T, 8>::plain v = *reinterpret_cast<const typename VecOf<T, 8>::type*>(row + c);
        return __builtin_convertvector(v, f8);
    }
    f8 r = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < cols) r[i] = (float)row[c + i];
    return r;
}

// The same in two halves: the load, and what waits for it.
template <typename T>
struct Raw8 {
    typename VecOf<T, 8>::plain v;
    __device__ __forceinline__ void load(const T* __restrict__ row, int64_t c, int64_t cols) {
        if (c + 8 <= cols) {
            v = *reinterpret_cast<const typename VecOf<T, 8>::type*>(row + c);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? row[c + i] : (T)0.f;
    }
    __device__ __forceinline__ f8 get() const { return __builtin_convertvector(v, f8); }
};

template <typename T>
__device__ __forceinline__ void store8(T* __restrict__ row, int64_t c, int64_t cols, f8 v) {
    typedef typename VecOf<T, 8>::plain V;
    const V w = __builtin_convertvector(v, V);
    if (c + 8 <= cols) {
        *reinterpret_cast<typename VecOf<T, 8>::type*>(row + c) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < cols) row[c + i] = w[i];
}

// The same of a type that is known at run time (DT_*).
__device__ __forceinline__ f8 load8_dt(const void* p, int dt, int64_t off, int64_t c, int64_t cols) {
    if (dt == DT_F32) return load8((const float*)p + off, c, cols);
    if (dt == DT_BF16) return load8((const bf16*)p + off, c, cols);
    return load8((const f16*)p + off, c, cols);
}
__device__ __forceinline__ void store8_dt(void* p, int dt, int64_t off, int64_t c, int64_t cols, f8 v) {
    if (dt == DT_F32) store8((float*)p + off, c, cols, v);
    else if (dt == DT_BF16) store8((bf16*)p + off, c, cols, v);
    else store8((f16*)p + off, c, cols, v);
}

// ---------------------------------------------------------------- 8-bit copies
// The byte s = e + 127 of a group whose largest magnitude has these bits: e is the
// exponent less 6, one more where the significand passes 127/64; at least -126,
// so that 2^e and 2^-e are normal. Bits are compared as integers, by which a NaN is
// the largest: a group with an infinity or a NaN has s = 255.
__device__ __forceinline__ unsigned pack_scale(unsigned amax_bits) {
    const int ex = (int)(amax_bits >> 23);
    if (ex == 255) return 255u;
    const int s = ex - 6 + ((amax_bits & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    return (unsigned)(s < 1 ? 1 : s);
}
// 2^-e, or 0 for s = 255 (every q of the group is then 0 by the caller's select).
__device__ __forceinline__ float pack_inverse(unsigned s) { return __uint_as_float((254u - s) << 23); }
// 2^e; NaN for s = 255.
__device__ __forceinline__ float unpack_scale(unsigned s) {
    return s == 255u ? __uint_as_float(0x7fc00000u) : s == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23);
}
__device__ __forceinline__ unsigned abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

__device__ __forceinline__ unsigned max_bits8(f8 v) {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, abs_bits(v[i]));
    return m;
}

// Four values as int8 in a word, the lowest first; scaled by 2^-e. Added to 3 * 2^22 a value
// is rounded to an integer (ties to even), whose low byte is the sum's. With e = 122 a
// value may round to 64, and 64 * 2^122 is no fp32 value: 63 then.
__device__ __forceinline__ unsigned quant4(float a, float b, float c, float d, unsigned s) {
    const float r = pack_inverse(s), big = 12582912.f;
    unsigned ia = __float_as_uint(fmaf(a, r, big)), ib = __float_as_uint(fmaf(b, r, big));
    unsigned ic = __float_as_uint(fmaf(c, r, big)), id = __float_as_uint(fmaf(d, r, big));
    if (s >= 249u) {
        auto least = [](unsigned v) { return (unsigned)max(-63, min(63, (int)(int8_t)v)); };
        ia = least(ia), ib = least(ib), ic = least(ic), id = least(id);
    }
    const unsigned lo = __builtin_amdgcn_perm(ib, ia, 0x0c0c0400u), hi = __builtin_amdgcn_perm(id, ic, 0x04000c0cu);
    return s == 255u ? 0u : lo | hi;
}

struct __attribute__((packed, aligned(1))) Bytes8 {
    unsigned lo, hi;
};

struct RawPacked8 {
    Bytes8 b;
    unsigned s;
    __device__ __forceinline__ void load(const int8_t* __restrict__ qrow, const uint8_t* __restrict__ srow, int64_t c,
                                         int64_t cols) {
        b = Bytes8{0, 0};
        s = 127;
        if (c >= cols) return;
        s = srow[c >> 5];
        if (c + 8 <= cols) {
            b = *reinterpret_cast<const Bytes8*>(qrow + c);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) (i < 4 ? b.lo : b.hi) |= (unsigned)(uint8_t)qrow[c + i] << (8 * (i & 3));
    }
    __device__ __forceinline__ f8 get() const {
        f8 r;
        const float sc = unpack_scale(s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r[i] = (float)(int8_t)(b.lo >> (8 * i)) * sc;
            r[4 + i] = (float)(int8_t)(b.hi >> (8 * i)) * sc;
        }
        return r;
    }
};

// Columns c .. c + 7 of a copy's row: q * 2^e.
__device__ __forceinline__ f8 load_packed8(const int8_t* __restrict__ qrow, const uint8_t* __restrict__ srow, int64_t c,
                                           int64_t cols) {
    RawPacked8 r;
    r.load(qrow, srow, c, cols);
    return r.get();
}

// Eight values of a group whose scale byte is s, columns c .. c + 7.
__device__ __forceinline__ void store_packed8(int8_t* __restrict__ qrow, int64_t c, int64_t cols, f8 v, unsigned s) {
    Bytes8 b;
    b.lo = quant4(v[0], v[1], v[2], v[3], s);
    b.hi = quant4(v[4], v[5], v[6], v[7], s);
    if (c + 8 <= cols) {
        *reinterpret_cast<Bytes8*>(qrow + c) = b;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i < cols) qrow[c + i] = (int8_t)((i < 4 ? b.lo : b.hi) >> (8 * (i & 3)));
}

// The copy of 32 values held by four neighbouring lanes, eight each (zeros past
// the row's end). Every lane of the four takes part.
__device__ __forceinline__ void pack_group(int8_t* __restrict__ qrow, uint8_t* __restrict__ srow, int64_t c, int64_t cols,
                                           f8 v) {
    unsigned m = max_bits8(v);
    m = max(m, dpp<DPP_XOR1>(m));
    m = max(m, dpp<DPP_XOR2>(m));
    const unsigned s = pack_scale(m);
    if (c >= cols) return;
    store_packed8(qrow, c, cols, v, s);
    if ((c & 31) == 0) srow[c >> 5] = (uint8_t)s;
}

// ---------------------------------------------------------------- activations
// exp(x) through the hardware's 2^x (1 ulp); the arguments here are at most 0 or
// saturate to 0 and infinity as the formulas want.
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

// 1 - erf(y) for y >= 0 as t poly(t) exp(-y^2), t = 1 / (1 + 0.3 y): poly of degree 8 fitted to the
// least largest relative error of exp(y^2) (1 - erf(y)) over y <= 10.6, past which exp(-y^2) is 0. 2.0e-8 of the
// value, 4.4e-7 with the roundings, so the normal distribution function keeps its digits in the negative tail;
// ex = exp(-y^2) is passed in, since the slope of z Phi(z) needs it too.
__device__ __forceinline__ float erfc_pos(float y, float ex) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, y, 1.f));
    float p = fmaf(-0.129555672f, t, 0.485735327f);
    p = fmaf(p, t, -0.51266557f);
    p = fmaf(p, t, 0.5482077f);
    p = fmaf(p, t, -0.0950254649f);
    p = fmaf(p, t, 0.215105802f);
    p = fmaf(p, t, 0.1482867f);
    p = fmaf(p, t, 0.170723736f);
    p = fmaf(p, t, 0.169187412f);
    return p * t * ex;
}

// The forward activations as three formulas, so that a kernel holds three and not five:
// max(z, lo), lo = -inf or 0; z / (1 + 2^(z (p + q z^2))), for x / (1 + exp(-x)) and
// (1 + tanh u) / 2 = 1 / (1 + exp(-2u)), z^2 kept finite so that q = 0 times it is 0 at an
// infinite z too; z Phi(z).
struct ActForward {
    int formula;
    float p, q;
};
__device__ __forceinline__ ActForward act_forward(int act) {
    if (act == 4) return {1, -1.44269504088896341f, 0.f};
    if (act == 3) return {1, -2.30220819813644130f, -0.10294323980544930f};   // -2 log2(e) sqrt(2/pi) (1, 0.044715)
    return {act == 2 ? 2 : 0, act == 1 ? 0.f : -__builtin_inff(), 0.f};
}
// N values of one formula under one uniform branch.
template <typename V, int N>
__device__ __forceinline__ void act_apply(const ActForward& f, V (&z)[N]) {
    constexpr int W = sizeof(V) / 4;
    if (f.formula == 1) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float x = z[j][i];
                const float x2 = fminf(x * x, __FLT_MAX__);
                z[j][i] = x * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * fmaf(f.q, x2, f.p)));
            }
    } else if (f.formula == 2) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float x = z[j][i];
                const float h = 0.5f * erfc_pos(fabsf(x) * 0.70710678118654752f, exp_fast(-0.5f * x * x));
                z[j][i] = x * (x < 0.f ? h : 1.f - h);
            }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < W; ++i) z[j][i] = z[j][i] < f.p ? f.p : z[j][i];   // a NaN stays one
    }
}

// act'(z), and act(z) in *a.
template <int ACT>
__device__ __forceinline__ float act_slope(float z, float* a) {
    if constexpr (ACT == 1) {
        *a = z > 0.f || z != z ? z : 0.f;
        return z > 0.f ? 1.f : z != z ? z : 0.f;
    }
    if constexpr (ACT == 2) {
        const float ex = exp_fast(-0.5f * z * z);
        const float h = 0.5f * erfc_pos(fabsf(z) * 0.70710678118654752f, ex);
        const float p = z < 0.f ? h : 1.f - h;
        *a = z * p;
        return fmaf(z * 0.39894228040143268f, ex, p);
    }
    // With e = exp(-2u) or exp(-z) and p = 1 / (1 + e), 1 - p as e p: as a difference it would be
    // off by 2^-25, which z u' makes 1.5e-6 of gelu_tanh's slope at z = 5. An infinite e, for which
    // p is 0, and z^2 are kept finite, so that 0 times them is 0.
    if constexpr (ACT == 3) {
        const float z2 = fminf(z * z, 1e30f);
        const float e = __builtin_amdgcn_exp2f(z * fmaf(-0.10294323980544930f, z2, -2.30220819813644130f));
        const float p = __builtin_amdgcn_rcpf(1.f + e);
        *a = z * p;
        return fmaf(p * (fminf(e, __FLT_MAX__) * p) * z, fmaf(0.21406444881780073f, z2, 1.595769121605731f), p);
    }
    if constexpr (ACT == 4) {
        const float e = exp_fast(-z);
        const float p = __builtin_amdgcn_rcpf(1.f + e);
        *a = z * p;
        return fmaf(p * (fminf(e, __FLT_MAX__) * p), z, p);
    }
    *a = z;
    return 1.f;
}

// f(integral constant of the activation): one uniform branch around the code of each.
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (act) {
        case 1: f(std::integral_constant<int, 1>()); break;
        case 2: f(std::integral_constant<int, 2>()); break;
        case 3: f(std::integral_constant<int, 3>()); break;
        case 4: f(std::integral_constant<int, 4>()); break;
        default: f(std::integral_constant<int, 0>()); break;
    }
}

// The gate of a gated layer, backward: of N values g, u and da, dg = da u act'(g), du = da act(g), a = act(g) u, in the
// places of da, u and g. As three formulas, as forward (the products' epilogue holds this code for each sixteen rows): of
// act_slope's, relu and none as one, and gelu_tanh and silu as z / (1 + e), e = 2^(z (p + q z^2)), whose slope is
// P + P (1 - P) z (r + s z^2), P = 1 / (1 + e).
template <typename V, int N>
__device__ __forceinline__ void gate_slopes(int act, V (&g)[N], V (&u)[N], V (&da)[N]) {
    constexpr int W = sizeof(V) / 4;
    auto each = [&](auto f) {
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                float a;
                const float slope = f(g[j][i], a), x = u[j][i], d = da[j][i];
                da[j][i] = d * x * slope;
                u[j][i] = d * a;
                g[j][i] = a * x;
            }
    };
    const ActForward f = act_forward(act);
    if (f.formula == 1) {
        const float r = act == 4 ? 1.f : 1.595769121605731f, s = act == 4 ? 0.f : 0.21406444881780073f;
        each([&](float z, float& a) {
            const float z2 = fminf(z * z, 1e30f);
            const float e = __builtin_amdgcn_exp2f(z * fmaf(f.q, z2, f.p));
            const float p = __builtin_amdgcn_rcpf(1.f + e);
            a = z * p;
            return fmaf(p * (fminf(e, __FLT_MAX__) * p) * z, fmaf(s, z2, r), p);
        });
    } else if (f.formula == 2) {
        each([&](float z, float& a) { return act_slope<2>(z, &a); });
    } else {
        each([&](float z, float& a) {
            a = z < f.p ? f.p : z;   // a NaN stays one
            return act == 0 || z > 0.f ? 1.f : z != z ? z : 0.f;
        });
    }
}

// What the rounding of v to T leaves, as it is stored beside it: times 2^11 in fp16, whose range would cut it (a gradient of
// 2^-10 leaves 2^-21, and fp16 has steps of 2^-24). In bf16 it has the range of v. Products take the factor out again.
template <typename T>
constexpr float REST_SCALE = std::is_same_v<T, f16> ? 2048.f : 1.f;
template <typename T, typename V>
__device__ __forceinline__ V rest_of(V v) {
    typedef typename VecOf<T, sizeof(V) / 4>::plain R;
    return (v - __builtin_convertvector(__builtin_convertvector(v, R), V)) * REST_SCALE<T>;
}

// v in 16-bit parts, each what the rounding of those before it leaves: one or two of 16-bit data, three bf16 ones of fp32,
// of which the first is cut at bf16's largest value (see k_lay_out_split in linear.hip).
template <typename T>
__device__ __forceinline__ void store_parts(void* base, int64_t part, int parts, int64_t off, int64_t c, int64_t cols, f8 v) {
    using R = std::conditional_t<sizeof(T) == 4, bf16, T>;
    typedef typename VecOf<R, 8>::plain V;
    for (int p = 0; p < parts; ++p) {
        f8 x = v;
        if (sizeof(T) == 4 && p == 0)
            x = __builtin_elementwise_min(__builtin_elementwise_max(x, f8(-0x1.fep127f)), f8(0x1.fep127f));
        const f8 r = __builtin_convertvector(__builtin_convertvector(x, V), f8);
        store8((R*)((char*)base + p * part) + off, c, cols, r);
        v = (v - r) * REST_SCALE<R>;
    }
}
// Columns c .. c + 7 of row m of dz = [d u] and a (N columns each, d, u and a zeros past them), and zeros up to the rows' ends.
template <typename T>
__device__ __forceinline__ void store_dz(const Epilogue& e, int64_t N, int64_t m, int64_t c, f8 d, f8 u, f8 a) {
    if constexpr (std::is_same_v<T, f16>)
        if (e.range) {
            d *= e.range[0];
            u *= e.range[0];
            a *= e.range[1];
        }
    if (e.out) {
        store_parts<T>(e.out, e.out_part, e.parts, m * e.ldo, c, N, d);
        store_parts<T>(e.out, e.out_part, e.parts, m * e.ldo + N, c, e.ldo - N, u);
        if (c + 8 >= N && c + 8 < e.ldo - N) store_parts<T>(e.out, e.out_part, e.parts, m * e.ldo + N, c + 8, e.ldo - N, f8{});
    }
    if (e.a) store_parts<T>(e.a, e.a_part, e.parts, m * e.lda, c, e.lda, a);
}

// ---------------------------------------------------------------- sums over a wave
__device__ __forceinline__ float wave_sum(float v) {
    v += __uint_as_float(dpp<DPP_XOR1>(__float_as_uint(v)));
    v += __uint_as_float(dpp<DPP_XOR2>(__float_as_uint(v)));
    v += __uint_as_float(dpp<DPP_HALF_MIRROR>(__float_as_uint(v)));
    v += __uint_as_float(dpp<DPP_MIRROR>(__float_as_uint(v)));
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(h[0]) + __uint_as_float(h[1]);
}
__device__ __forceinline__ float sum8(f8 v) {
    return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}

}  // namespace
}  // namespace mfac
