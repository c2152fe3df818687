// The kernel of the large products (see linear.hip) and its launch, for the files that compile it: product_layer.hip,
// product_gated.hip and product_hidden.hip, each some of its epilogues.
#pragma once

#include <algorithm>
#include <utility>

#include "internal.h"
#include "train.h"
#include "train_util.h"

namespace mfac {

struct GemmArgs {
    const char *A, *B;       // 16-bit elements
    int64_t lda, ldb;        // bytes
    int64_t apl, bpl;        // bytes between planes
    int M, N, K;             // GATED: N columns of the result, from 2 N rows of B
    int64_t up;              // GATED: bytes from B's first row to row N
    int ksteps, nseg;        // BK-wide steps over K, and how often K is gone over (pairs of planes)
    unsigned pa, pb;         // planes of the pairs, 4 bits each
    int tiles_m, tiles_n, splits;
    float* part;             // [splits][M][N] sums (GATED: [M][2 N]), where splits > 1
    Epilogue e;
};

struct Operand {
    int planes;               // 16-bit parts: 3 of fp32, 2 of a value and what its rounding left
    bool lay_out;
    int64_t rows, cols, ld;   // as laid out in memory
    size_t bytes;             // in the workspace
};
struct Plan {
    bool skinny;
    Operand a, b;
    int tile, ksteps, nseg, splits;
    int64_t tiles_m, tiles_n;
    size_t part_bytes;
};

// Past the 256 MB of the last-level cache, outputs written through the caches push the operands
// out: 8192^3, dx and dW took 1003 and 1030 us with plain stores, 915 and 943 with nontemporal
// ones (both are faster now). Below, those are slower: dx of 8192 x 8192 over K = 2048 took
// 248 us, with them 271.
constexpr int64_t LAST_LEVEL_CACHE = int64_t(256) << 20;
// Whether a product's results are stored past the caches: in tiles of 256, where they and the operands exceed them.
// `kept`: bytes of a gated layer's pre-activations (bf16 8192 rows, 2048 to 8192, and the copies' return: 587 us so, 603 through
// the caches).
inline bool streams(const Product& p, const Plan& q, int out_dt, int64_t kept = 0) {
    const int64_t out = p.gate == GATE_FORWARD ? p.M * p.N / 2 : p.M * p.N;
    const int64_t bytes = (p.M * p.K + p.N * p.K) * 2 * (q.nseg > 1 ? 3 : 1) + out * dtype_bytes(out_dt) + kept;
    return q.tile == 256 && bytes > LAST_LEVEL_CACHE;
}
// Bytes that a gated layer stores of its pre-activations, of type dt or as copies.
inline int64_t kept_bytes(const Product& p, bool z, bool copies, int dt) {
    return z ? p.M * p.N * dtype_bytes(dt) : copies ? p.M * p.N : 0;
}

// Launches the tiles of a product; compiled in the files named above.
template <typename T, int KIND>
hipError_t run_product(const Product& p, const Plan& q, const GemmArgs& g, hipStream_t st);

namespace {

typedef float v4 __attribute__((ext_vector_type(4)));

template <int... I, typename F>
__device__ __forceinline__ void for_each_index(std::integer_sequence<int, I...>, F f) {
    (f(std::integral_constant<int, I>()), ...);
}

// ---------------------------------------------------------------- epilogue
// The products' epilogues; the fields of the others are unused.
// WEIGHT_PARTS is WEIGHT of an fp16 operand in two parts: a kernel of its own, since its look at every K step for the end of
// the second parts cost plain fp16 gradients 1 to 5% (2048 rows, 1024 to 1024: 16.8 us against 16.0).
enum : int { FORWARD = 0, INPUT = 1, WEIGHT = 2, GATED = 3, HIDDEN = 4, WEIGHT_PARTS = 5 };
constexpr bool is_weight(int kind) { return kind == WEIGHT || kind == WEIGHT_PARTS; }
constexpr bool a_is_col(int kind) { return is_weight(kind); }
constexpr bool b_is_col(int kind) { return kind == INPUT || is_weight(kind) || kind == HIDDEN; }
constexpr int HIDDEN_COLS = 64;   // HIDDEN's N is a multiple of a wave's columns in every tile

// What an epilogue reads for columns n .. n + 7, whichever the row.
struct OfColumn {
    f8 bias, beta;   // bias, or gamma
};
template <int KIND>
__device__ __forceinline__ OfColumn of_column(const Epilogue& e, int64_t N, int64_t n) {
    OfColumn o{};
    if (KIND == FORWARD && e.bias) o.bias = load8_dt(e.bias, e.bias_dt, 0, n, N);
    if (KIND == WEIGHT && e.gamma) {
        o.bias = load8(e.gamma, n, N);
        if (e.beta) o.beta = load8(e.beta, n, N);
    }
    return o;
}
// And for (m, n .. n + 7).
struct OfPlace {
    f8 add;
    float db;
};
template <int KIND>
__device__ __forceinline__ OfPlace of_place(const Epilogue& e, int64_t N, bool in, int64_t m, int64_t n) {
    OfPlace o{};
    if (KIND != WEIGHT && e.add && in) o.add = load8_dt(e.add, e.io_dt, m * e.ldadd, n, N);
    if (KIND == WEIGHT && e.beta && in) o.db = e.db[m];
    return o;
}

// The sums c at (m, n .. n + 7) become outputs. Four neighbouring lanes hold 32
// neighbouring n of one row; every lane of a wave takes part (in: whether m is a row).
template <int KIND>
__device__ __forceinline__ void finish8(const Epilogue& e, int64_t N, bool in, int64_t m, int64_t n, f8 c,
                                        const OfColumn& col, const OfPlace& at) {
    if (!in) n = N;
    if constexpr (KIND == FORWARD) {
        c += col.bias;
        if (e.p.q) {
            f8 v = c;
            if (n + 8 > N)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (n + i >= N) v[i] = 0.f;
            pack_group(e.p.q + m * e.p.ldq, e.p.s + m * ((N + 31) / 32), n, N, v);
        }
        if (e.z && n < N) store8_dt(e.z, e.io_dt, m * e.ldz, n, N, c);
        f8 one[1] = {c};
        act_apply(act_forward(e.act), one);
        c = one[0];
    }
    if constexpr (KIND == WEIGHT)
        if (e.gamma) c = c * col.bias + at.db * col.beta;
    if constexpr (KIND != WEIGHT) c += at.add;
    if (n < N) store8_dt(e.out, e.out_dt, m * e.ldo, n, N, c);
}
template <int KIND>
__device__ __forceinline__ void finish8(const Epilogue& e, int64_t N, bool in, int64_t m, int64_t n, f8 c) {
    finish8<KIND>(e, N, in, m, n, c, of_column<KIND>(e, N, n), of_place<KIND>(e, N, in, m, n));
}

// The same of a gated layer: the gate's and the other projection's sums for columns n .. n + 7 of N.
__device__ __forceinline__ void finish_gated8(const Epilogue& e, int64_t N, bool in, int64_t m, int64_t n, f8 g, f8 u) {
    if (!in) n = N;
    if (e.bias) {
        g += load8_dt(e.bias, e.bias_dt, 0, n, N);
        u += load8_dt(e.bias, e.bias_dt, N, n, N);
    }
    if (e.p.q) {
        f8 v[2] = {g, u};
        if (n + 8 > N)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (n + i >= N) v[0][i] = v[1][i] = 0.f;
        const int64_t ng = (N + 31) / 32;
        pack_group(e.p.q + m * e.p.ldq, e.p.s + m * ng, n, N, v[0]);
        pack_group(e.p2.q + m * e.p2.ldq, e.p2.s + m * ng, n, N, v[1]);
    }
    if (n >= N) return;
    if (e.z) {
        store8_dt(e.z, e.io_dt, m * e.ldz, n, N, g);
        store8_dt(e.z2, e.io_dt, m * e.ldz, n, N, u);
    }
    f8 one[1] = {g};
    act_apply(act_forward(e.act), one);
    store8_dt(e.out, e.out_dt, m * e.ldo, n, N, one[0] * u);
}
// And of the gradient of its output, c: dz and a.
__device__ __forceinline__ void finish_hidden8(const Epilogue& e, int64_t N, bool in, int64_t m, int64_t n, f8 c) {
    if (!in || n >= N) return;
    f8 d[1] = {c}, g[1], u[1];
    if (e.p.q) {
        const int64_t ng = (N + 31) / 32;
        g[0] = load_packed8(e.p.q + m * e.p.ldq, e.p.s + m * ng, n, N);
        u[0] = load_packed8(e.p2.q + m * e.p2.ldq, e.p2.s + m * ng, n, N);
    } else {
        g[0] = load8_dt(e.z, e.io_dt, m * e.ldz, n, N);
        u[0] = load8_dt(e.z2, e.io_dt, m * e.ldz, n, N);
    }
    gate_slopes(e.act, g, u, d);
    if (e.io_dt == DT_F32) store_dz<float>(e, N, m, n, d[0], u[0], g[0]);
    else if (e.io_dt == DT_BF16) store_dz<bf16>(e, N, m, n, d[0], u[0], g[0]);
    else store_dz<f16>(e, N, m, n, d[0], u[0], g[0]);
}

// Four sums at a time, as the matrix cores leave them: lane l has columns n .. n + 3, n = 4 (l / 16)
// of 16, of row l % 16. EDGE: columns past N are possible; tiles without them run code
// without their checks, which would be most of it (and more than the instruction
// cache holds). Values are fp32 or of the operands' type T.
template <bool EDGE, typename T>
__device__ __forceinline__ v4 load4(const T* row, int64_t n, int64_t N) {
    if (!EDGE || n + 4 <= N) {
        const typename VecOf<T, 4>::plain v = *reinterpret_cast<const typename VecOf<T, 4>::type*>(row + n);
        return __builtin_convertvector(v, v4);
    }
    v4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < N) r[i] = (float)row[n + i];
    return r;
}
template <bool EDGE, typename T>
__device__ __forceinline__ v4 load4_dt(const void* p, int dt, int64_t off, int64_t n, int64_t N) {
    return dt == DT_F32 ? load4<EDGE>((const float*)p + off, n, N) : load4<EDGE>((const T*)p + off, n, N);
}
// STREAM: nontemporal stores, which leave the caches to the operands but take longer
// (see LAST_LEVEL_CACHE).
template <bool STREAM, typename V, typename P>
__device__ __forceinline__ void put(V v, P* p) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <bool EDGE, bool STREAM>
__device__ __forceinline__ void store4(float* row, int64_t n, int64_t N, v4 v) {
    if (!EDGE || n + 4 <= N) {
        put<STREAM>(v, reinterpret_cast<VecOf<float, 4>::type*>(row + n));
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < N) row[n + i] = v[i];
}
// Of two tiles of 16 columns, a in the first and b in the second: lanes with an even l / 16
// get their neighbour's a beside their own, those with an odd one their neighbour's b.
__device__ __forceinline__ void swap_rows(unsigned& a, unsigned& b) {
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
template <bool EDGE, bool STREAM, typename T>
__device__ __forceinline__ void store_pair16(T* row, int64_t n, int64_t N, int lane, v4 a, v4 b) {
    typedef typename VecOf<T, 4>::plain V;
    typedef unsigned u2 __attribute__((ext_vector_type(2)));
    typedef unsigned u4 __attribute__((ext_vector_type(4)));
    u2 x = __builtin_bit_cast(u2, __builtin_convertvector(a, V)), y = __builtin_bit_cast(u2, __builtin_convertvector(b, V));
    unsigned x0 = x[0], x1 = x[1], y0 = y[0], y1 = y[1];
    swap_rows(x0, y0);
    swap_rows(x1, y1);
    n += (lane >> 4 & 1) * 12;   // an odd l / 16: 16 further, less 4
    const u4 v = {x0, x1, y0, y1};
    const auto w = __builtin_bit_cast(typename VecOf<T, 8>::plain, v);
    if (!EDGE || n + 8 <= N) {
        put<STREAM>(w, reinterpret_cast<typename VecOf<T, 8>::type*>(row + n));
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (n + i < N) row[n + i] = w[i];
}
template <bool EDGE, bool STREAM, typename T, int NTL>
__device__ __forceinline__ void store_quads(void* p, int dt, int64_t off, int64_t n, int64_t N, int lane,
                                            const v4 (&c)[NTL]) {
    if (dt == DT_F32) {
#pragma unroll
        for (int j = 0; j < NTL; ++j) store4<EDGE, STREAM>((float*)p + off, n + j * 16, N, c[j]);
    } else {
#pragma unroll
        for (int j = 0; j < NTL; j += 2)
            store_pair16<EDGE, STREAM>((T*)p + off, n + j * 16, N, lane, c[j], c[j + 1]);
    }
}
// The 8-bit copy of a row's 32 columns from two such tiles, a and b.
template <bool EDGE>
__device__ __forceinline__ void pack_quads(int8_t* qrow, uint8_t* srow, int64_t n, int64_t N, int lane, v4 a, v4 b) {
    if constexpr (EDGE)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (n + i >= N) a[i] = 0.f;
            if (n + 16 + i >= N) b[i] = 0.f;
        }
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max(abs_bits(a[i]), abs_bits(b[i])));
    unsigned o = m;
    swap_rows(m, o);
    m = o = max(m, o);
    const auto r = __builtin_amdgcn_permlane32_swap(m, o, false, false);
    const unsigned s = pack_scale(max(r[0], r[1]));
    unsigned x = quant4(a[0], a[1], a[2], a[3], s), y = quant4(b[0], b[1], b[2], b[3], s);
    swap_rows(x, y);
    if (lane < 16 && (!EDGE || n < N)) srow[n >> 5] = (uint8_t)s;
    n += (lane >> 4 & 1) * 12;
    if (!EDGE || n + 8 <= N) {
        *reinterpret_cast<Bytes8*>(qrow + n) = Bytes8{x, y};
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (n + i < N) qrow[n + i] = (int8_t)((i < 4 ? x : y) >> (8 * (i & 3)));
}

// ---------------------------------------------------------------- large products
// Operand tile of R rows (of C's m or n) by BK = 64 k in LDS, in pieces of 16 bytes.
// [row][k] in memory: row r at piece 8 r, its piece p at p ^ (r % 8): the 16 rows that a
// fragment read touches at one p lie in all banks. [k][row] in memory: k at piece
// k R/8, its piece p at p ^ 2 f(k), f(k) = (k & 3) | (k >> 1 & 4): the eight k that
// half a wave's transposing read touches lie in all banks.
constexpr int BK = 64;
constexpr unsigned OUT_OF_RANGE = 0x80000000u;   // past every buffer's size: the copy writes zeros

__device__ __forceinline__ int row_swizzle(int r) { return r & 7; }
template <int R>
__device__ __forceinline__ int col_swizzle(int k) {
    return ((k & 3) | (k >> 1 & 4)) << 1 & (R / 8 - 1);   // 64 rows: four of the eight k
}

// What a thread copies of an operand tile: NI pieces, NT * 16 bytes apart in LDS. GATE: the tile's rows are by turns GATE
// of the gate's (from row0) and the same GATE of the other projection's; the eight rows that a wave copies at a time
// lie on one side, so the sides differ in the scalar address only.
template <int R, int NT, bool COL, int GATE = 0>
struct Copier {
    static_assert(GATE % 8 == 0 && (GATE & (GATE - 1)) == 0, "");
    static constexpr int NI = R * BK / 8 / NT;
    unsigned off[NI];
    int k[COL ? NI : 1];
    int64_t step;   // bytes from one K step to the next
    __device__ __forceinline__ void init(int t, int row0, int rows, int64_t ld) {
        if constexpr (COL) {
            step = BK * ld;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int l = i * NT + t, kk = l / (R / 8), c = ((l % (R / 8)) ^ col_swizzle<R>(kk)) * 8;
                k[i] = kk;
                off[i] = row0 + c < rows ? (unsigned)(kk * ld + c * 2) : OUT_OF_RANGE;
            }
        } else {
            step = BK * 2;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int l = i * NT + t, r = l >> 3;
                const int kc = ((l & 7) ^ row_swizzle(r)) * 8;
                k[0] = kc;   // the same for every i
                const int at = GATE ? r / (2 * GATE + !GATE) * GATE + r % (GATE + !GATE) : r;
                // a row past the end reads the last one: its sums are not stored
                off[i] = (unsigned)(min(at, rows - 1 - row0) * ld + kc * 2);
            }
        }
    }
    // base: the tile's first element at this step; left: K's elements from there on. In
    // assembly because the compiler waits for the builtin's copies before the next transposing
    // read of LDS, whichever buffer that reads (dx and dW of 8192^3: 899 and 921 us with it);
    // the kernel's own waits are all that is needed. Nothing is loaded into registers, and an
    // offset past the buffer's size writes zeros.
    __device__ __forceinline__ void issue(const char* base, int left, unsigned lds, int wave, int64_t up = 0) const {
        typedef int i4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            uint64_t b = (uint64_t)base;
            if (GATE && ((i * (NT / 8) + wave * 8) & GATE)) b += up;
            // base, stride 0, size OUT_OF_RANGE, raw 32-bit data
            const i4 r = {__builtin_amdgcn_readfirstlane((int)b), __builtin_amdgcn_readfirstlane((int)(b >> 32)),
                          (int)OUT_OF_RANGE, 0x00020000};
            const unsigned o = left >= BK || k[COL ? i : 0] < left ? off[i] : OUT_OF_RANGE;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                         :
                         : "s"(__builtin_amdgcn_readfirstlane(lds + (i * NT + wave * 64) * 16)), "v"(o), "s"(r)
                         : "memory", "m0");
        }
    }
};

template <typename T>
struct Frag {
    typedef typename VecOf<T, 8>::plain type;
};
__device__ __forceinline__ v4 mma(VecOf<bf16, 8>::plain a, VecOf<bf16, 8>::plain b, v4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ v4 mma(VecOf<f16, 8>::plain a, VecOf<f16, 8>::plain b, v4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Fragment of 16 rows (from row0) and k 32 kk .. + 31: lane l holds row l % 16 and eight k
// from 8 (l / 16).
template <typename T, int R, bool COL>
__device__ __forceinline__ typename Frag<T>::type read_frag(const char* lds, int row0, int kk, int lane) {
    if constexpr (COL) {
        typedef short s4 __attribute__((ext_vector_type(4)));
        typedef short s8 __attribute__((ext_vector_type(8)));
        const int k = kk * 32 + (lane >> 4) * 8 + ((lane & 15) >> 2), r = row0 + 4 * (lane & 3);
        const int at = k * R * 2 + ((r >> 3) ^ col_swizzle<R>(k)) * 16 + (r & 4) * 2;
        typedef __attribute__((address_space(3))) s4* P;
        const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + at));
        const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + at + 4 * R * 2));
        const s8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(typename Frag<T>::type, v);
    } else {
        const int r = row0 + (lane & 15), p = kk * 4 + (lane >> 4);
        return *reinterpret_cast<const typename Frag<T>::type*>(lds + r * (BK * 2) + (p ^ row_swizzle(r)) * 16);
    }
}

// The sums of a wave's tile into outputs; (m, n): this lane's first place. Straight from the
// registers: through LDS, whole rows of a tile stored together, it took 11 us a tile of
// 256 x 256, this way 7, of which 5 are the memory's (bf16, every CU at once).
template <typename T, int KIND, bool EDGE, bool STREAM, int MT, int NTL>
__device__ __forceinline__ void epilogue(const GemmArgs& g, float* part, int lane, int64_t m0, int64_t n,
                                         v4 (&acc)[MT][NTL]) {
    constexpr bool FWD = KIND == FORWARD, WGT = is_weight(KIND);
    const Epilogue& e = g.e;
    const int64_t N = g.N;
    v4 bias[NTL], beta[WGT ? NTL : 1];   // bias, or gamma
    ActForward act{};
    if constexpr (FWD) act = act_forward(e.act);
#pragma unroll
    for (int j = 0; j < NTL; ++j) {
        bias[j] = v4{0.f, 0.f, 0.f, 0.f};
        if (FWD && e.bias) bias[j] = load4_dt<EDGE, T>(e.bias, e.bias_dt, 0, n + j * 16, N);
        if constexpr (WGT)
            if (e.gamma) {
                bias[j] = load4<EDGE>(e.gamma, n + j * 16, N);
                beta[j] = v4{0.f, 0.f, 0.f, 0.f};
                if (e.beta) beta[j] = load4<EDGE>(e.beta, n + j * 16, N);
            }
    }
    // by templates: the body is past what the compiler unrolls, and acc must stay in registers
    for_each_index(std::make_integer_sequence<int, MT>(), [&](auto tag) {
        constexpr int i = decltype(tag)::value;
        const int64_t m = m0 + i * 16;
        if (m >= g.M) return;   // the four lanes of a row leave together
        if (part) {
#pragma unroll
            for (int j = 0; j < NTL; ++j) store4<EDGE, false>(part + m * N, n + j * 16, N, acc[i][j]);
            return;
        }
        if constexpr (FWD) {
#pragma unroll
            for (int j = 0; j < NTL; ++j) acc[i][j] += bias[j];
            if (e.p.q)
#pragma unroll
                for (int j = 0; j < NTL; j += 2)
                    pack_quads<EDGE>(e.p.q + m * e.p.ldq, e.p.s + m * ((N + 31) / 32), n + j * 16, N, lane, acc[i][j],
                                     acc[i][j + 1]);
            if (e.z) store_quads<EDGE, STREAM, T>(e.z, e.io_dt, m * e.ldz, n, N, lane, acc[i]);
            act_apply(act, acc[i]);
        }
        if constexpr (WGT)
            if (e.gamma) {
                const float db = e.beta ? e.db[m] : 0.f;
#pragma unroll
                for (int j = 0; j < NTL; ++j) acc[i][j] = acc[i][j] * bias[j] + db * beta[j];
            }
        if constexpr (!WGT)
            if (e.add)
#pragma unroll
                for (int j = 0; j < NTL; ++j)
                    acc[i][j] += load4_dt<EDGE, T>(e.add, e.io_dt, m * e.ldadd, n + j * 16, N);
        store_quads<EDGE, STREAM, T>(e.out, e.out_dt, m * e.ldo, n, N, lane, acc[i]);
    });
}

// The same of a gated layer: the first half of a wave's columns are the gate's, the second the other projection's, for
// the same N columns of the result. A tile's two halves of C meet in registers, so the pre-activations reach the memory only
// where they are kept: bf16 8192 rows, 2048 to 8192, both kept in 8 bits, 499 to 515 us (1.07 to 1.10 PFLOP/s).
template <typename T, bool EDGE, bool STREAM, int MT, int NTL>
__device__ __forceinline__ void epilogue_gated(const GemmArgs& g, float* part, int lane, int64_t m0, int64_t n,
                                               v4 (&acc)[MT][NTL]) {
    constexpr int H = NTL / 2;
    const Epilogue& e = g.e;
    const int64_t N = g.N;
    v4 bias[NTL];
    const ActForward act = act_forward(e.act);
#pragma unroll
    for (int j = 0; j < H; ++j) {
        bias[j] = bias[H + j] = v4{0.f, 0.f, 0.f, 0.f};
        if (e.bias) {
            bias[j] = load4_dt<EDGE, T>(e.bias, e.bias_dt, 0, n + j * 16, N);
            bias[H + j] = load4_dt<EDGE, T>(e.bias, e.bias_dt, N, n + j * 16, N);
        }
    }
    for_each_index(std::make_integer_sequence<int, MT>(), [&](auto tag) {
        constexpr int i = decltype(tag)::value;
        const int64_t m = m0 + i * 16;
        if (m >= g.M) return;   // the four lanes of a row leave together
        if (part) {
#pragma unroll
            for (int j = 0; j < H; ++j) {
                store4<EDGE, false>(part + m * 2 * N, n + j * 16, N, acc[i][j]);
                store4<EDGE, false>(part + m * 2 * N + N, n + j * 16, N, acc[i][H + j]);
            }
            return;
        }
        v4 a[H], u[H];
#pragma unroll
        for (int j = 0; j < H; ++j) {
            a[j] = acc[i][j] + bias[j];
            u[j] = acc[i][H + j] + bias[H + j];
        }
        if (e.p.q) {
            const int64_t ng = (N + 31) / 32;
#pragma unroll
            for (int j = 0; j < H; j += 2) {
                pack_quads<EDGE>(e.p.q + m * e.p.ldq, e.p.s + m * ng, n + j * 16, N, lane, a[j], a[j + 1]);
                pack_quads<EDGE>(e.p2.q + m * e.p2.ldq, e.p2.s + m * ng, n + j * 16, N, lane, u[j], u[j + 1]);
            }
        }
        if (e.z) {
            store_quads<EDGE, STREAM, T>(e.z, e.io_dt, m * e.ldz, n, N, lane, a);
            store_quads<EDGE, STREAM, T>(e.z2, e.io_dt, m * e.ldz, n, N, lane, u);
        }
        act_apply(act, a);
#pragma unroll
        for (int j = 0; j < H; ++j) a[j] *= u[j];
        store_quads<EDGE, STREAM, T>(e.out, e.out_dt, m * e.ldo, n, N, lane, a);
    });
}

// Eight neighbouring pre-activations as loaded, or of an 8-bit copy.
template <typename T>
struct RawEight {
    typedef unsigned u4 __attribute__((ext_vector_type(4)));
    u4 w;
    __device__ __forceinline__ void load(const void* z, int64_t ldz, const Packed& p, int64_t m, int64_t n, int64_t N) {
        if (p.q) {
            const Bytes8 b = *reinterpret_cast<const Bytes8*>(p.q + m * p.ldq + n);
            w[0] = b.lo;
            w[1] = b.hi;
            w[2] = p.s[m * (N / 32) + (n >> 5)];
        } else {
            const typename VecOf<T, 8>::plain v = *reinterpret_cast<const typename VecOf<T, 8>::type*>((const T*)z + m * ldz + n);
            w = __builtin_bit_cast(u4, v);
        }
    }
    __device__ __forceinline__ f8 get(bool packed) const {
        if (packed) return RawPacked8{{w[0], w[1]}, w[2]}.get();
        return __builtin_convertvector(__builtin_bit_cast(typename VecOf<T, 8>::plain, w), f8);
    }
};

// The gradient da of a gated layer's output becomes dz and a, of 16-bit data, in one part or two. The sums of two tiles of
// 16 columns are exchanged first, so that a lane has eight neighbours and takes 16 bytes of z at a time; the pre-activations
// of the next sixteen rows are on their way while these are worked on. N is a multiple of the columns that a wave has
// (HIDDEN_COLS), so a wave has them all or none: with checks for each column this code would be twice as long, and a wave runs
// all of it once a tile.
template <typename T, int MT, int NTL>
__device__ __forceinline__ void epilogue_hidden(const GemmArgs& g, int lane, int64_t m0, int64_t n,
                                                v4 (&acc)[MT][NTL]) {
    constexpr int H = NTL / 2;
    typedef typename VecOf<T, 8>::plain V;
    const Epilogue& e = g.e;
    const int64_t N = g.N;
    const bool packed = e.p.q;
    n += (lane >> 4 & 1) * 12;   // an odd l / 16: 16 further, less 4
    RawEight<T> zg[H], zu[H];
    auto load = [&](int64_t m) {
        m = min(m, (int64_t)g.M - 1);
#pragma unroll
        for (int j = 0; j < H; ++j) {
            zg[j].load(e.z, e.ldz, e.p, m, n + j * 32, N);
            zu[j].load(e.z2, e.ldz, e.p2, m, n + j * 32, N);
        }
    };
    float dz_by = 1.f, a_by = 1.f;
    if constexpr (std::is_same_v<T, f16>)
        if (e.range) {
            dz_by = e.range[0];
            a_by = e.range[1];
        }
    auto store = [&](void* base, int64_t apart, int64_t off, f8 v, float by) {
        T* at = (T*)base + off;
        if constexpr (std::is_same_v<T, f16>) v *= by;
        const V first = __builtin_convertvector(v, V);
        *reinterpret_cast<typename VecOf<T, 8>::type*>(at) = first;
        if (e.parts == 1) return;
        at = (T*)((char*)at + apart);
        *reinterpret_cast<typename VecOf<T, 8>::type*>(at) = __builtin_convertvector(rest_of<T>(v), V);
    };
    load(m0);
    for_each_index(std::make_integer_sequence<int, MT>(), [&](auto tag) {
        constexpr int i = decltype(tag)::value;
        const int64_t m = m0 + i * 16;
        f8 d[H], a[H], u[H];
#pragma unroll
        for (int j = 0; j < H; ++j) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                unsigned x = __float_as_uint(acc[i][2 * j][k]), y = __float_as_uint(acc[i][2 * j + 1][k]);
                swap_rows(x, y);
                d[j][k] = __uint_as_float(x);
                d[j][4 + k] = __uint_as_float(y);
            }
            a[j] = zg[j].get(packed);
            u[j] = zu[j].get(packed);
        }
        if (i + 1 < MT) load(m + 16);
        if (m >= g.M) return;
        gate_slopes(e.act, a, u, d);
#pragma unroll
        for (int j = 0; j < H; ++j) {
            if (e.out) {
                store(e.out, e.out_part, m * e.ldo + n + j * 32, d[j], dz_by);
                store(e.out, e.out_part, m * e.ldo + N + n + j * 32, u[j], dz_by);
            }
            if (e.a) store(e.a, e.a_part, m * e.lda + n + j * 32, a[j], a_by);
        }
    });
}

// A work-group's TM x TN tile of C, one part of K; each wave (TM/WM) x (TN/WN) of it. The
// MFMA's rows are n and its columns m, so that a lane's four sums are neighbours in a
// row of C. 256 x 256 by eight waves of 128 x 64, K steps of 64 (whole 128-byte lines of a
// row) in two stages fill 128 KB of LDS and 240 registers: the widest tile, because the
// operands' way from L2 to LDS is what narrower ones wait for (two work-groups of 256 x 128
// with steps of 32 on a CU took 1061 us for 8192^3 against 826).
// bf16 8192^3: y 790 us, dx 805, dW 821 (1392, 1365, 1339 TFLOP/s; a large library product
// reaches 1270 to 1330); the matrix cores are busy for 66% of the cycles, at the clock that
// the card's power leaves (2.0 GHz). Over K = 2048, 8192 x 8192: y 222 to 237 us, of which
// the four rounds of epilogues take 24.
// The sums stay in the MFMA's accumulators over all of K: against 64 bits an fp32 dW of
// random bf16 operands is off by 1.9e-7 (relative, 2-norm) over 8192 rows, 2.8e-7
// over 16384.
template <typename T, int KIND, int TM, int TN, int WM, int WN, int STAGES, bool STREAM>
__global__ __launch_bounds__(WM* WN * 64, 2) void k_product(GemmArgs g) {
    constexpr int NT = WM * WN * 64, MT = TM / WM / 16, NTL = TN / WN / 16;
    constexpr int STAGE = (TM + TN) * BK * 2;
    constexpr bool ACOL = a_is_col(KIND), BCOL = b_is_col(KIND);
    constexpr int GATE = KIND == GATED ? TN / WN / 2 : 0;   // columns of the result that a wave has
    constexpr int COLS = KIND == GATED ? TN / 2 : TN;
    __shared__ __attribute__((aligned(1024))) char lds[STAGES * STAGE];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave / WN, wn = wave % WN;

    // Tile and part of K of this work-group. Work-groups go round-robin over the 8 XCDs, each
    // with its own L2: an XCD takes neighbours of a list that has the tiles of one part
    // of K together, in bands of 8 tile rows.
    const int ntile = g.tiles_m * g.tiles_n, total_wgs = ntile * g.splits;
    const int xcd = blockIdx.x % 8, each = total_wgs / 8, more = total_wgs % 8;
    const int at = xcd * each + min(xcd, more) + blockIdx.x / 8;
    const int k_part = at / ntile, p = at - k_part * ntile;
    constexpr int BAND = 8;
    const int band = p / (BAND * g.tiles_n), in_band = p % (BAND * g.tiles_n);
    const int height = min(BAND, g.tiles_m - band * BAND);
    const int m0 = (band * BAND + in_band % height) * TM, n0 = in_band / height * COLS;

    Copier<TM, NT, ACOL> ca;
    Copier<TN, NT, BCOL, GATE> cb;
    ca.init(t, m0, g.M, g.lda);
    cb.init(t, n0, g.N, g.ldb);
    const int64_t a0 = ACOL ? (int64_t)m0 * 2 : m0 * g.lda, b0 = BCOL ? (int64_t)n0 * 2 : n0 * g.ldb;

    const int total = g.ksteps * g.nseg;
    const int s_begin = (int)((int64_t)total * k_part / g.splits);
    const int s_end = (int)((int64_t)total * (k_part + 1) / g.splits);
    int seg = s_begin / g.ksteps, ks = s_begin % g.ksteps;
    const unsigned lds_at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    auto issue = [&](int stage) {
        const char* a = g.A + (g.pa >> (4 * seg) & 15) * g.apl + a0 + ks * ca.step;
        const char* b = g.B + (g.pb >> (4 * seg) & 15) * g.bpl + b0 + ks * cb.step;
        ca.issue(a, g.K - ks * BK, lds_at + stage * STAGE, wave);
        cb.issue(b, g.K - ks * BK, lds_at + stage * STAGE + TM * BK * 2, wave, g.up);
        if (++ks == g.ksteps) {
            ks = 0;
            ++seg;
        }
    };

    v4 acc[MT][NTL];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NTL; ++j) acc[i][j] = v4{0.f, 0.f, 0.f, 0.f};

    // Two halves of a step, 32 k each. While the matrix cores work on one half's fragments,
    // the other's are read from LDS. Between the halves, the next step's copies have
    // landed, and this step's buffer is free for those of STAGES steps on.
    typename Frag<T>::type fa[2][MT], fb[2][NTL];
    auto read = [&](int stage, int kk) {
        const char* la = lds + stage * STAGE;
        const char* lb = la + TM * BK * 2;
#pragma unroll
        for (int j = 0; j < NTL; ++j) fb[kk][j] = read_frag<T, TN, BCOL>(lb, wn * (TN / WN) + j * 16, kk, lane);
#pragma unroll
        for (int i = 0; i < MT; ++i) fa[kk][i] = read_frag<T, TM, ACOL>(la, wm * (TM / WM) + i * 16, kk, lane);
    };
    auto multiply = [&](int kk) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NTL; ++j) acc[i][j] = mma(fb[kk][j], fa[kk][i], acc[i][j]);
        // one LDS read, then two products, and so on
        constexpr int READS = MT * (ACOL ? 2 : 1) + NTL * (BCOL ? 2 : 1), PER = MT * NTL / READS;
        if constexpr (PER > 0) {
#pragma unroll
            for (int i = 0; i < READS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, MT * NTL - READS * PER, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // This wave's copies of the step that is read next have landed (they land in order, `behind`
    // of them may be on their way after it) and its LDS reads are in registers; then every
    // wave's. The builtin's wait, unlike one in assembly, is one that the compiler counts: it
    // puts none of its own before the products.
    constexpr int PER_STEP = Copier<TM, NT, ACOL>::NI + Copier<TN, NT, BCOL>::NI;
    auto wait_all = [&](auto behind) {
        constexpr int N = decltype(behind)::value;
        static_assert(N < 16, "the low four bits of the count");
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070 | N);   // vmcnt(N) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr std::integral_constant<int, (STAGES - 2) * PER_STEP> rest{};
    constexpr std::integral_constant<int, 0> none{};

    const int steps = s_end - s_begin;
    // The second parts of fp16 come first, as stored: after their last step the sums lose their factor.
    constexpr bool RESTS = KIND == WEIGHT_PARTS;
    const int rests = RESTS ? min(g.ksteps - s_begin, steps) : 0;
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (i < steps) issue(i);
    if (STAGES > 2 && steps >= STAGES - 1) wait_all(rest);
    else wait_all(none);
    if (STAGES - 1 < steps) issue(STAGES - 1);
    read(0, 0);
    int stage = 0;
    for (int s = 0; s < steps; ++s) {
        const int next = stage + 1 == STAGES ? 0 : stage + 1;
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): the fragments of the first half
        read(stage, 1);
        multiply(0);
        if (STAGES > 2 && s + STAGES <= steps) wait_all(rest);
        else wait_all(none);
        if (s + STAGES < steps) issue(stage);
        __builtin_amdgcn_sched_barrier(0);
        read(next, 0);   // after the last step, of what lies there: not used
        multiply(1);
        stage = next;
        if (RESTS && s + 1 == rests)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NTL; ++j) acc[i][j] *= 1.f / REST_SCALE<T>;
    }

    if constexpr (KIND == WEIGHT_PARTS || (KIND == INPUT && std::is_same_v<T, f16>))
        if (g.e.times) {   // dz or a was stored times a factor
            const float by = *g.e.times;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NTL; ++j) acc[i][j] *= by;
        }

    float* part = g.splits > 1 ? g.part + (int64_t)k_part * g.M * g.N * (KIND == GATED ? 2 : 1) : nullptr;
    const int m = m0 + wm * (TM / WM) + (lane & 15), n = n0 + wn * (COLS / WN) + 4 * (lane >> 4);
    if constexpr (KIND == HIDDEN) {
        if (n < g.N) epilogue_hidden<T>(g, lane, m, n, acc);
        return;
    }
    auto finish = [&](auto edge) {
        constexpr bool EDGE = decltype(edge)::value;
        if constexpr (KIND == GATED) epilogue_gated<T, EDGE, STREAM>(g, part, lane, m, n, acc);
        else if constexpr (KIND != HIDDEN) epilogue<T, KIND, EDGE, STREAM>(g, part, lane, m, n, acc);
    };
    if (n0 + COLS <= g.N) finish(std::false_type());
    else finish(std::true_type());
}

}  // namespace

template <typename T, int KIND>
hipError_t run_product(const Product& p, const Plan& q, const GemmArgs& g, hipStream_t st) {
    const unsigned grid = (unsigned)(q.tiles_m * q.tiles_n * q.splits);
    // 64 x 64 tiles stage three steps: 512 x 1024 over K = 4096, 128 work-groups, takes 22 us with
    // three or four and 35 with two; 128 x 128 with three leave a CU one work-group, 31 us for
    // 2048^3 against 27
    // (a gated layer's waves have 32 columns of the result, one group of an 8-bit copy: four waves of 16 rows then)
    constexpr int WM = KIND == GATED ? 4 : 2;
    const int64_t kept = KIND == GATED ? kept_bytes(p, g.e.z, g.e.p.q, g.e.io_dt) : 0;
    // HIDDEN writes three to six times what it reads, past what the caches hold in any case: bf16 8192 rows, 2048 to 8192, two
    // parts each, take 527 us with plain stores, 548 with nontemporal ones
    if (q.tile == 64) k_product<T, KIND, 64, 64, WM, 4 / WM, 3, false><<<grid, 256, 0, st>>>(g);
    else if (q.tile == 128) k_product<T, KIND, 128, 128, 2, 2, 2, false><<<grid, 256, 0, st>>>(g);
    else if (KIND == HIDDEN || !streams(p, q, g.e.out_dt, kept))
        k_product<T, KIND, 256, 256, 2, 4, 2, false><<<grid, 512, 0, st>>>(g);
    else if constexpr (KIND != HIDDEN) k_product<T, KIND, 256, 256, 2, 4, 2, true><<<grid, 512, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace mfac
