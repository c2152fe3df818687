// Matrix products of a linear layer and its gradients, C (M x N) = A B^T over K:
//
//   forward   y = act(x W^T + b) + res     A = x [m][k],   B = W [n][k]
//   input     dx = dz W + add              A = dz [m][k],  B = W [k][n]
//   weight    dW = dz^T x                  A = dz [k][m],  B = x [k][n]
//
// Three kernels share one epilogue:
//   k_product  16-bit operands on v_mfma_f32_16x16x32, tiles of C in registers,
//              operand tiles copied from memory straight into LDS;
//   k_skinny   few rows of C: W streams through registers once, no LDS;
//   k_finish   joins the K parts of a product that was split over work-groups.
// Operands that the copies into LDS cannot take as they are (rows that do not start
// 16-byte aligned, 8-bit copies, fp32) are laid out first in the workspace: fp32 as
// three bf16 planes, hi + mid + lo, of whose nine products six are summed (|mid| is at most
// 2^-8 and |lo| 2^-17 of the value's power of two, so the others are at most
// 2^-24 (1 + 2^-10) of |a b| together: one fp32 rounding).
#include <algorithm>
#include <utility>

#include "../../include/mfac.h"
#include "internal.h"
#include "train.h"
#include "train_util.h"

namespace mfac {
namespace {

typedef float v4 __attribute__((ext_vector_type(4)));

template <int... I, typename F>
__device__ __forceinline__ void for_each_index(std::integer_sequence<int, I...>, F f) {
    (f(std::integral_constant<int, I>()), ...);
}

// ---------------------------------------------------------------- epilogue
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

// The three products' epilogues; the fields of the others are unused.
enum : int { FORWARD = 0, INPUT = 1, WEIGHT = 2 };

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
        o.beta = load8(e.beta, n, N);
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
    if (KIND == WEIGHT && e.gamma && in) o.db = e.db[m];
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

struct GemmArgs {
    const char *A, *B;       // 16-bit elements
    int64_t lda, ldb;        // bytes
    int64_t apl, bpl;        // bytes between planes
    int M, N, K;
    int ksteps, nseg;        // BK-wide steps over K, and how often K is gone over (pairs of planes)
    unsigned pa, pb;         // planes of the pairs, 4 bits each
    int tiles_m, tiles_n, splits;
    float* part;             // [splits][M][N] sums, where splits > 1
    Epilogue e;
};

// What a thread copies of an operand tile: NI pieces, NT * 16 bytes apart in LDS.
template <int R, int NT, bool COL>
struct Copier {
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
                // a row past the end reads the last one: its sums are not stored
                off[i] = (unsigned)(min(r, rows - 1 - row0) * ld + kc * 2);
            }
        }
    }
    // base: the tile's first element at this step; left: K's elements from there on. In
    // assembly because the compiler waits for the builtin's copies before the next transposing
    // read of LDS, whichever buffer that reads (dx and dW of 8192^3: 899 and 921 us with it);
    // the kernel's own waits are all that is needed. Nothing is loaded into registers, and an
    // offset past the buffer's size writes zeros.
    __device__ __forceinline__ void issue(const char* base, int left, unsigned lds, int wave) const {
        typedef int i4 __attribute__((ext_vector_type(4)));
        const uint64_t b = (uint64_t)base;
        // base, stride 0, size OUT_OF_RANGE, raw 32-bit data
        const i4 r = {__builtin_amdgcn_readfirstlane((int)b), __builtin_amdgcn_readfirstlane((int)(b >> 32)),
                      (int)OUT_OF_RANGE, 0x00020000};
#pragma unroll
        for (int i = 0; i < NI; ++i) {
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
    constexpr bool FWD = KIND == FORWARD, WGT = KIND == WEIGHT;
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
                beta[j] = load4<EDGE>(e.beta, n + j * 16, N);
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
                const float db = e.db[m];
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
template <typename T, bool ACOL, bool BCOL, int TM, int TN, int WM, int WN, int STAGES, bool STREAM>
__global__ __launch_bounds__(WM* WN * 64, 2) void k_product(GemmArgs g) {
    constexpr int NT = WM * WN * 64, MT = TM / WM / 16, NTL = TN / WN / 16;
    constexpr int STAGE = (TM + TN) * BK * 2, KIND = ACOL ? WEIGHT : BCOL ? INPUT : FORWARD;
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
    const int m0 = (band * BAND + in_band % height) * TM, n0 = in_band / height * TN;

    Copier<TM, NT, ACOL> ca;
    Copier<TN, NT, BCOL> cb;
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
        cb.issue(b, g.K - ks * BK, lds_at + stage * STAGE + TM * BK * 2, wave);
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
    }

    float* part = g.splits > 1 ? g.part + (int64_t)k_part * g.M * g.N : nullptr;
    const int m = m0 + wm * (TM / WM) + (lane & 15), n = n0 + wn * (TN / WN) + 4 * (lane >> 4);
    if (n0 + TN <= g.N) epilogue<T, KIND, false, STREAM>(g, part, lane, m, n, acc);
    else epilogue<T, KIND, true, STREAM>(g, part, lane, m, n, acc);
}

// Joins the K parts in order and finishes.
template <int KIND>
__global__ __launch_bounds__(256) void k_finish(const float* __restrict__ part, int splits, int64_t M, int64_t N,
                                                Epilogue e) {
    const int64_t pieces = (N + 31) / 32 * 4, total = M * pieces;
    // whole waves go around together (the exchanges of an 8-bit copy)
    for (int64_t u0 = (int64_t)blockIdx.x * 256; u0 < total; u0 += (int64_t)gridDim.x * 256) {
        const int64_t u = u0 + threadIdx.x, m = u / pieces, n = (u - m * pieces) * 8;
        const bool in = m < M;
        f8 v = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (in)
            for (int z = 0; z < splits; ++z) v += load8(part + (z * M + m) * N, n, N);
        finish8<KIND>(e, N, in, m, n, v);
    }
}

// ---------------------------------------------------------------- few rows
// C (M <= 16 rows) = x W^T. A work-group takes 16 NH rows of W (or 8) and all of K, which its NW
// waves share out in pieces of 16 bytes a row; lane l holds row l % 16 of x and of W, and
// the k of piece l / 16. The waves' sums are joined through LDS. 16-bit types on
// v_mfma_f32_16x16x32, fp32 on v_mfma_f32_16x16x4. Bound by reading W, 33.5 MB in 9.4 us. A CU
// takes in about 20 bytes a ns from beyond its L2, so all of them are wanted: narrow
// layers take 8 rows a work-group, the other half of the lanes reading the eighth again.
// Sharing K out over work-groups would be a launch more, which costs the host 3 us and the
// device 4.
template <typename T>
struct Piece {
    static constexpr int K = 16 / sizeof(T);   // values in 16 bytes
    typedef typename VecOf<T, K>::plain type;
};
__device__ __forceinline__ v4 mma_piece(VecOf<bf16, 8>::plain a, VecOf<bf16, 8>::plain b, v4 c) { return mma(a, b, c); }
__device__ __forceinline__ v4 mma_piece(VecOf<f16, 8>::plain a, VecOf<f16, 8>::plain b, v4 c) { return mma(a, b, c); }
__device__ __forceinline__ v4 mma_piece(VecOf<float, 4>::plain a, VecOf<float, 4>::plain b, v4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

template <typename T>
__device__ __forceinline__ typename Piece<T>::type load_piece(const T* __restrict__ row, int64_t k, int64_t K) {
    constexpr int N = Piece<T>::K;
    if (k + N <= K) return *reinterpret_cast<const typename VecOf<T, N>::type*>(row + k);
    typename Piece<T>::type r;
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = k + i < K ? row[k + i] : (T)0.f;
    return r;
}

struct SkinnyArgs {
    const void *x, *w;
    int64_t ldx, ldw, M, N, K;
    int rows;   // of W a work-group: 16 NH, or 8
    Epilogue e;
};

constexpr int NW = 16;   // whatever NH, so that a sum's order does not depend on it
template <typename T, int NH>
__global__ __launch_bounds__(NW * 64) void k_skinny(SkinnyArgs g) {
    constexpr int KP = 4 * Piece<T>::K;   // k of one MFMA step
    constexpr int U = 8 / NH;             // steps in flight
    __shared__ float red[NW][16 * NH][17];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * g.rows;
    const int64_t nsteps = (g.K + KP - 1) / KP;
    const int64_t s0 = nsteps * wave / NW, s1 = nsteps * (wave + 1) / NW;
    const T* x = (const T*)g.x + min((int64_t)(lane & 15), g.M - 1) * g.ldx;
    const T* w[NH];
    v4 c[NH];
#pragma unroll
    for (int h = 0; h < NH; ++h) {
        w[h] = (const T*)g.w + min(n0 + min(16 * h + (lane & 15), g.rows - 1), g.N - 1) * g.ldw;
        c[h] = v4{0.f, 0.f, 0.f, 0.f};
    }
    const int64_t kl = (lane >> 4) * Piece<T>::K;
    typedef typename Piece<T>::type V;
    typedef typename VecOf<T, Piece<T>::K>::type Unaligned;
    // U steps at a time while they lie within K, then one by one with a check (code that is
    // not run still has to be fetched past: checks on every load cost 2 us a launch)
    int64_t s = s0;
    for (const int64_t whole = min(s1, g.K / KP); s + U <= whole; s += U) {
        V xv[U], a[U][NH];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t k = (s + u) * KP + kl;
#pragma unroll
            for (int h = 0; h < NH; ++h) a[u][h] = *reinterpret_cast<const Unaligned*>(w[h] + k);
            xv[u] = *reinterpret_cast<const Unaligned*>(x + k);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < NH; ++h) c[h] = mma_piece(a[u][h], xv[u], c[h]);
    }
#pragma unroll 1
    for (; s < s1; ++s) {
        V a[NH];
#pragma unroll
        for (int h = 0; h < NH; ++h) a[h] = load_piece(w[h], s * KP + kl, g.K);
        const V xv = load_piece(x, s * KP + kl, g.K);
#pragma unroll
        for (int h = 0; h < NH; ++h) c[h] = mma_piece(a[h], xv, c[h]);
    }
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) red[wave][16 * h + 4 * (lane >> 4) + i][lane & 15] = c[h][i];
    __syncthreads();
    if (threadIdx.x < 256 * NH) {   // a thread to a sum
        const int n = threadIdx.x >> 4, m = threadIdx.x & 15;
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < NW; ++q) s += red[q][n][m];
        red[0][n][m] = s;
    }
    __syncthreads();
    const int across = g.rows / 8;   // lanes to a row of C, eight columns each
    if ((int)threadIdx.x >= 16 * across) return;
    const int m = lane / across, n = lane % across * 8;
    f8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = red[0][n + i][m];
    finish8<FORWARD>(g.e, g.N, m < g.M, m, n0 + n, v);
}

// ---------------------------------------------------------------- operands into the workspace
// dst (rows of ld elements, ld a multiple of 8) <- src, zeros past cols.
template <typename T>
__global__ __launch_bounds__(256) void k_lay_out(const T* __restrict__ src, int64_t lds, int64_t rows, int64_t cols,
                                                 T* __restrict__ dst, int64_t ld) {
    const int64_t pieces = ld / 8, total = rows * pieces;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        const int64_t r = u / pieces, c = (u - r * pieces) * 8;
        store8(dst + r * ld, c, ld, load8(src + r * lds, c, cols));
    }
}
// The same from fp32 into three bf16 planes, `plane` elements apart.
__global__ __launch_bounds__(256) void k_lay_out_split(const float* __restrict__ src, int64_t lds, int64_t rows,
                                                       int64_t cols, bf16* __restrict__ dst, int64_t ld, int64_t plane) {
    typedef VecOf<bf16, 8>::plain b8;
    const int64_t pieces = ld / 8, total = rows * pieces;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        const int64_t r = u / pieces, c = (u - r * pieces) * 8;
        f8 x = load8(src + r * lds, c, cols);
        bf16* d = dst + r * ld + c;
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            // the first part cut at bf16's largest value, to which the second adds the rest: rounded, a
            // value past it would be infinite (infinities and NaN come through in the second part)
            const f8 v = p ? x : __builtin_elementwise_min(__builtin_elementwise_max(x, f8(-0x1.fep127f)), f8(0x1.fep127f));
            const b8 h = __builtin_convertvector(v, b8);
            *reinterpret_cast<b8*>(d + p * plane) = h;
            x -= __builtin_convertvector(h, f8);
        }
    }
}

// ---------------------------------------------------------------- host
constexpr int64_t SKINNY_ROWS = 16;
constexpr int64_t CUS = 256;
// Past the 256 MB of the last-level cache, outputs written through the caches push the operands
// out: 8192^3, dx and dW took 1003 and 1030 us with plain stores, 915 and 943 with nontemporal
// ones (both are faster now). Below, those are slower: dx of 8192 x 8192 over K = 2048 took
// 248 us, with them 271.
constexpr int64_t LAST_LEVEL_CACHE = int64_t(256) << 20;

// Rows of `cols` elements that the copies into LDS take as they are.
bool plain16(const void* p, int64_t ld, int64_t cols) {
    return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && cols % 8 == 0 && ld <= (int64_t(1) << 21);
}

struct Operand {
    bool planes, lay_out;
    int64_t rows, cols, ld;   // as laid out in memory
    size_t bytes;             // in the workspace
};
Operand operand_of(int dt, const void* p, int64_t ld, bool packed, int64_t rows, int64_t cols) {
    Operand o{dt == DT_F32 && !packed, true, rows, cols, round_up(cols, 8), 0};
    o.lay_out = o.planes || packed || !plain16(p, ld, cols);
    if (!o.lay_out) o.ld = ld;
    else o.bytes = (size_t)round_up(rows * o.ld * 2 * (o.planes ? 3 : 1), 256);
    return o;
}

struct Plan {
    bool skinny;
    Operand a, b;
    int tile, ksteps, nseg, splits;
    int64_t tiles_m, tiles_n;
    size_t part_bytes;
};

// What a product takes in tiles of `tile`, its `total` K steps in `splits` parts: us, fitted to
// launches of 64 to 16384 rows (within 15% of most). A K step of a CU's work-groups (one of
// 256 x 256, up to two of 128 x 128, up to four of 64 x 64) takes step[their number]; dW, with both
// operands read transposed, a little longer. Joining parts is a launch and their traffic.
float product_time(const Product& p, int tile, int64_t total, int splits) {
    struct Cost {
        int wgs;
        float step[4], start;
    };
    static constexpr Cost c256{1, {1.5f}, 8.f}, c128{2, {0.68f, 1.0f}, 5.f}, c64{4, {0.3f, 0.48f, 0.62f, 0.82f}, 3.f};
    const Cost& c = tile == 256 ? c256 : tile == 128 ? c128 : c64;
    const int64_t wgs = ceil_div(p.M, tile) * ceil_div(p.N, tile) * splits;
    const int64_t on_cu = std::min<int64_t>(c.wgs, ceil_div(wgs, CUS));
    const float side = p.a_col ? 1.05f : 1.f;
    const float main = (float)ceil_div(wgs, CUS * on_cu) * ((float)ceil_div(total, splits) * c.step[on_cu - 1] * side + c.start);
    return splits == 1 ? main : main + 5.f + (float)splits * (float)(p.M * p.N) * (8.f / 8e6f);
}

Plan plan_of(int dt, const Product& p) {
    Plan q{};
    q.skinny = p.M <= SKINNY_ROWS && !p.a_col && !p.b_col;
    q.splits = 1;
    if (q.skinny) return q;
    q.a = p.a_col ? operand_of(dt, p.A, p.lda, false, p.K, p.M) : operand_of(dt, p.A, p.lda, false, p.M, p.K);
    const bool packed = p.bp.q != nullptr;
    q.b = p.b_col ? operand_of(dt, p.B, p.ldb, packed, p.K, p.N) : operand_of(dt, p.B, p.ldb, packed, p.N, p.K);
    q.ksteps = (int)ceil_div(p.K, BK);
    q.nseg = q.a.planes ? (q.b.planes ? 6 : 3) : 1;
    const int64_t total = (int64_t)q.ksteps * q.nseg;
    float best = 0.f;
    for (int tile : {256, 128, 64})
        for (int splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if (splits > total || (splits > 1 && p.M * p.N * splits > (int64_t(1) << 26))) break;
            const float t = product_time(p, tile, total, splits);
            if (q.tile && t >= best) continue;
            best = t;
            q.tile = tile;
            q.splits = splits;
        }
    q.tiles_m = ceil_div(p.M, q.tile);
    q.tiles_n = ceil_div(p.N, q.tile);
    if (q.splits > 1) q.part_bytes = (size_t)round_up(p.M * p.N * q.splits * 4, 256);
    return q;
}

hipError_t lay_out(int dt, const Operand& o, const void* src, int64_t ld, Packed p, void* dst, hipStream_t st) {
    if (p.q) return launch_unpack8(dt == DT_F16 ? DT_F16 : DT_BF16, o.rows, o.cols, p, dst, o.ld, st);
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(o.rows * (o.ld / 8), 256), 4096);
    if (o.planes)
        k_lay_out_split<<<grid, 256, 0, st>>>((const float*)src, ld, o.rows, o.cols, (bf16*)dst, o.ld, o.rows * o.ld);
    else if (dt == DT_BF16)
        k_lay_out<bf16><<<grid, 256, 0, st>>>((const bf16*)src, ld, o.rows, o.cols, (bf16*)dst, o.ld);
    else
        k_lay_out<f16><<<grid, 256, 0, st>>>((const f16*)src, ld, o.rows, o.cols, (f16*)dst, o.ld);
    return hipGetLastError();
}

// Whether a product's results are stored past the caches: in tiles of 256, where they and the operands exceed them.
bool streams(const Product& p, const Plan& q, int out_dt) {
    const int64_t bytes = (p.M * p.K + p.N * p.K) * 2 * (q.nseg > 1 ? 3 : 1) + p.M * p.N * dtype_bytes(out_dt);
    return q.tile == 256 && bytes > LAST_LEVEL_CACHE;
}

template <typename T, bool ACOL, bool BCOL>
hipError_t run_product(const Product& p, const Plan& q, const GemmArgs& g, hipStream_t st) {
    const unsigned grid = (unsigned)(q.tiles_m * q.tiles_n * q.splits);
    // 64 x 64 tiles stage three steps: 512 x 1024 over K = 4096, 128 work-groups, takes 22 us with
    // three or four and 35 with two; 128 x 128 with three leave a CU one work-group, 31 us for
    // 2048^3 against 27
    if (q.tile == 64) k_product<T, ACOL, BCOL, 64, 64, 2, 2, 3, false><<<grid, 256, 0, st>>>(g);
    else if (q.tile == 128) k_product<T, ACOL, BCOL, 128, 128, 2, 2, 2, false><<<grid, 256, 0, st>>>(g);
    else if (!streams(p, q, g.e.out_dt)) k_product<T, ACOL, BCOL, 256, 256, 2, 4, 2, false><<<grid, 512, 0, st>>>(g);
    else k_product<T, ACOL, BCOL, 256, 256, 2, 4, 2, true><<<grid, 512, 0, st>>>(g);
    return hipGetLastError();
}
template <typename T>
hipError_t run_product(const Product& p, const Plan& q, const GemmArgs& g, hipStream_t st) {
    if (p.a_col) return run_product<T, true, true>(p, q, g, st);
    return p.b_col ? run_product<T, false, true>(p, q, g, st) : run_product<T, false, false>(p, q, g, st);
}

hipError_t run_finish(const Product& p, const float* part, int splits, const Epilogue& e, hipStream_t st) {
    const int64_t pieces = ceil_div(p.N, 32) * 4;
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(p.M * pieces, 256), 8192);
    if (p.a_col) k_finish<WEIGHT><<<grid, 256, 0, st>>>(part, splits, p.M, p.N, e);
    else if (p.b_col) k_finish<INPUT><<<grid, 256, 0, st>>>(part, splits, p.M, p.N, e);
    else k_finish<FORWARD><<<grid, 256, 0, st>>>(part, splits, p.M, p.N, e);
    return hipGetLastError();
}

template <typename F>
void by_operand(int dt, F f) {
    if (dt == DT_F32) f((float*)nullptr);
    else if (dt == DT_BF16) f((bf16*)nullptr);
    else f((f16*)nullptr);
}

}  // namespace

size_t product_workspace_bytes(int dt, const Product& p) {
    const Plan q = plan_of(dt, p);
    return q.a.bytes + q.b.bytes + q.part_bytes;
}

hipError_t launch_product(int dt, const Product& p, const Epilogue& e, void* ws, hipStream_t st) {
    const Plan q = plan_of(dt, p);
    char* w = (char*)ws;
    hipError_t err;
    if (q.skinny) {
        SkinnyArgs g{p.A, p.B, p.lda, p.ldb, p.M, p.N, p.K, 16, e};
        // Rows of W a work-group: the 32 columns of a group in one for an 8-bit copy of z; else so
        // that the work-groups are about as many as CUs. 1024 x 4096, 12 rows: fp32 14.6 us with 16,
        // 13.4 with 8 (a quarter of it the fp32 MFMAs); bf16 9.4 and 8.2.
        if (e.p.q || p.N > 16 * CUS) g.rows = 32;
        else if (p.N <= 8 * CUS) g.rows = 8;
        const unsigned grid = (unsigned)ceil_div(p.N, g.rows);
        by_operand(dt, [&](auto* t) {
            using T = std::remove_reference_t<decltype(*t)>;
            if (g.rows == 32) k_skinny<T, 2><<<grid, NW * 64, 0, st>>>(g);
            else k_skinny<T, 1><<<grid, NW * 64, 0, st>>>(g);
        });
        err = hipGetLastError();
    } else {
        GemmArgs g{};
        g.A = (const char*)p.A;
        g.B = (const char*)p.B;
        if (q.a.lay_out) {
            if ((err = lay_out(dt, q.a, p.A, p.lda, Packed{}, w, st)) != hipSuccess) return err;
            g.A = w;
            w += q.a.bytes;
        }
        if (q.b.lay_out) {
            if ((err = lay_out(dt, q.b, p.B, p.ldb, p.bp, w, st)) != hipSuccess) return err;
            g.B = w;
            w += q.b.bytes;
        }
        g.lda = q.a.ld * 2;
        g.ldb = q.b.ld * 2;
        g.apl = q.a.rows * q.a.ld * 2;
        g.bpl = q.b.rows * q.b.ld * 2;
        g.M = (int)p.M;
        g.N = (int)p.N;
        g.K = (int)p.K;
        g.ksteps = q.ksteps;
        g.nseg = q.nseg;
        // pairs of planes, the small products first
        if (q.nseg == 6) {   // hi mid lo = 0 1 2; (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
            g.pa = 2u | 0u << 4 | 1u << 8 | 1u << 12 | 0u << 16 | 0u << 20;
            g.pb = 0u | 2u << 4 | 1u << 8 | 0u << 12 | 1u << 16 | 0u << 20;
        } else if (q.nseg == 3) {
            g.pa = 2u | 1u << 4 | 0u << 8;
        }
        g.tiles_m = (int)q.tiles_m;
        g.tiles_n = (int)q.tiles_n;
        g.splits = q.splits;
        g.part = (float*)w;
        g.e = e;
        err = dt == DT_F16 ? run_product<f16>(p, q, g, st) : run_product<bf16>(p, q, g, st);
    }
    if (err != hipSuccess || q.splits == 1) return err;
    return run_finish(p, (const float*)w, q.splits, e, st);
}

}  // namespace mfac

extern "C" __attribute__((visibility("default"))) mfac_status mfac_linear_plan(mfac_dtype type, mfac_dtype otype,
                                                                               mfac_product product, int64_t rows,
                                                                               int64_t cin, int64_t cout,
                                                                               int32_t packed, int32_t plan[3]) {
    using namespace mfac;
    constexpr int64_t most = int64_t(1) << 21;
    if (type < MFAC_F32 || type > MFAC_F16 || (otype != MFAC_F32 && otype != type) || product < MFAC_PRODUCT_FORWARD ||
        product > MFAC_PRODUCT_WEIGHT || rows < 1 || rows > (int64_t(1) << 30) || cin < 1 || cin > most || cout < 1 ||
        cout > most || (packed && product != MFAC_PRODUCT_WEIGHT) || !plan)
        return MFAC_EINVAL;
    Product p{};   // the plan is one of sizes and types; addresses only decide what is laid out first
    p.M = product == MFAC_PRODUCT_WEIGHT ? cout : rows;
    p.N = product == MFAC_PRODUCT_FORWARD ? cout : cin;
    p.K = product == MFAC_PRODUCT_FORWARD ? cin : product == MFAC_PRODUCT_INPUT ? cout : rows;
    p.a_col = product == MFAC_PRODUCT_WEIGHT;
    p.b_col = product != MFAC_PRODUCT_FORWARD;
    int8_t some;
    if (packed) p.bp.q = &some;
    const Plan q = plan_of(type, p);
    plan[0] = q.tile;
    plan[1] = q.splits;
    plan[2] = q.splits == 1 && streams(p, q, otype);   // parts are joined by plain stores
    return MFAC_OK;
}
