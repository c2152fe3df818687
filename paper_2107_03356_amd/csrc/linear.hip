// Matrix products of a linear layer and its gradients, C (M x N) = A B^T over K:
//
//   forward   y = act(x W^T + b) + res     A = x [m][k],   B = W [n][k]
//   input     dx = dz W + add              A = dz [m][k],  B = W [k][n]
//   weight    dW = dz^T x                  A = dz [k][m],  B = x [k][n]
//
// and of a gated layer, whose W has the gate's rows and then the other projection's:
//
//   gated     y = act(x Wg^T + bg) (x Wu^T + bu)     a tile of C has half its columns from each
//   hidden    da = dy W2, of which the epilogue forms dz = [da zu act'(zg), da act(zg)] and a = act(zg) zu
//
// The kernels finish their sums alike (finish8 and the epilogues of product.h):
//   k_product  16-bit operands on v_mfma_f32_16x16x32, tiles of C in registers,
//              operand tiles copied from memory straight into LDS (product.h);
//   k_skinny   few rows of C: W streams through registers once, no LDS;
//   k_finish   joins the K parts of a product that was split over work-groups
//              (k_finish_gated those of a gated layer).
// Operands that the copies into LDS cannot take as they are (rows that do not start
// 16-byte aligned, 8-bit copies, fp32) are laid out first in the workspace: fp32 as
// three bf16 planes, hi + mid + lo, of whose nine products six are summed (|mid| is at most
// 2^-8 and |lo| 2^-17 of the value's power of two, so the others are at most
// 2^-24 (1 + 2^-10) of |a b| together: one fp32 rounding).
#include <algorithm>
#include <utility>

#include "../../include/mfac.h"
#include "internal.h"
#include "product.h"
#include "train.h"

namespace mfac {

// compiled in product_layer.hip, product_gated.hip, product_hidden.hip
extern template hipError_t run_product<bf16, FORWARD>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
extern template hipError_t run_product<f16, FORWARD>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
extern template hipError_t run_product<bf16, INPUT>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
extern template hipError_t run_product<f16, INPUT>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
extern template hipError_t run_product<bf16, WEIGHT>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
extern template hipError_t run_product<f16, WEIGHT>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
extern template hipError_t run_product<f16, WEIGHT_PARTS>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
extern template hipError_t run_product<bf16, GATED>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
extern template hipError_t run_product<f16, GATED>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
extern template hipError_t run_product<bf16, HIDDEN>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
extern template hipError_t run_product<f16, HIDDEN>(const Product&, const Plan&, const GemmArgs&, hipStream_t);

namespace {

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
// The same of a gated layer (KIND GATED or HIDDEN): a work-group has 256 / GROUPS pieces of eight columns, of which its GROUPS
// groups of threads sum every GROUPS-th part, joined in order. Where there are many parts there are few sums, and a CU takes
// in about 20 bytes a ns: 64 parts of 181 x 276 sums took 46 us in 15 work-groups.
template <int KIND, int GROUPS>
__global__ __launch_bounds__(256) void k_finish_gated(const float* __restrict__ part, int splits, int64_t M, int64_t N,
                                                      Epilogue e) {
    constexpr int EACH = 256 / GROUPS, SIDES = KIND == GATED ? 2 : 1;   // sides: N sums each for N of the result
    __shared__ __attribute__((aligned(32))) float of[GROUPS > 1 ? SIDES : 1][GROUPS > 1 ? 256 * 8 : 1];
    const int64_t pieces = (N + 31) / 32 * 4, total = M * pieces;
    const int group = threadIdx.x / EACH;
    for (int64_t u0 = (int64_t)blockIdx.x * EACH; u0 < total; u0 += (int64_t)gridDim.x * EACH) {
        const int64_t u = u0 + threadIdx.x % EACH, m = u / pieces, n = (u - m * pieces) * 8;
        const bool in = m < M;
        f8 v[SIDES];
#pragma unroll
        for (int k = 0; k < SIDES; ++k) v[k] = f8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int z = group; in && z < splits; z += GROUPS * 4) {
            f8 a[4][SIDES];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (z + i * GROUPS < splits)
#pragma unroll
                    for (int k = 0; k < SIDES; ++k) a[i][k] = load8(part + (((z + i * GROUPS) * M + m) * SIDES + k) * N, n, N);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (z + i * GROUPS < splits)
#pragma unroll
                    for (int k = 0; k < SIDES; ++k) v[k] += a[i][k];
        }
        if constexpr (GROUPS > 1) {
            __syncthreads();   // what the turn before this one left has been read
#pragma unroll
            for (int k = 0; k < SIDES; ++k) *reinterpret_cast<f8*>(&of[k][threadIdx.x * 8]) = v[k];
            __syncthreads();
            if (group == 0)
#pragma unroll
                for (int k = 0; k < SIDES; ++k)
                    for (int q = 1; q < GROUPS; ++q) v[k] += *reinterpret_cast<const f8*>(&of[k][(q * EACH + threadIdx.x) * 8]);
        }
        if (group == 0) {   // whole groups of four lanes (the exchanges of an 8-bit copy)
            if constexpr (KIND == GATED) finish_gated8(e, N, in, m, n, v[0], v[1]);
            else finish_hidden8(e, N, in, m, n, v[0]);
        }
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

// A gated layer: columns n0 .. of the result, half of the 16 NH rows the gate's and half the other projection's.
struct SkinnyArgs {
    const void *x, *w;
    int64_t ldx, ldw, M, N, K;
    int rows;   // columns of the result a work-group: 16 NH (a gated layer 8 NH), or 8
    Epilogue e;
};

constexpr int NW = 16;   // whatever NH, so that a sum's order does not depend on it
template <typename T, int NH, bool GATE>
__global__ __launch_bounds__(NW * 64) void k_skinny(SkinnyArgs g) {
    constexpr int H = GATE ? NH / 2 : NH;
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
        const int64_t n = min(n0 + min(16 * (h % H) + (lane & 15), g.rows - 1), g.N - 1);
        w[h] = (const T*)g.w + (n + h / H * g.N) * g.ldw;
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
    static_assert(256 * NH <= NW * 64, "");
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
    if constexpr (GATE) {
        f8 u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = red[0][16 * H + n + i][m];
        finish_gated8(g.e, g.N, m < g.M, m, n0 + n, v, u);
    } else {
        finish8<FORWARD>(g.e, g.N, m < g.M, m, n0 + n, v);
    }
}

// ---------------------------------------------------------------- operands into the workspace
// Up to four matrices in one launch (blockIdx.y), since a launch takes longer than a small matrix, or one:
// dst (rows of ld elements, ld a multiple of 8) <- src, zeros past cols.
struct LayOuts {
    LayOut of[4];
};
__device__ __forceinline__ const LayOut& this_one(const LayOut& j) { return j; }
__device__ __forceinline__ const LayOut& this_one(const LayOuts& j) { return j.of[blockIdx.y]; }
template <typename T, typename J>
__global__ __launch_bounds__(256) void k_lay_out(J jobs) {
    const LayOut& j = this_one(jobs);
    const T* __restrict__ src = (const T*)j.src;
    T* __restrict__ dst = (T*)j.dst;
    const int64_t pieces = j.ld / 8, total = j.rows * pieces;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        const int64_t r = u / pieces, c = (u - r * pieces) * 8;
        store8(dst + r * j.ld, c, j.ld, load8(src + r * j.lds, c, j.cols));
    }
}
// The same from fp32 into three bf16 planes, one after another.
template <typename J>
__global__ __launch_bounds__(256) void k_lay_out_split(J jobs) {
    typedef VecOf<bf16, 8>::plain b8;
    const LayOut& j = this_one(jobs);
    const float* __restrict__ src = (const float*)j.src;
    bf16* __restrict__ dst = (bf16*)j.dst;
    const int64_t pieces = j.ld / 8, total = j.rows * pieces, plane = j.rows * j.ld;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < total; u += (int64_t)gridDim.x * 256) {
        const int64_t r = u / pieces, c = (u - r * pieces) * 8;
        f8 x = load8(src + r * j.lds, c, j.cols);
        bf16* d = dst + r * j.ld + c;
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
// Rows of `cols` elements that the copies into LDS take as they are.
bool plain16(const void* p, int64_t ld, int64_t cols) {
    return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && cols % 8 == 0 && ld <= (int64_t(1) << 21);
}

Operand operand_of(int dt, const void* p, int laid_out, int64_t ld, bool packed, int64_t rows, int64_t cols) {
    Operand o{laid_out ? laid_out : dt == DT_F32 && !packed ? 3 : 1, true, rows, cols, round_up(cols, 8), 0};
    o.lay_out = !laid_out && (o.planes == 3 || packed || !plain16(p, ld, cols));
    if (!o.lay_out) o.ld = ld;
    else o.bytes = (size_t)round_up(rows * o.ld * 2 * o.planes, 256);
    return o;
}

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
    const int64_t ar = p.a_col ? p.K : p.M, ac = p.a_col ? p.M : p.K, br = p.b_col ? p.K : p.N, bc = p.b_col ? p.N : p.K;
    q.a = operand_of(dt, p.A, p.a_parts, p.lda, false, ar, ac);
    q.b = operand_of(dt, p.B, p.b_parts, p.ldb, p.bp.q != nullptr, br, bc);
    q.ksteps = (int)ceil_div(p.K, BK);
    q.nseg = q.a.planes * q.b.planes == 9 ? 6 : q.a.planes * q.b.planes;   // not both of two parts
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
    q.tiles_n = p.gate == GATE_FORWARD ? ceil_div(p.N / 2, q.tile / 2) : ceil_div(p.N, q.tile);
    if (q.splits > 1) q.part_bytes = (size_t)round_up(p.M * p.N * q.splits * 4, 256);
    return q;
}

template <typename T>
hipError_t run_product(const Product& p, const Plan& q, const GemmArgs& g, hipStream_t st) {
    if (p.gate == GATE_FORWARD) return run_product<T, GATED>(p, q, g, st);
    if (p.gate == GATE_HIDDEN && q.splits == 1) return run_product<T, HIDDEN>(p, q, g, st);   // else when its parts are joined
    if constexpr (std::is_same_v<T, f16>)
        if (p.a_col && q.nseg == 2) return run_product<T, WEIGHT_PARTS>(p, q, g, st);
    if (p.a_col) return run_product<T, WEIGHT>(p, q, g, st);
    return p.b_col ? run_product<T, INPUT>(p, q, g, st) : run_product<T, FORWARD>(p, q, g, st);
}

template <int KIND>
void run_finish_gated(const float* part, int splits, int64_t M, int64_t N, const Epilogue& e, hipStream_t st) {
    const int64_t total = M * (ceil_div(N, 32) * 4);
    if (splits < 8)
        k_finish_gated<KIND, 1><<<(unsigned)std::min<int64_t>(ceil_div(total, 256), 8192), 256, 0, st>>>(part, splits, M, N, e);
    else
        k_finish_gated<KIND, 16><<<(unsigned)std::min<int64_t>(ceil_div(total, 16), 8192), 256, 0, st>>>(part, splits, M, N, e);
}
hipError_t run_finish(const Product& p, const float* part, int splits, const Epilogue& e, hipStream_t st) {
    const int64_t pieces = ceil_div(p.N, 32) * 4;
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(p.M * pieces, 256), 8192);
    if (p.gate == GATE_FORWARD) run_finish_gated<GATED>(part, splits, p.M, p.N / 2, e, st);
    else if (p.gate == GATE_HIDDEN) run_finish_gated<HIDDEN>(part, splits, p.M, p.N, e, st);
    else if (p.a_col) k_finish<WEIGHT><<<grid, 256, 0, st>>>(part, splits, p.M, p.N, e);
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

hipError_t launch_lay_out(int dt, int n, const LayOut* jobs, hipStream_t st) {
    if (n == 0) return hipSuccess;
    LayOuts all{};
    int64_t most = 1;
    for (int i = 0; i < n; ++i) {
        all.of[i] = jobs[i];
        most = std::max(most, ceil_div(jobs[i].rows * (jobs[i].ld / 8), 256));
    }
    const dim3 grid((unsigned)std::min<int64_t>(most, 4096), (unsigned)n);
    auto run = [&](const auto& j) {
        using J = std::decay_t<decltype(j)>;
        if (dt == DT_F32) k_lay_out_split<J><<<grid, 256, 0, st>>>(j);
        else if (dt == DT_BF16) k_lay_out<bf16, J><<<grid, 256, 0, st>>>(j);
        else k_lay_out<f16, J><<<grid, 256, 0, st>>>(j);
    };
    if (n == 1) run(jobs[0]);
    else run(all);
    return hipGetLastError();
}

int product_splits(int dt, const Product& p) { return plan_of(dt, p).splits; }
size_t product_workspace_bytes(int dt, const Product& p) {
    const Plan q = plan_of(dt, p);
    return q.a.bytes + q.b.bytes + q.part_bytes;
}

hipError_t launch_product(int dt, const Product& p, const Epilogue& e, void* ws, hipStream_t st) {
    const Plan q = plan_of(dt, p);
    char* w = (char*)ws;
    hipError_t err = hipSuccess;
    if (q.skinny) {
        const bool gated = p.gate == GATE_FORWARD;
        SkinnyArgs g{p.A, p.B, p.lda, p.ldb, p.M, gated ? p.N / 2 : p.N, p.K, 16, e};
        // Rows of W a work-group: the 32 columns of a group in one for an 8-bit copy of z; else so
        // that the work-groups are about as many as CUs. 1024 x 4096, 12 rows: fp32 14.6 us with 16,
        // 13.4 with 8 (a quarter of it the fp32 MFMAs); bf16 9.4 and 8.2. A gated layer has twice the rows of W to
        // one: 8192 columns, bf16 over 2048, 13.5 us with 16, 14.7 with 32, 17.2 with 8. More work-groups than CUs are a second
        // turn, so 8 end at 2048 columns: bf16 over 2048, one row, 2048 columns 5.6 with 8 and 6.8 with 16, 2304 8.8 and 6.9,
        // 2816 8.9 and 7.0, 4096 9.3 and 7.0; fp32, 12 rows, 2048 10.6 and 13.0, 2816 17.9 and 13.1.
        if (e.p.q || (!gated && g.N > 16 * CUS)) g.rows = 32;
        else if (g.N <= 8 * CUS) g.rows = 8;
        const unsigned grid = (unsigned)ceil_div(g.N, g.rows);
        by_operand(dt, [&](auto* t) {
            using T = std::remove_reference_t<decltype(*t)>;
            if (gated && g.rows == 32) k_skinny<T, 4, true><<<grid, NW * 64, 0, st>>>(g);
            else if (gated) k_skinny<T, 2, true><<<grid, NW * 64, 0, st>>>(g);
            else if (g.rows == 32) k_skinny<T, 2, false><<<grid, NW * 64, 0, st>>>(g);
            else k_skinny<T, 1, false><<<grid, NW * 64, 0, st>>>(g);
        });
        err = hipGetLastError();
    } else {
        GemmArgs g{};
        g.A = (const char*)p.A;
        g.B = (const char*)p.B;
        LayOut jobs[2];
        int njobs = 0;
        if (q.a.lay_out) {
            jobs[njobs++] = LayOut{p.A, p.lda, q.a.rows, q.a.cols, w, q.a.ld};
            g.A = w;
            w += q.a.bytes;
        }
        if (q.b.lay_out) {
            if (!p.bp.q) jobs[njobs++] = LayOut{p.B, p.ldb, q.b.rows, q.b.cols, w, q.b.ld};
            else err = launch_unpack8(dt == DT_F16 ? DT_F16 : DT_BF16, q.b.rows, q.b.cols, p.bp, w, q.b.ld, st);
            if (err != hipSuccess) return err;
            g.B = w;
            w += q.b.bytes;
        }
        if ((err = launch_lay_out(dt, njobs, jobs, st)) != hipSuccess) return err;
        g.lda = q.a.ld * 2;
        g.ldb = q.b.ld * 2;
        g.apl = p.a_parts ? p.a_part : q.a.rows * q.a.ld * 2;
        g.bpl = p.b_parts ? p.b_part : q.b.rows * q.b.ld * 2;
        g.M = (int)p.M;
        g.N = (int)(p.gate == GATE_FORWARD ? p.N / 2 : p.N);
        g.up = g.N * g.ldb;
        g.K = (int)p.K;
        g.ksteps = q.ksteps;
        g.nseg = q.nseg;
        // pairs of planes, the small products first
        if (q.nseg == 6) {   // hi mid lo = 0 1 2; (2,0) (0,2) (1,1) (1,0) (0,1) (0,0)
            g.pa = 2u | 0u << 4 | 1u << 8 | 1u << 12 | 0u << 16 | 0u << 20;
            g.pb = 0u | 2u << 4 | 1u << 8 | 0u << 12 | 1u << 16 | 0u << 20;
        } else if (q.nseg == 3) {
            (q.a.planes == 3 ? g.pa : g.pb) = 2u | 1u << 4 | 0u << 8;
        } else if (q.nseg == 2) {
            (q.a.planes == 2 ? g.pa : g.pb) = 1u | 0u << 4;
        }
        g.tiles_m = (int)q.tiles_m;
        g.tiles_n = (int)q.tiles_n;
        g.splits = q.splits;
        g.part = (float*)w;
        g.e = e;
        if (p.gate == GATE_HIDDEN && e.range) {
            const int64_t sums = p.K;
            err = launch_gate_range({p.A, p.lda, p.M, p.K, DT_F16}, {p.B, p.ldb, sums, p.N, DT_F16}, sums, p.M, p.N, e, st);
            if (err != hipSuccess) return err;
        }
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

extern "C" __attribute__((visibility("default"))) mfac_status mfac_gated_plan(mfac_dtype type, int32_t product, int64_t rows,
                                                                              int64_t cin, int64_t hidden, int32_t plan[3]) {
    using namespace mfac;
    constexpr int64_t most = int64_t(1) << 21;
    if (type < MFAC_F32 || type > MFAC_F16 || product < MFAC_GATED_FORWARD || product > MFAC_GATED_HIDDEN_SUMS || rows < 1 ||
        rows > (int64_t(1) << 30) || cin < 1 || cin > most || hidden < 1 || hidden > most / 2 || !plan)
        return MFAC_EINVAL;
    const bool backward = product == MFAC_GATED_HIDDEN || product == MFAC_GATED_HIDDEN_SUMS;
    Product p{};
    p.M = rows;
    p.N = backward ? hidden : 2 * hidden;
    p.K = cin;
    p.b_col = backward;
    p.gate = backward ? GATE_HIDDEN : GATE_FORWARD;
    const Plan q = plan_of(type, p);
    plan[0] = q.tile;
    plan[1] = q.splits;
    if (backward)   // where dz is not formed in it, the product stores da in fp32
        plan[2] = q.splits == 1 && !(product == MFAC_GATED_HIDDEN && hidden_fused(type, q.splits, hidden)) && streams(p, q, DT_F32);
    else
        plan[2] = q.splits == 1 &&
                  streams(p, q, type, kept_bytes(p, product == MFAC_GATED_FORWARD_Z, product == MFAC_GATED_FORWARD_COPIES, type));
    return MFAC_OK;
}
