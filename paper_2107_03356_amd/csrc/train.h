// Launchers of the training operators (norm.hip, pack8.hip, linear.hip; gated.hip, residual.hip, dropout.hip), called by
// train_capi.hip and gated_capi.hip once the arguments have been checked.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mfac {

enum : int { DT_F32 = 0, DT_BF16 = 1, DT_F16 = 2 };
inline int64_t dtype_bytes(int t) { return t == DT_F32 ? 4 : 2; }

// An 8-bit copy of a matrix; q == nullptr: none.
struct Packed {
    int8_t* q;
    int64_t ldq;
    uint8_t* s;
};

hipError_t launch_pack8(int dt, int64_t rows, int64_t cols, const void* x, int64_t ldx, Packed p, hipStream_t st);
hipError_t launch_unpack8(int dt, int64_t rows, int64_t cols, Packed p, void* y, int64_t ldy, hipStream_t st);

hipError_t launch_layer_norm(int dt, int wt, int64_t rows, int64_t cols, const void* x, int64_t ldx, const void* w,
                             const void* b, float eps, void* y, int64_t ldy, float* mean, float* rstd, Packed p,
                             hipStream_t st);
// part: norm_bwd_parts(rows, cols) * 2 * cols floats (unused if dw and db are null)
int64_t norm_bwd_parts(int64_t rows, int64_t cols);
hipError_t launch_layer_norm_bwd(int dt, int wt, int64_t rows, int64_t cols, const void* dy, int64_t lddy,
                                 const void* x, int64_t ldx, const float* mean, const float* rstd, Packed p,
                                 const void* w, const void* add, int64_t ldadd, void* dx, int64_t lddx, void* dw,
                                 void* db, float* part, hipStream_t st);

// part: act_bwd_parts(rows, cols) * cols floats (unused if db is null)
int64_t act_bwd_parts(int64_t rows, int64_t cols);
hipError_t launch_act_bwd(int dt, int act, int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* z,
                          int64_t ldz, Packed p, void* dz, int64_t lddz, void* a, int64_t lda, float* db, float* part,
                          hipStream_t st);
// out_a[c] = sum over p < nparts of part[p * stride + c], out_b likewise from part + cols (either may be null)
hipError_t launch_column_sums(const float* part, int64_t nparts, int64_t stride, int64_t cols, int out_dt, void* out_a,
                              void* out_b, hipStream_t st);

hipError_t launch_zero_matrix(int dt, int64_t rows, int64_t cols, void* y, int64_t ldy, hipStream_t st);

// What a product's epilogue does with an fp32 sum c at (m, n); see linear.hip.
struct Epilogue {
    int out_dt;          // type of out
    int io_dt;           // type of add and z
    int act;
    int bias_dt;
    void* out;
    int64_t ldo;
    const void* bias;    // over n
    const void* add;     // added after the activation
    int64_t ldadd;
    void* z;             // c + bias, before the activation
    int64_t ldz;
    Packed p;            // the same as an 8-bit copy
    const float *gamma, *beta;  // over n: c gamma + db[m] beta
    const float* db;
    // a gated layer (Product::gate): z and p are the gate's pre-activation, these the other one's, of the same strides
    void* z2;
    Packed p2;
    void* a;             // act(z) z2, where HIDDEN forms it (null: not wanted)
    int64_t lda;
    // out and a in this many 16-bit parts (1, 2; of fp32 3), each what the rounding of those before it leaves, bytes apart
    int parts;
    int64_t out_part, a_part;
    // of fp16 data in two parts: GATE_RANGE floats for the factors that keep dz and a within fp16's range, formed before the
    // pass (gated.hip); null: 1
    float* range;
    const float* times;  // an fp16 product's sums are multiplied by this one (null: 1)
};

// Of Epilogue::range: dz and a are stored times [0] and [1], and [2] and [3] take these out again (powers of two, at most
// and at least 1); behind them the maxima they are formed from.
constexpr int RANGE_WGS = 1024, GATE_RANGE = 4 + 4 * RANGE_WGS;
struct Magnitudes {
    const void* p;       // rows x cols, of type dt, or an 8-bit copy's bytes s (dt < 0)
    int64_t ld, rows, cols;
    int dt;
};
// d: dy, with w of `sums` rows (the next layer's weight), or da itself (w.p null)
hipError_t launch_gate_range(const Magnitudes& d, const Magnitudes& w, int64_t sums, int64_t rows, int64_t hidden, const Epilogue& e,
                             hipStream_t st);

// What a product's N columns are.
enum : int {
    GATE_NONE = 0,
    GATE_FORWARD = 1,  // of a forward product: 2 hidden rows of W, the gate's and the other projection's; out is rows x hidden
    GATE_HIDDEN = 2    // of an input product: hidden columns of da, whose epilogue writes dz (out, rows x 2 hidden)
};

// C (M x N) = A B^T summed over K; A is [m][k] (a_col false) or [k][m], B likewise over n.
struct Product {
    int64_t M, N, K;
    const void* A;
    int64_t lda;
    bool a_col;
    const void* B;
    int64_t ldb;
    bool b_col;
    Packed bp;  // B as an 8-bit copy (B null)
    int gate;   // GATE_*; N counts what the product has, 2 hidden or hidden
    // operands that are laid out already: in so many 16-bit parts (0: not), bytes apart, rows 16-byte aligned and zeros
    // up to the next multiple of 8 columns
    int a_parts;
    int64_t a_part;
    int b_parts;
    int64_t b_part;
};
size_t product_workspace_bytes(int dt, const Product& p);
// Whether dz and a come straight from the product that forms da, in so many parts of K (no column sums wanted): where its
// parts are joined, and in its epilogue of 16-bit data where a wave's columns are all there or none (fp32's epilogue would
// write 18 bytes a sum).
inline bool hidden_fused(int dt, int splits, int64_t hidden) { return splits > 1 || (dt != DT_F32 && hidden % 64 == 0); }
int product_splits(int dt, const Product& p);   // parts of K, of rows > 0
// A matrix as the products take it: ld elements a row, a multiple of 8; of fp32 three parts, one after another.
struct LayOut {
    const void* src;
    int64_t lds, rows, cols;
    void* dst;
    int64_t ld;
};
hipError_t launch_lay_out(int dt, int n, const LayOut* jobs, hipStream_t st);   // n <= 4
hipError_t launch_product(int dt, const Product& p, const Epilogue& e, void* ws, hipStream_t st);

// The gate's part of a backward pass; da is of type da_dt, dt or fp32, or null where out and db are (a alone is formed). Of the epilogue act, z, p, z2, p2, out (dz), a and
// their parts are used; out and a are 16-bit (bf16 for fp32 data), ldo and lda multiples of 8, zeros past their columns.
// part: gated_bwd_parts(rows, hidden) * 2 * hidden floats (unused if db is null)
int64_t gated_bwd_parts(int64_t rows, int64_t hidden);
hipError_t launch_gated_act_bwd(int dt, int da_dt, int64_t rows, int64_t hidden, const void* da, int64_t ldda,
                                const Epilogue& e, float* db, float* part, hipStream_t st);

// Dropout's mask; threshold 0: none.
struct Drop {
    unsigned threshold;
    float scale;
    const int64_t* at;   // seed, offset
};
hipError_t launch_dropout(int dt, int64_t rows, int64_t cols, const void* x, int64_t ldx, Drop d, void* y, int64_t ldy,
                          hipStream_t st);

// n = N_post(y), s = scale r + gate drop(n), h = N_pre(s); see residual_fwd.h. Pointers of what is absent or not
// wanted are null.
struct Residual {
    int norms;           // MFAC_NORM_*
    int64_t rows, cols;
    const void* y;
    int64_t ldy;
    const void *w1, *b1, *w2, *b2, *gate;   // of the post norm, the pre norm; cols values each, of type wt
    const void* gates;   // rows x cols, like y
    int64_t ldgates;
    const void* r;
    int64_t ldr;
    float scale, eps;
    Drop drop;
    void* s;
    int64_t lds;
    void* h;
    int64_t ldh;
    float *mean1, *rstd1, *mean2, *rstd2;
    Packed p;            // the 8-bit copy of the pre norm's xhat
};
hipError_t launch_residual(int dt, int wt, const Residual& g, hipStream_t st);

// Its gradients: of Residual the inputs (s an input too, or p), and
struct ResidualBwd {
    const void* ds;
    int64_t ldds;
    const void* dh;
    int64_t lddh;
    void* dy;
    int64_t lddy;
    void* dr;
    int64_t lddr;
    void* dgates;
    int64_t lddgates;
    void *dw1, *db1, *dw2, *db2, *dgate;   // of type wt
    float* part;         // residual_bwd_parts(dt, norms, rows, cols) * residual_sums(norms) * cols (unused if these are null)
};
int64_t residual_bwd_parts(int dt, int norms, int64_t rows, int64_t cols);
int residual_sums(int norms);
hipError_t launch_residual_bwd(int dt, int wt, const Residual& g, const ResidualBwd& b, hipStream_t st);

}  // namespace mfac
