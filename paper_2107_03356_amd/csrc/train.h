// Launchers of the training operators (norm.hip, pack8.hip, linear.hip), called
// by train_capi.hip once the arguments have been checked.
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
};
size_t product_workspace_bytes(int dt, const Product& p);
hipError_t launch_product(int dt, const Product& p, const Epilogue& e, void* ws, hipStream_t st);

}  // namespace mfac
