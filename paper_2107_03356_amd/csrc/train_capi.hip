// C ABI of the training operators (include/mfac.h): argument checks and the
// launches of norm.hip, pack8.hip and linear.hip.
#include <math.h>

#include <algorithm>

#include "../../include/mfac.h"
#include "checks.h"
#include "internal.h"
#include "train.h"

using namespace mfac;

namespace {

bool layer_ok(int64_t rows, int64_t cin, int64_t cout) {
    return size_ok(rows, cin) && size_ok(rows, cout) && cin <= MOST_WIDTH && cout <= MOST_WIDTH;
}

Product forward_product(int64_t rows, int64_t cin, int64_t cout, const void* x, int64_t ldx, const void* w,
                        int64_t ldw) {
    return Product{rows, cout, cin, x, ldx, false, w, ldw, false, Packed{}};
}
Product input_product(int64_t rows, int64_t cin, int64_t cout, const void* dz, int64_t lddz, const void* w,
                      int64_t ldw) {
    return Product{rows, cin, cout, dz, lddz, false, w, ldw, true, Packed{}};
}
Product weight_product(int64_t rows, int64_t cin, int64_t cout, const void* dz, int64_t lddz, const void* x,
                       int64_t ldx, Packed p) {
    return Product{cout, cin, rows, dz, lddz, true, x, ldx, true, p};
}

}  // namespace

MFAC_API mfac_status mfac_pack8(mfac_dtype type, int64_t rows, int64_t cols, const void* x, int64_t ldx, int8_t* q,
                                int64_t ldq, uint8_t* s, hipStream_t stream) {
    if (!type_ok(type) || !size_ok(rows, cols)) return MFAC_EINVAL;
    if (rows == 0) return MFAC_OK;
    if (!matrix_ok(x, type, ldx, cols) || !packed_ok(q, ldq, s, cols, false)) return MFAC_EINVAL;
    return done(launch_pack8(type, rows, cols, x, ldx, Packed{q, ldq, s}, stream));
}

MFAC_API mfac_status mfac_unpack8(mfac_dtype type, int64_t rows, int64_t cols, const int8_t* q, int64_t ldq,
                                  const uint8_t* s, void* y, int64_t ldy, hipStream_t stream) {
    if (!type_ok(type) || !size_ok(rows, cols)) return MFAC_EINVAL;
    if (rows == 0) return MFAC_OK;
    if (!matrix_ok(y, type, ldy, cols) || !packed_ok(q, ldq, s, cols, false)) return MFAC_EINVAL;
    return done(launch_unpack8(type, rows, cols, Packed{const_cast<int8_t*>(q), ldq, const_cast<uint8_t*>(s)}, y, ldy,
                               stream));
}

MFAC_API mfac_status mfac_layer_norm(mfac_dtype type, mfac_dtype wtype, int64_t rows, int64_t cols, const void* x,
                                     int64_t ldx, const void* w, const void* b, double eps, void* y, int64_t ldy,
                                     float* mean_out, float* rstd_out, int8_t* q, int64_t ldq, uint8_t* s,
                                     hipStream_t stream) {
    if (!type_ok(type) || !param_type_ok(wtype, type) || !size_ok(rows, cols) || !(eps >= 0) || !isfinite(eps))
        return MFAC_EINVAL;
    if (rows == 0) return MFAC_OK;
    if (!matrix_ok(x, type, ldx, cols) || !matrix_ok(y, type, ldy, cols) || !vector_ok(w, wtype) ||
        !vector_ok(b, wtype) || !packed_ok(q, ldq, s, cols, true) || !vector_ok(mean_out, MFAC_F32) ||
        !vector_ok(rstd_out, MFAC_F32))
        return MFAC_EINVAL;
    return done(launch_layer_norm(type, wtype, rows, cols, x, ldx, w, b, (float)eps, y, ldy, mean_out, rstd_out,
                                  Packed{q, ldq, s}, stream));
}

MFAC_API size_t mfac_layer_norm_bwd_workspace_bytes(int64_t rows, int64_t cols) {
    if (!size_ok(rows, cols)) return 0;
    return (size_t)round_up(norm_bwd_parts(std::max<int64_t>(rows, 1), cols) * 2 * cols * 4, 256);
}

MFAC_API mfac_status mfac_layer_norm_bwd(mfac_dtype type, mfac_dtype wtype, int64_t rows, int64_t cols, const void* dy,
                                         int64_t lddy, const void* x, int64_t ldx, const float* mean,
                                         const float* rstd, const int8_t* q, int64_t ldq, const uint8_t* s,
                                         const void* w, const void* add, int64_t ldadd, void* dx, int64_t lddx,
                                         void* dw, void* db, void* workspace, size_t workspace_bytes,
                                         hipStream_t stream) {
    if (!type_ok(type) || !param_type_ok(wtype, type) || !size_ok(rows, cols)) return MFAC_EINVAL;
    if (!vector_ok(w, wtype) || !vector_ok(dw, wtype) || !vector_ok(db, wtype)) return MFAC_EINVAL;
    if (rows > 0) {
        if (!matrix_ok(dy, type, lddy, cols) || !matrix_ok(dx, type, lddx, cols) || !rstd ||
            !vector_ok(rstd, MFAC_F32) || !packed_ok(q, ldq, s, cols, true))
            return MFAC_EINVAL;
        if (q ? x || mean : !mean || !vector_ok(mean, MFAC_F32) || !matrix_ok(x, type, ldx, cols)) return MFAC_EINVAL;
        if (add && !matrix_ok(add, type, ldadd, cols)) return MFAC_EINVAL;
    }
    if (dw || db) {
        const mfac_status e =
            check_workspace(mfac_layer_norm_bwd_workspace_bytes(rows, cols), workspace, workspace_bytes);
        if (e != MFAC_OK) return e;
    }
    return done(launch_layer_norm_bwd(type, wtype, rows, cols, dy, lddy, x, ldx, mean, rstd,
                                      Packed{const_cast<int8_t*>(q), ldq, const_cast<uint8_t*>(s)}, w, add, ldadd, dx,
                                      lddx, dw, db, (float*)workspace, stream));
}

MFAC_API size_t mfac_linear_workspace_bytes(mfac_dtype type, int64_t rows, int64_t cin, int64_t cout, const void* x,
                                            int64_t ldx, const void* w, int64_t ldw) {
    if (!type_ok(type) || !layer_ok(rows, cin, cout) || rows == 0) return 0;
    return product_workspace_bytes(type, forward_product(rows, cin, cout, x, ldx, w, ldw));
}

MFAC_API mfac_status mfac_linear(mfac_dtype type, mfac_dtype btype, mfac_act act, int64_t rows, int64_t cin,
                                 int64_t cout, const void* x, int64_t ldx, const void* w, int64_t ldw,
                                 const void* bias, const void* res, int64_t ldres, void* y, int64_t ldy, void* z_out,
                                 int64_t ldz, int8_t* q, int64_t ldq, uint8_t* s, void* workspace,
                                 size_t workspace_bytes, hipStream_t stream) {
    if (!type_ok(type) || !param_type_ok(btype, type) || !act_ok(act) || !layer_ok(rows, cin, cout))
        return MFAC_EINVAL;
    if (rows == 0) return MFAC_OK;
    if (!matrix_ok(x, type, ldx, cin) || !matrix_ok(w, type, ldw, cin) || !matrix_ok(y, type, ldy, cout) ||
        !vector_ok(bias, btype) || (res && !matrix_ok(res, type, ldres, cout)) ||
        (z_out && !matrix_ok(z_out, type, ldz, cout)) || !packed_ok(q, ldq, s, cout, true) || (z_out && q))
        return MFAC_EINVAL;
    const Product p = forward_product(rows, cin, cout, x, ldx, w, ldw);
    const mfac_status st = check_workspace(product_workspace_bytes(type, p), workspace, workspace_bytes);
    if (st != MFAC_OK) return st;
    Epilogue e{};
    e.out_dt = e.io_dt = type;
    e.act = act;
    e.bias_dt = btype;
    e.out = y;
    e.ldo = ldy;
    e.bias = bias;
    e.add = res;
    e.ldadd = ldres;
    e.z = z_out;
    e.ldz = ldz;
    e.p = Packed{q, ldq, s};
    return done(launch_product(type, p, e, workspace, stream));
}

MFAC_API size_t mfac_act_bwd_workspace_bytes(int64_t rows, int64_t cols) {
    if (!size_ok(rows, cols)) return 0;
    return (size_t)round_up(act_bwd_parts(std::max<int64_t>(rows, 1), cols) * cols * 4, 256);
}

MFAC_API mfac_status mfac_act_bwd(mfac_dtype type, mfac_act act, int64_t rows, int64_t cols, const void* dy,
                                  int64_t lddy, const void* z, int64_t ldz, const int8_t* q, int64_t ldq,
                                  const uint8_t* s, void* dz, int64_t lddz, void* a, int64_t lda, float* db,
                                  void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!type_ok(type) || !act_ok(act) || !size_ok(rows, cols) || !vector_ok(db, MFAC_F32)) return MFAC_EINVAL;
    if (rows > 0) {
        if (!matrix_ok(dy, type, lddy, cols) || (dz && !matrix_ok(dz, type, lddz, cols)) ||
            (a && !matrix_ok(a, type, lda, cols)) || !packed_ok(q, ldq, s, cols, true))
            return MFAC_EINVAL;
        if (act == MFAC_ACT_NONE ? z || q || a : (q != nullptr) == (z != nullptr) || !dz) return MFAC_EINVAL;
        if (z && !matrix_ok(z, type, ldz, cols)) return MFAC_EINVAL;
    }
    if (db) {
        const mfac_status e = check_workspace(mfac_act_bwd_workspace_bytes(rows, cols), workspace, workspace_bytes);
        if (e != MFAC_OK) return e;
    }
    if (!db && !dz && !a) return MFAC_OK;
    return done(launch_act_bwd(type, act, rows, cols, dy, lddy, z, ldz,
                               Packed{const_cast<int8_t*>(q), ldq, const_cast<uint8_t*>(s)}, dz, lddz, a, lda, db,
                               (float*)workspace, stream));
}

MFAC_API size_t mfac_linear_bwd_input_workspace_bytes(mfac_dtype type, int64_t rows, int64_t cin, int64_t cout,
                                                      const void* dz, int64_t lddz, const void* w, int64_t ldw) {
    if (!type_ok(type) || !layer_ok(rows, cin, cout) || rows == 0) return 0;
    return product_workspace_bytes(type, input_product(rows, cin, cout, dz, lddz, w, ldw));
}

MFAC_API mfac_status mfac_linear_bwd_input(mfac_dtype type, int64_t rows, int64_t cin, int64_t cout, const void* dz,
                                           int64_t lddz, const void* w, int64_t ldw, const void* add, int64_t ldadd,
                                           void* dx, int64_t lddx, void* workspace, size_t workspace_bytes,
                                           hipStream_t stream) {
    if (!type_ok(type) || !layer_ok(rows, cin, cout)) return MFAC_EINVAL;
    if (rows == 0) return MFAC_OK;
    if (!matrix_ok(dz, type, lddz, cout) || !matrix_ok(w, type, ldw, cin) || !matrix_ok(dx, type, lddx, cin) ||
        (add && !matrix_ok(add, type, ldadd, cin)))
        return MFAC_EINVAL;
    const Product p = input_product(rows, cin, cout, dz, lddz, w, ldw);
    const mfac_status st = check_workspace(product_workspace_bytes(type, p), workspace, workspace_bytes);
    if (st != MFAC_OK) return st;
    Epilogue e{};
    e.out_dt = e.io_dt = type;
    e.out = dx;
    e.ldo = lddx;
    e.add = add;
    e.ldadd = ldadd;
    return done(launch_product(type, p, e, workspace, stream));
}

MFAC_API size_t mfac_linear_bwd_weight_workspace_bytes(mfac_dtype type, int64_t rows, int64_t cin, int64_t cout,
                                                       const void* dz, int64_t lddz, const void* x, int64_t ldx) {
    if (!type_ok(type) || !layer_ok(rows, cin, cout) || rows == 0) return 0;
    int8_t some;   // an 8-bit copy, by its presence alone
    return product_workspace_bytes(
        type, weight_product(rows, cin, cout, dz, lddz, x, ldx, x ? Packed{} : Packed{&some, cin, nullptr}));
}

MFAC_API mfac_status mfac_linear_bwd_weight(mfac_dtype type, mfac_dtype gtype, int64_t rows, int64_t cin, int64_t cout,
                                            const void* dz, int64_t lddz, const void* x, int64_t ldx, const int8_t* q,
                                            int64_t ldq, const uint8_t* s, const float* gamma, const float* beta,
                                            const float* db, void* dw, int64_t lddw, void* workspace,
                                            size_t workspace_bytes, hipStream_t stream) {
    if (!type_ok(type) || !param_type_ok(gtype, type) || !layer_ok(rows, cin, cout))
        return MFAC_EINVAL;
    if (!matrix_ok(dw, gtype, lddw, cin)) return MFAC_EINVAL;
    if (rows == 0) return done(launch_zero_matrix(gtype, cout, cin, dw, lddw, stream));
    if (!matrix_ok(dz, type, lddz, cout) || !packed_ok(q, ldq, s, cin, true) || (q != nullptr) == (x != nullptr) ||
        (x && !matrix_ok(x, type, ldx, cin)))
        return MFAC_EINVAL;
    if ((gamma != nullptr) != (beta != nullptr) || (gamma && !db) || !vector_ok(gamma, MFAC_F32) ||
        !vector_ok(beta, MFAC_F32) || !vector_ok(db, MFAC_F32))
        return MFAC_EINVAL;
    const Product p = weight_product(rows, cin, cout, dz, lddz, x, ldx,
                                     Packed{const_cast<int8_t*>(q), ldq, const_cast<uint8_t*>(s)});
    const mfac_status st = check_workspace(product_workspace_bytes(type, p), workspace, workspace_bytes);
    if (st != MFAC_OK) return st;
    Epilogue e{};
    e.out_dt = gtype;
    e.io_dt = type;
    e.out = dw;
    e.ldo = lddw;
    e.gamma = gamma;
    e.beta = beta;
    e.db = db;
    return done(launch_product(type, p, e, workspace, stream));
}
