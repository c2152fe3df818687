// C ABI of a gated block's operators (include/mfac.h): argument checks and the launches of linear.hip, gated.hip,
// residual.hip and dropout.hip.
#include <math.h>

#include <algorithm>

#include "../../include/mfac.h"
#include "internal.h"
#include "train.h"

#define MFAC_API extern "C" __attribute__((visibility("default")))

using namespace mfac;

namespace {

constexpr int64_t MOST = int64_t(1) << 30, MOST_WIDTH = int64_t(1) << 21, MOST_HELD = int64_t(1) << 15;

bool type_ok(int t) { return t == MFAC_F32 || t == MFAC_BF16 || t == MFAC_F16; }
bool param_type_ok(int t, int data) { return t == MFAC_F32 || t == data; }
bool act_ok(int a) { return a >= MFAC_ACT_NONE && a <= MFAC_ACT_SILU; }
// hidden: 2 hidden rows of W are a layer's width
bool gated_ok(int64_t rows, int64_t cin, int64_t hidden) {
    return rows >= 0 && rows <= MOST && cin >= 1 && cin <= MOST_WIDTH && hidden >= 1 && hidden <= MOST_WIDTH / 2;
}
bool layer_ok(int64_t rows, int64_t cin, int64_t cout) {
    return rows >= 0 && rows <= MOST && cin >= 1 && cin <= MOST_WIDTH && cout >= 1 && cout <= MOST_WIDTH;
}
bool aligned(const void* p, int type) { return (uintptr_t)p % (type == MFAC_F32 ? 4 : 2) == 0; }
bool matrix_ok(const void* p, int type, int64_t ld, int64_t cols) {
    return p && ld >= cols && ld <= (int64_t(1) << 33) && aligned(p, type);
}
bool matrix_or_none(const void* p, int type, int64_t ld, int64_t cols) { return !p || matrix_ok(p, type, ld, cols); }
bool vector_ok(const void* p, int type) { return !p || aligned(p, type); }
bool copy_ok(const void* q, int64_t ldq, const void* s, int64_t cols) {
    return q && s && ldq >= cols && ldq <= (int64_t(1) << 33);
}

mfac_status done(hipError_t e) { return e == hipSuccess ? MFAC_OK : MFAC_EHIP; }

mfac_status check_workspace(size_t need, const void* ws, size_t bytes) {
    if (need == 0) return MFAC_OK;
    if (bytes < need) return MFAC_EWORKSPACE;
    return ws && ((uintptr_t)ws & 255) == 0 ? MFAC_OK : MFAC_EINVAL;
}

Product gated_product(int64_t rows, int64_t cin, int64_t hidden, const void* x, int64_t ldx, const void* w, int64_t ldw) {
    return Product{rows, 2 * hidden, cin, x, ldx, false, w, ldw, false, Packed{}, GATE_FORWARD};
}
Product hidden_product(int64_t rows, int64_t hidden, int64_t cout, const void* dy, int64_t lddy, const void* w, int64_t ldw) {
    return Product{rows, hidden, cout, dy, lddy, false, w, ldw, true, Packed{}, GATE_HIDDEN};
}

Product da_product(int64_t rows, int64_t hidden, int64_t cout, const void* dy, int64_t lddy, const void* w, int64_t ldw) {
    return Product{rows, hidden, cout, dy, lddy, false, w, ldw, true, Packed{}};
}
Product weight_product(int64_t rows, int64_t cin, int64_t cout, const void* dz, const void* dz_lo, int64_t lddz,
                       const void* x, const void* x_lo, int64_t ldx, Packed p) {
    return Product{cout, cin, rows, dz, lddz, true, x, ldx, true, p, GATE_NONE, dz_lo, x_lo};
}

// Both pre-activations as tensors, or both as copies; `absent_ok`: or neither.
bool pair_ok(int type, int64_t hidden, const void* zg, const void* zu, int64_t ldz, const void* qg, const void* sg,
             const void* qu, const void* su, int64_t ldq, bool absent_ok) {
    const bool z = zg || zu, q = qg || sg || qu || su;
    if (z && q) return false;
    if (z) return matrix_ok(zg, type, ldz, hidden) && matrix_ok(zu, type, ldz, hidden);
    if (q) return copy_ok(qg, ldq, sg, hidden) && copy_ok(qu, ldq, su, hidden);
    return absent_ok;
}
Packed packed(const int8_t* q, int64_t ldq, const uint8_t* s) {
    return Packed{const_cast<int8_t*>(q), ldq, const_cast<uint8_t*>(s)};
}

// What forms dz and a from da.
Epilogue gate_epilogue(int type, int act, const void* zg, const void* zu, int64_t ldz, Packed pg, Packed pu, void* dz,
                       void* dz_lo, int64_t lddz, void* a, void* a_lo, int64_t lda) {
    Epilogue e{};
    e.out_dt = e.io_dt = type;
    e.act = act;
    e.out = dz;
    e.out_lo = dz_lo;
    e.ldo = lddz;
    e.z = const_cast<void*>(zg);
    e.z2 = const_cast<void*>(zu);
    e.ldz = ldz;
    e.p = pg;
    e.p2 = pu;
    e.a = a;
    e.a_lo = a_lo;
    e.lda = lda;
    return e;
}

// The workspace of mfac_gated_hidden_bwd. Where db is wanted, or hidden is not a multiple of what a wave of the fused
// product holds, da is formed in fp32 and read again: in the product's epilogue the column sums of dz would have to be joined
// over the tiles, and the checks for each column would double a code that is run through once a tile. bf16, 8192
// rows, hidden 8192, cout 2048: TIME_FUSED us fused, TIME_UNFUSED so.
struct HiddenWorkspace {
    bool fused;
    size_t product, da, total;
};
HiddenWorkspace hidden_workspace(int type, int64_t rows, int64_t hidden, int64_t cout, const void* dy, int64_t lddy,
                                 const void* w, int64_t ldw, bool want_db) {
    HiddenWorkspace n{!want_db && hidden % 64 == 0, 0, 0, 0};
    const Product p = n.fused ? hidden_product(rows, hidden, cout, dy, lddy, w, ldw)
                              : da_product(rows, hidden, cout, dy, lddy, w, ldw);
    if (rows > 0) n.product = product_workspace_bytes(type, p);
    n.total = n.product;
    if (n.fused) return n;
    n.da = (size_t)round_up(rows * hidden * 4, 256);
    n.total += n.da + (want_db ? mfac_gated_act_bwd_workspace_bytes(rows, hidden) : 0);
    return n;
}

// p: the probability of a value to be dropped, in units of 2^-16.
bool drop_of(double p, const int64_t* at, Drop& d) {
    if (!(p >= 0 && p <= 1) || (uintptr_t)at % 8) return false;
    d.threshold = (unsigned)floor(65536 * p + 0.5);
    d.scale = d.threshold < 65536 ? (float)(65536.0 / (65536 - (int)d.threshold)) : 0.f;
    d.at = at;
    return d.threshold == 0 || at;
}

bool norms_ok(int32_t norms) {
    return norms >= 0 && norms <= 7 && norms != MFAC_NORM_LAYER;
}

}  // namespace

// ---------------------------------------------------------------- gated layers
MFAC_API size_t mfac_gated_linear_workspace_bytes(mfac_dtype type, int64_t rows, int64_t cin, int64_t hidden,
                                                  const void* x, int64_t ldx, const void* w, int64_t ldw) {
    if (!type_ok(type) || !gated_ok(rows, cin, hidden) || rows == 0) return 0;
    return product_workspace_bytes(type, gated_product(rows, cin, hidden, x, ldx, w, ldw));
}

MFAC_API mfac_status mfac_gated_linear(mfac_dtype type, mfac_dtype btype, mfac_act act, int64_t rows, int64_t cin,
                                       int64_t hidden, const void* x, int64_t ldx, const void* w, int64_t ldw,
                                       const void* bias, void* y, int64_t ldy, void* zg, void* zu, int64_t ldz,
                                       int8_t* qg, uint8_t* sg, int8_t* qu, uint8_t* su, int64_t ldq, void* workspace,
                                       size_t workspace_bytes, hipStream_t stream) {
    if (!type_ok(type) || !param_type_ok(btype, type) || !act_ok(act) || !gated_ok(rows, cin, hidden)) return MFAC_EINVAL;
    if (rows == 0) return MFAC_OK;
    if (!matrix_ok(x, type, ldx, cin) || !matrix_ok(w, type, ldw, cin) || !vector_ok(bias, btype) ||
        !matrix_ok(y, type, ldy, hidden) || !pair_ok(type, hidden, zg, zu, ldz, qg, sg, qu, su, ldq, true))
        return MFAC_EINVAL;
    const Product p = gated_product(rows, cin, hidden, x, ldx, w, ldw);
    const mfac_status st = check_workspace(product_workspace_bytes(type, p), workspace, workspace_bytes);
    if (st != MFAC_OK) return st;
    Epilogue e{};
    e.out_dt = e.io_dt = type;
    e.act = act;
    e.bias_dt = btype;
    e.out = y;
    e.ldo = ldy;
    e.bias = bias;
    e.z = zg;
    e.z2 = zu;
    e.ldz = ldz;
    e.p = Packed{qg, ldq, sg};
    e.p2 = Packed{qu, ldq, su};
    return done(launch_product(type, p, e, workspace, stream));
}

MFAC_API size_t mfac_gated_act_bwd_workspace_bytes(int64_t rows, int64_t hidden) {
    if (!gated_ok(rows, 1, hidden)) return 0;
    return (size_t)round_up(gated_bwd_parts(std::max<int64_t>(rows, 1), hidden) * 2 * hidden * 4, 256);
}

MFAC_API mfac_status mfac_gated_act_bwd(mfac_dtype type, mfac_act act, int64_t rows, int64_t hidden, const void* da,
                                        int64_t ldda, const void* zg, const void* zu, int64_t ldz, const int8_t* qg,
                                        const uint8_t* sg, const int8_t* qu, const uint8_t* su, int64_t ldq, void* dz,
                                        void* dz_lo, int64_t lddz, void* a, void* a_lo, int64_t lda, float* db,
                                        void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!type_ok(type) || !act_ok(act) || !gated_ok(rows, 1, hidden) || !vector_ok(db, MFAC_F32) ||
        (type == MFAC_F32 && (dz_lo || a_lo)) || (a_lo && !a))
        return MFAC_EINVAL;
    if (rows > 0 && (!matrix_ok(da, type, ldda, hidden) || !matrix_ok(dz, type, lddz, 2 * hidden) ||
                     !matrix_or_none(dz_lo, type, lddz, 2 * hidden) || !matrix_or_none(a, type, lda, hidden) ||
                     !matrix_or_none(a_lo, type, lda, hidden) ||
                     !pair_ok(type, hidden, zg, zu, ldz, qg, sg, qu, su, ldq, false)))
        return MFAC_EINVAL;
    if (db) {
        const mfac_status e =
            check_workspace(mfac_gated_act_bwd_workspace_bytes(rows, hidden), workspace, workspace_bytes);
        if (e != MFAC_OK) return e;
    }
    const Epilogue e = gate_epilogue(type, act, zg, zu, ldz, packed(qg, ldq, sg), packed(qu, ldq, su), dz, dz_lo, lddz, a,
                                     a_lo, lda);
    return done(launch_gated_act_bwd(type, type, rows, hidden, da, ldda, e, db, (float*)workspace, stream));
}

MFAC_API size_t mfac_gated_hidden_bwd_workspace_bytes(mfac_dtype type, int64_t rows, int64_t hidden, int64_t cout,
                                                      const void* dy, int64_t lddy, const void* w, int64_t ldw,
                                                      int32_t want_db) {
    if (!type_ok(type) || !gated_ok(rows, cout, hidden)) return 0;
    return hidden_workspace(type, rows, hidden, cout, dy, lddy, w, ldw, want_db != 0).total;
}

MFAC_API mfac_status mfac_gated_hidden_bwd(mfac_dtype type, mfac_act act, int64_t rows, int64_t hidden, int64_t cout,
                                           const void* dy, int64_t lddy, const void* w, int64_t ldw, const void* zg,
                                           const void* zu, int64_t ldz, const int8_t* qg, const uint8_t* sg,
                                           const int8_t* qu, const uint8_t* su, int64_t ldq, void* dz, void* dz_lo,
                                           int64_t lddz, void* a, void* a_lo, int64_t lda, float* db, void* workspace,
                                           size_t workspace_bytes, hipStream_t stream) {
    if (!type_ok(type) || !act_ok(act) || !gated_ok(rows, cout, hidden) || !vector_ok(db, MFAC_F32) ||
        (type == MFAC_F32 && (dz_lo || a_lo)) || (a_lo && !a))
        return MFAC_EINVAL;
    if (rows > 0 && (!matrix_ok(dy, type, lddy, cout) || !matrix_ok(w, type, ldw, hidden) ||
                     !matrix_ok(dz, type, lddz, 2 * hidden) || !matrix_or_none(dz_lo, type, lddz, 2 * hidden) ||
                     !matrix_or_none(a, type, lda, hidden) || !matrix_or_none(a_lo, type, lda, hidden) ||
                     !pair_ok(type, hidden, zg, zu, ldz, qg, sg, qu, su, ldq, false)))
        return MFAC_EINVAL;
    if (rows == 0 && !db) return MFAC_OK;
    const HiddenWorkspace need = hidden_workspace(type, rows, hidden, cout, dy, lddy, w, ldw, db != nullptr);
    const mfac_status st = check_workspace(need.total, workspace, workspace_bytes);
    if (st != MFAC_OK) return st;
    const Epilogue e = gate_epilogue(type, act, zg, zu, ldz, packed(qg, ldq, sg), packed(qu, ldq, su), dz, dz_lo, lddz, a,
                                     a_lo, lda);
    char* ws = (char*)workspace;
    if (need.fused) return done(launch_product(type, hidden_product(rows, hidden, cout, dy, lddy, w, ldw), e, ws, stream));
    // da in fp32, then the gate's pass over it
    float* da = (float*)(ws + need.product);
    if (rows > 0) {
        Epilogue plain{};
        plain.out_dt = MFAC_F32;
        plain.io_dt = type;
        plain.out = da;
        plain.ldo = hidden;
        const hipError_t err = launch_product(type, da_product(rows, hidden, cout, dy, lddy, w, ldw), plain, ws, stream);
        if (err != hipSuccess) return done(err);
    }
    return done(launch_gated_act_bwd(type, MFAC_F32, rows, hidden, da, hidden, e, db, (float*)(ws + need.product + need.da),
                                     stream));
}

// ---------------------------------------------------------------- weight gradients from two parts
MFAC_API size_t mfac_linear_bwd_weight_parts_workspace_bytes(mfac_dtype type, int64_t rows, int64_t cin, int64_t cout,
                                                             const void* dz, const void* dz_lo, int64_t lddz, const void* x,
                                                             const void* x_lo, int64_t ldx) {
    if ((type != MFAC_BF16 && type != MFAC_F16) || !layer_ok(rows, cin, cout) || rows == 0) return 0;
    int8_t some;   // an 8-bit copy, by its presence alone
    return product_workspace_bytes(type, weight_product(rows, cin, cout, dz, dz_lo, lddz, x, x_lo, ldx,
                                                        x ? Packed{} : Packed{&some, cin, nullptr}));
}

MFAC_API mfac_status mfac_linear_bwd_weight_parts(mfac_dtype type, mfac_dtype gtype, int64_t rows, int64_t cin, int64_t cout,
                                                  const void* dz, const void* dz_lo, int64_t lddz, const void* x,
                                                  const void* x_lo, int64_t ldx, const int8_t* q, int64_t ldq,
                                                  const uint8_t* s, const float* gamma, const float* beta, const float* db,
                                                  void* dw, int64_t lddw, void* workspace, size_t workspace_bytes,
                                                  hipStream_t stream) {
    if ((type != MFAC_BF16 && type != MFAC_F16) || !param_type_ok(gtype, type) || !layer_ok(rows, cin, cout) ||
        !matrix_ok(dw, gtype, lddw, cin))
        return MFAC_EINVAL;
    if (rows == 0) return done(launch_zero_matrix(gtype, cout, cin, dw, lddw, stream));
    const bool copy = q || s;
    if (!matrix_ok(dz, type, lddz, cout) || !matrix_or_none(dz_lo, type, lddz, cout) || copy == (x != nullptr) ||
        (copy ? !copy_ok(q, ldq, s, cin) : !matrix_ok(x, type, ldx, cin)) || !matrix_or_none(x_lo, type, ldx, cin) ||
        (dz_lo != nullptr) == (x_lo != nullptr) || (x_lo && !x))
        return MFAC_EINVAL;
    if ((gamma != nullptr) != (beta != nullptr) || (gamma && !db) || !vector_ok(gamma, MFAC_F32) ||
        !vector_ok(beta, MFAC_F32) || !vector_ok(db, MFAC_F32))
        return MFAC_EINVAL;
    const Product p = weight_product(rows, cin, cout, dz, dz_lo, lddz, x, x_lo, ldx, packed(q, ldq, s));
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

// ---------------------------------------------------------------- between two blocks
MFAC_API mfac_status mfac_residual_norm(mfac_dtype type, mfac_dtype wtype, int32_t norms, int64_t rows, int64_t cols,
                                        const void* y, int64_t ldy, const void* post_w, const void* post_b,
                                        const void* gate, const void* gates, int64_t ldgates, const void* res,
                                        int64_t ldres, double scale, double p, const int64_t* at, const void* pre_w,
                                        const void* pre_b, double eps, void* s, int64_t lds, void* h, int64_t ldh,
                                        float* post_mean, float* post_rstd, float* pre_mean, float* pre_rstd, int8_t* q,
                                        int64_t ldq, uint8_t* sq, hipStream_t stream) {
    Residual g{};
    if (!type_ok(type) || !param_type_ok(wtype, type) || !norms_ok(norms) || rows < 0 || rows > MOST || cols < 1 ||
        cols > MOST_HELD || !(eps >= 0) || !isfinite(eps) || !isfinite(scale) || !drop_of(p, at, g.drop))
        return MFAC_EINVAL;
    const bool post = norms & MFAC_NORM_POST, pre = norms & MFAC_NORM_PRE, layer = norms & MFAC_NORM_LAYER;
    if ((!post && (post_w || post_b || post_mean || post_rstd)) || (!layer && (post_b || pre_b || post_mean || pre_mean)) ||
        (!pre && (pre_w || pre_b || pre_mean || pre_rstd || h || q || sq)) || (gate && gates))
        return MFAC_EINVAL;
    if (rows == 0) return MFAC_OK;
    for (const void* v : {post_w, post_b, gate, pre_w, pre_b})
        if (!vector_ok(v, wtype)) return MFAC_EINVAL;
    for (const void* v : {post_mean, post_rstd, pre_mean, pre_rstd})
        if (!vector_ok(v, MFAC_F32)) return MFAC_EINVAL;
    if (!matrix_ok(y, type, ldy, cols) || !matrix_or_none(gates, type, ldgates, cols) ||
        !matrix_or_none(res, type, ldres, cols) || !matrix_or_none(s, type, lds, cols) ||
        (pre && !matrix_ok(h, type, ldh, cols)) || ((q || sq) && !copy_ok(q, ldq, sq, cols)) || (!s && !h))
        return MFAC_EINVAL;
    g.norms = norms;
    g.rows = rows;
    g.cols = cols;
    g.y = y;
    g.ldy = ldy;
    g.w1 = post_w;
    g.b1 = post_b;
    g.w2 = pre_w;
    g.b2 = pre_b;
    g.gate = gate;
    g.gates = gates;
    g.ldgates = ldgates;
    g.r = res;
    g.ldr = ldres;
    g.scale = (float)scale;
    g.eps = (float)eps;
    g.s = s;
    g.lds = lds;
    g.h = h;
    g.ldh = ldh;
    g.mean1 = post_mean;
    g.rstd1 = post_rstd;
    g.mean2 = pre_mean;
    g.rstd2 = pre_rstd;
    g.p = Packed{q, ldq, sq};
    return done(launch_residual(type, wtype, g, stream));
}

MFAC_API size_t mfac_residual_norm_bwd_workspace_bytes(mfac_dtype type, int32_t norms, int64_t rows,
                                                       int64_t cols) {
    if (!type_ok(type) || !norms_ok(norms) || rows < 0 || rows > MOST || cols < 1 || cols > MOST_HELD) return 0;
    return (size_t)round_up(residual_bwd_parts(type, std::max<int64_t>(rows, 1), cols) * residual_sums(norms) * cols * 4, 256);
}

MFAC_API mfac_status mfac_residual_norm_bwd(mfac_dtype type, mfac_dtype wtype, int32_t norms, int64_t rows, int64_t cols,
                                            const void* ds, int64_t ldds, const void* dh, int64_t lddh, const void* y,
                                            int64_t ldy, const float* post_mean, const float* post_rstd, const void* s,
                                            int64_t lds, const int8_t* q, int64_t ldq, const uint8_t* sq,
                                            const float* pre_mean, const float* pre_rstd, const void* post_w,
                                            const void* post_b, const void* gate, const void* gates, int64_t ldgates,
                                            double scale, double p, const int64_t* at, const void* pre_w, void* dy,
                                            int64_t lddy, void* dres, int64_t lddres, void* dgates, int64_t lddgates,
                                            void* dpost_w, void* dpost_b, void* dgate, void* dpre_w, void* dpre_b,
                                            void* workspace, size_t workspace_bytes, hipStream_t stream) {
    Residual g{};
    if (!type_ok(type) || !param_type_ok(wtype, type) || !norms_ok(norms) || rows < 0 || rows > MOST || cols < 1 ||
        cols > MOST_HELD || !isfinite(scale) || !drop_of(p, at, g.drop))
        return MFAC_EINVAL;
    const bool post = norms & MFAC_NORM_POST, pre = norms & MFAC_NORM_PRE, layer = norms & MFAC_NORM_LAYER;
    if ((!post && (post_w || post_b || post_mean || post_rstd || dpost_w || dpost_b)) ||
        (!layer && (post_b || post_mean || pre_mean || dpost_b || dpre_b)) ||
        (!pre && (dh || s || q || sq || pre_w || pre_mean || pre_rstd || dpre_w || dpre_b)) || (gate && gates) ||
        (dgate && !gate) || (dgates && !gates))
        return MFAC_EINVAL;
    for (const void* v : {post_w, post_b, gate, pre_w, (const void*)dpost_w, (const void*)dpost_b, (const void*)dgate,
                          (const void*)dpre_w, (const void*)dpre_b})
        if (!vector_ok(v, wtype)) return MFAC_EINVAL;
    if (rows > 0) {
        for (const void* v : {post_mean, post_rstd, pre_mean, pre_rstd})
            if (!vector_ok(v, MFAC_F32)) return MFAC_EINVAL;
        if (!matrix_or_none(ds, type, ldds, cols) || !matrix_or_none(dy, type, lddy, cols) ||
            !matrix_or_none(dres, type, lddres, cols) || !matrix_or_none(gates, type, ldgates, cols) ||
            !matrix_or_none(dgates, type, lddgates, cols) || !matrix_or_none(y, type, ldy, cols))
            return MFAC_EINVAL;
        if (!ds && !pre) return MFAC_EINVAL;
        if (!y && (post || dgate || dgates)) return MFAC_EINVAL;
        if (post && (!post_rstd || (layer && !post_mean))) return MFAC_EINVAL;
        if (pre) {
            const bool copy = q || sq;
            if (!matrix_ok(dh, type, lddh, cols) || !pre_rstd || copy == (s != nullptr)) return MFAC_EINVAL;
            if (copy ? !copy_ok(q, ldq, sq, cols) || pre_mean : !matrix_ok(s, type, lds, cols) || (layer && !pre_mean))
                return MFAC_EINVAL;
        }
    }
    if (dpost_w || dpost_b || dgate || dpre_w || dpre_b) {
        const mfac_status e =
            check_workspace(mfac_residual_norm_bwd_workspace_bytes(type, norms, rows, cols), workspace, workspace_bytes);
        if (e != MFAC_OK) return e;
    }
    g.norms = norms;
    g.rows = rows;
    g.cols = cols;
    g.y = post || dgate || dgates ? y : nullptr;
    g.ldy = ldy;
    g.w1 = post_w;
    g.b1 = post_b;
    g.w2 = pre_w;
    g.gate = gate;
    g.gates = gates;
    g.ldgates = ldgates;
    g.scale = (float)scale;
    g.s = const_cast<void*>(s);
    g.lds = lds;
    g.mean1 = const_cast<float*>(post_mean);
    g.rstd1 = const_cast<float*>(post_rstd);
    g.mean2 = const_cast<float*>(pre_mean);
    g.rstd2 = const_cast<float*>(pre_rstd);
    g.p = packed(q, ldq, sq);
    ResidualBwd b{ds, ldds, dh, lddh, dy, lddy, dres, lddres, dgates, lddgates, dpost_w, dpost_b, dpre_w, dpre_b, dgate,
                  (float*)workspace};
    return done(launch_residual_bwd(type, wtype, g, b, stream));
}

// ---------------------------------------------------------------- dropout
MFAC_API mfac_status mfac_dropout(mfac_dtype type, int64_t rows, int64_t cols, const void* x, int64_t ldx, double p,
                                  const int64_t* at, void* y, int64_t ldy, hipStream_t stream) {
    Drop d{};
    if (!type_ok(type) || rows < 0 || rows > MOST || cols < 1 || cols > MOST || !drop_of(p, at, d)) return MFAC_EINVAL;
    if (rows == 0) return MFAC_OK;
    if (!matrix_ok(x, type, ldx, cols) || !matrix_ok(y, type, ldy, cols) || !at) return MFAC_EINVAL;
    return done(launch_dropout(type, rows, cols, x, ldx, d, y, ldy, stream));
}
