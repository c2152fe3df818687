// C ABI of a gated block's operators (include/mfac.h): argument checks and the launches of linear.hip, gated.hip,
// residual.hip and dropout.hip.
#include <math.h>

#include <algorithm>

#include "../../include/mfac.h"
#include "checks.h"
#include "internal.h"
#include "train.h"

using namespace mfac;

namespace {

constexpr int64_t MOST_HELD = int64_t(1) << 15;

// hidden: 2 hidden rows of W are a layer's width
bool gated_ok(int64_t rows, int64_t cin, int64_t hidden) {
    return size_ok(rows, cin) && cin <= MOST_WIDTH && hidden >= 1 && hidden <= MOST_WIDTH / 2;
}
bool matrix_or_none(const void* p, int type, int64_t ld, int64_t cols) { return !p || matrix_ok(p, type, ld, cols); }
bool copy_ok(const void* q, int64_t ldq, const void* s, int64_t cols) { return packed_ok(q, ldq, s, cols, false); }

Product gated_product(int64_t rows, int64_t cin, int64_t hidden, const void* x, int64_t ldx, const void* w, int64_t ldw) {
    return Product{rows, 2 * hidden, cin, x, ldx, false, w, ldw, false, Packed{}, GATE_FORWARD};
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

// A gated layer's backward pass: what it takes, what it forms.
struct GatedBwd {
    int type, gtype, act;
    int64_t rows, cin, hidden, cout;   // cout 0: dy is the gradient of the gated layer's own output
    const void* dy;
    int64_t lddy;
    const void* w2;
    int64_t ldw2;
    const void* x;
    int64_t ldx;
    Packed xp;
    const float *gamma, *beta;
    const void* w1;
    int64_t ldw1;
    bool dx, dw1, db1, dw2;
    // places in the workspace: dy as the products take it, da in fp32, dz and a in parts, db and its parts, the products'
    bool fused;
    int parts;
    int64_t lddy_in, ldw2_in, ldx_in, ldw1_in, lddz, lda;
    size_t dy_in, w2_in, x_in, w1_in, da, dz, a, db, db_part, range, product, total;

    bool da_given() const { return cout == 0; }
    bool sums() const { return db1 || (dw1 && beta); }
    bool dz_wanted() const { return dx || dw1; }
    bool da_wanted() const { return dz_wanted() || db1; }   // a is formed without it
    bool ranged() const { return type == MFAC_F16 && parts == 2; }   // dz and a may need factors to be in two parts
    int64_t dy_part() const { return rows * lddy_in * 2; }
    int64_t dz_part() const { return rows * lddz * 2; }
    int64_t a_part() const { return rows * lda * 2; }

    // The products, dy, dz and a being at these addresses; ws: the workspace (or null, where only sizes are looked at).
    Product da_product(const void* at, const char* ws) const {
        Product p{rows, hidden, cout, at, dy_laid_out() ? lddy_in : lddy, false, w2, ldw2, true, Packed{},
                  fused ? GATE_HIDDEN : GATE_NONE};
        if (dy_laid_out()) p.a_parts = type == MFAC_F32 ? 3 : 1, p.a_part = dy_part();
        if (type == MFAC_F32) p.B = ws ? ws + w2_in : nullptr, p.ldb = ldw2_in, p.b_parts = 3, p.b_part = cout * ldw2_in * 2;
        return p;
    }
    Product dw2_product(const void* at, const void* a_at) const {
        Product p{cout, hidden, rows, at, dy_laid_out() ? lddy_in : lddy, true, a_at, lda, true, Packed{}};
        if (dy_laid_out()) p.a_parts = type == MFAC_F32 ? 3 : 1, p.a_part = dy_part();
        p.b_parts = parts, p.b_part = a_part();
        return p;
    }
    // dx is of 16-bit data from dz's first part: in two it would be no nearer after its own rounding
    Product dx_product(const void* dz_at, const char* ws) const {
        Product p{rows, cin, 2 * hidden, dz_at, lddz, false, w1, ldw1, true, Packed{}};
        p.a_parts = type == MFAC_F32 ? 3 : 1, p.a_part = dz_part();
        if (type == MFAC_F32) p.B = ws ? ws + w1_in : nullptr, p.ldb = ldw1_in, p.b_parts = 3, p.b_part = 2 * hidden * ldw1_in * 2;
        return p;
    }
    Product dw1_product(const void* dz_at, const char* ws) const {
        Product p{2 * hidden, cin, rows, dz_at, lddz, true, x, ldx, true, xp};
        p.a_parts = parts, p.a_part = dz_part();
        if (type == MFAC_F32 && x) p.B = ws ? ws + x_in : nullptr, p.ldb = ldx_in, p.b_parts = 3, p.b_part = rows * ldx_in * 2;
        return p;
    }
    // What is laid out before the products, in one launch: fp32, split once, and dy where its rows are not 16-byte aligned.
    int lay_outs(char* ws, LayOut (&jobs)[4]) const {
        int n = 0;
        if (dy_laid_out()) jobs[n++] = LayOut{dy, lddy, rows, cout, ws + dy_in, lddy_in};
        if (type != MFAC_F32) return n;
        if (!da_given() && da_wanted()) jobs[n++] = LayOut{w2, ldw2, cout, hidden, ws + w2_in, ldw2_in};
        if (dw1 && x) jobs[n++] = LayOut{x, ldx, rows, cin, ws + x_in, ldx_in};
        if (dx) jobs[n++] = LayOut{w1, ldw1, 2 * hidden, cin, ws + w1_in, ldw1_in};
        return n;
    }
    bool dy_laid_out() const {
        return !da_given() && (type == MFAC_F32 || ((uintptr_t)dy & 15) || lddy % 8 || cout % 8 || lddy > MOST_WIDTH);
    }

    void place() {
        fused = parts = 0;
        lddy_in = round_up(std::max<int64_t>(cout, 1), 8);
        lddz = round_up(2 * hidden, 8);
        lda = ldw2_in = round_up(hidden, 8);
        ldx_in = ldw1_in = round_up(cin, 8);
        dy_in = w2_in = x_in = w1_in = da = dz = a = db = db_part = range = product = total = 0;
        if (!(dx || dw1 || db1 || dw2)) return;
        // Gradients of 16-bit weights' data in fp32 are formed from dz and a in two parts: rounded to one, they leave
        // the gradient 2.3e-3 from 64 bits (relative, 2-norm), in two 3e-6. It doubles these two products.
        parts = type == MFAC_F32 ? 3 : gtype == MFAC_F32 && (dw1 || dw2) ? 2 : 1;
        // dz straight from the product that forms da, without db, whose sums would have to be joined over the tiles.
        // Otherwise da is stored in fp32 and read again.
        fused = !da_given() && da_wanted() && !sums() && rows > 0;
        fused = fused && hidden_fused(type, product_splits(type, da_product(nullptr, nullptr)), hidden);
        auto take = [&](size_t bytes) {
            const size_t at = total;
            total += (size_t)round_up((int64_t)bytes, 256);
            return at;
        };
        if (dy_laid_out()) dy_in = take((size_t)dy_part() * (type == MFAC_F32 ? 3 : 1));
        if (type == MFAC_F32) {
            if (!da_given() && da_wanted()) w2_in = take((size_t)cout * ldw2_in * 6);
            if (dw1 && x) x_in = take((size_t)rows * ldx_in * 6);
            if (dx) w1_in = take((size_t)hidden * ldw1_in * 12);
        }
        if (!da_given() && da_wanted() && !fused) da = take((size_t)rows * hidden * 4);
        if (dz_wanted()) dz = take((size_t)dz_part() * parts);
        if (dw2) a = take((size_t)a_part() * parts);
        if (sums()) {
            db = take((size_t)hidden * 8);
            db_part = take((size_t)gated_bwd_parts(std::max<int64_t>(rows, 1), hidden) * hidden * 8);
        }
        if (ranged()) range = take(GATE_RANGE * 4);
        if (rows > 0) {   // one after another in the same place; addresses in the workspace are aligned, and not looked at
            if (!da_given() && da_wanted()) need(da_product(dy_laid_out() ? nullptr : dy, nullptr));
            if (dx) need(dx_product(nullptr, nullptr));
            if (dw1) need(dw1_product(nullptr, nullptr));
            if (dw2) need(dw2_product(dy_laid_out() ? nullptr : dy, nullptr));
        }
        const size_t at = total;
        total += product;
        product = at;
    }
    void need(const Product& p) { product = std::max(product, product_workspace_bytes(type, p)); }
};

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

MFAC_API size_t mfac_gated_bwd_workspace_bytes(mfac_dtype type, mfac_dtype gtype, int64_t rows, int64_t cin, int64_t hidden,
                                               int64_t cout, const void* dy, int64_t lddy, const void* w2, int64_t ldw2,
                                               const void* x, int64_t ldx, const void* w1, int64_t ldw1, uint32_t wanted) {
    if (!type_ok(type) || !param_type_ok(gtype, type) || !gated_ok(rows, cin, hidden) || cout < 0 || cout > MOST_WIDTH ||
        wanted > 31)
        return 0;
    int8_t some;   // an 8-bit copy and a norm's parameters, by their presence alone
    float one;
    GatedBwd g{type, gtype, MFAC_ACT_NONE, rows, cin, hidden, cout, dy, lddy, w2, ldw2, x, ldx,
               x ? Packed{} : Packed{&some, cin, nullptr}, &one, wanted & MFAC_GATED_BETA ? &one : nullptr, w1, ldw1,
               (wanted & MFAC_GATED_DX) != 0, (wanted & MFAC_GATED_DW1) != 0, (wanted & MFAC_GATED_DB1) != 0,
               (wanted & MFAC_GATED_DW2) != 0};
    g.place();
    return g.total;
}

MFAC_API mfac_status mfac_gated_bwd(mfac_dtype type, mfac_dtype gtype, mfac_act act, int64_t rows, int64_t cin,
                                    int64_t hidden, int64_t cout, const void* dy, int64_t lddy, const void* w2, int64_t ldw2,
                                    const void* x, int64_t ldx, const int8_t* q, int64_t ldq, const uint8_t* s,
                                    const float* gamma, const float* beta, const void* w1, int64_t ldw1, const void* zg,
                                    const void* zu, int64_t ldz, const int8_t* qg, const uint8_t* sg, const int8_t* qu,
                                    const uint8_t* su, int64_t ldqz, void* dx, int64_t lddx, void* dw1, int64_t lddw1,
                                    float* db1, void* dw2, int64_t lddw2, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream) {
    if (!type_ok(type) || !param_type_ok(gtype, type) || !act_ok(act) || !gated_ok(rows, cin, hidden) || cout < 0 ||
        cout > MOST_WIDTH || (cout == 0 && dw2) || !matrix_or_none(dw1, gtype, lddw1, cin) || !vector_ok(db1, MFAC_F32) ||
        !matrix_or_none(dw2, gtype, lddw2, hidden))
        return MFAC_EINVAL;
    if (!dx && !dw1 && !db1 && !dw2) return MFAC_OK;
    if (rows > 0) {
        const bool copy = q || s;
        if (!matrix_ok(dy, type, lddy, cout ? cout : hidden) || (cout && (dx || dw1 || db1) && !matrix_ok(w2, type, ldw2, hidden)) ||
            !pair_ok(type, hidden, zg, zu, ldz, qg, sg, qu, su, ldqz, false) ||
            (dx && (!matrix_ok(w1, type, ldw1, cin) || !matrix_ok(dx, type, lddx, cin))))
            return MFAC_EINVAL;
        if (dw1 && (copy == (x != nullptr) || (copy ? !copy_ok(q, ldq, s, cin) : !matrix_ok(x, type, ldx, cin)) ||
                    (beta && !gamma) || !vector_ok(gamma, MFAC_F32) || !vector_ok(beta, MFAC_F32)))
            return MFAC_EINVAL;
    }
    GatedBwd g{type, gtype, act, rows, cin, hidden, cout, dy, lddy, w2, ldw2, x, ldx, packed(q, ldq, s), gamma, beta, w1, ldw1,
               dx != nullptr, dw1 != nullptr, db1 != nullptr, dw2 != nullptr};
    g.place();
    const mfac_status st = check_workspace(g.total, workspace, workspace_bytes);
    if (st != MFAC_OK) return st;
    char* ws = (char*)workspace;
    hipError_t err = hipSuccess;
    if (rows == 0) {
        if (dw1) err = launch_zero_matrix(gtype, 2 * hidden, cin, dw1, lddw1, stream);
        if (err == hipSuccess && dw2) err = launch_zero_matrix(gtype, cout, hidden, dw2, lddw2, stream);
        if (err == hipSuccess && db1) err = launch_zero_matrix(MFAC_F32, 1, 2 * hidden, db1, 2 * hidden, stream);
        return done(err);
    }
    LayOut jobs[4];
    const int njobs = g.lay_outs(ws, jobs);
    const void* dy_at = g.dy_laid_out() ? ws + g.dy_in : g.dy;
    if ((err = launch_lay_out(type, njobs, jobs, stream)) != hipSuccess) return done(err);
    Epilogue e{};   // what forms dz and a from da
    e.out_dt = e.io_dt = type;
    e.act = act;
    e.z = const_cast<void*>(zg);
    e.z2 = const_cast<void*>(zu);
    e.ldz = ldz;
    e.p = packed(qg, ldqz, sg);
    e.p2 = packed(qu, ldqz, su);
    e.out = g.dz_wanted() ? ws + g.dz : nullptr;
    e.ldo = g.lddz;
    e.a = dw2 ? ws + g.a : nullptr;
    e.lda = g.lda;
    e.parts = g.parts;
    e.out_part = g.dz_part();
    e.a_part = g.a_part();
    float* const range = g.ranged() ? (float*)(ws + g.range) : nullptr;
    e.range = range;
    float* db = db1 ? db1 : g.sums() ? (float*)(ws + g.db) : nullptr;
    if (!g.da_wanted()) {
        err = launch_gated_act_bwd(type, type, rows, hidden, nullptr, 0, e, nullptr, nullptr, stream);
    } else if (g.fused) {
        err = launch_product(type, g.da_product(dy_at, ws), e, ws + g.product, stream);
    } else if (g.da_given()) {
        err = launch_gated_act_bwd(type, type, rows, hidden, dy, lddy, e, db, (float*)(ws + g.db_part), stream);
    } else {
        Epilogue plain{};
        plain.out_dt = MFAC_F32;
        plain.io_dt = type;
        plain.out = ws + g.da;
        plain.ldo = hidden;
        err = launch_product(type, g.da_product(dy_at, ws), plain, ws + g.product, stream);
        if (err == hipSuccess)
            err = launch_gated_act_bwd(type, MFAC_F32, rows, hidden, ws + g.da, hidden, e, db, (float*)(ws + g.db_part), stream);
    }
    auto product = [&](const Product& p, int out_dt, void* out, int64_t ldo, bool affine, int factor) {
        Epilogue o{};
        o.times = range ? range + factor : nullptr;
        o.out_dt = out_dt;
        o.io_dt = type;
        o.out = out;
        o.ldo = ldo;
        if (affine) {
            o.gamma = gamma;
            o.beta = beta;
            o.db = db;
        }
        if (err == hipSuccess) err = launch_product(type, p, o, ws + g.product, stream);
    };
    if (dw2) product(g.dw2_product(dy_at, ws + g.a), gtype, dw2, lddw2, false, 3);
    if (dx) product(g.dx_product(ws + g.dz, ws), type, dx, lddx, false, 2);
    if (dw1) product(g.dw1_product(ws + g.dz, ws), gtype, dw1, lddw1, true, 2);
    return done(err);
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
    return (size_t)round_up(residual_bwd_parts(type, norms, std::max<int64_t>(rows, 1), cols) * residual_sums(norms) * cols * 4, 256);
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
    if (!type_ok(type) || !size_ok(rows, cols) || !drop_of(p, at, d)) return MFAC_EINVAL;
    if (rows == 0) return MFAC_OK;
    if (!matrix_ok(x, type, ldx, cols) || !matrix_ok(y, type, ldy, cols) || !at) return MFAC_EINVAL;
    return done(launch_dropout(type, rows, cols, x, ldx, d, y, ldy, stream));
}
