// Host-side check of the gated block's C ABI (csrc/gated_capi.hip) under AddressSanitizer and
// UndefinedBehaviorSanitizer, without a GPU: the calls are linked against stubs of the kernel launchers,
// which check what they are given against the workspace. Every call is made once as it should be, over the
// combinations of what may be wanted, and once with a launch that fails (MFAC_EHIP). Exit status 0 and "host check ok"
// on success.
#include <stdio.h>
#include <string.h>

#include "../../include/mfac.h"
#include "../../paper_2107_03356_amd/csrc/train.h"

namespace {
int failures = 0, launches = 0;
bool fail_launch = false;
const char *ws_from = nullptr, *ws_to = nullptr;
hipError_t launched() {
    ++launches;
    return fail_launch ? hipErrorUnknown : hipSuccess;
}
#define CHECK(c)                                                                        \
    do {                                                                                \
        if (!(c)) {                                                                     \
            fprintf(stderr, "host check failed: %s (%s:%d)\n", #c, __FILE__, __LINE__); \
            ++failures;                                                                 \
        }                                                                               \
    } while (0)
// A range that lies in the workspace as a whole, or outside of it.
void range(const void* p, int64_t bytes) {
    const char* c = (const char*)p;
    if (c >= ws_from && c < ws_to) CHECK(c + bytes <= ws_to);
}
}  // namespace

namespace mfac {
int64_t act_bwd_parts(int64_t rows, int64_t) { return rows < 3 ? rows : 3; }
int64_t gated_bwd_parts(int64_t rows, int64_t cols) { return act_bwd_parts(rows, cols); }
hipError_t launch_gated_act_bwd(int dt, int da_dt, int64_t rows, int64_t hidden, const void* da, int64_t ldda, const Epilogue& e,
                                float* db, float* part, hipStream_t) {
    CHECK(e.ldo % 8 == 0 && e.lda % 8 == 0 && e.ldo >= 2 * hidden && e.lda >= hidden && ((uintptr_t)e.out & 15) == 0);
    CHECK(e.parts == 1 || e.parts == (dt == DT_F32 ? 3 : 2));
    range(da, ((rows - 1) * ldda + hidden) * dtype_bytes(da_dt));
    range(e.out, e.out_part * (e.parts - 1) + rows * e.ldo * 2);
    if (e.a) range(e.a, e.a_part * (e.parts - 1) + rows * e.lda * 2);
    if (db) {
        range(db, hidden * 8);
        range(part, gated_bwd_parts(rows, hidden) * hidden * 8);
    }
    return launched();
}
hipError_t launch_zero_matrix(int, int64_t, int64_t, void*, int64_t, hipStream_t) { return launched(); }
int product_splits(int, const Product& p) { return 1 + (p.M + p.N) % 2; }   // either, by the sizes
size_t product_workspace_bytes(int, const Product& p) { return (size_t)(p.M + p.N + p.K); }
hipError_t launch_product(int dt, const Product& p, const Epilogue& e, void* ws, hipStream_t) {
    CHECK((const char*)ws + product_workspace_bytes(dt, p) <= ws_to || !ws_from);
    const int64_t ar = p.a_col ? p.K : p.M, ac = p.a_col ? p.M : p.K, br = p.b_col ? p.K : p.N, bc = p.b_col ? p.N : p.K;
    if (p.a_parts) {
        CHECK(((uintptr_t)p.A & 15) == 0 && p.lda % 8 == 0 && p.lda >= ac);
        range(p.A, p.a_part * (p.a_parts - 1) + ar * p.lda * 2);
    }
    if (p.b_parts) {
        CHECK(((uintptr_t)p.B & 15) == 0 && p.ldb % 8 == 0 && p.ldb >= bc);
        range(p.B, p.b_part * (p.b_parts - 1) + br * p.ldb * 2);
    }
    CHECK(p.a_parts * p.b_parts != 4);   // not both in two parts
    const int64_t width = p.gate == GATE_HIDDEN ? 2 * p.N : p.gate == GATE_FORWARD ? p.N / 2 : p.N;
    CHECK(e.ldo >= width);
    if (p.gate != GATE_HIDDEN) range(e.out, ((p.M - 1) * e.ldo + width) * dtype_bytes(e.out_dt));
    if (p.gate == GATE_HIDDEN) {
        CHECK(product_splits(dt, p) > 1 || (dt != DT_F32 && p.N % 64 == 0));
        CHECK(dt == DT_F32 ? e.parts == 3 : e.parts == 1 || e.parts == 2);
        if (e.out) range(e.out, e.out_part * (e.parts - 1) + p.M * e.ldo * 2);
        if (e.a) range(e.a, e.a_part * (e.parts - 1) + p.M * e.lda * 2);
    }
    if (e.beta) CHECK(e.gamma && e.db);
    return launched();
}
hipError_t launch_lay_out(int dt, int n, const LayOut* jobs, hipStream_t) {
    CHECK(n >= 0 && n <= 4);
    for (int i = 0; i < n; ++i) {
        CHECK(jobs[i].ld % 8 == 0 && jobs[i].ld >= jobs[i].cols && jobs[i].lds >= jobs[i].cols);
        range(jobs[i].dst, jobs[i].rows * jobs[i].ld * 2 * (dt == DT_F32 ? 3 : 1));
    }
    return fail_launch && n ? hipErrorUnknown : hipSuccess;
}
hipError_t launch_dropout(int, int64_t, int64_t, const void*, int64_t, Drop d, void*, int64_t, hipStream_t) {
    CHECK(d.threshold <= 65536);
    return launched();
}
hipError_t launch_residual(int, int, const Residual&, hipStream_t) { return launched(); }
int64_t residual_bwd_parts(int, int, int64_t rows, int64_t) { return rows < 5 ? rows : 5; }
int residual_sums(int norms) { return norms & 4 ? 4 : 2; }
hipError_t launch_residual_bwd(int, int, const Residual&, const ResidualBwd&, hipStream_t) { return launched(); }
}  // namespace mfac

int main() {
    char* const P = (char*)(1 << 20);
    float* const F = (float*)P;
    // the backward pass over types, sizes with and without what the products need, and everything that may be wanted
    for (int type = 0; type < 3; ++type)
        for (int gtype : {0, type})
            for (int64_t hidden : {1, 5, 40, 64, 131})
                for (int64_t cout : {0, 7, 48})
                    for (unsigned wanted = 0; wanted < 32; ++wanted) {
                        if (cout == 0 && (wanted & MFAC_GATED_DW2)) continue;
                        const bool beta = wanted & MFAC_GATED_BETA, copy = wanted % 3 == 0;
                        const int64_t rows = 9, cin = 33, width = cout ? cout : hidden;
                        for (int64_t off : {0, 2}) {   // 16-byte aligned rows, or not
                            const char* dy = P + (type ? off : 2 * off);
                            const void* x = copy ? nullptr : P;
                            const size_t need = mfac_gated_bwd_workspace_bytes((mfac_dtype)type, (mfac_dtype)gtype, rows, cin, hidden,
                                                                               cout, dy, width, P, hidden, x, cin, P, cin, wanted);
                            char* ws = (char*)(1ll << 40);
                            ws_from = ws;
                            ws_to = ws + need;
                            auto call = [&](size_t bytes) {
                                return mfac_gated_bwd(
                                    (mfac_dtype)type, (mfac_dtype)gtype, MFAC_ACT_SILU, rows, cin, hidden, cout, dy, width,
                                    cout ? P : nullptr, hidden, x, cin, copy ? (int8_t*)P : nullptr, cin, copy ? (uint8_t*)P : nullptr,
                                    F, beta ? F : nullptr, P, cin, P, P, 2 * hidden, nullptr, nullptr, nullptr, nullptr, 0,
                                    wanted & MFAC_GATED_DX ? P : nullptr, cin, wanted & MFAC_GATED_DW1 ? P : nullptr, cin,
                                    wanted & MFAC_GATED_DB1 ? F : nullptr, wanted & MFAC_GATED_DW2 ? P : nullptr, hidden, ws, bytes,
                                    nullptr);
                            };
                            launches = 0;
                            CHECK(call(need) == MFAC_OK);
                            CHECK((launches == 0) == ((wanted & 15) == 0));
                            if (need) CHECK(call(need - 1) == MFAC_EWORKSPACE);
                            if (wanted & 15) {
                                fail_launch = true;
                                CHECK(call(need) == MFAC_EHIP);
                                fail_launch = false;
                            }
                        }
                    }
    ws_from = ws_to = nullptr;
    // the largest sizes: no overflow on the way
    CHECK(mfac_gated_bwd_workspace_bytes(MFAC_F32, MFAC_F32, 1ll << 30, 1 << 21, 1 << 20, 1 << 21, P, 1ll << 33, P, 1 << 20, P, 1 << 21,
                                         P, 1 << 21, 31) > (size_t)1 << 52);
    for (int norms : {0, 1, 2, 3, 5, 6, 7})
        for (double p : {0.0, 0.3, 1.0, 1e-9}) {
            launches = 0;
            const bool post = norms & 1, pre = norms & 2;
            CHECK(mfac_residual_norm(MFAC_F16, MFAC_F32, norms, 3, 50, P, 50, post ? P : nullptr, nullptr, nullptr, nullptr, 0, P, 50, 1.0, p,
                                     (int64_t*)P, pre ? P : nullptr, nullptr, 1e-5, P, 50, pre ? P : nullptr, 50, nullptr, nullptr, nullptr,
                                     nullptr, nullptr, 0, nullptr, nullptr) == MFAC_OK);
            CHECK(mfac_dropout(MFAC_F16, 3, 50, P, 50, p, (int64_t*)P, P, 50, nullptr) == MFAC_OK);
            CHECK(launches == 2);
            CHECK(mfac_residual_norm_bwd_workspace_bytes(MFAC_F32, norms, 1ll << 30, 1 << 15) > 0);
        }
    if (failures) {
        fprintf(stderr, "%d failures\n", failures);
        return 1;
    }
    printf("host check ok\n");
    return 0;
}
