// Host-side check of the training operators' C ABI (csrc/train_capi.hip) under
// AddressSanitizer and UndefinedBehaviorSanitizer, without a GPU.
//
// The calls are linked against stubs of the kernel launchers, which record what
// they were given. Every call is made once as it should be (its launcher must
// run), once with a launch that fails (MFAC_EHIP), and with each of its pointers
// and sizes wrong in turn (no launcher may run). Exit status 0 and "host check
// ok" on success.
#include <stdio.h>
#include <string.h>

#include "../../include/mfac.h"
#include "../../paper_2107_03356_amd/csrc/train.h"

namespace {
int failures = 0, launches = 0;
bool fail_launch = false;
hipError_t launched() {
    ++launches;
    return fail_launch ? hipErrorUnknown : hipSuccess;
}
#define CHECK(c)                                                                    \
    do {                                                                            \
        if (!(c)) {                                                                 \
            fprintf(stderr, "host check failed: %s (%s:%d)\n", #c, __FILE__, __LINE__); \
            ++failures;                                                             \
        }                                                                           \
    } while (0)
}  // namespace

namespace mfac {
hipError_t launch_pack8(int, int64_t, int64_t, const void*, int64_t, Packed, hipStream_t) { return launched(); }
hipError_t launch_unpack8(int, int64_t, int64_t, Packed, void*, int64_t, hipStream_t) { return launched(); }
hipError_t launch_layer_norm(int, int, int64_t, int64_t, const void*, int64_t, const void*, const void*, float, void*,
                             int64_t, float*, float*, Packed, hipStream_t) {
    return launched();
}
int64_t norm_bwd_parts(int64_t, int64_t) { return 3; }
hipError_t launch_layer_norm_bwd(int, int, int64_t, int64_t, const void*, int64_t, const void*, int64_t, const float*,
                                 const float*, Packed, const void*, const void*, int64_t, void*, int64_t, void*, void*,
                                 float*, hipStream_t) {
    return launched();
}
int64_t act_bwd_parts(int64_t, int64_t) { return 2; }
hipError_t launch_act_bwd(int, int, int64_t, int64_t, const void*, int64_t, const void*, int64_t, Packed, void*, int64_t,
                          void*, int64_t, float*, float*, hipStream_t) {
    return launched();
}
hipError_t launch_zero_matrix(int, int64_t, int64_t, void*, int64_t, hipStream_t) { return launched(); }
Product last{};
Epilogue last_epilogue{};
size_t product_workspace_bytes(int, const Product& p) { return p.K == 1 ? 0 : 512; }
hipError_t launch_product(int, const Product& p, const Epilogue& e, void*, hipStream_t) {
    last = p;
    last_epilogue = e;
    return launched();
}
}  // namespace mfac

// Makes the call `f` (a lambda of its arguments by reference) as it should be, then with each
// change of `args` in turn.
template <typename Args, typename Call, typename... Change>
void drive(const Args& good, Call call, Change... change) {
    launches = 0;
    CHECK(call(good) == MFAC_OK);
    CHECK(launches == 1);
    fail_launch = true;
    CHECK(call(good) == MFAC_EHIP);
    fail_launch = false;
    launches = 0;
    int index = 0;
    (
        [&](auto f) {
            Args a = good;
            f(a);
            const mfac_status s = call(a);
            if (s != MFAC_EINVAL && s != MFAC_EWORKSPACE) {
                fprintf(stderr, "change %d was taken (%d)\n", index, (int)s);
                ++failures;
            }
            ++index;
        }(change),
        ...);
    CHECK(launches == 0);
}

struct A {
    int type = MFAC_BF16, ptype = MFAC_F32, act = MFAC_ACT_GELU;
    int64_t rows = 8, cols = 64, cin = 64, cout = 32;
    char *x = (char*)4096, *w = (char*)4096, *b = (char*)4096, *y = (char*)4096, *ws = (char*)4096;
    int64_t ldx = 64, ldw = 64, ldy = 64;
    int8_t* q = nullptr;
    int64_t ldq = 64;
    uint8_t* s = nullptr;
    float *mean = (float*)4096, *rstd = (float*)4096, *db = (float*)4096;
    double eps = 1e-5;
    size_t bytes = 1 << 20;
};
#define BAD(change) [](A& a) { change; }
#define T(v) (mfac_dtype)(v)

int main() {
    A p;
    p.q = (int8_t*)4096;
    p.s = (uint8_t*)4096;
    drive(p, [](const A& a) { return mfac_pack8(T(a.type), a.rows, a.cols, a.x, a.ldx, a.q, a.ldq, a.s, nullptr); },
          BAD(a.type = 3), BAD(a.rows = -1), BAD(a.cols = 0), BAD(a.cols = (1 << 30) + 1), BAD(a.x = nullptr),
          BAD(a.x += 1), BAD(a.ldx = 63), BAD(a.q = nullptr), BAD(a.s = nullptr), BAD(a.ldq = 63));
    drive(p, [](const A& a) { return mfac_unpack8(T(a.type), a.rows, a.cols, a.q, a.ldq, a.s, a.y, a.ldy, nullptr); },
          BAD(a.type = 7), BAD(a.y = nullptr), BAD(a.ldy = 0), BAD(a.q = nullptr), BAD(a.s = nullptr));
    A n;
    drive(n,
          [](const A& a) {
              return mfac_layer_norm(T(a.type), T(a.ptype), a.rows, a.cols, a.x, a.ldx, a.w, a.b, a.eps, a.y, a.ldy,
                                     a.mean, a.rstd, a.q, a.ldq, a.s, nullptr);
          },
          BAD(a.ptype = MFAC_F16), BAD(a.eps = -1), BAD(a.eps = 1.0 / 0.0), BAD(a.x = nullptr), BAD(a.y = nullptr),
          BAD(a.w += 1), BAD(a.q = (int8_t*)1), BAD(a.mean = (float*)((char*)a.mean + 1)), BAD(a.cols = 1ll << 40));
    CHECK(mfac_layer_norm_bwd_workspace_bytes(8, 64) == 3 * 2 * 64 * 4);
    drive(n,
          [](const A& a) {
              return mfac_layer_norm_bwd(T(a.type), T(a.ptype), a.rows, a.cols, a.y, a.ldy, a.x, a.ldx, a.mean, a.rstd, a.q,
                                         a.ldq, a.s, a.w, nullptr, 0, a.y, a.ldy, a.b, a.b, a.ws, a.bytes, nullptr);
          },
          BAD(a.rstd = nullptr), BAD(a.mean = nullptr), BAD(a.x = nullptr), BAD(a.bytes = 10), BAD(a.ws += 16),
          BAD(a.q = (int8_t*)4096), BAD(a.ldy = 3), BAD(a.b += 2));
    A l;
    l.ldy = 32;
    drive(l,
          [](const A& a) {
              return mfac_linear(T(a.type), T(a.ptype), (mfac_act)a.act, a.rows, a.cin, a.cout, a.x, a.ldx, a.w, a.ldw, a.b,
                                 nullptr, 0, a.y, a.ldy, nullptr, 0, a.q, a.ldq, a.s, a.ws, a.bytes, nullptr);
          },
          BAD(a.act = 5), BAD(a.act = -1), BAD(a.x = nullptr), BAD(a.w = nullptr), BAD(a.ldw = 1), BAD(a.ldy = 31),
          BAD(a.bytes = 511), BAD(a.ws = nullptr), BAD(a.s = (uint8_t*)1), BAD(a.cin = (1 << 21) + 1), BAD(a.rows = 1ll << 31));
    CHECK(mfac::last.M == 8 && mfac::last.N == 32 && mfac::last.K == 64 && !mfac::last.a_col && !mfac::last.b_col);
    A z;
    drive(z,
          [](const A& a) {
              return mfac_act_bwd(T(a.type), (mfac_act)a.act, a.rows, a.cols, a.y, a.ldy, a.x, a.ldx, a.q, a.ldq, a.s, a.y,
                                  a.ldy, nullptr, 0, a.db, a.ws, a.bytes, nullptr);
          },
          BAD(a.x = nullptr), BAD(a.act = MFAC_ACT_NONE), BAD(a.bytes = 0), BAD(a.y = nullptr), BAD(a.q = (int8_t*)4096));
    drive(l,
          [](const A& a) {
              return mfac_linear_bwd_input(T(a.type), a.rows, a.cin, a.cout, a.y, a.ldy, a.w, a.ldw, nullptr, 0, a.x, a.ldx,
                                           a.ws, a.bytes, nullptr);
          },
          BAD(a.y = nullptr), BAD(a.w = nullptr), BAD(a.x = nullptr), BAD(a.ldx = 2), BAD(a.bytes = 1));
    CHECK(mfac::last.M == 8 && mfac::last.N == 64 && mfac::last.K == 32 && mfac::last.b_col);
    drive(l,
          [](const A& a) {
              return mfac_linear_bwd_weight(T(a.type), T(a.ptype), a.rows, a.cin, a.cout, a.y, a.ldy, a.x, a.ldx, a.q, a.ldq,
                                            a.s, a.mean, a.rstd, a.db, a.w, a.ldw, a.ws, a.bytes, nullptr);
          },
          BAD(a.x = nullptr), BAD(a.q = (int8_t*)4096; a.s = (uint8_t*)4096), BAD(a.mean = nullptr), BAD(a.db = nullptr),
          BAD(a.ptype = MFAC_F16), BAD(a.w = nullptr), BAD(a.ldw = 63), BAD(a.bytes = 0));
    CHECK(mfac::last.M == 32 && mfac::last.N == 64 && mfac::last.K == 8 && mfac::last.a_col && mfac::last.b_col);
    CHECK(mfac::last_epilogue.out_dt == MFAC_F32 && mfac::last_epilogue.gamma && mfac::last_epilogue.beta);
    // no rows: nothing to launch, but gradients of weights are zeroed
    launches = 0;
    CHECK(mfac_pack8(MFAC_F32, 0, 5, nullptr, 0, nullptr, 0, nullptr, nullptr) == MFAC_OK);
    CHECK(mfac_linear(MFAC_F32, MFAC_F32, MFAC_ACT_NONE, 0, 5, 5, nullptr, 0, nullptr, 0, nullptr, nullptr, 0, nullptr, 0,
                      nullptr, 0, nullptr, 0, nullptr, nullptr, 0, nullptr) == MFAC_OK);
    CHECK(launches == 0);
    CHECK(mfac_linear_bwd_weight(MFAC_F32, MFAC_F32, 0, 5, 5, nullptr, 0, nullptr, 0, nullptr, 0, nullptr, nullptr, nullptr,
                                 nullptr, (void*)4096, 5, nullptr, 0, nullptr) == MFAC_OK);
    CHECK(launches == 1);
    if (failures) {
        fprintf(stderr, "%d failures\n", failures);
        return 1;
    }
    printf("host check ok\n");
    return 0;
}
