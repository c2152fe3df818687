// Argument checks of the training operators' C calls (train_capi.hip, gated_capi.hip).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/mfac.h"

#define MFAC_API extern "C" __attribute__((visibility("default")))

namespace mfac {
namespace {

constexpr int64_t MOST = int64_t(1) << 30;
// A layer's widths are at most this: the products' copies address a tile of 256 rows in 32 bits.
constexpr int64_t MOST_WIDTH = int64_t(1) << 21;

bool type_ok(int t) { return t == MFAC_F32 || t == MFAC_BF16 || t == MFAC_F16; }
// Parameters come in fp32 or in the type of the data.
bool param_type_ok(int t, int data) { return t == MFAC_F32 || t == data; }
bool act_ok(int a) { return a >= MFAC_ACT_NONE && a <= MFAC_ACT_SILU; }
bool size_ok(int64_t rows, int64_t cols) { return rows >= 0 && rows <= MOST && cols >= 1 && cols <= MOST; }

bool vector_ok(const void* p, int type) { return !p || (uintptr_t)p % (type == MFAC_F32 ? 4 : 2) == 0; }
// A matrix of rows x cols with ld elements between rows.
bool matrix_ok(const void* p, int type, int64_t ld, int64_t cols) {
    return p && ld >= cols && ld <= (int64_t(1) << 33) && vector_ok(p, type);
}
// q and s both given, or (where it may be absent) neither.
bool packed_ok(const void* q, int64_t ldq, const void* s, int64_t cols, bool absent_ok) {
    if (!q && !s) return absent_ok;
    return q && s && ldq >= cols && ldq <= (int64_t(1) << 33);
}

mfac_status done(hipError_t e) { return e == hipSuccess ? MFAC_OK : MFAC_EHIP; }

// The workspace a call needs: MFAC_OK, or what is wrong with the one given.
mfac_status check_workspace(size_t need, const void* ws, size_t bytes) {
    if (need == 0) return MFAC_OK;
    if (bytes < need) return MFAC_EWORKSPACE;
    return ws && ((uintptr_t)ws & 255) == 0 ? MFAC_OK : MFAC_EINVAL;
}

}  // namespace
}  // namespace mfac
