// Dropout: y = x where the mask keeps a value, times 65536 / (65536 - T), and 0 elsewhere. The gradient is the same
// of dy, so one kernel serves both passes. The memory's rate bounds it, 16 bits of the mask's words to a value (drop.h): bf16
// 8192 x 8192 takes 42 us, 6.4 TB/s of x and y.
#include "drop.h"
#include "internal.h"
#include "strips.h"
#include "train.h"

namespace mfac {
namespace {

template <typename T>
__global__ __launch_bounds__(256) void k_dropout(Strips s, Drop d, const T* x, int64_t ldx, T* y, int64_t ldy) {
    const DropKey k = drop_key(d);
    for_strips(s, [&](int64_t row, int64_t c) {
        if (row >= s.rows || c >= s.cols) return;
        const f8 v = load8(x + row * ldx, c, s.cols);
        store8(y + row * ldy, c, s.cols, drop8(d, k, (unsigned)row, (unsigned)(c >> 3), v));
    });
}

}  // namespace

hipError_t launch_dropout(int dt, int64_t rows, int64_t cols, const void* x, int64_t ldx, Drop d, void* y, int64_t ldy,
                          hipStream_t st) {
    const Strips s = strips_of(rows, cols);
    auto run = [&](auto* t) {
        using T = std::remove_reference_t<decltype(*t)>;
        k_dropout<T><<<strip_grid(s), 256, 0, st>>>(s, d, (const T*)x, ldx, (T*)y, ldy);
        return hipGetLastError();
    };
    return dt == DT_F32 ? run((float*)nullptr) : dt == DT_BF16 ? run((bf16*)nullptr) : run((f16*)nullptr);
}

}  // namespace mfac
