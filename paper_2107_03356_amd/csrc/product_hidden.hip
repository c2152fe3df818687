// The large products of the gradient of a gated layer's output, compiled.
#include "product.h"

namespace mfac {
template hipError_t run_product<bf16, HIDDEN>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
template hipError_t run_product<f16, HIDDEN>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
}  // namespace mfac
