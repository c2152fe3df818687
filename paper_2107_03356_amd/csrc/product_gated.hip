// The large products of a gated layer, compiled.
#include "product.h"

namespace mfac {
template hipError_t run_product<bf16, GATED>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
template hipError_t run_product<f16, GATED>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
}  // namespace mfac
