// The large products of a linear layer and its gradients, compiled.
#include "product.h"

namespace mfac {
template hipError_t run_product<bf16, FORWARD>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
template hipError_t run_product<f16, FORWARD>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
template hipError_t run_product<bf16, INPUT>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
template hipError_t run_product<f16, INPUT>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
template hipError_t run_product<bf16, WEIGHT>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
template hipError_t run_product<f16, WEIGHT>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
template hipError_t run_product<f16, WEIGHT_PARTS>(const Product&, const Plan&, const GemmArgs&, hipStream_t);
}  // namespace mfac
