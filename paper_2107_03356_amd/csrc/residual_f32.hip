// What lies between two blocks, for data of this type (a file for each: they take a minute to compile together).
#include "residual_bwd.h"
#include "residual_fwd.h"

namespace mfac {
template hipError_t residual_fwd<float>(int, const Residual&, hipStream_t);
template hipError_t residual_bwd<float>(int, const Residual&, const ResidualBwd&, hipStream_t);
}  // namespace mfac
