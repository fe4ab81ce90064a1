// The norms around a block in bf16, rows in registers: backward.
#include "residual_norm_kernel.h"

namespace convfwd {

hipError_t residual_norm_bwd_bf16(const ResidualNormArgs& a, const ResidualNormForm& f, hipStream_t s) { return residual_norm_bwd_held<CONV_BF16>(a, f, s); }

}  // namespace convfwd
