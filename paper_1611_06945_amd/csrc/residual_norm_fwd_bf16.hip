// The norms around a block in bf16, rows in registers: forward.
#include "residual_norm_kernel.h"

namespace convfwd {

hipError_t residual_norm_fwd_bf16(const ResidualNormArgs& a, const ResidualNormForm& f, hipStream_t s) { return residual_norm_fwd_held<CONV_BF16>(a, f, s); }

}  // namespace convfwd
