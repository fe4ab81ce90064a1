// The norms around a block in f32, rows in registers: forward.
#include "residual_norm_kernel.h"

namespace convfwd {

hipError_t residual_norm_fwd_f32(const ResidualNormArgs& a, const ResidualNormForm& f, hipStream_t s) { return residual_norm_fwd_held<CONV_F32>(a, f, s); }

}  // namespace convfwd
