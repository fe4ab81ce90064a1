// Products of a first operand in two f16 parts: the gradients of linear layers behind GELU and SiLU.
#include "linear_common.h"

namespace convfwd {

hipError_t launch_product_parts_f16(const ProductArgs& g, const LinearOut& e, ProductLayout layout, ProductForm form, int splits, hipStream_t s)
{
    if (splits > 1) {
        const PartialSums::Args arg = {};
        CONVFWD_PARTS_LAYOUTS(launch_product_form, CONV_F16, PartialSums)
    }
    const LinearOut& arg = e;
    CONVFWD_PARTS_LAYOUTS(launch_product_form, CONV_F16, LinearEpi<CONV_F16>)
}

}  // namespace convfwd
