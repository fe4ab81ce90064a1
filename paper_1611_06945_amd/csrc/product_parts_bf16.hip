// Products of a first operand in two bf16 parts: the gradients of linear layers behind GELU and SiLU.
#include "linear_common.h"

namespace convfwd {

hipError_t launch_product_parts_bf16(const ProductArgs& g, const LinearOut& e, ProductLayout layout, ProductForm form, int splits, hipStream_t s)
{
    if (splits > 1) {
        const PartialSums::Args arg = {};
        CONVFWD_PARTS_LAYOUTS(launch_product_form, CONV_BF16, PartialSums)
    }
    const LinearOut& arg = e;
    CONVFWD_PARTS_LAYOUTS(launch_product_form, CONV_BF16, LinearEpi<CONV_BF16>)
}

}  // namespace convfwd
