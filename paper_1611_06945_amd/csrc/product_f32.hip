// Products of fp32 rows as sums of three bf16 planes: the tiles of linear layers and their gradients.
#include "linear_common.h"

namespace convfwd {

hipError_t launch_product_f32(const ProductArgs& g, const LinearOut& e, ProductLayout layout, ProductForm form, int splits, hipStream_t s)
{
    if (splits > 1) {
        // (the same sums of bf16 operands whatever they stand for)
        return launch_product_bf16(g, e, layout, form, splits, s);
    }
    const LinearOut& arg = e;
    CONVFWD_PRODUCT_LAYOUTS(launch_product_direct, CONV_BF16, LinearEpi<CONV_F32>)
}

}  // namespace convfwd
