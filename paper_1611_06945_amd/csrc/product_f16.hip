// Products of f16 rows: the tiles of linear layers and their gradients.
#include "linear_common.h"

namespace convfwd {

hipError_t launch_product_f16(const ProductArgs& g, const LinearOut& e, ProductLayout layout, ProductForm form, int splits, hipStream_t s)
{
    if (splits > 1) {
        const PartialSums::Args arg = {};
        CONVFWD_PRODUCT_LAYOUTS(launch_product_form, CONV_F16, PartialSums)
    }
    const LinearOut& arg = e;
    CONVFWD_PRODUCT_LAYOUTS(launch_product_form, CONV_F16, LinearEpi<CONV_F16>)
}

}  // namespace convfwd
