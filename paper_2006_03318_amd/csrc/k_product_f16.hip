// Products of float16 with aligned operands.
#define DD_PRODUCT_KERNEL
#include "dd_product.h"

namespace dd {
template void launch_tiles<f16_t, true>(const Product &, const Plan &, float *, hipStream_t);
template void launch_two<f16_t>(const Product &, const Product &, hipStream_t);
}
