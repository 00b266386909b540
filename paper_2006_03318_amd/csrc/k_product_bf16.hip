// Products of bfloat16 with aligned operands.
#define DD_PRODUCT_KERNEL
#include "dd_product.h"

namespace dd {
template void launch_tiles<bf16_t, true>(const Product &, const Plan &, float *, hipStream_t);
template void launch_two<bf16_t>(const Product &, const Product &, hipStream_t);
}
