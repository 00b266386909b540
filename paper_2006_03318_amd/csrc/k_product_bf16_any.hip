// Products of bfloat16 with operands of any alignment.
#define DD_PRODUCT_KERNEL
#include "dd_product.h"

namespace dd {
template void launch_tiles<bf16_t, false>(const Product &, const Plan &, float *, hipStream_t);
}
