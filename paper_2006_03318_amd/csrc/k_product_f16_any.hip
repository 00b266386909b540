// Products of float16 with operands of any alignment.
#define DD_PRODUCT_KERNEL
#include "dd_product.h"

namespace dd {
template void launch_tiles<f16_t, false>(const Product &, const Plan &, float *, hipStream_t);
}
