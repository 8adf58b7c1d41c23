// Products with 4-bit group-scaled weights for f16 activations.
#include <hip/hip_runtime.h>

#include "group_product.hpp"

namespace samd {

int launch_group_product_f16(const GroupProduct &p, hipStream_t s) { return launch_product_of<half_t>(p, s); }

}  // namespace samd
