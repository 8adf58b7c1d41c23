// Products with 4-bit group-scaled weights for bf16 activations.
#include <hip/hip_runtime.h>

#include "group_product.hpp"

namespace samd {

int launch_group_product_bf16(const GroupProduct &p, hipStream_t s) { return launch_product_of<bf16_t>(p, s); }

}  // namespace samd
