// Products of bf16 activations with 4-bit group-scaled weights.
#include <hip/hip_runtime.h>

#include "group_product.hpp"

namespace samd {

int launch_group_product_bf16(const GroupProduct &p, hipStream_t s) { return launch_product<bf16_t, 1>(p, s); }

}  // namespace samd
