// Products of f32 activations with 4-bit group-scaled weights.
#include <hip/hip_runtime.h>

#include "group_product.hpp"

namespace samd {

int launch_group_product_f32(const GroupProduct &p, hipStream_t s) { return launch_product<float, 1>(p, s); }

}  // namespace samd
