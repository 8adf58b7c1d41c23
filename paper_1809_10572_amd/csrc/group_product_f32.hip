// Products with 4-bit group-scaled weights for f32 activations.
#include <hip/hip_runtime.h>

#include "group_product.hpp"

namespace samd {

int launch_group_product_f32(const GroupProduct &p, hipStream_t s) { return launch_product_of<float>(p, s); }

}  // namespace samd
