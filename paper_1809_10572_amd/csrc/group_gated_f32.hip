// The gated block on 4-bit group-scaled weights for f32 activations.
#include <hip/hip_runtime.h>

#include "group_product.hpp"

namespace samd {

int launch_group_gated_f32(const GroupProduct &p, hipStream_t s) { return launch_product<float, 2>(p, s); }

}  // namespace samd
