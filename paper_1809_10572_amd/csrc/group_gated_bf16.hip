// The gated block on 4-bit group-scaled weights for bf16 activations.
#include <hip/hip_runtime.h>

#include "group_product.hpp"

namespace samd {

int launch_group_gated_bf16(const GroupProduct &p, hipStream_t s) { return launch_product<bf16_t, 2>(p, s); }

}  // namespace samd
