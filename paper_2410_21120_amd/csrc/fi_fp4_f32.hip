// Attention over a paged cache of 4-bit values for fp32 queries.
#include <hip/hip_runtime.h>

#include "fi_fp4_device.h"

namespace fi {

int launch_fp4_tree_f32(const fi_fp4_tree_attention_args& a, void* stream) { return launch_fp4_type<float>(a, static_cast<hipStream_t>(stream)); }

}  // namespace fi
