// Instances of the attention core's dK/dV kernel for bf16.
#include "core_attn_kernels.hpp"

namespace imattn {

void launch_core_dkv_bf16(bool few, const CoreArgs& a, unsigned grid, hipStream_t st) { core_widths<bf16_t, CORE_DKV>(few, a, grid, st); }

}  // namespace imattn
