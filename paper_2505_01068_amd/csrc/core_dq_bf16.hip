// Instances of the attention core's dQ kernel for bf16.
#include "core_attn_kernels.hpp"

namespace imattn {

void launch_core_dq_bf16(bool few, const CoreArgs& a, unsigned grid, hipStream_t st) { core_widths<bf16_t, CORE_DQ>(few, a, grid, st); }

}  // namespace imattn
