// Instances of the attention core's dQ kernel for fp32.
#include "core_attn_kernels.hpp"

namespace imattn {

void launch_core_dq_f32(bool few, const CoreArgs& a, unsigned grid, hipStream_t st) { core_widths<float, CORE_DQ>(few, a, grid, st); }

}  // namespace imattn
