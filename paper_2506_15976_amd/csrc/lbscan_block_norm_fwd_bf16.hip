#include "lbscan_block_norm.inc"

namespace lbscan {
hipError_t launch_block_norm_fwd_bf16(const BlockNormParams& p, hipStream_t stream) { return launch_typed<bf16_t>(p, stream); }
}  // namespace lbscan
