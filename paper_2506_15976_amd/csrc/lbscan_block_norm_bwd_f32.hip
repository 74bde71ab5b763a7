#define LBSCAN_BLOCK_NORM_BACKWARD
#include "lbscan_block_norm.inc"

namespace lbscan {
hipError_t launch_block_norm_bwd_f32(const BlockNormParams& p, hipStream_t stream) { return launch_typed<float>(p, stream); }
}  // namespace lbscan
