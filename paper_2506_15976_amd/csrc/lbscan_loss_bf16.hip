#include "lbscan_loss_tile.inc"

namespace lbscan {
hipError_t launch_loss_tiles_bf16(LossKind kind, const LossTiles& p, int few, int loose, hipStream_t stream)
{
    return launch_typed<bf16_t>(kind, p, few, loose, stream);
}
}  // namespace lbscan
