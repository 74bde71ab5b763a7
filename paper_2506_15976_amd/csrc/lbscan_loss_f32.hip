#include "lbscan_loss_tile.inc"

namespace lbscan {
hipError_t launch_loss_tiles_f32(LossKind kind, const LossTiles& p, int few, hipStream_t stream)
{
    return launch_typed<float>(kind, p, few, stream);
}
}  // namespace lbscan
