// Launches of the norms around a block: the kernel for the storage type, the blocks' shares of the weights' gradients.
#include "lbscan_block_norm.h"
#include "lbscan_norm.h"

namespace lbscan {

size_t block_norm_bwd_floats(const BlockNormParams& p)
{
    if (p.rows <= 0) return 0;
    return (size_t)block_norm_shares(p) * 2 * p.dim + (block_norm_shape(p, true).packs == 0 ? p.rows : 0);
}

hipError_t launch_block_norm_fwd(const BlockNormParams& p, hipStream_t stream)
{
    return p.dtype == 0 ? launch_block_norm_fwd_f32(p, stream) : launch_block_norm_fwd_bf16(p, stream);
}

hipError_t launch_block_norm_bwd(BlockNormParams p, float* workspace, hipStream_t stream)
{
    p.shares = block_norm_shares(p);
    p.part = workspace;
    p.means = workspace + (size_t)p.shares * 2 * p.dim;
    const hipError_t e = p.dtype == 0 ? launch_block_norm_bwd_f32(p, stream) : launch_block_norm_bwd_bf16(p, stream);
    if (e != hipSuccess || (!p.dweight && !p.dbranch)) return e;
    return launch_norm_reduce(workspace, p.dweight, p.dbranch, p.dim, p.shares, stream);
}

}  // namespace lbscan
