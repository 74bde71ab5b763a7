// The norms around a block, with its gate and its residual stream, over the last axis of (rows, dim): what the kernels and
// the entry points share.
//     v = x SiLU(gate) (x without one)              vhat = v rv,  rv = 1 / sqrt(mean v^2 + eps)  (1 without norm_branch)
//     s = vhat branch_weight + residual_scale residual
//     y = s rs weight,  rs = 1 / sqrt(mean s^2 + eps)  (y = s without norm_stream)
// Backwards, shat = s rs, g = dy weight:
//     ds = rs (g - shat mean(g shat)) + dsum  (dy + dsum without norm_stream)     dweight = sum over rows of dy shat
//     dresidual = residual_scale ds           h = ds branch_weight               dbranch = sum over rows of ds vhat
//     dv = rv (h - vhat mean(h vhat))  (h without norm_branch)
//     dx = dv SiLU(gate),  dgate = dv x SiLU'(gate)
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lbscan {

struct BlockNormParams {
    long rows;
    int dim, dtype;
    int norm_branch, norm_stream;
    float eps, residual_scale;
    const void* x;
    const void* gate;             // nullable
    const float* residual;        // forward, nullable
    const float* branch_weight;   // (dim), nullable: 1
    const float* weight;          // (dim), nullable: 1; with norm_stream only
    void* y;
    float* sum;                   // with a residual: s; backward: read
    float *rv, *rs;               // (rows), of the norms that there are; forward: nullable
    const void* dy;
    const float* dsum;            // nullable
    void* dx;
    void* dgate;                  // with a gate
    float* dresidual;             // with a residual, nullable
    float* part;                  // (shares, 2, dim) sums of a block's rows
    float* means;                 // (rows) mean(g shat), rows too long for registers
    float *dweight, *dbranch;     // nullable
    int with_residual;
    int shares;
};

hipError_t launch_block_norm_fwd(const BlockNormParams& p, hipStream_t stream);
hipError_t launch_block_norm_bwd(BlockNormParams p, float* workspace, hipStream_t stream);
size_t block_norm_bwd_floats(const BlockNormParams& p);

// One translation unit for each storage type and direction (lbscan_block_norm.inc).
hipError_t launch_block_norm_fwd_f32(const BlockNormParams& p, hipStream_t stream);
hipError_t launch_block_norm_fwd_bf16(const BlockNormParams& p, hipStream_t stream);
hipError_t launch_block_norm_bwd_f32(const BlockNormParams& p, hipStream_t stream);
hipError_t launch_block_norm_bwd_bf16(const BlockNormParams& p, hipStream_t stream);

// The rows' teams: `lanes` lanes of each of `waves` waves, `packs` packs of `pack` elements a lane.  packs 0: rows that
// registers do not hold.
struct BlockNormShape { int pack, lanes, waves, packs; };
inline BlockNormShape block_norm_shape(const BlockNormParams& p, bool backward)
{
    const int full = p.with_residual || p.dtype == 0 ? 4 : 8;      // 16 bytes of the widest tensor
    BlockNormShape s{p.dim < full ? 1 : full, 64, 1, 1};
    const int n = (p.dim + s.pack - 1) / s.pack;
    if (n <= 16) { s.lanes = 16; return s; }
    // at most 16 elements a lane; in the widest teams 24, which the gradients have registers for without gate and residual only
    // (gradients with a residual hold so much that a compute unit has one block of 16 elements a lane, whose reductions nothing
    // covers: 8 elements in twice the waves where that makes teams of four to sixteen.  MI355X, us, gradients, 16 / 8: 8192 x 2048
    // bf16 with everything 94.9 / 74.9, 4096 x 4096 bf16 without a gate 80.9 / 62.2, 2048 x 8192 the norm in front alone 71.6 / 59.8;
    // sixteen waves do not have the registers for a gate)
    const bool narrow = backward && p.with_residual && n > 256 && n <= (p.gate ? 1024 : 2048);
    const int most = narrow ? 2 : 16 / s.pack;
    for (s.waves = 1; s.waves <= (narrow ? 16 : 8); s.waves *= 2) {
        s.packs = (n + 64 * s.waves - 1) / (64 * s.waves);
        if (s.packs <= most) return s;
    }
    s.waves = 8;
    if (s.packs <= most * 3 / 2 && !(backward && (p.gate || p.with_residual))) { s.packs = most * 3 / 2; return s; }
    s.packs = 0;
    return s;
}
// Teams that a block has room for.
inline int block_norm_teams(const BlockNormShape& s) { return s.packs == 0 || s.waves > 4 ? 1 : 4 / s.waves * (64 / s.lanes); }
inline int block_norm_shares(const BlockNormParams& p)
{
    const BlockNormShape s = block_norm_shape(p, true);
    const long teams = block_norm_teams(s), whole = (p.rows + teams - 1) / teams, most = s.waves >= 8 || s.packs == 0 ? 256 : 512;
    return (int)(whole < most ? whole : most);
}

}  // namespace lbscan
