// Gated linear recurrence: what its kernels and their launchers share.
//
// Per (b, d), over the tokens of a row in scan order:
//     r = sigma(gate_a)      i = sigma(gate_x)      la = -rate softplus(decay) r
//     a = exp(la)            beta = sqrt(1 - a^2)
//     h_t = a_t h_{t-1} + beta_t i_t x_t            (starts[t]: h_{t-1} counts as zero)
// Backwards, with s_t the gradient arriving at h_t and psi_t = a_t s_t what it passes on to h_{t-1}
// (nothing where a sequence starts):
//     s_t = dout_t + psi_{t+1}
//     dx = s beta i          dgate_x = s beta i (1 - i) x
//     q = la dL/dla = s (a h_{t-1} la - a^2 (la / beta) i x)
//     dgate_a = q (1 - r)    ddecay = sigma(decay) / softplus(decay) * sum of q
// la / beta has the limit 0 where the gate closes (la -> 0, beta ~ sqrt(-2 la)): every gradient is finite.
#pragma once
#include "lbscan_gated_plan.h"

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lbscan {

struct GatedParams : GatedShape {
    int batch, dim, seqlen;
    int dtype, reverse;
    float rate;
    const void* x;
    const void* gate_a;
    const void* gate_x;
    const float* decay;         // (D)
    const uint8_t* starts;      // (B, L), nullable
    const float* h0;            // (B, D), nullable: zeros
    void* y;                    // nullable: states are not wanted (checkpoint launch)
    float* hT;                  // (B, D), nullable
    float* ckpt;                // (B * D, ntiles), nullable: state entering each tile
    float* seg_prod;            // cut rows: (nseg, B * D): product of a over the segment (-0: a sequence starts in it)
    float* seg_state;           // (nseg, B * D): the state that it reaches from zero
    float* seg_psi;             // (nseg, B * D): the gradient that it passes on to the left from zero
    // backward
    const void* dout;
    const float* dhT;           // (B, D), nullable
    void* dx;
    void* dgate_a;
    void* dgate_x;
    float* dh0;                 // (B, D), nullable
    float* qsum;                // (nseg, B * D): sums of q
    float* ddecay;              // (D)
};

// Fills lanes, waves, ntiles, nseg, seg_tiles from the sizes.
void gated_shape(GatedParams& p);
// Floats of scratch: summaries of cut rows (forward); those, sums of q and, unless the caller saved them,
// checkpoints (backward).
size_t gated_fwd_floats(const GatedParams& p);
size_t gated_bwd_floats(const GatedParams& p, bool saved);
size_t gated_saved_floats(const GatedParams& p);
hipError_t launch_gated_fwd(GatedParams p, float* workspace, hipStream_t stream);
hipError_t launch_gated_bwd(GatedParams p, float* workspace, const float* saved, hipStream_t stream);

// One translation unit per storage type and direction of the scan (lbscan_gated.inc).
enum class GatedPass { forward, summary, backward, backward_summary };
hipError_t launch_gated_f32(const GatedParams& p, GatedPass pass, hipStream_t stream);
hipError_t launch_gated_f32_rev(const GatedParams& p, GatedPass pass, hipStream_t stream);
hipError_t launch_gated_bf16(const GatedParams& p, GatedPass pass, hipStream_t stream);
hipError_t launch_gated_bf16_rev(const GatedParams& p, GatedPass pass, hipStream_t stream);

}  // namespace lbscan
