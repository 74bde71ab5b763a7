// Gated linear recurrence: launch shapes, scratch and the launches of a call.
#include "lbscan_gated.h"
#include "lbscan_internal.h"

namespace lbscan {
namespace {

// ddecay[d] = sigma(decay) / softplus(decay) * sum over batch entries and segments of the rows' sums, in a
// fixed order.  64 channels a block, four threads to a channel.
__global__ __launch_bounds__(256) void gated_decay_kernel(const float* __restrict__ qsum, const float* __restrict__ decay,
                                                          float* __restrict__ ddecay, int dim, int shares)
{
    __shared__ float part[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (d < dim)
        for (int k = wave; k < shares; k += 4) s += qsum[(long)k * dim + d];
    part[wave][lane] = s;
    __syncthreads();
    if (wave || d >= dim) return;
    float slope;
    const float soft = softplus_f32(decay[d], slope);
    // (both go with e^decay where it is small, down to where they underflow)
    const float ratio = decay[d] < -16.0f ? 1.0f : slope / soft;
    ddecay[d] = ((part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane])) * ratio;
}

hipError_t launch_kernels(const GatedParams& p, GatedPass pass, hipStream_t stream)
{
    if (p.dtype == 0) return p.reverse ? launch_gated_f32_rev(p, pass, stream) : launch_gated_f32(p, pass, stream);
    return p.reverse ? launch_gated_bf16_rev(p, pass, stream) : launch_gated_bf16(p, pass, stream);
}

long rows_of_call(const GatedParams& p) { return (long)p.batch * p.dim; }

}  // namespace

void gated_shape(GatedParams& p)
{
    const int v = gated_lane_tokens(p.dtype), L = p.seqlen;
    const long rows = rows_of_call(p);
    p.nseg = 1;
    p.waves = 1;
    if (L < kGatedShort) {
        p.lanes = 1;
        p.ntiles = p.seg_tiles = 1;
        return;
    }
    p.lanes = 8;
    while (p.lanes < 64 && p.lanes * v < L) p.lanes *= 2;
    const int wave_tiles = (L + 64 * v - 1) / (64 * v);
    if (wave_tiles > 2) {
        if (rows < 4096 && wave_tiles >= 9) p.waves = 16;
        else if (rows < 8192) p.waves = 4;
    }
    const int tile = p.lanes * p.waves * v;
    p.ntiles = p.seg_tiles = (L + tile - 1) / tile;
    if (rows < 256 && p.ntiles > 1) {
        int want = (int)((512 + rows - 1) / rows);
        want = want < 64 ? want : 64;                      // a lane folds a segment
        want = want < p.ntiles ? want : p.ntiles;
        p.seg_tiles = (p.ntiles + want - 1) / want;
        p.nseg = (p.ntiles + p.seg_tiles - 1) / p.seg_tiles;
    }
}

size_t gated_saved_floats(const GatedParams& p)
{
    return p.ntiles > 1 ? (size_t)rows_of_call(p) * p.ntiles : 0;
}
size_t gated_fwd_floats(const GatedParams& p)
{
    // the segments' maps, and the leaving state where it takes the place of the entering one
    return p.nseg > 1 ? (size_t)rows_of_call(p) * (p.nseg * 2 + 1) : 0;
}
size_t gated_bwd_floats(const GatedParams& p, bool saved)
{
    // sums of q; of cut rows the maps both ways
    const size_t n = (size_t)rows_of_call(p) * p.nseg;
    return n + (p.nseg > 1 ? 3 * n : 0) + (saved ? 0 : gated_saved_floats(p));
}

hipError_t launch_gated_fwd(GatedParams p, float* workspace, hipStream_t stream)
{
    const size_t n = (size_t)rows_of_call(p) * p.nseg;
    if (p.nseg == 1) return launch_kernels(p, GatedPass::forward, stream);
    p.seg_prod = workspace;
    p.seg_state = workspace + n;
    hipError_t e = launch_kernels(p, GatedPass::summary, stream);
    if (e != hipSuccess) return e;
    // every segment reads h0, also after the last one has written hT
    float* const hT = p.hT;
    const bool in_place = hT && hT == p.h0;
    if (in_place) p.hT = workspace + 2 * n;
    if ((e = launch_kernels(p, GatedPass::forward, stream)) != hipSuccess || !in_place) return e;
    return launch_copy(hT, p.hT, rows_of_call(p), stream);
}

hipError_t launch_gated_bwd(GatedParams p, float* workspace, const float* saved, hipStream_t stream)
{
    const size_t n = (size_t)rows_of_call(p) * p.nseg;
    p.qsum = workspace;
    float* rest = workspace + n;
    hipError_t e;
    if (p.nseg > 1) {
        p.seg_prod = rest;
        p.seg_state = rest + n;
        p.seg_psi = rest + 2 * n;
        rest += 3 * n;
    }
    p.ckpt = const_cast<float*>(saved);
    if (!saved && gated_saved_floats(p)) {
        // states at the tiles' starts, as the forward call leaves them
        GatedParams f = p;
        f.ckpt = p.ckpt = rest;
        f.y = nullptr;
        f.hT = nullptr;
        if (p.nseg > 1 && (e = launch_kernels(f, GatedPass::summary, stream)) != hipSuccess) return e;
        if ((e = launch_kernels(f, GatedPass::forward, stream)) != hipSuccess) return e;
    }
    if (p.nseg > 1 && (e = launch_kernels(p, GatedPass::backward_summary, stream)) != hipSuccess) return e;
    if ((e = launch_kernels(p, GatedPass::backward, stream)) != hipSuccess) return e;
    gated_decay_kernel<<<(p.dim + 63) / 64, 256, 0, stream>>>(p.qsum, p.decay, p.ddecay, p.dim, p.nseg * p.batch);
    return hipGetLastError();
}

}  // namespace lbscan
