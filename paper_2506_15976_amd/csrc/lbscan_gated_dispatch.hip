// Gated linear recurrence: launch shapes, scratch and the launches of a call.
#include "lbscan_gated.h"
#include "lbscan_internal.h"

namespace lbscan {
namespace {

// ddecay[d] = sigma(decay) / softplus(decay) * sum over batch entries and segments of the rows' sums, in a
// fixed order.  16 channels a block, 16 threads to a channel.
__global__ __launch_bounds__(256) void gated_decay_kernel(const float* __restrict__ qsum, const float* __restrict__ decay,
                                                          float* __restrict__ ddecay, unsigned first, unsigned dim, int shares)
{
    __shared__ float part[16][17];
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const unsigned d = (first + blockIdx.x) * 16 + lane;
    float s = 0.0f, slope = 0.0f, soft = 1.0f, own = 0.0f;
    if (d < dim) {
        own = decay[d];
        soft = softplus_f32(own, slope);
#pragma unroll 4
        for (int k = group; k < shares; k += 16) s += qsum[(long)k * dim + d];
    }
    part[group][lane] = s;
    __syncthreads();
    if (group || d >= dim) return;
#pragma unroll
    for (int g = 1; g < 16; ++g) s += part[g][lane];
    // (both go with e^decay where it is small, down to where they underflow)
    ddecay[d] = s * (own < -16.0f ? 1.0f : slope / soft);
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
    static_cast<GatedShape&>(p) = gated_shape_of(rows_of_call(p), p.seqlen, p.dtype);
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
    const unsigned blocks = ((unsigned)p.dim + 15) / 16;
    constexpr unsigned most = (unsigned)most_blocks(256);
    for (unsigned first = 0; e == hipSuccess && first < blocks; first += most) {
        gated_decay_kernel<<<blocks - first < most ? blocks - first : most, 256, 0, stream>>>(p.qsum, p.decay, p.ddecay, first,
                                                                                              (unsigned)p.dim, p.nseg * p.batch);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace lbscan
