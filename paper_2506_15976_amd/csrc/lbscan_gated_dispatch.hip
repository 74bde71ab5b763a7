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

// Waves of a row's team, for a row of so many wave tiles (the tokens of 64 lanes).  As few idle lanes as possible
// first: a tile that the row does not fill costs as much as a full one.  Among equals a tile that holds the
// whole row (nothing is carried along: 88 registers instead of 115 in the backward kernel), then the order below.  Fewer
// waves than 8 a CU do not keep the memory busy, and sixteen to a team leave room for one
// team a CU with 2-byte storage (there they are for few rows only).  MI355X, us, forward / backward, by waves a
// team:
//     8 x 768 x 4096 bf16     1: 39.7 / 78.9    4: 40.3 / 75.5    8: 37.1 / 68.7    16: 61.6 / 137.8
//     8 x 768 x 4096 fp32     1: 82.1 / 151.7   4: 78.8 / 141.4   8: 73.5 / 134.5   16: 71.6 / 132.2
//     1 x 768 x 8192 bf16     1: 16.0 / 30.6    4: 11.6 / 22.1    8: 11.9 / 23.0    16: 11.2 / 26.3
//     1 x 256 x 65536 fp32    1: 194.6 / 453.4  4: 59.4 / 130.5   8: 48.6 / 105.0   16: 49.5 / 98.2
//     1 x 384 x 20000 bf16    1: 35.9 / 64.1    4: 17.7 / 31.2    8: 15.5 / 28.9    16: 18.7 / 33.0
//     4 x 1000 x 3001 bf16    1: 21.6 / 35.6    4: 24.7 / 42.6    8: 23.9 / 49.9    16: 43.4 / 100.0
//     16 x 512 x 700 bf16     1: 13.3 / 23.9    2: 12.6 / 24.5    4: 20.2 / 37.7
int team_waves(int wave_tiles, long rows, int dtype)
{
    int best = 0, padded = 0;
    for (const int w : {8, 4, 1, 2, 16}) {
        if (w > 1 && w >= 2 * wave_tiles) continue;                    // half of it would idle
        if (w < 16 && w < wave_tiles && rows * w <= 2048) continue;
        if (w == 16 && best && dtype != 0) continue;
        const int n = (wave_tiles + w - 1) / w * w;
        if (!best || n < padded || (n == padded && n == w)) { best = w; padded = n; }
    }
    return best;
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
    if (wave_tiles > 1) p.waves = team_waves(wave_tiles, rows, p.dtype);
    const int tile = p.lanes * p.waves * v;
    p.ntiles = p.seg_tiles = (L + tile - 1) / tile;
    // A row is cut where there are too few for the CUs and it is long; the maps of the pieces cost another pass over three
    // of the tensors.  MI355X, us, forward / backward, whole and cut: 1 x 64 x 65536 bf16 21.1 / 35.7 and 16.1 / 21.2,
    // 1 x 16 x 65536 fp32 22.4 / 39.8 and 9.6 / 14.2, 1 x 128 x 65536 fp32 29.7 / 56.0 and 40.1 / 60.7, and of three
    // tiles 2 x 24 x 9000 fp32 6.4 / 12.1 and 7.8 / 11.6.
    if (rows <= 96 && p.ntiles > 3) {
        int want = (int)((256 + rows - 1) / rows);
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
