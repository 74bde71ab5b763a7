// Layer norm over the last axis of (rows, dim): what its kernels and the entry points share.
//     s = x + residual (x itself without one)      hat = (s - mean) rstd,  rstd = 1 / sqrt(var + eps)
//     y = hat weight + bias
// Backwards, g = dy weight:
//     ds = rstd (g - mean(g) - hat mean(g hat)) + dsum      (dx and dresidual)
//     dweight = sum over rows of dy hat                      dbias = sum over rows of dy
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lbscan {

struct NormParams {
    long rows;
    int dim, dtype;
    float eps;
    const void* x;            // forward: (rows, dim) in the storage type; backward without a residual: the same
    const float* residual;    // forward, nullable
    const float* weight;      // (dim), nullable: 1
    const float* bias;        // (dim), nullable: 0
    void* y;
    float* sum;               // forward with a residual: s; backward: read instead of x
    float* mean;              // (rows), forward: nullable
    float* rstd;
    const void* dy;
    const float* dsum;        // nullable
    void* dx;                 // nullable when dresidual is not
    float* dresidual;         // nullable
    float* part;              // (shares, 2, dim) sums of a block's rows
    float* dweight;           // nullable
    float* dbias;             // nullable
    int with_residual;
    int shares;
};

hipError_t launch_norm_fwd(const NormParams& p, hipStream_t stream);
hipError_t launch_norm_bwd(NormParams p, float* workspace, hipStream_t stream);
size_t norm_bwd_floats(const NormParams& p);

}  // namespace lbscan
