// The scan and its convolution as serving calls them: what their kernels and the entry points share.
//     conv   pre = bias + sum_{k<K-1} weight_k before_k + weight_{K-1} x,  x' = SiLU(pre);  before moves on by one token
//     step   dt = softplus(delta + delta_bias),  h = exp(dt A) h + dt B x',  y = (sum_n C h + Dskip x') SiLU(z)
// Row b of a call has the states at slots[b] of the pools (at b without slots).  A row whose slot is outside the pool, or
// that an earlier row has, is padding: zeros come out and no state is touched.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lbscan {

struct StepParams {
    int batch, dim, dstate, pool;
    int dtype, softplus;
    int width, activation;                // width 0: no convolution
    long x_stride, delta_stride, z_stride, b_stride, c_stride;
    const void *x, *delta, *Bm, *Cm;
    const void* z;                        // nullable
    const float* A;
    const float *Dskip, *delta_bias;      // nullable
    const float* conv_weight;             // (dim, width)
    const float* conv_bias;               // nullable
    void* conv_state;                     // (pool, dim, width - 1), storage type
    const int32_t* slots;                 // nullable
    float* state;                         // (pool, dim, dstate)
    void* y;
};
hipError_t launch_step(const StepParams& p, hipStream_t stream);

struct PromptParams {
    int batch, dim, seqlen, width, pool;
    int dtype, activation;
    long x_stride;                        // elements from one batch entry to the next
    const void* x;                        // (batch, dim, seqlen)
    const float* weight;
    const float* bias;                    // nullable
    void* state;                          // (pool, dim, width - 1); none for width 1
    const int32_t* slots;                 // nullable
    const int32_t* lengths;               // nullable
    void* y;
};
hipError_t launch_prompt(const PromptParams& p, hipStream_t stream);

}  // namespace lbscan
