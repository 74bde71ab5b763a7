// Softmax cross entropy over a vocabulary with the product of rows and table included: what its kernels, its plan and the
// entry points share.  With l_tv = scale x_t . W_v:
//     lse_t = log sum_v exp l_tv        loss_t = lse_t - l_t,target(t)
//     G_tv = (g_t + e_t) exp(l_tv - lse_t) - g_t [v = target(t)],   g, e: gradients of loss and lse
//     dx_t = scale sum_v G_tv W_v       dW_v = scale sum_t G_tv x_t
// In bf16 G is rounded, a factor of products whose other one is bf16.  What is left at the targets, most of the gradient of flat
// logits, rest_t = G_t,target(t) - bf16(G_t,target(t)), is added by itself:
//     dx_t += scale rest_t W_target(t)  dW_v += scale sum of rest_t x_t over the tokens t with target v
// (2-norm of the error of dx and dweight over that of the result, 16384 x 50000 x 768: 2.4e-3 without, 1.7e-3 with, of which
// their own rounding is 1.66e-3).  The other terms' rounding stays.  Of many small ones that is little; a token that is sure of another
// word than its target has large ones, and the error, with a result's own rounding, comes near that of two roundings: 4096 x 8000 x 256,
// logits of deviation 2, 4, 6, 12: dx 1.66e-3, 1.79e-3, 1.90e-3, 1.99e-3.  (G in two parts would be twice the products.)
// Tokens whose target is no row of the table are left out of all of it: the others (the live ones) are packed together first.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "lbscan_loss_plan.h"

namespace lbscan {

struct LossParams {
    long tokens;
    int vocab, dim, dtype, wide_ids;
    float scale;
    const void *x, *weight, *targets;
    float *loss, *lse;                // backward: lse is read
    const float *dloss, *dlse;        // nullable: zeros
    void *dx, *dweight;               // nullable
};

LossPlan loss_plan(const LossParams& p, bool backward);
hipError_t launch_loss_fwd(const LossParams& p, const LossPlan& plan, void* workspace, hipStream_t stream);
hipError_t launch_loss_bwd(const LossParams& p, const LossPlan& plan, void* workspace, hipStream_t stream);

// The products' launches, one translation unit for each storage type (lbscan_loss_tile.inc).
struct LossTiles {
    const LossChoice* choice;
    const void* w;                    // (vocab, ldw), rows of whole steps along dim; loose: of dim, at any element's address
    const void* x;                    // (rows, dimp): the live rows, then zeros to a whole tile
    void* g;                          // (rows, piece)
    const int* targets;               // (rows)
    const float *lse2, *both;         // (rows) lse log2(e), g + e
    const float* down;                // (rows) fp32: g; bf16: the rounded slope at the target
    const int *tokens_of, *slot;      // bf16, dweight: tokens of each row of the table, and its place in the list
    const void* list;                 // (.., dimp) sums of rest_t x_t
    float* own;                       // (rows) x_t . W_target
    float2* part;                     // (chunks, live rows) maximum and sum of a chunk of the vocabulary
    float* acc;                       // (splits, live rows, dimp)
    float* share;                     // (splits, count in whole tiles, dimp)
    void* dweight;
    int vocab, dim, dimp, ldw, piece;
    int first, count;                 // columns of the vocabulary that this launch has
    int last;                         // of the pieces
    int add;                          // dx: added to what is there
    float scale;
};
enum class LossKind { lse, slope, dx, dweight };
hipError_t launch_loss_tiles_f32(LossKind kind, const LossTiles& p, int few, int loose, hipStream_t stream);
hipError_t launch_loss_tiles_bf16(LossKind kind, const LossTiles& p, int few, int loose, hipStream_t stream);

}  // namespace lbscan
