// Token embedding: what its kernels and the entry points share.
//     out_i = scale weight[ids_i]        (zeros where ids_i is no row of the table)
//     dweight[v] = scale * sum of dout_i over the tokens i with ids_i = v, in the order of i
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lbscan {

struct EmbedParams {
    long tokens;
    int vocab, dim, dtype;
    int wide_ids;             // 1: int64, 0: int32
    float scale;
    const void* ids;
    const void* weight;
    void* out;
    const void* dout;
    void* dweight;
    // scratch of the gradient: the valid tokens' places sorted by row, their rows, the number of tokens of
    // each row, the number of valid tokens, and the sums of rows that go on in the next piece
    int* place;
    int* row;
    int* count;               // (vocab)
    int* valid;
    int* share_total;         // tokens of (share of the tokens, block of rows), and of each of its rows
    int* share_count;
    int blocks_log2, shares;  // the sort's grid
    int piece;                // sorted tokens that a wave adds
    float* part;              // (pieces, 2, dim)
};

hipError_t launch_embed_fwd(const EmbedParams& p, hipStream_t stream);
hipError_t launch_embed_bwd(EmbedParams p, void* workspace, hipStream_t stream);
size_t embed_bwd_bytes(const EmbedParams& p);

}  // namespace lbscan
