// C entry points of the operators of state space language models (single steps and prompts, norms around a block, the
// loss over the vocabulary):
// argument checks and the launches of a call.  Everything a kernel's indexing assumes is checked here first.
#include "../../include/lbscan.h"
#include "lbscan_block_norm.h"
#include "lbscan_internal.h"
#include "lbscan_loss.h"
#include "lbscan_step.h"

#include <math.h>

namespace {

using lbscan::hip_fail;

bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// Present, or absent where it may be, and aligned to its element type.
bool good(const void* p, size_t n, bool optional = false) { return p ? aligned_to(p, n) : optional; }
size_t element_bytes(int dtype) { return dtype == LBSCAN_FP32 ? 4 : 2; }
bool known_type(int dtype) { return dtype == LBSCAN_FP32 || dtype == LBSCAN_BF16; }
bool is_flag(int v) { return v == 0 || v == 1; }
bool enough(const void* workspace, size_t have, size_t need)
{
    return need == 0 || (workspace && have >= need && aligned_to(workspace, 4));
}
int done(hipError_t e, const char* where) { return e == hipSuccess ? LBSCAN_OK : hip_fail(e, where); }

// Values of a row of x: whole blocks of a row's end still count in 32 bits.
constexpr int64_t kMostValues = 0x7fffffff - 4095;
constexpr int kMostSlots = 65536;             // rows of a batch whose slots each row looks through

// Rows of the batch and of the pools.
int check_pool(int batch, int pool, const int32_t* slots)
{
    if (pool < 0 || !good(slots, 4, true) || (!slots && pool < batch)) return LBSCAN_EINVAL;
    return slots && batch > kMostSlots ? LBSCAN_EUNSUPPORTED : LBSCAN_OK;
}
// Distance of the rows of a (B, n) tensor, 0: dense.
bool good_stride(int64_t stride, int64_t n) { return stride == 0 || (stride >= n && stride < ((int64_t)1 << 40)); }

int check_block_norm(const lbscan_block_norm_args* a)
{
    if (!a) return LBSCAN_EINVAL;
    if (a->rows < 0 || a->dim < 0) return LBSCAN_EINVAL;
    if (!known_type(a->dtype)) return LBSCAN_EUNSUPPORTED;
    if (!is_flag(a->norm_branch) || !is_flag(a->norm_stream)) return LBSCAN_EINVAL;
    if (!isfinite(a->eps) || a->eps < 0 || isnan(a->residual_scale)) return LBSCAN_EINVAL;
    if (a->dim > (1 << 23) || a->rows > ((int64_t)1 << 31) - 1) return LBSCAN_EUNSUPPORTED;
    if (a->weight && !a->norm_stream) return LBSCAN_EINVAL;
    return LBSCAN_OK;
}
lbscan::BlockNormParams block_norm_params(const lbscan_block_norm_args* a)
{
    lbscan::BlockNormParams p{};
    p.rows = a->rows; p.dim = a->dim; p.dtype = a->dtype;
    p.norm_branch = a->norm_branch; p.norm_stream = a->norm_stream;
    p.eps = a->eps; p.residual_scale = a->residual_scale;
    p.x = a->x; p.gate = a->gate; p.residual = a->residual;
    p.branch_weight = a->branch_weight; p.weight = a->weight;
    p.y = a->y; p.sum = a->sum; p.rv = a->branch_rstd; p.rs = a->stream_rstd;
    p.with_residual = a->residual != nullptr;
    return p;
}

int check_loss(const lbscan_loss_args* a)
{
    if (!a) return LBSCAN_EINVAL;
    if (a->tokens < 0 || a->vocab < 0 || a->dim < 0) return LBSCAN_EINVAL;
    if (!known_type(a->dtype)) return LBSCAN_EUNSUPPORTED;
    if (a->ids_type != LBSCAN_IDS_INT32 && a->ids_type != LBSCAN_IDS_INT64) return LBSCAN_EUNSUPPORTED;
    if (!isfinite(a->scale)) return LBSCAN_EINVAL;
    if (a->tokens > (1 << 24) || a->vocab >= (1 << 30) || a->dim < 1 || a->dim > 65536) return LBSCAN_EUNSUPPORTED;
    return LBSCAN_OK;
}
lbscan::LossParams loss_params(const lbscan_loss_args* a)
{
    lbscan::LossParams p{};
    p.tokens = a->tokens; p.vocab = a->vocab; p.dim = a->dim; p.dtype = a->dtype;
    p.wide_ids = a->ids_type == LBSCAN_IDS_INT64; p.scale = a->scale;
    p.x = a->x; p.weight = a->weight; p.targets = a->targets;
    p.loss = a->loss; p.lse = a->lse;
    return p;
}
bool good_loss_inputs(const lbscan_loss_args* a)
{
    const size_t e = element_bytes(a->dtype);
    return good(a->x, e) && good(a->weight, e, a->vocab == 0) && good(a->targets, a->ids_type == LBSCAN_IDS_INT64 ? 8 : 4) && good(a->lse, 4);
}
size_t loss_bytes(const lbscan::LossParams& p, const lbscan::LossPlan& plan) { return p.tokens && p.vocab ? plan.total : 0; }
bool enough_wide(const void* workspace, size_t have, size_t need)
{
    return need == 0 || (workspace && have >= need && aligned_to(workspace, 16));
}

}  // namespace

extern "C" {

int lbscan_step(const lbscan_step_args* a, void* hip_stream)
{
    if (!a) return LBSCAN_EINVAL;
    if (a->batch < 0 || a->dim < 0 || a->dstate < 0 || a->conv_width < 0) return LBSCAN_EINVAL;
    if (!known_type(a->dtype)) return LBSCAN_EUNSUPPORTED;
    if (!is_flag(a->delta_softplus) || !is_flag(a->conv_activation)) return LBSCAN_EINVAL;
    if (a->conv_width > 4 || (int64_t)a->batch * a->dim > kMostValues) return LBSCAN_EUNSUPPORTED;
    const int rc = check_pool(a->batch, a->pool, a->slots);
    if (rc != LBSCAN_OK) return rc;
    if (a->batch == 0 || a->dim == 0) return LBSCAN_OK;
    if (a->dstate < 1 || a->dstate > LBSCAN_MAX_DSTATE) return LBSCAN_EUNSUPPORTED;
    const size_t e = element_bytes(a->dtype);
    const int K = a->conv_width;
    // (a pool of no rows has no memory: every row is padding then)
    if (!good(a->x, e) || !good(a->delta, e) || !good(a->Bm, e) || !good(a->Cm, e) || !good(a->z, e, true) || !good(a->A, 4) ||
        !good(a->Dskip, 4, true) || !good(a->delta_bias, 4, true) || !good(a->state, 4, a->pool == 0) || !good(a->y, e) ||
        !good(a->conv_weight, 4, K == 0) || !good(a->conv_bias, 4, true) || !good(a->conv_state, e, K <= 1 || a->pool == 0))
        return LBSCAN_EINVAL;
    if (!good_stride(a->x_stride, a->dim) || !good_stride(a->delta_stride, a->dim) || !good_stride(a->z_stride, a->dim) ||
        !good_stride(a->b_stride, a->dstate) || !good_stride(a->c_stride, a->dstate))
        return LBSCAN_EINVAL;
    lbscan::StepParams p{};
    p.batch = a->batch; p.dim = a->dim; p.dstate = a->dstate; p.pool = a->pool;
    p.dtype = a->dtype; p.softplus = a->delta_softplus; p.width = K; p.activation = a->conv_activation;
    p.x_stride = a->x_stride ? a->x_stride : a->dim;
    p.delta_stride = a->delta_stride ? a->delta_stride : a->dim;
    p.z_stride = a->z_stride ? a->z_stride : a->dim;
    p.b_stride = a->b_stride ? a->b_stride : a->dstate;
    p.c_stride = a->c_stride ? a->c_stride : a->dstate;
    p.x = a->x; p.delta = a->delta; p.Bm = a->Bm; p.Cm = a->Cm; p.z = a->z;
    p.A = a->A; p.Dskip = a->Dskip; p.delta_bias = a->delta_bias;
    p.conv_weight = a->conv_weight; p.conv_bias = a->conv_bias; p.conv_state = a->conv_state;
    p.slots = a->slots; p.state = a->state; p.y = a->y;
    return done(lbscan::launch_step(p, static_cast<hipStream_t>(hip_stream)), "lbscan_step");
}

int lbscan_conv1d_prompt(const lbscan_conv_state_args* a, void* hip_stream)
{
    if (!a) return LBSCAN_EINVAL;
    if (a->batch < 0 || a->dim < 0 || a->seqlen < 0) return LBSCAN_EINVAL;
    if (!known_type(a->dtype) || a->width < 1 || a->width > 4) return LBSCAN_EUNSUPPORTED;
    if (!is_flag(a->activation)) return LBSCAN_EINVAL;
    if ((int64_t)a->dim * a->seqlen > kMostValues) return LBSCAN_EUNSUPPORTED;
    const int rc = check_pool(a->batch, a->pool, a->slots);
    if (rc != LBSCAN_OK) return rc;
    if (a->batch == 0 || a->dim == 0 || a->seqlen == 0) return LBSCAN_OK;
    const size_t e = element_bytes(a->dtype);
    if (!good(a->x, e) || !good(a->weight, 4) || !good(a->bias, 4, true) ||
        !good(a->state, e, a->width == 1 || a->pool == 0) || !good(a->lengths, 4, true) || !good(a->y, e) ||
        !good_stride(a->x_stride, (int64_t)a->dim * a->seqlen))
        return LBSCAN_EINVAL;
    lbscan::PromptParams p{};
    p.batch = a->batch; p.dim = a->dim; p.seqlen = a->seqlen; p.width = a->width; p.pool = a->pool;
    p.dtype = a->dtype; p.activation = a->activation;
    p.x_stride = a->x_stride ? a->x_stride : (long)a->dim * a->seqlen;
    p.x = a->x; p.weight = a->weight; p.bias = a->bias; p.state = a->state;
    p.slots = a->slots; p.lengths = a->lengths; p.y = a->y;
    return done(lbscan::launch_prompt(p, static_cast<hipStream_t>(hip_stream)), "lbscan_conv1d_prompt");
}

int lbscan_block_norm_fwd(const lbscan_block_norm_args* args, void* hip_stream)
{
    const int rc = check_block_norm(args);
    if (rc != LBSCAN_OK) return rc;
    if (args->rows == 0 || args->dim == 0) return LBSCAN_OK;
    const size_t e = element_bytes(args->dtype);
    if (!good(args->x, e) || !good(args->gate, e, true) || !good(args->residual, 4, true) || !good(args->branch_weight, 4, true) ||
        !good(args->weight, 4, true) || !good(args->y, e) || !good(args->sum, 4, !args->residual) ||
        !good(args->branch_rstd, 4, true) || !good(args->stream_rstd, 4, true))
        return LBSCAN_EINVAL;
    return done(lbscan::launch_block_norm_fwd(block_norm_params(args), static_cast<hipStream_t>(hip_stream)), "lbscan_block_norm_fwd");
}

int lbscan_block_norm_bwd(const lbscan_block_norm_args* args, const void* dout, const float* dsum, void* dx, void* dgate,
                          float* dresidual, float* dweight, float* dbranch, void* hip_stream)
{
    const int rc = check_block_norm(args);
    if (rc != LBSCAN_OK) return rc;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (!good(dweight, 4, true) || !good(dbranch, 4, true) || (dweight && !args->norm_stream)) return LBSCAN_EINVAL;
    if (args->dim == 0) return LBSCAN_OK;
    if (args->rows == 0) {
        hipError_t e = hipSuccess;
        if (dweight) e = lbscan::launch_zero(dweight, args->dim, stream);
        if (e == hipSuccess && dbranch) e = lbscan::launch_zero(dbranch, args->dim, stream);
        return done(e, "lbscan_block_norm_bwd");
    }
    const size_t e = element_bytes(args->dtype);
    const bool residual = args->residual != nullptr;
    if (!good(args->x, e) || !good(args->gate, e, true) || !good(args->branch_weight, 4, true) || !good(args->weight, 4, true) ||
        !good(args->sum, 4, !(residual && args->norm_stream)) || !good(args->branch_rstd, 4, !args->norm_branch) ||
        !good(args->stream_rstd, 4, !args->norm_stream) || !good(dout, e) || !good(dsum, 4, true) || !good(dx, e) ||
        !good(dgate, e, !args->gate) || !good(dresidual, 4, true))
        return LBSCAN_EINVAL;
    if ((!residual && (dsum || dresidual)) || (!args->gate && dgate)) return LBSCAN_EINVAL;
    lbscan::BlockNormParams p = block_norm_params(args);
    if (!enough(args->workspace, args->workspace_bytes, lbscan::block_norm_bwd_floats(p) * sizeof(float))) return LBSCAN_EWORKSPACE;
    p.dy = dout; p.dsum = dsum; p.dx = dx; p.dgate = dgate; p.dresidual = dresidual; p.dweight = dweight; p.dbranch = dbranch;
    return done(lbscan::launch_block_norm_bwd(p, static_cast<float*>(args->workspace), stream), "lbscan_block_norm_bwd");
}

size_t lbscan_block_norm_workspace_bytes(const lbscan_block_norm_args* args)
{
    if (check_block_norm(args) != LBSCAN_OK || args->rows == 0 || args->dim == 0) return 0;
    return lbscan::block_norm_bwd_floats(block_norm_params(args)) * sizeof(float);
}

int lbscan_loss_fwd(const lbscan_loss_args* args, void* hip_stream)
{
    const int rc = check_loss(args);
    if (rc != LBSCAN_OK) return rc;
    if (args->tokens == 0) return LBSCAN_OK;
    if (!good_loss_inputs(args) || !good(args->loss, 4)) return LBSCAN_EINVAL;
    const lbscan::LossParams p = loss_params(args);
    const lbscan::LossPlan plan = lbscan::loss_plan(p, false);
    if (!enough_wide(args->workspace, args->workspace_bytes, loss_bytes(p, plan))) return LBSCAN_EWORKSPACE;
    return done(lbscan::launch_loss_fwd(p, plan, args->workspace, static_cast<hipStream_t>(hip_stream)), "lbscan_loss_fwd");
}

int lbscan_loss_bwd(const lbscan_loss_args* args, const float* dloss, const float* dlse, void* dx, void* dweight, void* hip_stream)
{
    const int rc = check_loss(args);
    if (rc != LBSCAN_OK) return rc;
    const size_t e = element_bytes(args->dtype);
    if (!good(dweight, e, true) || !good(dx, e, true)) return LBSCAN_EINVAL;
    if (args->tokens && (!good_loss_inputs(args) || !good(dloss, 4, true) || !good(dlse, 4, true))) return LBSCAN_EINVAL;
    lbscan::LossParams p = loss_params(args);
    p.dloss = dloss; p.dlse = dlse; p.dx = dx; p.dweight = dweight;
    if (!dx && !dweight) return LBSCAN_OK;
    const lbscan::LossPlan plan = lbscan::loss_plan(p, true);
    if (!enough_wide(args->workspace, args->workspace_bytes, loss_bytes(p, plan))) return LBSCAN_EWORKSPACE;
    return done(lbscan::launch_loss_bwd(p, plan, args->workspace, static_cast<hipStream_t>(hip_stream)), "lbscan_loss_bwd");
}

size_t lbscan_loss_workspace_bytes(const lbscan_loss_args* args, int which)
{
    if (check_loss(args) != LBSCAN_OK || (which != LBSCAN_WS_FWD && which != LBSCAN_WS_BWD)) return 0;
    lbscan::LossParams p = loss_params(args);
    char wanted;
    p.dx = p.dweight = &wanted;                        // (never written: both gradients are planned for)
    return loss_bytes(p, lbscan::loss_plan(p, which == LBSCAN_WS_BWD));
}

}  // extern "C"
