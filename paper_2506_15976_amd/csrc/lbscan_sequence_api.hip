// C entry points of the operators around the scan (gated linear recurrence, layer norm, token embedding):
// argument checks and the launches of a call.  Everything a kernel's indexing assumes is checked here first.
#include "../../include/lbscan.h"
#include "lbscan_embed.h"
#include "lbscan_gated.h"
#include "lbscan_internal.h"
#include "lbscan_norm.h"

#include <math.h>

namespace {

using lbscan::hip_fail;

bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// Present, or absent where it may be, and aligned to its element type.
bool good(const void* p, size_t n, bool optional = false) { return p ? aligned_to(p, n) : optional; }
size_t element_bytes(int dtype) { return dtype == LBSCAN_FP32 ? 4 : 2; }
bool known_type(int dtype) { return dtype == LBSCAN_FP32 || dtype == LBSCAN_BF16; }
bool enough(const void* workspace, size_t have, size_t need)
{
    return need == 0 || (workspace && have >= need && aligned_to(workspace, 4));
}

// ---- gated linear recurrence -----------------------------------------------------------------------
int check_gated(const lbscan_gated_args* a)
{
    if (!a) return LBSCAN_EINVAL;
    if (a->batch < 0 || a->dim < 0 || a->seqlen < 0) return LBSCAN_EINVAL;
    if (!known_type(a->dtype)) return LBSCAN_EUNSUPPORTED;
    if (a->reverse != 0 && a->reverse != 1) return LBSCAN_EINVAL;
    if (!isfinite(a->rate) || a->rate < 0) return LBSCAN_EINVAL;
    if (a->seqlen > (1 << 28) || (int64_t)a->batch * a->dim > 0x7fffffff) return LBSCAN_EUNSUPPORTED;
    return LBSCAN_OK;
}
int check_gated_inputs(const lbscan_gated_args* a)
{
    const size_t e = element_bytes(a->dtype);
    return good(a->x, e) && good(a->gate_a, e) && good(a->gate_x, e) && good(a->decay, 4) && good(a->h0, 4, true) ? LBSCAN_OK
                                                                                                              : LBSCAN_EINVAL;
}
lbscan::GatedParams gated_params(const lbscan_gated_args* a)
{
    lbscan::GatedParams p{};
    p.batch = a->batch; p.dim = a->dim; p.seqlen = a->seqlen;
    p.dtype = a->dtype; p.reverse = a->reverse; p.rate = a->rate;
    p.x = a->x; p.gate_a = a->gate_a; p.gate_x = a->gate_x; p.decay = a->decay; p.starts = a->starts;
    p.h0 = a->h0; p.y = a->y; p.hT = a->hT;
    lbscan::gated_shape(p);
    return p;
}
bool gated_empty(const lbscan_gated_args* a) { return a->batch == 0 || a->dim == 0 || a->seqlen == 0; }

// ---- layer norm ------------------------------------------------------------------------------------
int check_norm(const lbscan_norm_args* a)
{
    if (!a) return LBSCAN_EINVAL;
    if (a->rows < 0 || a->dim < 0) return LBSCAN_EINVAL;
    if (!known_type(a->dtype)) return LBSCAN_EUNSUPPORTED;
    if (!isfinite(a->eps) || a->eps < 0) return LBSCAN_EINVAL;
    if (a->dim > (1 << 23) || a->rows > ((int64_t)1 << 31) - 1) return LBSCAN_EUNSUPPORTED;
    return LBSCAN_OK;
}
lbscan::NormParams norm_params(const lbscan_norm_args* a)
{
    lbscan::NormParams p{};
    p.rows = a->rows; p.dim = a->dim; p.dtype = a->dtype; p.eps = a->eps;
    p.x = a->x; p.residual = a->residual; p.weight = a->weight; p.bias = a->bias;
    p.y = a->y; p.sum = a->sum; p.mean = a->mean; p.rstd = a->rstd;
    p.with_residual = a->residual != nullptr;
    return p;
}

// ---- token embedding ---------------------------------------------------------------------------------
int check_embed(const lbscan_embed_args* a)
{
    if (!a) return LBSCAN_EINVAL;
    if (a->tokens < 0 || a->vocab < 0 || a->dim < 0) return LBSCAN_EINVAL;
    if (!known_type(a->dtype)) return LBSCAN_EUNSUPPORTED;
    if (a->ids_type != LBSCAN_IDS_INT32 && a->ids_type != LBSCAN_IDS_INT64) return LBSCAN_EUNSUPPORTED;
    if (isnan(a->scale)) return LBSCAN_EINVAL;
    if (a->tokens > 0x7fff0000L || a->dim > (1 << 23)) return LBSCAN_EUNSUPPORTED;
    return LBSCAN_OK;
}
lbscan::EmbedParams embed_params(const lbscan_embed_args* a)
{
    lbscan::EmbedParams p{};
    p.tokens = a->tokens; p.vocab = a->vocab; p.dim = a->dim; p.dtype = a->dtype;
    p.wide_ids = a->ids_type == LBSCAN_IDS_INT64; p.scale = a->scale;
    p.ids = a->ids; p.weight = a->weight; p.out = a->out;
    return p;
}

int done(hipError_t e, const char* where) { return e == hipSuccess ? LBSCAN_OK : hip_fail(e, where); }

}  // namespace

extern "C" {

int lbscan_gated_fwd(const lbscan_gated_args* args, void* hip_stream)
{
    int rc = check_gated(args);
    if (rc != LBSCAN_OK) return rc;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (gated_empty(args)) {
        // no steps: the state passes through
        const long n = (long)args->batch * args->dim;
        if (!args->hT || n == 0 || args->hT == args->h0) return LBSCAN_OK;
        if (!good(args->hT, 4) || !good(args->h0, 4, true)) return LBSCAN_EINVAL;
        return done(lbscan::launch_copy(args->hT, args->h0, n, stream), "lbscan_gated_fwd");
    }
    if ((rc = check_gated_inputs(args)) != LBSCAN_OK) return rc;
    if (!good(args->y, element_bytes(args->dtype)) || !good(args->hT, 4, true)) return LBSCAN_EINVAL;
    lbscan::GatedParams p = gated_params(args);
    if (!enough(args->workspace, args->workspace_bytes, lbscan::gated_fwd_floats(p) * sizeof(float))) return LBSCAN_EWORKSPACE;
    if (args->saved_state) {
        const size_t need = lbscan::gated_saved_floats(p) * sizeof(float);
        if (!enough(args->saved_state, args->saved_state_bytes, need)) return LBSCAN_EWORKSPACE;
        if (need) p.ckpt = static_cast<float*>(args->saved_state);
    }
    return done(lbscan::launch_gated_fwd(p, static_cast<float*>(args->workspace), stream), "lbscan_gated_fwd");
}

int lbscan_gated_bwd(const lbscan_gated_args* args, const void* dout, const float* dhT, void* dx, void* dgate_a,
                     void* dgate_x, float* ddecay, float* dh0, void* hip_stream)
{
    int rc = check_gated(args);
    if (rc != LBSCAN_OK) return rc;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (gated_empty(args)) {
        hipError_t e = hipSuccess;
        const long n = (long)args->batch * args->dim;
        if (args->dim && !good(ddecay, 4)) return LBSCAN_EINVAL;
        if (!good(dh0, 4, true) || !good(dhT, 4, true)) return LBSCAN_EINVAL;
        if (args->dim) e = lbscan::launch_zero(ddecay, args->dim, stream);
        if (e == hipSuccess && dh0 && n && dh0 != dhT) e = lbscan::launch_copy(dh0, dhT, n, stream);
        return done(e, "lbscan_gated_bwd");
    }
    if ((rc = check_gated_inputs(args)) != LBSCAN_OK) return rc;
    const size_t e = element_bytes(args->dtype);
    if (!good(dout, e) || !good(dx, e) || !good(dgate_a, e) || !good(dgate_x, e) || !good(ddecay, 4) || !good(dhT, 4, true) ||
        !good(dh0, 4, true))
        return LBSCAN_EINVAL;
    lbscan::GatedParams p = gated_params(args);
    const size_t saved = args->saved_state ? lbscan::gated_saved_floats(p) * sizeof(float) : 0;
    if (saved && !enough(args->saved_state, args->saved_state_bytes, saved)) return LBSCAN_EWORKSPACE;
    if (!enough(args->workspace, args->workspace_bytes, lbscan::gated_bwd_floats(p, saved != 0) * sizeof(float)))
        return LBSCAN_EWORKSPACE;
    p.dout = dout; p.dhT = dhT; p.dx = dx; p.dgate_a = dgate_a; p.dgate_x = dgate_x; p.ddecay = ddecay; p.dh0 = dh0;
    return done(lbscan::launch_gated_bwd(p, static_cast<float*>(args->workspace),
                                         saved ? static_cast<const float*>(args->saved_state) : nullptr, stream),
                "lbscan_gated_bwd");
}

size_t lbscan_gated_workspace_bytes(const lbscan_gated_args* args, int which)
{
    if (check_gated(args) != LBSCAN_OK || gated_empty(args)) return 0;
    const lbscan::GatedParams p = gated_params(args);
    switch (which) {
        case LBSCAN_WS_FWD: return lbscan::gated_fwd_floats(p) * sizeof(float);
        case LBSCAN_WS_BWD: return lbscan::gated_bwd_floats(p, args->saved_state != nullptr) * sizeof(float);
        case LBSCAN_WS_SAVED: return lbscan::gated_saved_floats(p) * sizeof(float);
        default: return 0;
    }
}

int lbscan_norm_fwd(const lbscan_norm_args* args, void* hip_stream)
{
    int rc = check_norm(args);
    if (rc != LBSCAN_OK) return rc;
    if (args->rows == 0 || args->dim == 0) return LBSCAN_OK;
    const size_t e = element_bytes(args->dtype);
    if (!good(args->x, e) || !good(args->y, e) || !good(args->residual, 4, true) || !good(args->weight, 4, true) ||
        !good(args->bias, 4, true) || !good(args->sum, 4, !args->residual) || !good(args->mean, 4, true) ||
        !good(args->rstd, 4, true) || !args->mean != !args->rstd)
        return LBSCAN_EINVAL;
    return done(lbscan::launch_norm_fwd(norm_params(args), static_cast<hipStream_t>(hip_stream)), "lbscan_norm_fwd");
}

int lbscan_norm_bwd(const lbscan_norm_args* args, const void* dout, const float* dsum, void* dx, float* dresidual,
                    float* dweight, float* dbias, void* hip_stream)
{
    int rc = check_norm(args);
    if (rc != LBSCAN_OK) return rc;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (!good(dweight, 4, true) || !good(dbias, 4, true)) return LBSCAN_EINVAL;
    if (args->dim == 0) return LBSCAN_OK;
    if (args->rows == 0) {
        hipError_t e = hipSuccess;
        if (dweight) e = lbscan::launch_zero(dweight, args->dim, stream);
        if (e == hipSuccess && dbias) e = lbscan::launch_zero(dbias, args->dim, stream);
        return done(e, "lbscan_norm_bwd");
    }
    const size_t e = element_bytes(args->dtype);
    const bool residual = args->residual != nullptr;
    if (!(residual ? good(args->sum, 4) : good(args->x, e)) || !good(args->mean, 4) || !good(args->rstd, 4) ||
        !good(args->weight, 4, true) || !good(dout, e) || !good(dsum, 4, true) || !good(dx, e, residual) ||
        !good(dresidual, 4, true))
        return LBSCAN_EINVAL;
    if (!residual && (dsum || dresidual)) return LBSCAN_EINVAL;
    lbscan::NormParams p = norm_params(args);
    if (!enough(args->workspace, args->workspace_bytes, lbscan::norm_bwd_floats(p) * sizeof(float))) return LBSCAN_EWORKSPACE;
    p.dy = dout; p.dsum = dsum; p.dx = dx; p.dresidual = dresidual; p.dweight = dweight; p.dbias = dbias;
    return done(lbscan::launch_norm_bwd(p, static_cast<float*>(args->workspace), stream), "lbscan_norm_bwd");
}

size_t lbscan_norm_workspace_bytes(const lbscan_norm_args* args)
{
    if (check_norm(args) != LBSCAN_OK || args->rows == 0 || args->dim == 0) return 0;
    return lbscan::norm_bwd_floats(norm_params(args)) * sizeof(float);
}

int lbscan_embed_fwd(const lbscan_embed_args* args, void* hip_stream)
{
    int rc = check_embed(args);
    if (rc != LBSCAN_OK) return rc;
    if (args->tokens == 0 || args->dim == 0) return LBSCAN_OK;
    const size_t e = element_bytes(args->dtype);
    if (args->vocab < 1 || !good(args->ids, args->ids_type == LBSCAN_IDS_INT64 ? 8 : 4) || !good(args->weight, e) ||
        !good(args->out, e))
        return LBSCAN_EINVAL;
    return done(lbscan::launch_embed_fwd(embed_params(args), static_cast<hipStream_t>(hip_stream)), "lbscan_embed_fwd");
}

int lbscan_embed_bwd(const lbscan_embed_args* args, const void* dout, void* dweight, void* hip_stream)
{
    int rc = check_embed(args);
    if (rc != LBSCAN_OK) return rc;
    if (args->vocab == 0 || args->dim == 0) return args->tokens && args->dim ? LBSCAN_EINVAL : LBSCAN_OK;
    const size_t e = element_bytes(args->dtype);
    if (!good(dweight, e)) return LBSCAN_EINVAL;
    if (args->tokens && (!good(args->ids, args->ids_type == LBSCAN_IDS_INT64 ? 8 : 4) || !good(dout, e))) return LBSCAN_EINVAL;
    lbscan::EmbedParams p = embed_params(args);
    if (!enough(args->workspace, args->workspace_bytes, lbscan::embed_bwd_bytes(p))) return LBSCAN_EWORKSPACE;
    p.dout = dout; p.dweight = dweight;
    return done(lbscan::launch_embed_bwd(p, args->workspace, static_cast<hipStream_t>(hip_stream)), "lbscan_embed_bwd");
}

size_t lbscan_embed_workspace_bytes(const lbscan_embed_args* args)
{
    if (check_embed(args) != LBSCAN_OK || args->vocab == 0 || args->dim == 0) return 0;
    return lbscan::embed_bwd_bytes(embed_params(args));
}

}  // extern "C"
