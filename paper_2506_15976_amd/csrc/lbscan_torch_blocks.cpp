// The operators of state space language models for torch (single steps and prompts, norms around a block, the loss):
// argument checks, outputs and scratch, autograd nodes.  No arithmetic: every value is computed by the kernels behind include/lbscan.h.
#include "lbscan_torch.h"

namespace lbscan_torch {
namespace {

// A (B, n) tensor that may be columns of a wider one; its rows' distance.
int64_t expect_rows(const char* name, const Tensor& t, int64_t B, int64_t n, at::ScalarType type, const Tensor& like)
{
    if (t.dim() != 2 || t.size(0) != B || t.size(1) != n || t.scalar_type() != type)
        throw Failure(LBSCAN_EINVAL, std::string(name) + ": expected " + shape_of({B, n}) + " " + c10::toString(type) + ", got " +
                                         shape_of(t.sizes()) + " " + c10::toString(t.scalar_type()));
    const bool dense = t.is_contiguous();
    if (!t.is_cuda() || t.device() != like.device() || !(dense || ((n <= 1 || t.stride(1) == 1) && (B <= 1 || t.stride(0) >= n))))
        throw Failure(LBSCAN_EINVAL, std::string(name) + " must be a device tensor with contiguous rows, on the device of the others");
    return dense || B <= 1 ? 0 : t.stride(0);
}

// What a call writes to (an output or a state of the caller's) must not have memory of what it reads, or writes besides: other blocks
// may still have to read it.  A tensor that is written is dense; one that is read is, too, or has rows that may be columns of a wider
// tensor.
struct Memory {
    const char* name;
    uintptr_t begin = 0, end = 0;                  // the same where there is nothing
    uintptr_t row = 0, pitch = 0;                  // bytes of a row, and from one to the next; 0: dense
    Memory(const char* n, const Tensor& t) : name(n)
    {
        if (t.numel() == 0) return;
        begin = reinterpret_cast<uintptr_t>(t.data_ptr());
        if (t.is_contiguous()) {
            end = begin + t.nbytes();
        } else {
            row = t.size(1) * t.element_size();
            pitch = t.stride(0) * t.element_size();
            end = begin + (t.size(0) - 1) * pitch + row;
        }
    }
    Memory(const char* n, const Maybe& t) : name(n) { if (t) *this = Memory(n, *t); }
};
void expect_apart(const Memory& written, at::ArrayRef<Memory> others)
{
    if (written.begin == written.end) return;
    for (const Memory& o : others) {
        if (o.begin == o.end || o.begin >= written.end || written.begin >= o.end) continue;
        if (o.pitch && written.begin >= o.begin) {
            // between two rows: behind the one that begins before it, in front of the next
            const uintptr_t from = (written.begin - o.begin) % o.pitch;
            if (from >= o.row && from + (written.end - written.begin) <= o.pitch) continue;
        }
        throw Failure(LBSCAN_EINVAL, std::string(written.name) + " must not be, or share memory with, " + o.name);
    }
}

// A pool of states, and the rows' places in it.
int32_t expect_pool(const char* name, const Tensor& state, at::IntArrayRef rest, at::ScalarType type, const Maybe& slots, int64_t B,
                    const Tensor& like)
{
    const int64_t S = state.dim() ? state.size(0) : -1;
    c10::SmallVector<int64_t, 3> shape{S};
    shape.append(rest.begin(), rest.end());
    expect(name, state, shape, type, like);
    expect("slots", slots, {B}, at::kInt, like);
    if (!slots && S != B)
        throw Failure(LBSCAN_EINVAL, std::string(name) + ": expected " + std::to_string(B) + " rows (one for each row of x, without slots), got " +
                                         std::to_string(S));
    expect_writable(name, state);
    return size32(name, S);
}

// ---- single tokens through the scan ------------------------------------------------------------------------
Tensor step(Tensor x, Tensor delta, Tensor A, Tensor Bm, Tensor Cm, Tensor state, Maybe Dskip, Maybe z, Maybe delta_bias, bool softplus,
            Maybe conv_state, Maybe conv_weight, Maybe conv_bias, bool activation, Maybe slots, Maybe out, py::object stream_object)
{
    expect_axes("x", x, 2);
    expect_axes("A", A, 2);
    const int64_t B = x.size(0), D = x.size(1), N = A.size(1);
    const auto type = x.scalar_type();
    lbscan_step_args a{};
    a.dtype = type_code("x", type);
    a.x_stride = expect_rows("x", x, B, D, type, x);
    a.delta_stride = expect_rows("delta", delta, B, D, type, x);
    if (z) a.z_stride = expect_rows("z", *z, B, D, type, x);
    a.b_stride = expect_rows("Bm", Bm, B, N, type, x);
    a.c_stride = expect_rows("Cm", Cm, B, N, type, x);
    expect("A", A, {D, N}, at::kFloat, x);
    expect("Dskip", Dskip, {D}, at::kFloat, x);
    expect("delta_bias", delta_bias, {D}, at::kFloat, x);
    a.pool = expect_pool("state", state, {D, N}, at::kFloat, slots, B, x);
    if (conv_weight) {
        expect_axes("conv_weight", *conv_weight, 2);
        const int64_t K = conv_weight->size(1);
        expect("conv_weight", *conv_weight, {D, K}, at::kFloat, x);
        expect("conv_bias", conv_bias, {D}, at::kFloat, x);
        if (K < 1 || K > 4) throw Failure(LBSCAN_EUNSUPPORTED, "conv_weight: width " + std::to_string(K) + ", supported are 1 to 4");
        if (!conv_state) throw Failure(LBSCAN_EINVAL, "conv_weight needs a conv_state");
        if (expect_pool("conv_state", *conv_state, {D, K - 1}, type, slots, B, x) != a.pool)
            throw Failure(LBSCAN_EINVAL, "conv_state: expected as many rows as state, " + std::to_string(a.pool));
        a.conv_width = (int32_t)K;
    } else if (conv_state || conv_bias) {
        throw Failure(LBSCAN_EINVAL, "conv_state and conv_bias need a conv_weight");
    }
    c10::DeviceGuard guard(x.device());
    const Stream stream(stream_object, x);
    expect("out", out, {B, D}, type, x);
    expect_writable("out", out);
    const Memory states("state", state), conv_states("conv_state", conv_state);
    const Memory inputs[] = {{"x", x}, {"delta", delta}, {"z", z}, {"Bm", Bm}, {"Cm", Cm}, {"A", A}, {"Dskip", Dskip},
                             {"delta_bias", delta_bias}, {"conv_weight", conv_weight}, {"conv_bias", conv_bias}, {"slots", slots}};
    for (const Memory& written : {Memory("out", out), states, conv_states}) expect_apart(written, inputs);
    expect_apart({"out", out}, {states, conv_states});
    expect_apart(states, {conv_states});
    Tensor y = out ? *out : fresh(stream, {B, D}, x, type);
    a.batch = size32("x", B);
    a.dim = size32("x", D);
    a.dstate = size32("A", N);
    a.delta_softplus = softplus;
    a.conv_activation = activation;
    a.x = x.data_ptr(); a.delta = delta.data_ptr(); a.Bm = Bm.data_ptr(); a.Cm = Cm.data_ptr();
    a.z = address(z);
    a.A = address<float>(A);
    a.Dskip = address<float>(Dskip);
    a.delta_bias = address<float>(delta_bias);
    a.conv_weight = address<float>(conv_weight);
    a.conv_bias = address<float>(conv_bias);
    a.conv_state = address(conv_state);
    a.slots = address<int32_t>(slots);
    a.state = address<float>(state);
    a.y = y.data_ptr();
    check(lbscan_step(&a, stream.raw), "lbscan_step");
    written(out);
    written(state);
    written(conv_state);
    return y;
}

// x (B,D,L), or (B,D) for a single token.
Tensor conv1d_prompt(Tensor x, Maybe state, Tensor weight, Maybe bias, bool activation, Maybe lengths, Maybe slots, Maybe out,
                     bool single, py::object stream_object)
{
    const char* name = single ? "lbscan_conv1d_step" : "lbscan_conv1d_prompt";
    expect_axes("x", x, single ? 2 : 3);
    expect_axes("weight", weight, 2);
    const int64_t B = x.size(0), D = x.size(1), L = single ? 1 : x.size(2), K = weight.size(1);
    const auto type = x.scalar_type();
    lbscan_conv_state_args a{};
    a.dtype = type_code("x", type);
    if (K < 1 || K > 4) throw Failure(LBSCAN_EUNSUPPORTED, "weight: width " + std::to_string(K) + ", supported are 1 to 4");
    if (single) a.x_stride = expect_rows("x", x, B, D, type, x);
    else expect("x", x, x.sizes(), type, x);
    expect("weight", weight, {D, K}, at::kFloat, x);
    expect("bias", bias, {D}, at::kFloat, x);
    expect("lengths", lengths, {B}, at::kInt, x);
    if (!state) throw Failure(LBSCAN_EINVAL, "state is missing");
    a.pool = expect_pool("state", *state, {D, K - 1}, type, slots, B, x);
    c10::DeviceGuard guard(x.device());
    const Stream stream(stream_object, x);
    expect("out", out, x.sizes(), type, x);
    expect_writable("out", out);
    const Memory states("state", state);
    const Memory inputs[] = {{"x", x}, {"weight", weight}, {"bias", bias}, {"lengths", lengths}, {"slots", slots}};
    for (const Memory& written : {Memory("out", out), states}) expect_apart(written, inputs);
    expect_apart({"out", out}, {states});
    Tensor y = out ? *out : fresh(stream, x.sizes(), x, type);
    a.batch = size32("x", B);
    a.dim = size32("x", D);
    a.seqlen = size32("x", L);
    a.width = (int32_t)K;
    a.activation = activation;
    a.x = x.data_ptr();
    a.weight = address<float>(weight);
    a.bias = address<float>(bias);
    a.state = address(state);
    a.slots = address<int32_t>(slots);
    a.lengths = address<int32_t>(lengths);
    a.y = y.data_ptr();
    check(lbscan_conv1d_prompt(&a, stream.raw), name);
    written(out);
    written(state);
    return y;
}

// ---- norms around a block ------------------------------------------------------------------------------------
struct BlockNorm {
    Tensor x;
    Maybe weight, gate, branch_weight, residual;
    double residual_scale;
    bool norm_branch, norm_stream;
    double eps;

    lbscan_block_norm_args args() const
    {
        lbscan_block_norm_args a{};
        if (x.dim() < 1) throw Failure(LBSCAN_EINVAL, "x needs an axis to normalise");
        a.dtype = type_code("x", x.scalar_type());
        const int64_t D = x.size(-1);
        expect("x", x, x.sizes(), x.scalar_type(), x);
        expect("gate", gate, x.sizes(), x.scalar_type(), x);
        expect("residual", residual, x.sizes(), at::kFloat, x);
        expect("weight", weight, {D}, at::kFloat, x);
        expect("branch_weight", branch_weight, {D}, at::kFloat, x);
        if (weight && !norm_stream) throw Failure(LBSCAN_EINVAL, "weight belongs to the norm of the stream");
        a.dim = size32("x", D);
        a.rows = D ? x.numel() / D : 0;
        a.norm_branch = norm_branch;
        a.norm_stream = norm_stream;
        a.eps = (float)eps;
        a.residual_scale = (float)residual_scale;
        a.x = x.data_ptr();
        a.gate = address(gate);
        a.residual = address<float>(residual);
        a.branch_weight = address<float>(branch_weight);
        a.weight = address<float>(weight);
        return a;
    }
};

struct BlockNormResult { Tensor y, sum, rv, rs; };
BlockNormResult block_norm_run(const BlockNorm& n, bool stats, const Maybe& out, const Stream& stream)
{
    lbscan_block_norm_args a = n.args();
    const Tensor& x = n.x;
    c10::DeviceGuard guard(x.device());
    expect("out", out, x.sizes(), x.scalar_type(), x);
    expect_writable("out", out);
    expect_apart({"out", out}, {{"x", x}, {"the gate", n.gate}, {"the residual", n.residual}, {"weight", n.weight},
                                {"branch_weight", n.branch_weight}});
    BlockNormResult r;
    r.y = out ? *out : fresh(stream, x.sizes(), x, x.scalar_type());
    if (n.residual) r.sum = fresh(stream, x.sizes(), x, at::kFloat);
    if (stats) {
        const auto rows = x.sizes().slice(0, x.dim() - 1);
        for (auto [wanted, t] : {std::pair{n.norm_branch, &r.rv}, std::pair{n.norm_stream, &r.rs}}) {
            if (!wanted) continue;
            *t = fresh(stream, rows, x, at::kFloat);
            if (x.size(-1) == 0) {                       // rows of no columns: no kernel runs
                c10::OptionalStreamGuard on;
                if (stream.named) on.reset_stream(*stream.named);
                t->zero_();
            }
        }
    }
    a.y = r.y.data_ptr();
    a.sum = address<float>(r.sum);
    a.branch_rstd = address<float>(r.rv);
    a.stream_rstd = address<float>(r.rs);
    check(lbscan_block_norm_fwd(&a, stream.raw), "lbscan_block_norm_fwd");
    written(out);
    return r;
}

py::object block_norm_fwd(Tensor x, Maybe weight, Maybe gate, Maybe branch_weight, Maybe residual, double residual_scale, bool norm_branch,
                          bool norm_stream, double eps, bool stats, Maybe out, py::object stream)
{
    const BlockNormResult r = block_norm_run({x, weight, gate, branch_weight, residual, residual_scale, norm_branch, norm_stream, eps},
                                             stats, out, Stream(stream, x));
    if (!stats) return residual ? py::object(py::make_tuple(r.y, r.sum)) : py::cast(r.y);
    const py::tuple s = py::make_tuple(maybe(r.rv), maybe(r.rs));
    return residual ? py::make_tuple(r.y, r.sum, s[0], s[1]) : py::make_tuple(r.y, s[0], s[1]);
}

struct BlockNormGradients { Tensor dx, dgate, dresidual, dweight, dbranch; };
// n.residual: the sum that the forward call returned
BlockNormGradients block_norm_gradients(const BlockNorm& n, const Tensor& dout, const Maybe& dsum, const Maybe& rv, const Maybe& rs,
                                        bool with_weight, bool with_branch, const Stream& stream)
{
    lbscan_block_norm_args a = n.args();
    const Tensor& x = n.x;
    c10::DeviceGuard guard(x.device());
    const auto rows = x.sizes().slice(0, x.dim() - 1);
    expect("dout", dout, x.sizes(), x.scalar_type(), x);
    if (dsum && !n.residual) throw Failure(LBSCAN_EINVAL, "dsum belongs to a sum");
    expect("dsum", dsum, x.sizes(), at::kFloat, x);
    if (n.norm_branch != (bool)rv || n.norm_stream != (bool)rs)
        throw Failure(LBSCAN_EINVAL, "branch_rstd and stream_rstd: expected those of the norms that there are");
    expect("branch_rstd", rv, rows, at::kFloat, x);
    expect("stream_rstd", rs, rows, at::kFloat, x);
    a.sum = const_cast<float*>(a.residual);
    a.branch_rstd = address<float>(rv);
    a.stream_rstd = address<float>(rs);
    BlockNormGradients g;
    g.dx = fresh(stream, x.sizes(), x, x.scalar_type());
    if (n.gate) g.dgate = fresh(stream, x.sizes(), x, x.scalar_type());
    if (n.residual) g.dresidual = fresh(stream, x.sizes(), x, at::kFloat);
    if (with_weight) g.dweight = fresh(stream, {x.size(-1)}, x, at::kFloat);
    if (with_branch) g.dbranch = fresh(stream, {x.size(-1)}, x, at::kFloat);
    const size_t need = lbscan_block_norm_workspace_bytes(&a);
    const Tensor ws = scratch(stream, need, x);
    a.workspace = address(ws);
    a.workspace_bytes = need;
    check(lbscan_block_norm_bwd(&a, dout.data_ptr(), address<float>(dsum), g.dx.data_ptr(), address(g.dgate), address<float>(g.dresidual),
                                address<float>(g.dweight), address<float>(g.dbranch), stream.raw),
          "lbscan_block_norm_bwd");
    return g;
}

py::dict block_norm_bwd(Tensor x, Maybe weight, Tensor dout, Maybe gate, Maybe branch_weight, Maybe total, Maybe dsum, Maybe rv, Maybe rs,
                        double residual_scale, bool norm_branch, bool norm_stream, py::object stream)
{
    const BlockNormGradients g =
        block_norm_gradients({x, weight, gate, branch_weight, total, residual_scale, norm_branch, norm_stream, 0.0}, dout, dsum, rv, rs,
                             (bool)weight, (bool)branch_weight, Stream(stream, x));
    py::dict r;
    r["dx"] = g.dx;
    r["dgate"] = maybe(g.dgate);
    r["dresidual"] = maybe(g.dresidual);
    r["dweight"] = maybe(g.dweight);
    r["dbranch_weight"] = maybe(g.dbranch);
    return r;
}

struct BlockNormNode : torch::autograd::Function<BlockNormNode> {
    static variable_list forward(AutogradContext* ctx, Tensor x, Maybe weight, Maybe gate, Maybe branch_weight, Maybe residual,
                                 double residual_scale, bool norm_branch, bool norm_stream, double eps)
    {
        x = x.contiguous();
        if (gate) gate = gate->contiguous();
        if (residual) residual = residual->contiguous();
        if (!x.is_cuda()) throw Failure(LBSCAN_EINVAL, "x must be a device tensor");
        const BlockNormResult r = block_norm_run({x, weight, gate, branch_weight, residual, residual_scale, norm_branch, norm_stream, eps},
                                                 true, {}, Stream(x));
        ctx->save_for_backward({x, tensor(weight), tensor(gate), tensor(branch_weight), r.sum, r.rv, r.rs});
        ctx->saved_data["residual_scale"] = residual_scale;
        ctx->saved_data["norm_branch"] = norm_branch;
        ctx->saved_data["norm_stream"] = norm_stream;
        ctx->set_materialize_grads(false);
        return residual ? variable_list{r.y, r.sum} : variable_list{r.y};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        return backward_pass([&] { return gradients(ctx, grads); });
    }
    static variable_list gradients(AutogradContext* ctx, const variable_list& grads)
    {
        refuse_second_derivatives();
        const auto s = ctx->get_saved_variables();
        Tensor dout = grads[0], dsum = grads.size() > 1 ? grads[1] : Tensor();
        variable_list r(9);
        if (!dout.defined() && !dsum.defined()) return r;
        dout = dout.defined() ? dout.contiguous() : at::zeros_like(s[0]);
        if (dsum.defined()) dsum = dsum.contiguous();
        const BlockNormGradients g = block_norm_gradients(
            {s[0], maybe(s[1]), maybe(s[2]), maybe(s[3]), maybe(s[4]), ctx->saved_data["residual_scale"].toDouble(),
             ctx->saved_data["norm_branch"].toBool(), ctx->saved_data["norm_stream"].toBool(), 0.0},
            dout, maybe(dsum), maybe(s[5]), maybe(s[6]), s[1].defined(), s[3].defined(), Stream(s[0]));
        r[0] = g.dx; r[1] = g.dweight; r[2] = g.dgate; r[3] = g.dbranch; r[4] = g.dresidual;
        return r;
    }
};

py::object block_norm(Tensor x, Maybe weight, Maybe gate, Maybe branch_weight, Maybe residual, double residual_scale, bool norm_branch,
                      bool norm_stream, double eps)
{
    const auto r = BlockNormNode::apply(x, weight, gate, branch_weight, residual, residual_scale, norm_branch, norm_stream, eps);
    return r.size() > 1 ? py::object(py::make_tuple(r[0], r[1])) : py::cast(r[0]);
}

// ---- loss over the vocabulary ----------------------------------------------------------------------------------
lbscan_loss_args loss_args(const Tensor& x, const Tensor& weight, const Tensor& targets, double scale)
{
    lbscan_loss_args a{};
    expect_axes("weight", weight, 2);
    if (x.dim() < 1) throw Failure(LBSCAN_EINVAL, "x needs an axis of rows' elements");
    const auto type = targets.scalar_type();
    if (type != at::kLong && type != at::kInt)
        throw Failure(LBSCAN_EUNSUPPORTED, std::string("targets: expected int32 or int64, got ") + c10::toString(type));
    a.dtype = type_code("x", x.scalar_type());
    expect("x", x, x.sizes(), x.scalar_type(), x);
    expect("weight", weight, {weight.size(0), x.size(-1)}, x.scalar_type(), x);
    expect("targets", targets, x.sizes().slice(0, x.dim() - 1), type, x);
    a.ids_type = type == at::kLong ? LBSCAN_IDS_INT64 : LBSCAN_IDS_INT32;
    a.tokens = targets.numel();
    a.vocab = size32("weight", weight.size(0));
    a.dim = size32("x", x.size(-1));
    a.scale = (float)scale;
    a.x = x.data_ptr(); a.weight = weight.data_ptr(); a.targets = targets.data_ptr();
    return a;
}

std::pair<Tensor, Tensor> loss_run(const Tensor& x, const Tensor& weight, const Tensor& targets, double scale, const Stream& stream)
{
    lbscan_loss_args a = loss_args(x, weight, targets, scale);
    c10::DeviceGuard guard(x.device());
    Tensor loss = fresh(stream, targets.sizes(), x, at::kFloat), lse = fresh(stream, targets.sizes(), x, at::kFloat);
    a.loss = address<float>(loss);
    a.lse = address<float>(lse);
    const size_t need = lbscan_loss_workspace_bytes(&a, LBSCAN_WS_FWD);
    const Tensor ws = scratch(stream, need, x);
    a.workspace = address(ws);
    a.workspace_bytes = need;
    check(lbscan_loss_fwd(&a, stream.raw), "lbscan_loss_fwd");
    return {loss, lse};
}
py::tuple loss_fwd(Tensor x, Tensor weight, Tensor targets, double scale, py::object stream)
{
    auto [loss, lse] = loss_run(x, weight, targets, scale, Stream(stream, x));
    return py::make_tuple(loss, lse);
}

std::pair<Tensor, Tensor> loss_gradients(const Tensor& x, const Tensor& weight, const Tensor& targets, const Tensor& lse, const Maybe& dloss,
                                         const Maybe& dlse, double scale, bool want_dx, bool want_dw, const Stream& stream)
{
    lbscan_loss_args a = loss_args(x, weight, targets, scale);
    c10::DeviceGuard guard(x.device());
    expect("lse", lse, targets.sizes(), at::kFloat, x);
    expect("dloss", dloss, targets.sizes(), at::kFloat, x);
    expect("dlse", dlse, targets.sizes(), at::kFloat, x);
    a.lse = address<float>(lse);
    Tensor dx, dweight;
    if (want_dx) dx = fresh(stream, x.sizes(), x, x.scalar_type());
    if (want_dw) dweight = fresh(stream, weight.sizes(), x, x.scalar_type());
    const size_t need = lbscan_loss_workspace_bytes(&a, LBSCAN_WS_BWD);
    const Tensor ws = scratch(stream, need, x);
    a.workspace = address(ws);
    a.workspace_bytes = need;
    check(lbscan_loss_bwd(&a, address<float>(dloss), address<float>(dlse), address(dx), address(dweight), stream.raw), "lbscan_loss_bwd");
    return {dx, dweight};
}
py::dict loss_bwd(Tensor x, Tensor weight, Tensor targets, Tensor lse, Maybe dloss, Maybe dlse, double scale, py::object stream)
{
    auto [dx, dweight] = loss_gradients(x, weight, targets, lse, dloss, dlse, scale, true, true, Stream(stream, x));
    py::dict r;
    r["dx"] = dx;
    r["dweight"] = dweight;
    return r;
}

struct LossNode : torch::autograd::Function<LossNode> {
    static variable_list forward(AutogradContext* ctx, Tensor x, Tensor weight, Tensor targets, double scale, bool want_dx, bool want_dw)
    {
        x = x.contiguous();
        weight = weight.contiguous();
        targets = targets.contiguous();
        if (!x.is_cuda()) throw Failure(LBSCAN_EINVAL, "x must be a device tensor");
        auto [loss, lse] = loss_run(x, weight, targets, scale, Stream(x));
        ctx->save_for_backward({x, weight, targets, lse});
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["dx"] = want_dx;
        ctx->saved_data["dweight"] = want_dw;
        ctx->set_materialize_grads(false);
        return {loss, lse};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        return backward_pass([&] { return gradients(ctx, grads); });
    }
    static variable_list gradients(AutogradContext* ctx, const variable_list& grads)
    {
        refuse_second_derivatives();
        const auto s = ctx->get_saved_variables();
        variable_list r(6);
        if (!grads[0].defined() && !grads[1].defined()) return r;
        Maybe dloss, dlse;
        if (grads[0].defined()) dloss = grads[0].contiguous();
        if (grads[1].defined()) dlse = grads[1].contiguous();
        auto [dx, dweight] = loss_gradients(s[0], s[1], s[2], s[3], dloss, dlse, ctx->saved_data["scale"].toDouble(),
                                            ctx->saved_data["dx"].toBool(), ctx->saved_data["dweight"].toBool(), Stream(s[0]));
        r[0] = dx;
        r[1] = dweight;
        return r;
    }
};
py::tuple loss(Tensor x, Tensor weight, Tensor targets, double scale)
{
    const auto r = LossNode::apply(x, weight, targets, scale, x.requires_grad(), weight.requires_grad());
    return py::make_tuple(r[0], r[1]);
}

}  // namespace

void define_blocks(py::module_& m)
{
    m.def("loss_fwd", loss_fwd);
    m.def("loss_bwd", loss_bwd);
    m.def("loss", loss);
    m.def("step", step);
    m.def("conv1d_prompt", conv1d_prompt);
    m.def("block_norm_fwd", block_norm_fwd);
    m.def("block_norm_bwd", block_norm_bwd);
    m.def("block_norm", block_norm);
}

}  // namespace lbscan_torch
