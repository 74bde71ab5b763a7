// The operators around the scan for torch: argument checks, outputs and scratch from torch's allocator, the
// current stream, and autograd nodes.  No arithmetic: every value is computed by the kernels behind
// include/lbscan.h.
//
// Why not Python, as for the scan itself: these calls are short.  A norm of 64 x 384 and its gradients took 131 us of
// host time as a Python autograd function (the backward thread starts Python with cold caches), and the kernels
// take 10.
#include "../../include/lbscan.h"

#include <c10/core/DeviceGuard.h>
#include <c10/core/StreamGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/extension.h>

#include <optional>
#include <string>
#include <vector>

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;
using Maybe = std::optional<Tensor>;

// ---- errors ------------------------------------------------------------------------------------------
struct Failure : std::runtime_error {          // becomes binding.LbscanError
    int code;
    Failure(int c, const std::string& what) : std::runtime_error(what), code(c) {}
};

void check(int rc, const char* name)
{
    if (rc == LBSCAN_OK) return;
    std::string what = std::string(name) + " failed (" + std::to_string(rc) + "): " + lbscan_strerror(rc);
    if (rc == LBSCAN_EHIP) what += std::string(": ") + lbscan_last_error();
    throw Failure(rc, what);
}

std::string shape_of(at::IntArrayRef s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + ")";
}

int type_code(const char* name, at::ScalarType t)
{
    if (t == at::kFloat) return LBSCAN_FP32;
    if (t == at::kBFloat16) return LBSCAN_BF16;
    throw Failure(LBSCAN_EUNSUPPORTED, std::string(name) + ": unsupported tensor dtype " + c10::toString(t));
}

// Shape, type, layout and device of one tensor; `like` is the tensor whose device the call runs on.
void expect(const char* name, const Tensor& t, at::IntArrayRef shape, at::ScalarType type, const Tensor& like)
{
    if (t.sizes() != shape || t.scalar_type() != type)
        throw Failure(LBSCAN_EINVAL, std::string(name) + ": expected " + shape_of(shape) + " " + c10::toString(type) + ", got " +
                                         shape_of(t.sizes()) + " " + c10::toString(t.scalar_type()));
    if (!t.is_cuda() || !t.is_contiguous() || t.device() != like.device())
        throw Failure(LBSCAN_EINVAL, std::string(name) + " must be a contiguous device tensor, on the device of the others");
}
void expect(const char* name, const Maybe& t, at::IntArrayRef shape, at::ScalarType type, const Tensor& like)
{
    if (t) expect(name, *t, shape, type, like);
}
void expect_axes(const char* name, const Tensor& t, int64_t n)
{
    if (t.dim() != n) throw Failure(LBSCAN_EINVAL, std::string(name) + ": expected " + std::to_string(n) + " axes, got " + shape_of(t.sizes()));
}
int32_t size32(const char* name, int64_t n)
{
    if (n > INT32_MAX) throw Failure(LBSCAN_EINVAL, std::string(name) + ": size " + std::to_string(n) + " does not fit 32 bits");
    return (int32_t)n;
}

template <typename P = void> P* address(const Maybe& t) { return t ? static_cast<P*>(t->data_ptr()) : nullptr; }
template <typename P = void> P* address(const Tensor& t) { return t.defined() ? static_cast<P*>(t.data_ptr()) : nullptr; }
Maybe maybe(const Tensor& t) { return t.defined() ? Maybe(t) : Maybe(); }
Tensor tensor(const Maybe& t) { return t ? *t : Tensor(); }

// ---- streams -----------------------------------------------------------------------------------------
// The stream of a call: the current one of the tensors' device, or a torch.cuda.Stream that the caller names.  Memory
// that the call takes is the named stream's: a block of the current stream's may have been freed with kernels that
// use it still queued there, and the call does not wait for them.  Outputs are tied to the current stream, where the caller
// goes on with them.
struct Stream {
    void* raw;
    std::optional<c10::Stream> named, current;         // where they are different streams
    Stream(const py::object& s, const Tensor& like)
    {
        raw = like.is_cuda() ? c10::hip::getCurrentHIPStream(like.device().index()).stream() : nullptr;
        if (s.is_none() || !like.is_cuda()) return;
        const auto device = s.attr("device_index").cast<c10::DeviceIndex>();
        if (device != like.device().index())
            throw Failure(LBSCAN_EINVAL, "stream: of device " + std::to_string(device) + ", the tensors are on device " +
                                             std::to_string(like.device().index()));
        raw = reinterpret_cast<void*>(s.attr("cuda_stream").cast<uintptr_t>());
        const auto other = c10::Stream::unpack3(s.attr("stream_id").cast<int64_t>(), device, like.device().type());
        const auto here = c10::impl::VirtualGuardImpl(like.device().type()).getStream(like.device());
        if (other != here) {
            named = other;
            current = here;
        }
    }
    explicit Stream(const Tensor& like) : raw(c10::hip::getCurrentHIPStream(like.device().index()).stream()) {}
};

// An output, or what goes on to another call.
Tensor fresh(const Stream& stream, at::IntArrayRef shape, const Tensor& like, at::ScalarType type)
{
    if (!stream.named) return at::empty(shape, like.options().dtype(type));
    const c10::StreamGuard guard(*stream.named);
    Tensor t = at::empty(shape, like.options().dtype(type));
    if (t.numel()) t.record_stream(*stream.current);
    return t;
}
// Memory that goes back with the call.
Tensor scratch(const Stream& stream, size_t bytes, const Tensor& like)
{
    if (!bytes) return Tensor();
    c10::OptionalStreamGuard guard;
    if (stream.named) guard.reset_stream(*stream.named);
    return at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
}

// ---- tensors that a call overwrites --------------------------------------------------------------------
// The caller's own (a state, `out`): autograd has to know, by the tensor's version, as a backward pass may still need
// what was there; and there is no gradient of the old values.
void expect_writable(const char* name, const Maybe& t)
{
    if (t && t->requires_grad() && at::GradMode::is_enabled())
        throw Failure(LBSCAN_EINVAL, std::string(name) + " requires grad and cannot be overwritten");
}
void written(const Maybe& t)
{
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

// The Python error of a failure is set (the GIL is held).
void set_python_error(const Failure& e)
{
    const py::object type = py::module_::import("paper_2506_15976_amd.binding").attr("LbscanError");
    PyErr_SetObject(type.ptr(), type(e.code, e.what()).ptr());
}

// A node's backward pass.  Its errors cross torch's threads, which hand Python errors on as they are and make a RuntimeError
// of every other exception.
template <typename F>
variable_list backward_pass(const F& pass)
{
    try {
        return pass();
    } catch (const Failure& e) {
        const py::gil_scoped_acquire gil;
        set_python_error(e);
        python_error error;
        error.persist();
        throw error;
    }
}

// Gradients have no gradients of their own.  A backward pass that is itself recorded would leave them out of what
// is differentiated next without a word, so it is refused.
void refuse_second_derivatives()
{
    if (at::GradMode::is_enabled())
        throw Failure(LBSCAN_EUNSUPPORTED, "lbscan operators can be differentiated once: backward with create_graph is not supported");
}

// ---- gated linear recurrence ---------------------------------------------------------------------------
struct Gated {
    Tensor x, gate_a, gate_x, decay;
    Maybe starts, h0;
    double rate;
    bool reverse;

    // x, gate_a, gate_x (B,D,L), or (B,D) for a single token
    lbscan_gated_args args() const
    {
        const bool step = x.dim() == 2;
        if (!step) expect_axes("x", x, 3);
        const auto type = x.scalar_type();
        lbscan_gated_args a{};
        a.dtype = type_code("x", type);
        const int64_t B = x.size(0), D = x.size(1);
        expect("x", x, x.sizes(), type, x);
        expect("gate_a", gate_a, x.sizes(), type, x);
        expect("gate_x", gate_x, x.sizes(), type, x);
        expect("decay", decay, {D}, at::kFloat, x);
        if (starts) {
            const auto marks = starts->scalar_type();
            if (marks != at::kBool && marks != at::kByte)
                throw Failure(LBSCAN_EUNSUPPORTED, std::string("starts: expected bool or uint8, got ") + c10::toString(marks));
            if (step) expect("starts", *starts, {B}, marks, x);
            else expect("starts", *starts, {B, x.size(2)}, marks, x);
        }
        expect(step ? "state" : "h0", h0, {B, D}, at::kFloat, x);
        a.batch = size32("x", B);
        a.dim = size32("x", D);
        a.seqlen = step ? 1 : size32("x", x.size(2));
        a.reverse = reverse;
        a.rate = (float)rate;
        a.x = x.data_ptr(); a.gate_a = gate_a.data_ptr(); a.gate_x = gate_x.data_ptr();
        a.decay = address<float>(decay);
        a.starts = address<uint8_t>(starts);
        a.h0 = address<float>(h0);
        return a;
    }
};

void keep(lbscan_gated_args& a, const Maybe& saved, const Tensor& like)
{
    if (!saved) return;
    expect("saved_state", *saved, saved->sizes(), at::kFloat, like);
    a.saved_state = saved->data_ptr();
    a.saved_state_bytes = saved->numel() * 4;
}

Maybe gated_saved(const Tensor& x, bool reverse, const Stream& stream)
{
    expect_axes("x", x, 3);
    lbscan_gated_args a{};
    a.batch = size32("x", x.size(0)); a.dim = size32("x", x.size(1)); a.seqlen = size32("x", x.size(2));
    a.dtype = type_code("x", x.scalar_type());
    a.reverse = reverse;
    const size_t need = lbscan_gated_workspace_bytes(&a, LBSCAN_WS_SAVED);
    if (!need) return {};
    return fresh(stream, {(int64_t)(need / 4)}, x, at::kFloat);
}
Maybe gated_saved_state(Tensor x, bool reverse, py::object stream) { return gated_saved(x, reverse, Stream(stream, x)); }

std::pair<Tensor, Tensor> gated_run(const Gated& g, const Maybe& out, const Maybe& saved, bool return_state, const Stream& stream)
{
    lbscan_gated_args a = g.args();
    c10::DeviceGuard guard(g.x.device());
    expect("out", out, g.x.sizes(), g.x.scalar_type(), g.x);
    expect_writable("out", out);
    Tensor y = out ? *out : fresh(stream, g.x.sizes(), g.x, g.x.scalar_type()), hT;
    if (return_state) hT = fresh(stream, {g.x.size(0), g.x.size(1)}, g.x, at::kFloat);
    a.y = y.data_ptr();
    a.hT = address<float>(hT);
    keep(a, saved, g.x);
    const size_t need = lbscan_gated_workspace_bytes(&a, LBSCAN_WS_FWD);
    const Tensor ws = scratch(stream, need, g.x);
    a.workspace = address(ws);
    a.workspace_bytes = need;
    check(lbscan_gated_fwd(&a, stream.raw), "lbscan_gated_fwd");
    written(out);
    written(saved);
    return {y, hT};
}

py::object gated_fwd(Tensor x, Tensor gate_a, Tensor gate_x, Tensor decay, Maybe starts, Maybe h0, double rate, bool reverse,
                     bool return_state, Maybe out, Maybe saved, py::object stream)
{
    const Gated g{x, gate_a, gate_x, decay, starts, h0, rate, reverse};
    expect_axes("x", x, 3);
    auto [y, hT] = gated_run(g, out, saved, return_state, Stream(stream, x));
    return return_state ? py::object(py::make_tuple(y, hT)) : py::cast(y);
}

Tensor gated_step(Tensor x, Tensor gate_a, Tensor gate_x, Tensor decay, Tensor state, Maybe starts, double rate, Maybe out,
                  py::object stream_object)
{
    expect_axes("x", x, 2);
    lbscan_gated_args a = Gated{x, gate_a, gate_x, decay, starts, state, rate, false}.args();
    c10::DeviceGuard guard(x.device());
    const Stream stream(stream_object, x);
    expect("out", out, x.sizes(), x.scalar_type(), x);
    expect_writable("out", out);
    expect_writable("state", state);
    Tensor y = out ? *out : fresh(stream, x.sizes(), x, x.scalar_type());
    a.y = y.data_ptr();
    a.hT = address<float>(state);                    // updated in place
    check(lbscan_gated_fwd(&a, stream.raw), "lbscan_gated_step");
    written(out);
    written(state);
    return y;
}

struct GatedGradients { Tensor dx, dgate_a, dgate_x, ddecay, dh0; };
GatedGradients gated_gradients(const Gated& g, const Tensor& dout, const Maybe& dhT, const Maybe& saved, bool with_dh0,
                               const Stream& stream)
{
    const Tensor& x = g.x;
    expect_axes("x", x, 3);
    lbscan_gated_args a = g.args();
    c10::DeviceGuard guard(x.device());
    expect("dout", dout, x.sizes(), x.scalar_type(), x);
    expect("dhT", dhT, {x.size(0), x.size(1)}, at::kFloat, x);
    keep(a, saved, x);
    GatedGradients r{fresh(stream, x.sizes(), x, x.scalar_type()), fresh(stream, x.sizes(), x, x.scalar_type()),
                     fresh(stream, x.sizes(), x, x.scalar_type()), fresh(stream, {x.size(1)}, x, at::kFloat),
                     with_dh0 ? fresh(stream, {x.size(0), x.size(1)}, x, at::kFloat) : Tensor()};
    const size_t need = lbscan_gated_workspace_bytes(&a, LBSCAN_WS_BWD);
    const Tensor ws = scratch(stream, need, x);
    a.workspace = address(ws);
    a.workspace_bytes = need;
    check(lbscan_gated_bwd(&a, dout.data_ptr(), address<float>(dhT), address(r.dx), address(r.dgate_a), address(r.dgate_x),
                           address<float>(r.ddecay), address<float>(r.dh0), stream.raw),
          "lbscan_gated_bwd");
    return r;
}

py::dict gated_bwd(Tensor x, Tensor gate_a, Tensor gate_x, Tensor decay, Tensor dout, Maybe starts, Maybe h0, Maybe dhT, double rate,
                   bool reverse, Maybe saved, py::object stream)
{
    const bool with_dh0 = h0 || dhT;
    const GatedGradients r = gated_gradients({x, gate_a, gate_x, decay, starts, h0, rate, reverse}, dout, dhT, saved, with_dh0,
                                             Stream(stream, x));
    py::dict g;
    g["dx"] = r.dx; g["dgate_a"] = r.dgate_a; g["dgate_x"] = r.dgate_x; g["ddecay"] = r.ddecay;
    if (with_dh0) g["dh0"] = r.dh0;
    return g;
}

struct GatedNode : torch::autograd::Function<GatedNode> {
    static variable_list forward(AutogradContext* ctx, Tensor x, Tensor gate_a, Tensor gate_x, Tensor decay, Maybe starts, Maybe h0,
                                 double rate, bool reverse, bool return_state, bool keep_states)
    {
        x = x.contiguous(); gate_a = gate_a.contiguous(); gate_x = gate_x.contiguous();
        if (starts) starts = starts->contiguous();
        if (h0) h0 = h0->contiguous();
        expect_axes("x", x, 3);
        if (!x.is_cuda()) throw Failure(LBSCAN_EINVAL, "x must be a device tensor");
        const Stream stream(x);
        const Maybe saved = keep_states ? gated_saved(x, reverse, stream) : Maybe();
        auto [y, hT] = gated_run({x, gate_a, gate_x, decay, starts, h0, rate, reverse}, {}, saved, return_state, stream);
        ctx->save_for_backward({x, gate_a, gate_x, decay, tensor(starts), tensor(h0), tensor(saved)});
        ctx->saved_data["rate"] = rate;
        ctx->saved_data["reverse"] = reverse;
        ctx->set_materialize_grads(false);
        return return_state ? variable_list{y, hT} : variable_list{y};
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        return backward_pass([&] { return gradients(ctx, grads); });
    }
    static variable_list gradients(AutogradContext* ctx, const variable_list& grads)
    {
        refuse_second_derivatives();
        const auto s = ctx->get_saved_variables();
        Tensor dout = grads[0], dhT = grads.size() > 1 ? grads[1] : Tensor();
        variable_list r(10);
        if (!dout.defined() && !dhT.defined()) return r;
        dout = dout.defined() ? dout.contiguous() : at::zeros_like(s[0]);
        if (dhT.defined()) dhT = dhT.contiguous();
        const GatedGradients g =
            gated_gradients({s[0], s[1], s[2], s[3], maybe(s[4]), maybe(s[5]), ctx->saved_data["rate"].toDouble(),
                             ctx->saved_data["reverse"].toBool()},
                            dout, maybe(dhT), maybe(s[6]), s[5].defined(), Stream(s[0]));
        r[0] = g.dx; r[1] = g.dgate_a; r[2] = g.dgate_x; r[3] = g.ddecay; r[5] = g.dh0;
        return r;
    }
};

py::object gated(Tensor x, Tensor gate_a, Tensor gate_x, Tensor decay, Maybe starts, Maybe h0, double rate, bool reverse, bool return_state)
{
    const bool wanted = at::GradMode::is_enabled() && (x.requires_grad() || gate_a.requires_grad() || gate_x.requires_grad() ||
                                                       decay.requires_grad() || (h0 && h0->requires_grad()));
    const auto r = GatedNode::apply(x, gate_a, gate_x, decay, starts, h0, rate, reverse, return_state, wanted);
    return return_state ? py::object(py::make_tuple(r[0], r[1])) : py::cast(r[0]);
}

// ---- layer norm ------------------------------------------------------------------------------------------
lbscan_norm_args norm_args(const Tensor& x, const Maybe& weight, const Maybe& bias, double eps)
{
    lbscan_norm_args a{};
    if (x.dim() < 1) throw Failure(LBSCAN_EINVAL, "x needs an axis to normalise");
    a.dtype = type_code("x", x.scalar_type());
    const int64_t D = x.size(-1);
    expect("x", x, x.sizes(), x.scalar_type(), x);
    expect("weight", weight, {D}, at::kFloat, x);
    expect("bias", bias, {D}, at::kFloat, x);
    a.dim = size32("x", D);
    a.rows = D ? x.numel() / D : 0;
    a.eps = (float)eps;
    a.weight = address<float>(weight);
    a.bias = address<float>(bias);
    return a;
}

struct NormResult { Tensor y, sum, mean, rstd; };
NormResult norm_run(const Tensor& x, const Maybe& weight, const Maybe& bias, const Maybe& residual, double eps, bool stats,
                    const Maybe& out, const Stream& stream)
{
    lbscan_norm_args a = norm_args(x, weight, bias, eps);
    c10::DeviceGuard guard(x.device());
    expect("residual", residual, x.sizes(), at::kFloat, x);
    expect("out", out, x.sizes(), x.scalar_type(), x);
    expect_writable("out", out);
    NormResult r;
    r.y = out ? *out : fresh(stream, x.sizes(), x, x.scalar_type());
    if (residual) r.sum = fresh(stream, x.sizes(), x, at::kFloat);
    if (stats) {
        const auto rows = x.sizes().slice(0, x.dim() - 1);
        r.mean = fresh(stream, rows, x, at::kFloat);
        r.rstd = fresh(stream, rows, x, at::kFloat);
        if (x.size(-1) == 0) {                       // rows of no columns: no kernel runs
            c10::OptionalStreamGuard on;
            if (stream.named) on.reset_stream(*stream.named);
            r.mean.zero_();
            r.rstd.zero_();
        }
    }
    a.x = x.data_ptr();
    a.residual = address<float>(residual);
    a.y = r.y.data_ptr();
    a.sum = address<float>(r.sum);
    a.mean = address<float>(r.mean);
    a.rstd = address<float>(r.rstd);
    check(lbscan_norm_fwd(&a, stream.raw), "lbscan_norm_fwd");
    written(out);
    return r;
}

py::object norm_fwd(Tensor x, Maybe weight, Maybe bias, Maybe residual, double eps, bool stats, Maybe out, py::object stream)
{
    const NormResult r = norm_run(x, weight, bias, residual, eps, stats, out, Stream(stream, x));
    if (residual) return stats ? py::make_tuple(r.y, r.sum, r.mean, r.rstd) : py::make_tuple(r.y, r.sum);
    return stats ? py::object(py::make_tuple(r.y, r.mean, r.rstd)) : py::cast(r.y);
}

struct NormGradients { Tensor dx, dresidual, dweight, dbias; };
// x: without a residual; sum: with one.  The shape and the type are dout's.
NormGradients norm_gradients(const Maybe& x, const Maybe& weight, const Tensor& dout, const Tensor& mean, const Tensor& rstd,
                             bool with_bias, const Maybe& sum, const Maybe& dsum, const Stream& stream)
{
    if (!sum && (!x || dsum)) throw Failure(LBSCAN_EINVAL, "x is required without a sum, and dsum belongs to one");
    lbscan_norm_args a = norm_args(dout, weight, {}, 0.0);
    c10::DeviceGuard guard(dout.device());
    const auto rows = dout.sizes().slice(0, dout.dim() - 1);
    expect("x", x, dout.sizes(), dout.scalar_type(), dout);
    expect("sum", sum, dout.sizes(), at::kFloat, dout);
    expect("dsum", dsum, dout.sizes(), at::kFloat, dout);
    expect("mean", mean, rows, at::kFloat, dout);
    expect("rstd", rstd, rows, at::kFloat, dout);
    a.x = address(x);
    a.residual = a.sum = address<float>(sum);
    a.mean = address<float>(mean);
    a.rstd = address<float>(rstd);
    NormGradients g;
    if (sum) g.dresidual = fresh(stream, dout.sizes(), dout, at::kFloat);
    // in fp32 dx and dresidual are the same values
    const bool shared = sum && dout.scalar_type() == at::kFloat;
    g.dx = shared ? g.dresidual : fresh(stream, dout.sizes(), dout, dout.scalar_type());
    if (weight) g.dweight = fresh(stream, {dout.size(-1)}, dout, at::kFloat);
    if (with_bias) g.dbias = fresh(stream, {dout.size(-1)}, dout, at::kFloat);
    const size_t need = lbscan_norm_workspace_bytes(&a);
    const Tensor ws = scratch(stream, need, dout);
    a.workspace = address(ws);
    a.workspace_bytes = need;
    check(lbscan_norm_bwd(&a, dout.data_ptr(), address<float>(dsum), shared ? nullptr : g.dx.data_ptr(), address<float>(g.dresidual),
                          address<float>(g.dweight), address<float>(g.dbias), stream.raw),
          "lbscan_norm_bwd");
    return g;
}

py::dict norm_bwd(Maybe x, Maybe weight, Tensor dout, Tensor mean, Tensor rstd, bool with_bias, Maybe sum, Maybe dsum, py::object stream)
{
    const NormGradients g = norm_gradients(x, weight, dout, mean, rstd, with_bias, sum, dsum, Stream(stream, dout));
    py::dict r;
    r["dx"] = g.dx;
    r["dresidual"] = maybe(g.dresidual);
    r["dweight"] = maybe(g.dweight);
    r["dbias"] = maybe(g.dbias);
    return r;
}

struct NormNode : torch::autograd::Function<NormNode> {
    static variable_list forward(AutogradContext* ctx, Tensor x, Maybe weight, Maybe bias, Maybe residual, double eps)
    {
        x = x.contiguous();
        if (residual) residual = residual->contiguous();
        if (!x.is_cuda()) throw Failure(LBSCAN_EINVAL, "x must be a device tensor");
        const NormResult r = norm_run(x, weight, bias, residual, eps, true, {}, Stream(x));
        // (with a residual x is not read again)
        ctx->save_for_backward({residual ? Tensor() : x, tensor(weight), r.mean, r.rstd, r.sum});
        ctx->saved_data["bias"] = (bool)bias;
        ctx->saved_data["type"] = x.scalar_type();
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
        variable_list r(5);
        if (!dout.defined() && !dsum.defined()) return r;
        const Tensor& like = s[0].defined() ? s[0] : s[4];
        dout = dout.defined() ? dout.contiguous() : at::zeros(like.sizes(), like.options().dtype(ctx->saved_data["type"].toScalarType()));
        if (dsum.defined()) dsum = dsum.contiguous();
        const NormGradients g = norm_gradients(maybe(s[0]), maybe(s[1]), dout, s[2], s[3], ctx->saved_data["bias"].toBool(), maybe(s[4]),
                                               maybe(dsum), Stream(like));
        r[0] = g.dx; r[1] = g.dweight; r[2] = g.dbias; r[3] = g.dresidual;
        return r;
    }
};

py::object norm(Tensor x, Maybe weight, Maybe bias, Maybe residual, double eps)
{
    const auto r = NormNode::apply(x, weight, bias, residual, eps);
    return r.size() > 1 ? py::object(py::make_tuple(r[0], r[1])) : py::cast(r[0]);
}

// ---- token embedding ---------------------------------------------------------------------------------------
lbscan_embed_args embed_args(const Tensor& ids, int64_t vocab, int64_t dim, const Tensor& like, double scale)
{
    lbscan_embed_args a{};
    const auto type = ids.scalar_type();
    if (type != at::kLong && type != at::kInt)
        throw Failure(LBSCAN_EUNSUPPORTED, std::string("ids: expected int32 or int64, got ") + c10::toString(type));
    expect("ids", ids, ids.sizes(), type, like);
    a.ids_type = type == at::kLong ? LBSCAN_IDS_INT64 : LBSCAN_IDS_INT32;
    a.dtype = type_code("weight", like.scalar_type());
    a.tokens = ids.numel();
    a.vocab = size32("vocab", vocab);
    a.dim = size32("dim", dim);
    a.scale = (float)scale;
    a.ids = ids.data_ptr();
    return a;
}

Tensor embed_run(const Tensor& ids, const Tensor& weight, double scale, const Maybe& out, const Stream& stream)
{
    expect_axes("weight", weight, 2);
    lbscan_embed_args a = embed_args(ids, weight.size(0), weight.size(1), weight, scale);
    expect("weight", weight, weight.sizes(), weight.scalar_type(), weight);
    c10::DeviceGuard guard(weight.device());
    c10::SmallVector<int64_t, 6> shape(ids.sizes().begin(), ids.sizes().end());
    shape.push_back(weight.size(1));
    expect("out", out, shape, weight.scalar_type(), weight);
    expect_writable("out", out);
    Tensor y = out ? *out : fresh(stream, shape, weight, weight.scalar_type());
    a.weight = weight.data_ptr();
    a.out = y.data_ptr();
    check(lbscan_embed_fwd(&a, stream.raw), "lbscan_embed_fwd");
    written(out);
    return y;
}

Tensor embed_gradient(const Tensor& ids, const Tensor& dout, int64_t vocab, double scale, const Stream& stream)
{
    if (dout.dim() != ids.dim() + 1 || dout.sizes().slice(0, ids.dim()) != ids.sizes())
        throw Failure(LBSCAN_EINVAL, "dout: expected the shape of ids and one more axis, got " + shape_of(dout.sizes()));
    if (vocab < 0) throw Failure(LBSCAN_EINVAL, "vocab: " + std::to_string(vocab));
    lbscan_embed_args a = embed_args(ids, vocab, dout.size(-1), dout, scale);
    expect("dout", dout, dout.sizes(), dout.scalar_type(), dout);
    c10::DeviceGuard guard(dout.device());
    Tensor dweight = fresh(stream, {vocab, dout.size(-1)}, dout, dout.scalar_type());
    const size_t need = lbscan_embed_workspace_bytes(&a);
    const Tensor ws = scratch(stream, need, dout);
    a.workspace = address(ws);
    a.workspace_bytes = need;
    check(lbscan_embed_bwd(&a, dout.data_ptr(), dweight.data_ptr(), stream.raw), "lbscan_embed_bwd");
    return dweight;
}

Tensor embed_fwd(Tensor ids, Tensor weight, double scale, Maybe out, py::object stream)
{
    return embed_run(ids, weight, scale, out, Stream(stream, weight));
}
Tensor embed_bwd(Tensor ids, Tensor dout, int64_t vocab, double scale, py::object stream)
{
    return embed_gradient(ids, dout, vocab, scale, Stream(stream, dout));
}

struct EmbedNode : torch::autograd::Function<EmbedNode> {
    static Tensor forward(AutogradContext* ctx, Tensor ids, Tensor weight, double scale)
    {
        ids = ids.contiguous();
        weight = weight.contiguous();
        if (!weight.is_cuda()) throw Failure(LBSCAN_EINVAL, "weight must be a device tensor");
        ctx->save_for_backward({ids});
        ctx->saved_data["vocab"] = weight.dim() ? weight.size(0) : 0;
        ctx->saved_data["scale"] = scale;
        return embed_run(ids, weight, scale, {}, Stream(weight));
    }
    static variable_list backward(AutogradContext* ctx, variable_list grads)
    {
        return backward_pass([&] { return gradients(ctx, grads); });
    }
    static variable_list gradients(AutogradContext* ctx, const variable_list& grads)
    {
        refuse_second_derivatives();
        const Tensor dout = grads[0].contiguous();
        return {Tensor(), embed_gradient(ctx->get_saved_variables()[0], dout, ctx->saved_data["vocab"].toInt(),
                                         ctx->saved_data["scale"].toDouble(), Stream(dout)),
                Tensor()};
    }
};
Tensor embed(Tensor ids, Tensor weight, double scale) { return EmbedNode::apply(ids, weight, scale); }

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m)
{
    py::register_exception_translator([](std::exception_ptr p) {
        try {
            if (p) std::rethrow_exception(p);
        } catch (const Failure& e) {
            set_python_error(e);
        }
    });
    m.def("gated_fwd", gated_fwd);
    m.def("gated_step", gated_step);
    m.def("gated_bwd", gated_bwd);
    m.def("gated_saved", gated_saved_state);
    m.def("gated", gated);
    m.def("norm_fwd", norm_fwd);
    m.def("norm_bwd", norm_bwd);
    m.def("norm", norm);
    m.def("embed_fwd", embed_fwd);
    m.def("embed_bwd", embed_bwd);
    m.def("embed", embed);
}
