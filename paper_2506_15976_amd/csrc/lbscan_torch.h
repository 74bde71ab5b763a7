// What the torch sides of the operators share: errors, argument checks, outputs and scratch from torch's allocator,
// the current stream or a named one, backward passes.
#pragma once
#include "../../include/lbscan.h"

#include <c10/core/DeviceGuard.h>
#include <c10/core/StreamGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/extension.h>

#include <optional>
#include <string>
#include <vector>

namespace lbscan_torch {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;
using Maybe = std::optional<Tensor>;

// ---- errors ------------------------------------------------------------------------------------------
struct Failure : std::runtime_error {          // becomes binding.LbscanError
    int code;
    Failure(int c, const std::string& what) : std::runtime_error(what), code(c) {}
};

inline void check(int rc, const char* name)
{
    if (rc == LBSCAN_OK) return;
    std::string what = std::string(name) + " failed (" + std::to_string(rc) + "): " + lbscan_strerror(rc);
    if (rc == LBSCAN_EHIP) what += std::string(": ") + lbscan_last_error();
    throw Failure(rc, what);
}

inline std::string shape_of(at::IntArrayRef s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + ")";
}

inline int type_code(const char* name, at::ScalarType t)
{
    if (t == at::kFloat) return LBSCAN_FP32;
    if (t == at::kBFloat16) return LBSCAN_BF16;
    throw Failure(LBSCAN_EUNSUPPORTED, std::string(name) + ": unsupported tensor dtype " + c10::toString(t));
}

// Shape, type, layout and device of one tensor; `like` is the tensor whose device the call runs on.
inline void expect(const char* name, const Tensor& t, at::IntArrayRef shape, at::ScalarType type, const Tensor& like)
{
    if (t.sizes() != shape || t.scalar_type() != type)
        throw Failure(LBSCAN_EINVAL, std::string(name) + ": expected " + shape_of(shape) + " " + c10::toString(type) + ", got " +
                                         shape_of(t.sizes()) + " " + c10::toString(t.scalar_type()));
    if (!t.is_cuda() || !t.is_contiguous() || t.device() != like.device())
        throw Failure(LBSCAN_EINVAL, std::string(name) + " must be a contiguous device tensor, on the device of the others");
}
inline void expect(const char* name, const Maybe& t, at::IntArrayRef shape, at::ScalarType type, const Tensor& like)
{
    if (t) expect(name, *t, shape, type, like);
}
inline void expect_axes(const char* name, const Tensor& t, int64_t n)
{
    if (t.dim() != n) throw Failure(LBSCAN_EINVAL, std::string(name) + ": expected " + std::to_string(n) + " axes, got " + shape_of(t.sizes()));
}
inline int32_t size32(const char* name, int64_t n)
{
    if (n > INT32_MAX) throw Failure(LBSCAN_EINVAL, std::string(name) + ": size " + std::to_string(n) + " does not fit 32 bits");
    return (int32_t)n;
}

template <typename P = void> P* address(const Maybe& t) { return t ? static_cast<P*>(t->data_ptr()) : nullptr; }
template <typename P = void> P* address(const Tensor& t) { return t.defined() ? static_cast<P*>(t.data_ptr()) : nullptr; }
inline Maybe maybe(const Tensor& t) { return t.defined() ? Maybe(t) : Maybe(); }
inline Tensor tensor(const Maybe& t) { return t ? *t : Tensor(); }

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
inline Tensor fresh(const Stream& stream, at::IntArrayRef shape, const Tensor& like, at::ScalarType type)
{
    if (!stream.named) return at::empty(shape, like.options().dtype(type));
    const c10::StreamGuard guard(*stream.named);
    Tensor t = at::empty(shape, like.options().dtype(type));
    if (t.numel()) t.record_stream(*stream.current);
    return t;
}
// Memory that goes back with the call.
inline Tensor scratch(const Stream& stream, size_t bytes, const Tensor& like)
{
    if (!bytes) return Tensor();
    c10::OptionalStreamGuard guard;
    if (stream.named) guard.reset_stream(*stream.named);
    return at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
}

// ---- tensors that a call overwrites --------------------------------------------------------------------
// The caller's own (a state, `out`): autograd has to know, by the tensor's version, as a backward pass may still need
// what was there; and there is no gradient of the old values.
inline void expect_writable(const char* name, const Maybe& t)
{
    if (t && t->requires_grad() && at::GradMode::is_enabled())
        throw Failure(LBSCAN_EINVAL, std::string(name) + " requires grad and cannot be overwritten");
}
inline void written(const Maybe& t)
{
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

// The Python error of a failure is set (the GIL is held).
inline void set_python_error(const Failure& e)
{
    const py::object type = py::module_::import("paper_2506_15976_amd.binding").attr("LbscanError");
    PyErr_SetObject(type.ptr(), type(e.code, e.what()).ptr());
}

// A backward pass that is being recorded into a graph, and whose next node adds up a leaf's gradient on the default stream, where
// an eager graph that still lives has left it: torch would make the default stream wait for the recorded one, which ends
// the recording, or the process, from a thread that no caller sees.  (It makes no stream wait for nodes that the pass does not
// reach: other leaves may be in use elsewhere.)
inline void refuse_leaves_of_the_default_stream()
{
    const auto node = torch::autograd::get_current_node();
    if (!node) return;
    const auto& edges = node->next_edges();
    for (size_t k = 0; k < edges.size(); ++k) {
        if (!edges[k].function || !node->task_should_compute_output(k)) continue;
        const auto leaf = edges[k].function->stream();
        if (!leaf || leaf->device_type() != c10::DeviceType::CUDA) continue;
        const c10::impl::VirtualGuardImpl guard(leaf->device_type());
        hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
        if (*leaf != guard.getDefaultStream(leaf->device()) || *leaf == guard.getStream(leaf->device()) ||
            hipStreamIsCapturing(c10::hip::getCurrentHIPStream(leaf->device_index()).stream(), &status) != hipSuccess)
            continue;
        if (status == hipStreamCaptureStatusActive)
            throw Failure(LBSCAN_EUNSUPPORTED, "a backward pass cannot be captured while an eager graph of the same leaves, made on the "
                                               "default stream, lives: delete its outputs first");
    }
}

// A node's backward pass.  Its errors cross torch's threads, which hand Python errors on as they are and make a RuntimeError
// of every other exception.
template <typename F>
variable_list backward_pass(const F& pass)
{
    try {
        refuse_leaves_of_the_default_stream();
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
inline void refuse_second_derivatives()
{
    if (at::GradMode::is_enabled())
        throw Failure(LBSCAN_EUNSUPPORTED, "lbscan operators can be differentiated once: backward with create_graph is not supported");
}

// The operators of lbscan_torch_blocks.cpp.
void define_blocks(py::module_& m);

}  // namespace lbscan_torch
