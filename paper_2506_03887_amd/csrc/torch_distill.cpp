// The distillation loss as torch has it: its checks of tensors, and the loss as a node of the autograd graph.  In C++, because the
// engine runs a backward pass on a thread of its own, where a node in Python waits for the interpreter first and then runs in it: with
// the node in Python a step of 64 x 513 (the loss, and its gradient through the engine) took 98 us, of which kernels 10; with this one
// 54, of which the engine's way to its thread and back is some 45.
#include <torch/extension.h>

#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>

#include <algorithm>
#include <climits>
#include <optional>
#include <string>
#include <tuple>

#include "../../include/pre3.h"

namespace {

using torch::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;
using MaybeTensor = std::optional<Tensor>;

PyObject *pre3_error;                          // the package's exception, made from a status and a text; kept for the process

void expect(bool holds, const char *what) {
    if (holds) return;
    PyErr_SetString(PyExc_AssertionError, what);
    throw pybind11::error_already_set();
}
int32_t type_of_logits(at::ScalarType t) {
    switch (t) {
        case at::kBFloat16: case at::kUInt16: case at::kShort: return PRE3_LOGITS_BF16;      // (the patterns, in integers)
        case at::kHalf: return PRE3_LOGITS_F16;
        case at::kFloat: return PRE3_LOGITS_F32;
        default: return -1;
    }
}
bool on(const Tensor &t, const Tensor &logits) { return t.device() == logits.device(); }
bool is_word(const Tensor &t) { return t.scalar_type() == at::kInt || t.scalar_type() == at::kUInt32; }
void expect_kind(const Tensor &t, bool kind, const char *name) {
    if (t.is_cuda() && kind) return;
    PyErr_SetString(PyExc_TypeError, (std::string("expected a CUDA tensor of kind ") + name + ", got " + c10::toString(t.scalar_type()) + " on " + t.device().str()).c_str());
    throw pybind11::error_already_set();
}
void expect_fit(const Tensor &logits, const Tensor &ids, const Tensor &values, const MaybeTensor &mask) {
    expect(logits.dim() == 2 && (logits.stride(1) == 1 || logits.size(1) == 1) && logits.stride(0) >= 0, "logits: two dimensions, the second one contiguous");
    const int64_t rows = logits.size(0), vocab = logits.size(1);
    expect(rows <= INT_MAX && vocab <= INT_MAX, "logits: too many");
    expect(ids.dim() == 2 && ids.size(0) == rows && ids.size(1) <= INT_MAX && ids.is_contiguous(), "teacher_ids: [rows, k], contiguous");
    expect(values.sizes() == ids.sizes() && values.is_contiguous(), "teacher_logits: one for each id, contiguous");
    expect(on(ids, logits) && on(values, logits), "tensors on several devices");
    if (mask)
        expect(mask->dim() == 2 && mask->size(0) == rows && mask->size(1) == (vocab + 31) / 32 && mask->is_contiguous() && on(*mask, logits),
               "bitmask: [rows, ceil(vocab / 32)], contiguous, on the logits' device");
    expect_kind(logits, type_of_logits(logits.scalar_type()) >= 0, "logits");
    expect_kind(ids, ids.scalar_type() == at::kInt, "i32");
    expect_kind(values, type_of_logits(values.scalar_type()) >= 0, "logits");
    if (mask) expect_kind(*mask, is_word(*mask), "u32");
}
// (the stride of a single row may be anything)
int64_t row_stride(const Tensor &t) { return t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1)); }

// Tells autograd that `t` has been written, as torch's own operations in place do: a node that has saved it raises in its backward pass.
// (Tensors made in inference mode are saved by no node, and have no version.)
void written(const Tensor &t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// The call's arguments, of tensors that fit.
pre3_distill arguments(const Tensor &logits, const Tensor &ids, const Tensor &values, const MaybeTensor &mask, double temperature) {
    pre3_distill d{};
    d.logits = logits.data_ptr();
    d.bitmask = mask ? static_cast<const uint32_t *>(mask->data_ptr()) : nullptr;
    d.teacher_ids = static_cast<const int32_t *>(ids.data_ptr());
    d.teacher_logits = values.data_ptr();
    d.row_stride = row_stride(logits);
    d.logits_type = type_of_logits(logits.scalar_type());
    d.teacher_type = type_of_logits(values.scalar_type());
    d.rows = (int32_t)logits.size(0);
    d.vocab = (int32_t)logits.size(1);
    d.k = (int32_t)ids.size(1);
    d.temperature = temperature;
    return d;
}
// The workspace, which has to live until the launch: what the allocator gives away after that, it gives to the same stream.
Tensor workspace_of(pre3_distill &d, const Tensor &logits) {
    const int64_t need = pre3_distill_workspace_bytes(d.rows, d.vocab);
    if (need <= 0) return Tensor();
    Tensor workspace = at::empty({need}, logits.options().dtype(at::kByte).requires_grad(false));
    d.workspace = workspace.data_ptr();
    d.workspace_bytes = need;
    return workspace;
}
at::TensorOptions floats(const Tensor &like) { return like.options().dtype(at::kFloat).requires_grad(false); }
pre3_stream stream_of(const Tensor &t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }
std::string refusal(const char *call) { return std::string(call) + ": bad argument or launch failure"; }
void expect_ok(int status, const char *call) {
    if (status == PRE3_OK) return;
    const pybind11::object e = pybind11::reinterpret_borrow<pybind11::object>(pre3_error)(status, refusal(call));
    PyErr_SetObject(pre3_error, e.ptr());
    throw pybind11::error_already_set();
}

// The loss; with `stats`, what the backward pass needs.
Tensor loss_of(const Tensor &logits, const Tensor &ids, const Tensor &values, const MaybeTensor &mask, double temperature, Tensor *stats) {
    const c10::DeviceGuard guard(logits.device());             // (the library launches on the current device)
    pre3_distill d = arguments(logits, ids, values, mask, temperature);
    const Tensor workspace = workspace_of(d, logits);
    Tensor loss = at::empty({d.rows}, floats(logits));
    if (stats) *stats = at::empty({d.rows, 2}, floats(logits));
    expect_ok(pre3_distill_loss(&d, loss.data_ptr<float>(), stats ? stats->data_ptr<float>() : nullptr, stream_of(logits)), "pre3_distill_loss");
    return loss;
}

struct DistillLoss : torch::autograd::Function<DistillLoss> {
    static Tensor forward(AutogradContext *ctx, const Tensor &logits, const Tensor &ids, const Tensor &values, const MaybeTensor &mask, double temperature) {
        Tensor stats, loss = loss_of(logits, ids, values, mask, temperature, &stats);
        ctx->save_for_backward({logits, ids, values, mask ? *mask : Tensor(), stats});
        ctx->saved_data["temperature"] = temperature;
        return loss;
    }
    // On a thread of the engine's, without the interpreter.
    static variable_list backward(AutogradContext *ctx, variable_list upstream) {
        TORCH_CHECK(!at::GradMode::is_enabled(), "distill_loss is differentiable once");       // create_graph=True
        const variable_list saved = ctx->get_saved_variables();                                // (raises where one of them has been written since)
        const Tensor &logits = saved[0], weight = upstream[0];
        const MaybeTensor mask = saved[3].defined() ? MaybeTensor(saved[3]) : std::nullopt;
        const c10::DeviceGuard guard(logits.device());
        const pre3_distill d = arguments(logits, saved[1], saved[2], mask, ctx->saved_data["temperature"].toDouble());
        Tensor grad = at::empty({d.rows, d.vocab}, logits.options().requires_grad(false));
        const int status = pre3_distill_grad(&d, saved[4].data_ptr<float>(), weight.data_ptr<float>(), weight.stride(0), grad.data_ptr(), d.vocab, stream_of(logits));
        TORCH_CHECK(status == PRE3_OK, "pre3 status ", status, ": ", refusal("pre3_distill_grad"));
        return {grad, Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

Tensor distill_loss(const Tensor &logits, const Tensor &ids, const Tensor &values, const MaybeTensor &mask, double temperature) {
    expect_fit(logits, ids, values, mask);
    // (a tangent would be lost, and the loss read as constant)
    for (const Tensor *t : {&logits, &values}) TORCH_CHECK_NOT_IMPLEMENTED(!t->_fw_grad(0).defined(), "distill_loss has no forward-mode derivative");
    if (at::GradMode::is_enabled() && logits.requires_grad()) return DistillLoss::apply(logits, ids, values, mask, temperature);
    return loss_of(logits, ids, values, mask, temperature, nullptr);
}

std::tuple<Tensor, Tensor> distill_loss_grad(const Tensor &of, const Tensor &ids, const Tensor &values, const MaybeTensor &mask, double temperature,
                                             const MaybeTensor &row_weight, const MaybeTensor &out) {
    const Tensor logits = of.detach();
    expect_fit(logits, ids, values, mask);
    const int64_t rows = logits.size(0), vocab = logits.size(1);
    if (row_weight) {
        expect(row_weight->dim() == 1 && row_weight->size(0) == rows && on(*row_weight, logits), "row_weight: [rows], on the logits' device");
        expect_kind(*row_weight, row_weight->scalar_type() == at::kFloat, "f32");
    }
    if (out)
        expect(out->sizes() == logits.sizes() && out->scalar_type() == logits.scalar_type() && on(*out, logits) && (out->stride(1) == 1 || vocab == 1) && out->stride(0) >= 0,
               "out: of the logits' shape, type and device, the second dimension contiguous");
    const c10::DeviceGuard guard(logits.device());
    pre3_distill d = arguments(logits, ids, values, mask, temperature);
    const Tensor workspace = workspace_of(d, logits), grad = out ? *out : at::empty({rows, vocab}, logits.options());
    Tensor loss = at::empty({rows}, floats(logits));
    expect_ok(pre3_distill_loss_grad(&d, row_weight ? row_weight->data_ptr<float>() : nullptr, row_weight ? row_weight->stride(0) : 0, loss.data_ptr<float>(),
                                     grad.data_ptr(), row_stride(grad), stream_of(logits)),
              "pre3_distill_loss_grad");
    if (out) written(grad);
    return {loss, grad};
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
    m.def("distill_loss", &distill_loss);
    m.def("distill_loss_grad", &distill_loss_grad);
    m.def("raise_as", [](pybind11::object error) { pre3_error = error.release().ptr(); });
}
