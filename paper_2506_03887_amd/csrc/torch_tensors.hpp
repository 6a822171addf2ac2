// What the library's calls on torch's tensors share: checks, streams, errors.
#pragma once
#include <torch/extension.h>

#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>

#include <algorithm>
#include <optional>
#include <string>

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
// (the stride of a single row may be anything)
int64_t row_stride(const Tensor &t) { return t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1)); }

// Tells autograd that `t` has been written, as torch's own operations in place do: a node that has saved it raises in its backward pass.
// (Tensors made in inference mode are saved by no node, and have no version.)
void written(const Tensor &t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
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

}  // namespace
