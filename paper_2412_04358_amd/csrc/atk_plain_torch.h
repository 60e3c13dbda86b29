// What the extension modules that marshal calls on plain torch tensors share (atk_decode_torch.cpp, atk_quant_torch.cpp): host code against torch's own structures.
#pragma once
#include <Python.h>

#include <cmath>
#include <vector>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/version.h>

#include "../../include/atk_decode.h"

namespace {

bool plain_mode() {
    return !at::impl::torch_function_mode_enabled() && !c10::impl::TorchDispatchModeTLS::any_modes_set() && !torch::jit::tracer::isTracing();
}
// a plain tensor on that device (-1: any GPU, which it becomes); NULL if it is none
const at::Tensor *tensor(PyObject *o, int *device) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() ||
        t.key_set().has_any(c10::DispatchKeySet({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize})))
        return nullptr;
    if (*device < 0) *device = t.get_device();
    return t.get_device() == *device ? &t : nullptr;
}
const at::Tensor *ints(PyObject *o, int *device, std::initializer_list<int64_t> shape) {
    const at::Tensor *t = tensor(o, device);
    return t && t->scalar_type() == at::kInt && t->sizes() == at::IntArrayRef(shape) && t->is_contiguous() ? t : nullptr;
}
int type_of(const at::Tensor &t) {
    return t.scalar_type() == at::kFloat ? ATK_F32 : t.scalar_type() == at::kBFloat16 ? ATK_BF16 : t.scalar_type() == at::kHalf ? ATK_F16 : -1;
}
bool integer(PyObject *o, int64_t *out) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    *out = PyLong_AsLongLongAndOverflow(o, &over);
    return over == 0;
}
void *stream_of(int device) { return c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream(); }

// None for what `body` throws (no memory, say: the Python path meets the same and says so in torch's words)
template <typename BODY>
PyObject *plain(BODY body) {
    try {
        if (!plain_mode()) Py_RETURN_NONE;
        return body();
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// The table of a PageTables object, by the address of its argument structure.
const atk_page_tables *tables_of(PyObject *o) {
    int64_t at;
    return integer(o, &at) ? (const atk_page_tables *)(intptr_t)at : nullptr;
}
PyObject *said(int code) {  // 0 is a result here: what is None is not done yet
    return PyLong_FromLong(code);
}

}  // namespace
