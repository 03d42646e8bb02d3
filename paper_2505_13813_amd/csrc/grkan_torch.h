// Helpers of the native front end's sources: what a plain tensor is, streams, types, statuses as exceptions.
#ifndef GRKAN_TORCH_H_
#define GRKAN_TORCH_H_

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/csrc/utils/pybind.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <optional>

#include "../../include/grkan.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

constexpr c10::DispatchKeySet kNotPlain({
    c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot, c10::DispatchKey::FuncTorchBatched,
    c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::FuncTorchVmapMode, c10::DispatchKey::Batched,
    c10::DispatchKey::Functionalize, c10::DispatchKey::Negative, c10::DispatchKey::Conjugate,
    c10::DispatchKey::ZeroTensor});

bool plain(const Tensor &t, const c10::Device &dev)
{
    return t.defined() && t.device() == dev && t.layout() == at::kStrided && !t.key_set().has_any(kNotPlain) &&
           !t._fw_grad(0).defined();
}

bool plain_context()
{
    return !torch::jit::tracer::isTracing() && !c10::impl::TorchDispatchModeTLS::any_modes_set() &&
           !c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode);
}

bool on_current_gpu(const Tensor &t) { return t.is_cuda() && t.get_device() == c10::hip::current_device(); }

void *stream_of(const Tensor &t) { return c10::hip::getCurrentHIPStream(t.get_device()).stream(); }

std::optional<grkan_dtype_t> io_of(const Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return GRKAN_F32;
    case at::kBFloat16: return GRKAN_BF16;
    case at::kHalf: return GRKAN_F16;
    default: return std::nullopt;
    }
}

// A status of the library as the exception the Python functions raise for it.
void check(grkan_status_t st, const char *where)
{
    if (st == GRKAN_OK)
        return;
    pybind11::gil_scoped_acquire gil;
    const pybind11::object type = pybind11::module_::import("paper_2505_13813_amd.binding").attr("GrkanError");
    PyErr_SetObject(type.ptr(), type((int)st, where).ptr());
    python_error error;
    error.persist(); // (in the backward pass it crosses threads)
    throw error;
}

// No function mode, or device contexts alone (torch.set_default_device: they act on factory functions only).
bool no_function_mode()
{
    if (!at::impl::torch_function_mode_enabled())
        return true;
    const pybind11::object device_context = pybind11::module_::import("torch.utils._device").attr("DeviceContext");
    for (const pybind11::handle mode : pybind11::module_::import("torch.overrides").attr("_get_current_function_mode_stack")())
        if (reinterpret_cast<PyObject *>(Py_TYPE(mode.ptr())) != device_context.ptr())
            return false;
    return true;
}

// The arguments of an entry as tensors; `taken` is false if one is a tensor subclass (or no tensor at all), or if a
// function mode would see the calls of the Python route.
struct Arguments {
    bool taken = no_function_mode();

    Tensor tensor(pybind11::handle h)
    {
        if (!taken || !THPVariable_CheckExact(h.ptr())) {
            taken = false;
            return Tensor();
        }
        return THPVariable_Unpack(h.ptr());
    }
    std::optional<Tensor> optional(pybind11::handle h)
    {
        return h.is_none() ? std::nullopt : std::optional<Tensor>(tensor(h));
    }
    template <typename Entry> auto call(Entry &&entry) const -> decltype(entry())
    {
        if (!taken)
            return std::nullopt;
        pybind11::gil_scoped_release no_gil;
        return entry();
    }
};

} // namespace
#endif // GRKAN_TORCH_H_
