// What the native modules of the binding share: plain tensors, outputs and workspaces made with little host time, the
// interpreter lock.  Host code only.
#pragma once
#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <Python.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <optional>

#include "ccq.h"

namespace {

// (A subclass may have an idea of its own of what its attributes are: the general path asks it.)
const at::Tensor* tensor(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

// Outputs and workspaces are made past PyTorch's dispatcher.  Where someone looks on there (a TorchDispatchMode, a
// functorch transform) the general path makes them, through it.
bool looked_on() { return c10::impl::dispatch_mode_enabled() || c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode); }

bool plain_bf16(const at::Tensor* t) { return t && t->dim() == 2 && t->scalar_type() == at::kBFloat16 && t->is_cuda() && t->stride(1) == 1; }

void* current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// bf16 [rows][N] whose row stride is a multiple of 8 elements, as the entry points require.
at::Tensor new_output(int64_t rows, int64_t N, c10::Device device) {
  const int64_t ld = (N + 7) / 8 * 8;
  at::Tensor y = at::detail::empty_cuda({rows, ld}, at::kBFloat16, device, std::nullopt);
  if (ld != N) {
    const int64_t size[2] = {rows, N}, stride[2] = {ld, 1};
    y.unsafeGetTensorImpl()->set_sizes_and_strides(at::IntArrayRef(size, 2), at::IntArrayRef(stride, 2));
  }
  return y;
}

// Gives up the interpreter lock, as a foreign call through ctypes and torch.empty do: an allocation can wait for the device,
// a launch for room in its queue, and other threads run meanwhile.  Nothing of Python is touched inside.
class Unlocked {
 public:
  Unlocked() : state_(PyEval_SaveThread()) {}
  ~Unlocked() { PyEval_RestoreThread(state_); }
  Unlocked(const Unlocked&) = delete;
  Unlocked& operator=(const Unlocked&) = delete;

 private:
  PyThreadState* state_;
};

struct Workspace {
  at::Tensor held;
  void* ptr = nullptr;
  int64_t bytes = 0;
  // (contiguous memory of the operands' GPU: kernels write `bytes` bytes from ptr on)
  bool of(PyObject* given, const at::Tensor* x) {
    const at::Tensor* t = tensor(given);
    if (!t || t->device() != x->device() || !t->is_contiguous()) return false;
    ptr = t->data_ptr();
    bytes = (int64_t)t->nbytes();
    return true;
  }
  void make(int64_t need, c10::Device device) {
    if (need <= 0) return;
    held = at::detail::empty_cuda({need}, at::kByte, device, std::nullopt);
    ptr = held.data_ptr();
    bytes = need;
  }
};

PyObject* general() { Py_RETURN_NONE; }

}  // namespace
