// What the native modules take besides tensors: descriptors (ctypes structures of the binding), the GPU that one's memory is on, flags.  Host code only.
#pragma once
#include <c10/hip/HIPFunctions.h>

#include "call.h"

namespace {

// A ctypes structure of the binding.
template <typename T>
class Struct {
 public:
  explicit Struct(PyObject* o) {
    held_ = PyObject_GetBuffer(o, &view_, PyBUF_SIMPLE) == 0;
    if (!held_) PyErr_Clear();
    else if (view_.len == (Py_ssize_t)sizeof(T)) p = static_cast<const T*>(view_.buf);
  }
  ~Struct() {
    if (held_) PyBuffer_Release(&view_);
  }
  Struct(const Struct&) = delete;
  Struct& operator=(const Struct&) = delete;
  const T* p = nullptr;

 private:
  Py_buffer view_;
  bool held_ = false;
};

bool here(const at::Tensor* t) { return t->is_cuda() && t->device().index() == c10::hip::current_device(); }
// The GPU that a descriptor's memory is on, as its object has it.
bool here(PyObject* gpu) {
  int overflow = 0;
  return PyLong_Check(gpu) && PyLong_AsLongAndOverflow(gpu, &overflow) == c10::hip::current_device();
}
// (what is true without being True, the general path asks for its truth)
bool is_flag(PyObject* o) { return o == Py_True || o == Py_False; }

}  // namespace
