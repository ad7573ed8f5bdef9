// Python module _lists: lists of torch tensors as arrays of brsvd_tensor, for the calls that take all of a model's gradients.  A step of Python for each of a tensor's
// properties takes 40 ns, five of them and the comparisons for 500 tensors and 500 results 270 us; this takes what reading them from the objects takes.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <array>
#include <cstring>
#include <exception>

#include "brsvd.h"

namespace {

struct Object {
  PyObject* p;
  explicit Object(PyObject* q) : p(q) {}
  Object(const Object&) = delete;
  ~Object() { Py_XDECREF(p); }
};

int64_t dtype_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return BRSVD_DTYPE_F32;
    case at::kBFloat16: return BRSVD_DTYPE_BF16;
    case at::kHalf: return BRSVD_DTYPE_F16;
    default: return -1;
  }
}

// Whether two tensors of one shape, or a tensor itself where they are one, fill their memory without gaps, with their numbers in the same order
bool same_order(const at::Tensor& a, const at::Tensor& b) {
  constexpr int kMost = 64;
  const int64_t dims = a.dim();
  if (dims > kMost) return false;
  std::array<int, kMost> of;
  int n = 0;
  for (int64_t d = 0; d < dims; ++d)
    if (a.size(d) != 1) {
      if (a.stride(d) != b.stride(d)) return false;
      of[n++] = (int)d;
    }
  std::sort(of.begin(), of.begin() + n, [&](int x, int y) { return a.stride(x) < a.stride(y); });
  int64_t expected = 1;
  for (int i = 0; i < n; ++i) {
    if (a.stride(of[i]) != expected) return false;
    expected *= a.size(of[i]);
  }
  return true;
}
bool strided_rows(const at::Tensor& t) { return t.dim() == 2 && t.stride(1) == 1 && t.stride(0) >= t.size(1); }

// tables(tensors) or tables(tensors, out): a tuple of one bytes object for each list
PyObject* tables(PyObject*, PyObject* const* args, Py_ssize_t lists) {
  if (lists < 1 || lists > 2) return PyErr_Format(PyExc_TypeError, "one list or two");
  static const char* const names[2] = {"tensors", "out"};
  for (int l = 0; l < lists; ++l)
    if (!PyList_Check(args[l]) && !PyTuple_Check(args[l])) return PyErr_Format(PyExc_TypeError, "%s must be a list of CUDA tensors", names[l]);
  const Object first(PySequence_Tuple(args[0])), second(lists > 1 ? PySequence_Tuple(args[1]) : nullptr);      // they stay as they are
  if (!first.p || (lists > 1 && !second.p)) return nullptr;
  PyObject* const from[2] = {first.p, second.p};
  const Py_ssize_t n = PyTuple_GET_SIZE(first.p);
  if (lists > 1 && PyTuple_GET_SIZE(second.p) != n) return PyErr_Format(PyExc_ValueError, "out has %zd tensors, expected %zd", PyTuple_GET_SIZE(second.p), n);
  const Object a(PyBytes_FromStringAndSize(nullptr, n * (Py_ssize_t)sizeof(brsvd_tensor))), b(lists > 1 ? PyBytes_FromStringAndSize(nullptr, n * (Py_ssize_t)sizeof(brsvd_tensor)) : nullptr);
  if (!a.p || (lists > 1 && !b.p)) return nullptr;
  char* const to[2] = {PyBytes_AS_STRING(a.p), lists > 1 ? PyBytes_AS_STRING(b.p) : nullptr};
  try {
    for (Py_ssize_t i = 0; i < n; ++i) {
      const at::Tensor* t[2] = {nullptr, nullptr};
      bool dense = true, rows = true;
      for (int l = 0; l < lists; ++l) {
        PyObject* o = PyTuple_GET_ITEM(from[l], i);
        if (THPVariable_Check(o)) t[l] = &THPVariable_Unpack(o);
        if (PyErr_Occurred()) return nullptr;
        if (!t[l] || !t[l]->defined() || !t[l]->is_cuda() || t[l]->layout() != at::kStrided || dtype_of(*t[l]) < 0)
          return PyErr_Format(PyExc_TypeError, "%s[%zd] must be a CUDA tensor of dtype torch.float32, torch.bfloat16 or torch.float16", names[l], i);
        if (l && t[l]->sizes() != t[0]->sizes()) return PyErr_Format(PyExc_TypeError, "out[%zd] has another shape than tensors[%zd]", i, i);
        dense = dense && t[l]->is_contiguous();
      }
      const int64_t numbers = t[0]->numel();
      if (!dense && numbers) {
        for (int l = 0; l < lists; ++l) rows = rows && strided_rows(*t[l]);
        if (!rows && !(same_order(*t[0], *t[lists - 1])))
          return PyErr_Format(PyExc_TypeError, "tensors[%zd] must be dense, or a matrix with unit column stride%s", i, lists > 1 ? ", and out's laid out like it" : "");
      }
      const bool strided = !dense && numbers && rows;
      for (int l = 0; l < lists; ++l) {
        brsvd_tensor x{};
        x.data = numbers ? t[l]->data_ptr() : nullptr;
        x.rows = strided ? t[l]->size(0) : 1;
        x.cols = strided ? t[l]->size(1) : numbers;
        x.ld = strided ? t[l]->stride(0) : numbers;
        x.dtype = dtype_of(*t[l]);
        memcpy(to[l] + i * sizeof x, &x, sizeof x);
      }
    }
  } catch (const std::exception& e) {
    return PyErr_Format(PyExc_RuntimeError, "%s", e.what());
  }
  return lists > 1 ? PyTuple_Pack(2, a.p, b.p) : PyTuple_Pack(1, a.p);
}

PyMethodDef methods[] = {{"tables", (PyCFunction)(void (*)(void))tables, METH_FASTCALL, "arrays of brsvd_tensor of one or two lists of CUDA tensors"}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lists", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// torch_version: the torch whose objects it reads; another one's may be laid out differently.
PyMODINIT_FUNC PyInit__lists() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", BRSVD_TORCH_VERSION) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
