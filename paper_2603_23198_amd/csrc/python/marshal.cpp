// The binding's view of tensors: checked device pointers, one call per tensor (0.05 us; the same
// checks by attribute in Python take 0.3 us, of calls whose kernels take 3), and the entries of a
// list of gradients.
#include <torch/csrc/autograd/python_variable.h>

#include "../../../include/sfl.h"

namespace {

const char* const kNames[] = {"float32", "bfloat16", "int32", "float64"};  // SFL_F32, SFL_BF16, then by place

bool is_kind(const at::Tensor& t, long kind) {
  switch (kind) {
    case 0: return t.scalar_type() == at::kFloat;
    case 1: return t.scalar_type() == at::kBFloat16;
    case 2: return t.scalar_type() == at::kInt;
    case 3: return t.scalar_type() == at::kDouble;
    default: return false;
  }
}

// Whether the tensor is rows of `cols` elements: trailing dimensions of it, the first not among them,
// hold that many ([batch][token][cols] and [token][head][cols / heads] do), or it is flat.
bool in_rows(const at::Tensor& t, int64_t cols) {
  int64_t n = 1;
  for (int64_t i = t.dim() - 1; i > 0 && n != cols; --i) n *= t.size(i);
  return n == cols || t.dim() < 2;
}

// The tensor's pointer if it is a contiguous device tensor of the kind and n elements (any number
// where n < 0) in rows of cols (any where cols < 0); else false with a Python error set.
bool pointer(PyObject* o, long kind, long long n, long long cols, const void** p, int64_t* numel) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "expected a tensor, got %.80s", Py_TYPE(o)->tp_name);
    return false;
  }
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!is_kind(t, kind) || (n >= 0 && t.numel() != n) || !t.is_contiguous() || !t.is_cuda()) {
    PyErr_Format(PyExc_ValueError, "expected a contiguous %s tensor of %lld elements on the GPU, got %s of %lld%s%s",
                 kNames[kind], n >= 0 ? n : (long long)t.numel(), at::toString(t.scalar_type()), (long long)t.numel(),
                 t.is_contiguous() ? "" : ", not contiguous", t.is_cuda() ? "" : ", on the CPU");
    return false;
  }
  if (cols >= 0 && !in_rows(t, cols)) {
    PyErr_Format(PyExc_ValueError, "expected rows of %lld elements, got a last dimension of %lld", cols,
                 (long long)t.size(-1));
    return false;
  }
  *p = t.numel() ? t.data_ptr() : nullptr;
  *numel = t.numel();
  return true;
}

// C++ exceptions end here.
template <typename F> PyObject* guarded(F f) {
  try {
    return f();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// ptr(tensor or None, kind, n[, cols]) -> device pointer or None
PyObject* ptr(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    if (nargs != 3 && nargs != 4) {
      PyErr_SetString(PyExc_TypeError, "ptr(tensor, kind, n[, cols])");
      return nullptr;
    }
    if (a[0] == Py_None) Py_RETURN_NONE;
    const long kind = PyLong_AsLong(a[1]);
    const long long n = PyLong_AsLongLong(a[2]), cols = nargs == 4 ? PyLong_AsLongLong(a[3]) : -1;
    if (PyErr_Occurred()) return nullptr;
    if (kind < 0 || kind > 3) {
      PyErr_SetString(PyExc_ValueError, "unknown kind of tensor");
      return nullptr;
    }
    const void* p;
    int64_t numel;
    if (!pointer(a[0], kind, n, cols, &p, &numel)) return nullptr;
    return PyLong_FromVoidPtr(const_cast<void*>(p));
  });
}

// space(tensor or None) -> (device pointer or None, bytes) of a workspace of any type
PyObject* space(PyObject*, PyObject* o) {
  return guarded([&]() -> PyObject* {
    if (o == Py_None) return Py_BuildValue("(Oi)", Py_None, 0);
    if (!THPVariable_Check(o)) {
      PyErr_Format(PyExc_TypeError, "expected a tensor as workspace, got %.80s", Py_TYPE(o)->tp_name);
      return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_contiguous() || !t.is_cuda()) {
      PyErr_Format(PyExc_ValueError, "expected a contiguous workspace on the GPU, got one that is%s%s",
                   t.is_contiguous() ? "" : " not contiguous", t.is_cuda() ? "" : " on the CPU");
      return nullptr;
    }
    if (!t.numel()) return Py_BuildValue("(Oi)", Py_None, 0);
    return Py_BuildValue("(NK)", PyLong_FromVoidPtr(t.data_ptr()), (unsigned long long)t.nbytes());
  });
}

// grads(sequence of tensors, sequence of as many or None) -> bytearray of sfl_grad_t
PyObject* grads(PyObject*, PyObject* const* a, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    if (nargs != 2 || !(PyList_Check(a[0]) || PyTuple_Check(a[0])) ||
        !(a[1] == Py_None || PyList_Check(a[1]) || PyTuple_Check(a[1]))) {
      PyErr_SetString(PyExc_TypeError, "expected a list or tuple of tensors, and another or None");
      return nullptr;
    }
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[0]);
    const bool has_out = a[1] != Py_None;
    if (has_out && PySequence_Fast_GET_SIZE(a[1]) != n) {
      PyErr_SetString(PyExc_ValueError, "as many outputs as gradients are needed");
      return nullptr;
    }
    PyObject* rows = PyByteArray_FromStringAndSize(nullptr, n * (Py_ssize_t)sizeof(sfl_grad_t));
    if (!rows) return nullptr;
    sfl_grad_t* g = reinterpret_cast<sfl_grad_t*>(PyByteArray_AS_STRING(rows));
    for (Py_ssize_t i = 0; i < n; ++i) {
      PyObject* o = PySequence_Fast_GET_ITEM(a[0], i);
      const void *src = nullptr, *dst = nullptr;
      int64_t numel = 0, out_numel = 0;
      const long kind = THPVariable_Check(o) && THPVariable_Unpack(o).scalar_type() == at::kBFloat16 ? SFL_BF16 : SFL_F32;
      if (!pointer(o, kind, -1, -1, &src, &numel) ||
          (has_out && !pointer(PySequence_Fast_GET_ITEM(a[1], i), kind, numel, -1, &dst, &out_numel))) {
        Py_DECREF(rows);
        return nullptr;
      }
      g[i] = sfl_grad_t{src, const_cast<void*>(dst), numel, (int32_t)kind, 0};
    }
    return rows;
  });
}

PyMethodDef methods[] = {{"ptr", (PyCFunction)(void (*)(void))ptr, METH_FASTCALL, nullptr},
                         {"space", space, METH_O, nullptr},
                         {"grads", (PyCFunction)(void (*)(void))grads, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
