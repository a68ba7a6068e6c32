// Checks of the tensors that a call of the Python binding gets, and their
// addresses, in one call each instead of five per tensor (the checks of
// rope_append's 12 tensors took 6 of the 10 us of a call).
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <string>

namespace {

const at::Tensor* tensor_of(PyObject* o, const char* name) {
  if (THPVariable_Check(o)) return &THPVariable_Unpack(o);
  PyErr_Format(PyExc_TypeError, "%s: expected a tensor, but got %s", name, Py_TYPE(o)->tp_name);
  return nullptr;
}

std::string text(const at::IntArrayRef v) {
  std::string s = "(";
  for (size_t i = 0; i < v.size(); ++i) s += (i ? ", " : "") + std::to_string(v[i]);
  return s + ")";
}

std::string told(const at::Tensor& t) {
  return text(t.sizes()) + " " + std::string(t.dtype().name()) + " on " + t.device().str() + ", strides " +
         text(t.strides());
}

const char* type_name(at::ScalarType d) { return c10::toString(d); }

bool plain(const at::Tensor& t, long dev) {
  return t.layout() == at::kStrided && !t.is_neg() && (dev < 0 ? t.is_cpu() : t.is_cuda() && t.get_device() == dev);
}

at::ScalarType type_of(long code) {
  switch (code) {
    case 0: return at::kBFloat16;
    case 1: return at::kFloat;
    case 2: return at::kInt;
    case 3: return at::kChar;
    default: return at::ScalarType::Undefined;
  }
}

// dense(device, name, tensor, type code, elements, ...): the addresses of dense
// tensors of that device (-1: host), type and number of elements, as a tuple;
// 0 for None.
PyObject* dense_args(PyObject* const* args, Py_ssize_t n) {
  if (n < 1 || (n - 1) % 4 != 0) {
    PyErr_SetString(PyExc_TypeError, "dense(device, name, tensor, type, elements, ...)");
    return nullptr;
  }
  const long dev = PyLong_AsLong(args[0]);
  if (dev == -1 && PyErr_Occurred()) return nullptr;
  PyObject* out = PyTuple_New((n - 1) / 4);
  if (!out) return nullptr;
  for (Py_ssize_t i = 1; i < n; i += 4) {
    const char* name = PyUnicode_AsUTF8(args[i]);
    unsigned long long p = 0;
    bool ok = name != nullptr;
    if (ok && args[i + 1] != Py_None) {
      const at::Tensor* t = tensor_of(args[i + 1], name);
      const at::ScalarType type = type_of(PyLong_AsLong(args[i + 2]));
      const long long count = PyLong_AsLongLong(args[i + 3]);
      ok = t && !PyErr_Occurred();
      if (ok) {
        ok = plain(*t, dev) && t->scalar_type() == type && t->numel() == count && t->is_contiguous();
        if (ok) {
          p = reinterpret_cast<unsigned long long>(t->data_ptr());
          ok = p != 0 || count == 0;
        }
        if (!ok)
          PyErr_Format(PyExc_ValueError, "%s: expected %lld dense %s elements on %s:%ld, but got %s", name, count,
                       type_name(type), dev < 0 ? "cpu" : "cuda", dev < 0 ? 0 : dev, told(*t).c_str());
      }
    }
    PyObject* v = ok ? PyLong_FromUnsignedLongLong(p) : nullptr;
    if (!v) {
      Py_DECREF(out);
      return nullptr;
    }
    PyTuple_SET_ITEM(out, (i - 1) / 4, v);
  }
  return out;
}

// rows(device, name, tensor, T, H, D): address and row stride (elements; 0 where
// there is one row at most) of bf16 token rows [T, H, D] whose heads are dense
// and whose rows do not overlap.
PyObject* rows_args(PyObject* const* args, Py_ssize_t n) {
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "rows(device, name, tensor, T, H, D)");
    return nullptr;
  }
  const char* name = PyUnicode_AsUTF8(args[1]);
  if (!name) return nullptr;
  const at::Tensor* t = tensor_of(args[2], name);
  if (!t) return nullptr;
  const long dev = PyLong_AsLong(args[0]);
  const long long T = PyLong_AsLongLong(args[3]), H = PyLong_AsLongLong(args[4]), D = PyLong_AsLongLong(args[5]);
  if (PyErr_Occurred()) return nullptr;
  if (!(plain(*t, dev) && t->scalar_type() == at::kBFloat16 && t->dim() == 3 && t->size(0) == T && t->size(1) == H &&
        t->size(2) == D && t->stride(2) == 1 && (t->stride(1) == D || H == 1) && (T <= 1 || t->stride(0) >= H * D))) {
    PyErr_Format(PyExc_ValueError,
                 "%s: expected bf16 [%lld, %lld, %lld] on %s:%ld with dense, disjoint rows, but got %s", name, T, H, D,
                 dev < 0 ? "cpu" : "cuda", dev < 0 ? 0 : dev, told(*t).c_str());
    return nullptr;
  }
  return Py_BuildValue("KL", reinterpret_cast<unsigned long long>(t->data_ptr()),
                       static_cast<long long>(T > 1 ? t->stride(0) : 0));
}

// No C++ exception leaves an entry (tensors without memory of their own throw,
// or have no address).
template <PyObject* F(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    return F(args, n);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyMethodDef methods[] = {
    {"dense", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<dense_args>)), METH_FASTCALL,
     "addresses of dense tensors, checked"},
    {"rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<rows_args>)), METH_FASTCALL,
     "address and row stride of token rows, checked"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensor_args", "Checked tensor arguments of the binding.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_args(void) { return PyModule_Create(&module); }
