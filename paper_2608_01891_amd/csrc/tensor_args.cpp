// Calls of the C interface from the Python binding: checks the tensors, lays out
// the argument block and calls the entry point, in one native call. (Checked in
// Python and called through ctypes, rope_append with its 12 tensors took 9.7 us a
// call, now 6.4, most of it the launch.)
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <exception>
#include <string>

namespace {

std::string text(const at::IntArrayRef v) {
  std::string s = "(";
  for (size_t i = 0; i < v.size(); ++i) s += (i ? ", " : "") + std::to_string(v[i]);
  return s + ")";
}

std::string told(const at::Tensor& t) {
  return text(t.sizes()) + " " + std::string(t.dtype().name()) + " on " + t.device().str() + ", strides " +
         text(t.strides());
}

std::string place(long dev) { return dev < 0 ? "cpu" : "cuda:" + std::to_string(dev); }

bool plain(const at::Tensor& t, long dev) {
  return t.layout() == at::kStrided && !t.is_neg() && (dev < 0 ? t.is_cpu() : t.is_cuda() && t.get_device() == dev);
}

constexpr long kRows = 4;  // the other codes: the types of dense tensors

at::ScalarType type_of(long code) {
  constexpr at::ScalarType types[7] = {at::kBFloat16, at::kFloat, at::kInt,  at::kChar, at::ScalarType::Undefined,
                                       at::kLong,     at::kFloat8_e4m3fn};
  return code >= 0 && code < 7 ? types[code] : at::ScalarType::Undefined;
}

// The argument block as it is laid out: addresses of 8 bytes, numbers of 4.
struct Block {
  static constexpr size_t kMost = 256;
  alignas(8) unsigned char bytes[kMost] = {};
  size_t at = 0;
  long long stride[4];  // of the rows seen so far
  int strides = 0, taken = 0;

  template <class T>
  bool put(T v) {
    at = (at + sizeof(T) - 1) / sizeof(T) * sizeof(T);
    if (at + sizeof(T) > kMost) {
      PyErr_SetString(PyExc_TypeError, "argument block too long");
      return false;
    }
    memcpy(bytes + at, &v, sizeof(T));
    at += sizeof(T);
    return true;
  }
  bool put_int(long long v) {
    if (v != static_cast<int32_t>(v)) {
      PyErr_Format(PyExc_OverflowError, "%lld does not fit 32 bits", v);
      return false;
    }
    return put(static_cast<int32_t>(v));
  }
};

bool numbers(PyObject* const* args, int n, long long* out) {
  for (int i = 0; i < n; ++i) {
    out[i] = PyLong_AsLongLong(args[i]);
    if (out[i] == -1 && PyErr_Occurred()) return false;
  }
  return true;
}

// One item; how many arguments it takes, 0 on an error:
//   name, tensor, type code, elements   address of a dense tensor (0 for None)
//   name, tensor, kRows, T, H, D        address of bf16 token rows [T, H, D] whose heads are dense and
//                                       whose rows do not overlap; their stride (elements; 0 for one
//                                       row at most) is kept
//   None                                the next kept stride
//   int (or what stands for one, as numpy's integers do), float   a number of 4 bytes
Py_ssize_t item(PyObject* const* args, Py_ssize_t n, long dev, Block& b) {
  PyObject* o = args[0];
  if (PyIndex_Check(o)) {
    long long v;
    return numbers(args, 1, &v) && b.put_int(v);
  }
  if (PyFloat_Check(o)) return b.put(static_cast<float>(PyFloat_AS_DOUBLE(o)));
  if (o == Py_None) {
    if (b.taken < b.strides) return b.put_int(b.stride[b.taken++]);
    PyErr_SetString(PyExc_TypeError, "no stride is left");
    return 0;
  }
  const char* name = PyUnicode_Check(o) ? PyUnicode_AsUTF8(o) : nullptr;
  long long v[4];
  if (!name || n < 4 || !numbers(args + 2, 1, v) || (v[0] == kRows && n < 6)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "expected name, tensor, type, size");
    return 0;
  }
  const bool rows = v[0] == kRows;
  if (!numbers(args + 3, rows ? 3 : 1, v + 1)) return 0;
  if (args[1] == Py_None && !rows) return b.put(static_cast<uint64_t>(0)) ? 4 : 0;
  if (!THPVariable_Check(args[1])) {
    PyErr_Format(PyExc_TypeError, "%s: expected a tensor, but got %s", name, Py_TYPE(args[1])->tp_name);
    return 0;
  }
  const at::Tensor& t = THPVariable_Unpack(args[1]);
  if (rows) {
    const long long T = v[1], H = v[2], D = v[3];
    if (!(plain(t, dev) && t.scalar_type() == at::kBFloat16 && t.dim() == 3 && t.size(0) == T && t.size(1) == H &&
          t.size(2) == D && t.stride(2) == 1 && (t.stride(1) == D || H == 1) && (T <= 1 || t.stride(0) >= H * D))) {
      PyErr_Format(PyExc_ValueError,
                   "%s: expected bf16 [%lld, %lld, %lld] on %s with dense, disjoint rows, but got %s", name, T, H, D,
                   place(dev).c_str(), told(t).c_str());
      return 0;
    }
    if (b.strides == 4) {
      PyErr_SetString(PyExc_TypeError, "too many rows");
      return 0;
    }
    b.stride[b.strides++] = T > 1 ? t.stride(0) : 0;
  } else {
    const at::ScalarType type = type_of(v[0]);
    if (!(plain(t, dev) && t.scalar_type() == type && t.numel() == v[1] && t.is_contiguous() &&
          (v[1] == 0 || t.data_ptr() != nullptr))) {
      PyErr_Format(PyExc_ValueError, "%s: expected %lld dense %s elements on %s, but got %s", name, v[1],
                   c10::toString(type), place(dev).c_str(), told(t).c_str());
      return 0;
    }
  }
  return b.put(reinterpret_cast<uint64_t>(t.data_ptr())) ? (rows ? 6 : 4) : 0;
}

using Plain = int (*)(const void*, void*);
using WithWorkspace = int (*)(const void*, void*, size_t, void*);
using Query = int (*)(const void*, size_t*);

// call(entry, device, stream, workspace, bytes, item, ...): the entry point's
// status. workspace None: it takes none. stream None: it is the workspace query
// of an entry point, whose (status, bytes) come back.
PyObject* call(PyObject* const* args, Py_ssize_t n) {
  if (n < 5) {
    PyErr_SetString(PyExc_TypeError, "call(entry, device, stream, workspace, bytes, item, ...)");
    return nullptr;
  }
  void* fn = PyLong_AsVoidPtr(args[0]);
  const long dev = PyLong_AsLong(args[1]);
  const bool query = args[2] == Py_None, none = args[3] == Py_None;
  void* stream = query ? nullptr : PyLong_AsVoidPtr(args[2]);
  void* ws = none ? nullptr : PyLong_AsVoidPtr(args[3]);
  const size_t bytes = PyLong_AsSize_t(args[4]);
  if (PyErr_Occurred()) return nullptr;
  Block b;
  for (Py_ssize_t i = 5; i < n;) {
    const Py_ssize_t k = item(args + i, n - i, dev, b);
    if (k == 0) return nullptr;
    i += k;
  }
  int status;
  size_t need = 0;
  Py_BEGIN_ALLOW_THREADS;
  if (query)
    status = reinterpret_cast<Query>(fn)(b.bytes, &need);
  else if (none)
    status = reinterpret_cast<Plain>(fn)(b.bytes, stream);
  else
    status = reinterpret_cast<WithWorkspace>(fn)(b.bytes, ws, bytes, stream);
  Py_END_ALLOW_THREADS;
  return query ? Py_BuildValue("in", status, static_cast<Py_ssize_t>(need)) : PyLong_FromLong(status);
}

// No C++ exception leaves the entry (tensors without memory of their own throw,
// or have no address).
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    return call(args, n);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyMethodDef methods[] = {{"call", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry)), METH_FASTCALL,
                          "checked tensors and numbers as an argument block, and the call with it"},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensor_args", "Calls of the C interface with checked tensors.", -1,
                      methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_args(void) { return PyModule_Create(&module); }
