// Python module _binding: what the binding of the linear-attention block and of the
// 8-bit block does for each call, whose kernels for a few tokens take 3 to 7 us.
//
// at(), rows_at() and heads_at() give the address of a tensor that is as it has to be in 0.1
// us, where reading its shape, type, device, strides and address from Python
// takes 0.6.  They look at tensors through DLPack's exchange interface (a table of
// functions that torch offers as torch.Tensor.__dlpack_c_exchange_api__), so
// nothing of torch is compiled in.  What they find wrong, or do not know, goes to
// the Python functions of the same arguments, which say what it is.
//
// The entry points' own names call them with converted arguments, in 0.3 us where
// ctypes takes 1.4 for fifteen.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>
#include <limits>
#include <tuple>
#include <type_traits>
#include <utility>

#include "acid.h"

namespace {

// The interface's structs, as far as they are used.
struct Tensor {
  char* data;
  int32_t device_type, device_id, ndim;
  uint8_t code, bits;
  uint16_t lanes;
  const int64_t *shape, *strides;
  uint64_t byte_offset;
};
struct Exchange {
  uint32_t major, minor;
  const void* previous;
  void *allocate, *export_tensor, *import_tensor;
  int (*look)(void* object, Tensor* out);  // fills out; the object keeps what it points to
  void* stream;
};
constexpr int32_t kRocm = 10;

const Exchange* api = nullptr;
PyObject *tensor_type = nullptr, *slow_at = nullptr, *slow_rows = nullptr, *slow_heads = nullptr;
struct {
  PyObject* dtype;
  uint8_t code, bits;
} types[8];
int n_types = 0;

// args: GPU, name, tensor, shape, dtype.  Whether the tensor is on that GPU, of
// that shape and type.
bool look(PyObject* const* args, Py_ssize_t n, Tensor* t) {
  if (!api || n != 5 || !PyObject_TypeCheck(args[2], (PyTypeObject*)tensor_type) ||
      !PyLong_Check(args[0]) || !PyTuple_Check(args[3]))
    return false;
  if (api->look(args[2], t) != 0) {
    PyErr_Clear();
    return false;
  }
  if (t->device_type != kRocm || t->device_id != PyLong_AsLong(args[0]) || t->lanes != 1 ||
      t->ndim != PyTuple_GET_SIZE(args[3]) || (t->ndim && !t->strides))
    return false;
  int type = 0;
  while (type < n_types && types[type].dtype != args[4]) ++type;
  if (type == n_types || t->code != types[type].code || t->bits != types[type].bits) return false;
  for (int i = 0; i < t->ndim; ++i) {
    PyObject* want = PyTuple_GET_ITEM(args[3], i);
    if (!PyLong_Check(want) || PyLong_AsLongLong(want) != t->shape[i]) {
      PyErr_Clear();
      return false;
    }
  }
  return true;
}

PyObject* in_python(PyObject* f, PyObject* const* args, Py_ssize_t n) {
  if (f) return PyObject_Vectorcall(f, args, n, nullptr);
  PyErr_SetString(PyExc_RuntimeError, "bind() comes first");
  return nullptr;
}

PyObject* address(const Tensor& t) {
  return PyLong_FromUnsignedLongLong((uintptr_t)t.data + t.byte_offset);
}

PyObject* at(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n == 5 && args[2] == Py_None) Py_RETURN_NONE;
  Tensor t;
  if (look(args, n, &t)) {
    int64_t step = 1;
    bool contiguous = true, empty = false;
    for (int i = t.ndim - 1; i >= 0; --i) {
      contiguous = contiguous && (t.shape[i] == 1 || t.strides[i] == step);
      empty = empty || t.shape[i] == 0;
      step *= t.shape[i];
    }
    if (contiguous || empty) return address(t);
  }
  return in_python(slow_at, args, n);
}

PyObject* rows_at(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Tensor t;
  if (look(args, n, &t) && t.ndim == 2) {
    const int64_t rows = t.shape[0], cols = t.shape[1];
    const bool one = rows <= 1;
    if ((cols == 1 || t.strides[1] == 1) && (one || t.strides[0] >= cols)) {
      PyObject* out = PyTuple_New(2);
      if (!out) return nullptr;
      PyTuple_SET_ITEM(out, 0, address(t));
      PyTuple_SET_ITEM(out, 1, PyLong_FromLongLong(one ? (cols + 7) / 8 * 8 : t.strides[0]));
      if (PyTuple_GET_ITEM(out, 0) && PyTuple_GET_ITEM(out, 1)) return out;
      Py_DECREF(out);
      return nullptr;
    }
  }
  return in_python(slow_rows, args, n);
}

PyObject* heads_at(PyObject*, PyObject* const* args, Py_ssize_t n) {
  Tensor t;
  if (look(args, n, &t) && (t.ndim == 3 || t.ndim == 4) &&
      (t.shape[t.ndim - 1] == 1 || t.strides[t.ndim - 1] == 1)) {
    const int64_t seq = t.ndim == 4 && t.shape[0] > 1 ? t.strides[0] : 0;
    return Py_BuildValue("KLLL", (unsigned long long)((uintptr_t)t.data + t.byte_offset),
                         (long long)t.strides[t.ndim - 3], (long long)t.strides[t.ndim - 2],
                         (long long)seq);
  }
  return in_python(slow_heads, args, n);
}

// ------------------------------------------------------------- entry points

// An argument of a C function: addresses as integers, None (NULL) or bytes.
template <typename T>
T value(PyObject* o) {
  if constexpr (std::is_pointer_v<T>) {
    if (o == Py_None) return nullptr;
    if (PyBytes_Check(o)) return (T)(uintptr_t)PyBytes_AS_STRING(o);
    return (T)(uintptr_t)PyLong_AsUnsignedLongLong(o);
  } else if constexpr (std::is_floating_point_v<T>) {
    return (T)PyFloat_AsDouble(o);
  } else if constexpr (std::is_unsigned_v<T>) {
    return (T)PyLong_AsUnsignedLongLong(o);
  } else {
    const long long v = PyLong_AsLongLong(o);
    if (v < std::numeric_limits<T>::min() || v > std::numeric_limits<T>::max())
      PyErr_SetString(PyExc_OverflowError, "argument out of range");
    return (T)v;
  }
}

template <typename R, typename... A, size_t... I>
PyObject* convert_and_call(R (*f)(A...), PyObject* const* args, std::index_sequence<I...>) {
  const std::tuple<A...> v{value<A>(args[I])...};
  if (PyErr_Occurred()) return nullptr;
  R result;
  Py_BEGIN_ALLOW_THREADS;
  result = std::apply(f, v);
  Py_END_ALLOW_THREADS;
  return PyLong_FromLongLong((long long)result);
}
template <typename R, typename... A>
PyObject* call(R (*f)(A...), PyObject* const* args, Py_ssize_t n) {
  if (!f || n != (Py_ssize_t)sizeof...(A)) {
    PyErr_Format(PyExc_TypeError, f ? "%zd arguments, not %zd" : "bind() comes first",
                 (Py_ssize_t)sizeof...(A), n);
    return nullptr;
  }
  return convert_and_call(f, args, std::index_sequence_for<A...>());
}

// The library that ctypes has loaded gives the addresses.
#define ENTRIES(E) \
  E(linear_attention_workspace_needed) E(linear_attention) E(linear_attention_step)               \
  E(residual_norm) E(linear_w4) E(quantize_w4)                                                    \
  E(quantize_fp8) E(ln_modulate_fp8) E(quantize_fp8_weight) E(linear_fp8_workspace_needed)        \
  E(linear_fp8) E(rotary_qkv)
#define ENTRY(name)                                                       \
  decltype(&acid_##name) name##_address = nullptr;                        \
  PyObject* name(PyObject*, PyObject* const* args, Py_ssize_t n) {        \
    return call(name##_address, args, n);                                 \
  }
ENTRIES(ENTRY)
#undef ENTRY

// bind(exchange capsule or None, tensor type, Python's at, rows_at and heads_at,
// ((dtype, code, bits), ..), {entry point: address}): before the first call of
// the others.
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *capsule, *type, *py_at, *py_rows, *py_heads, *dtypes, *entries;
  if (!PyArg_ParseTuple(args, "OO!OOOO!O!", &capsule, &PyType_Type, &type, &py_at, &py_rows,
                        &py_heads, &PyTuple_Type, &dtypes, &PyDict_Type, &entries))
    return nullptr;
#define ENTRY(name)                                                                         \
  if (PyObject* address = PyDict_GetItemString(entries, "acid_" #name))                     \
    name##_address = (decltype(name##_address))(uintptr_t)PyLong_AsUnsignedLongLong(address);
  ENTRIES(ENTRY)
#undef ENTRY
  if (PyErr_Occurred()) return nullptr;
  const Exchange* x = nullptr;
  if (capsule != Py_None) {
    x = (const Exchange*)PyCapsule_GetPointer(capsule, "dlpack_exchange_api");
    if (!x) return nullptr;
    if (x->major != 1 || !x->look) x = nullptr;  // an interface of another layout
  }
  if (PyTuple_GET_SIZE(dtypes) > 8) {
    PyErr_SetString(PyExc_ValueError, "at most eight dtypes");
    return nullptr;
  }
  n_types = 0;
  for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(dtypes); ++i) {
    PyObject* d;
    if (!PyArg_ParseTuple(PyTuple_GET_ITEM(dtypes, i), "Obb", &d, &types[i].code, &types[i].bits))
      return nullptr;
    Py_INCREF(d);
    types[i].dtype = d;
    n_types = (int)i + 1;
  }
  Py_INCREF(type);
  Py_INCREF(py_at);
  Py_INCREF(py_rows);
  Py_INCREF(py_heads);
  tensor_type = type;
  slow_at = py_at;
  slow_rows = py_rows;
  slow_heads = py_heads;
  api = x;
  return PyBool_FromLong(x != nullptr);
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, "Where tensors are looked at, and what is called otherwise."},
    {"at", (PyCFunction)(void (*)())at, METH_FASTCALL,
     "Address of a contiguous tensor, or None: (gpu, name, tensor, shape, dtype)."},
    {"rows_at", (PyCFunction)(void (*)())rows_at, METH_FASTCALL,
     "(address, row stride) of a matrix: (gpu, name, tensor, shape, dtype)."},
    {"heads_at", (PyCFunction)(void (*)())heads_at, METH_FASTCALL,
     "(address, head, row and sequence stride) of heads: (gpu, name, tensor, shape, dtype)."},
#define ENTRY(name) {#name, (PyCFunction)(void (*)())name, METH_FASTCALL, "acid_" #name},
    ENTRIES(ENTRY)
#undef ENTRY
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
