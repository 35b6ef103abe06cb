// Operand checks of the Python binding, in native code: a stack call hands the
// library 40 to 70 tensors, and checking each from Python (0.8 us apiece) took
// longer than the call's kernels at small sizes.
//
//   pointers(tensors, count, shape, dtype, device) -> bytes or None
//
// The device addresses of tensors[0 .. count - 1] as an array of `void*`, if
// every one is a plain tensor of exactly `shape` and `dtype`, contiguous and on
// `device`; None otherwise (the binding then finds out what is wrong, and says
// so).
//
//   heads(tensor, shape, dtype, device) -> (address, stride) or None
//
// The same for one [batch, n, heads, head_dim] operand whose heads lie side by
// side and whose positions are evenly spaced over the whole batch: its address
// and the elements between two positions.  None entries of shape match any
// extent, device None any GPU.
#include <torch/csrc/Device.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

namespace {

constexpr int kMaxDims = 8;

PyObject* pointers(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 5) {
    PyErr_SetString(PyExc_TypeError, "pointers(tensors, count, shape, dtype, device)");
    return nullptr;
  }
  PyObject *seq = args[0], *shape = args[2];
  const Py_ssize_t count = PyLong_AsSsize_t(args[1]);
  if (count == -1 && PyErr_Occurred()) return nullptr;
  if (!(PyList_CheckExact(seq) || PyTuple_CheckExact(seq)) || !PyTuple_Check(shape) ||
      !THPDtype_Check(args[3]) || !THPDevice_Check(args[4]) ||
      PySequence_Fast_GET_SIZE(seq) < count || count < 0 || PyTuple_GET_SIZE(shape) > kMaxDims)
    Py_RETURN_NONE;
  int64_t dims[kMaxDims];
  const Py_ssize_t nd = PyTuple_GET_SIZE(shape);
  for (Py_ssize_t i = 0; i < nd; i++) {
    dims[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i));
    if (dims[i] == -1 && PyErr_Occurred()) return nullptr;
  }
  const auto dtype = reinterpret_cast<THPDtype*>(args[3])->scalar_type;
  const auto device = reinterpret_cast<THPDevice*>(args[4])->device;
  std::vector<void*> out((size_t)count);
  for (Py_ssize_t i = 0; i < count; i++) {
    PyObject* o = PySequence_Fast_ITEMS(seq)[i];
    if (!THPVariable_CheckExact(o)) Py_RETURN_NONE;
    const at::Tensor& t = THPVariable_Unpack(o);
    // strided storage with an address of its own (no fake, wrapped or meta tensor)
    bool ok = t.layout() == c10::kStrided && t.scalar_type() == dtype && t.device() == device &&
              device.type() == c10::kCUDA && !t.unsafeGetTensorImpl()->is_python_dispatch() &&
              t.has_storage() && !t.is_conj() && !t.is_neg() && t.dim() == nd &&
              t.is_contiguous();
    for (Py_ssize_t k = 0; ok && k < nd; k++) ok = t.size(k) == dims[k];
    if (!ok) Py_RETURN_NONE;
    out[(size_t)i] = t.data_ptr();
  }
  return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(out.data()),
                                   count * (Py_ssize_t)sizeof(void*));
}

// A plain tensor in GPU memory with an address of its own.
bool plain(const at::Tensor& t) {
  return t.layout() == c10::kStrided && t.device().type() == c10::kCUDA &&
         !t.unsafeGetTensorImpl()->is_python_dispatch() && t.has_storage() && !t.is_conj() &&
         !t.is_neg();
}

PyObject* heads(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 4) {
    PyErr_SetString(PyExc_TypeError, "heads(tensor, shape, dtype, device)");
    return nullptr;
  }
  PyObject* shape = args[1];
  if (!THPVariable_CheckExact(args[0]) || !PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != 4 ||
      !THPDtype_Check(args[2]) || (args[3] != Py_None && !THPDevice_Check(args[3])))
    Py_RETURN_NONE;
  const at::Tensor& t = THPVariable_Unpack(args[0]);
  if (!plain(t) || t.scalar_type() != reinterpret_cast<THPDtype*>(args[2])->scalar_type ||
      (args[3] != Py_None && t.device() != reinterpret_cast<THPDevice*>(args[3])->device) ||
      t.dim() != 4)
    Py_RETURN_NONE;
  for (int i = 0; i < 4; i++) {
    PyObject* e = PyTuple_GET_ITEM(shape, i);
    if (e == Py_None) continue;
    const int64_t want = PyLong_AsLongLong(e);
    if (want == -1 && PyErr_Occurred()) return nullptr;
    if (t.size(i) != want) Py_RETURN_NONE;
  }
  const int64_t b = t.size(0), n = t.size(1), h = t.size(2), d = t.size(3);
  const int64_t stride = n > 1 ? t.stride(1) : b > 1 ? t.stride(0) : h * d;
  if ((d > 1 && t.stride(3) != 1) || (h > 1 && t.stride(2) != d) ||
      (n > 1 && b > 1 && t.stride(0) != n * t.stride(1)) || stride < h * d)
    Py_RETURN_NONE;
  PyObject* out = PyTuple_New(2);
  if (!out) return nullptr;
  PyObject* p = PyLong_FromVoidPtr(t.data_ptr());
  PyObject* st = PyLong_FromLongLong(stride);
  PyTuple_SET_ITEM(out, 0, p);
  PyTuple_SET_ITEM(out, 1, st);
  if (!p || !st) {
    Py_DECREF(out);
    return nullptr;
  }
  return out;
}

PyObject* guarded_heads(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
  try {
    return heads(self, args, nargs);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

PyObject* guarded_pointers(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
  try {
    return pointers(self, args, nargs);
  } catch (...) {   // a tensor that has no such property: the binding's own checks decide
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

PyMethodDef methods[] = {
    {"pointers", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded_pointers)),
     METH_FASTCALL, "addresses of tensors that match, or None"},
    {"heads", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded_heads)), METH_FASTCALL,
     "address and position stride of an operand that matches, or None"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
