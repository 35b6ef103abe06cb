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
//
//   rotary, grouped_forward, grouped_backward, cache_append, cache_read,
//   cache_attention (library function, operands .., stream)
//
// The binding's calls of these names from checked operands to the library, for
// tensors on the current GPU: a decoding step is a handful of kernels of 3 to 5 us,
// and from Python a call took 10 us (of which the launch is 3), so 5.  The result as
// the binding returns it; the library's status, an int, if it refuses; None if an
// operand is not what it should be (the binding's own checks then say what).
#include <ATen/ops/empty.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <vector>

#include "hcmix.h"

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

// [batch, n, heads, head_dim] with its heads side by side and its positions evenly
// spaced: their address, the elements between two, the extents.
struct Heads {
  void* p;
  int64_t stride, size[4];
};

bool heads_of(PyObject* o, Heads* h) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!plain(t) || t.dim() != 4) return false;
  for (int i = 0; i < 4; i++) h->size[i] = t.size(i);
  const int64_t b = h->size[0], n = h->size[1], c = h->size[2], d = h->size[3];
  h->stride = n > 1 ? t.stride(1) : b > 1 ? t.stride(0) : c * d;
  if ((d > 1 && t.stride(3) != 1) || (c > 1 && t.stride(2) != d) ||
      (n > 1 && b > 1 && t.stride(0) != n * t.stride(1)) || h->stride < c * d)
    return false;
  h->p = t.data_ptr();
  return true;
}

PyObject* heads(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 4) {
    PyErr_SetString(PyExc_TypeError, "heads(tensor, shape, dtype, device)");
    return nullptr;
  }
  PyObject* shape = args[1];
  Heads h;
  if (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != 4 || !THPDtype_Check(args[2]) ||
      (args[3] != Py_None && !THPDevice_Check(args[3])) || !heads_of(args[0], &h))
    Py_RETURN_NONE;
  const at::Tensor& t = THPVariable_Unpack(args[0]);
  if (t.scalar_type() != reinterpret_cast<THPDtype*>(args[2])->scalar_type ||
      (args[3] != Py_None && t.device() != reinterpret_cast<THPDevice*>(args[3])->device))
    Py_RETURN_NONE;
  for (int i = 0; i < 4; i++) {
    PyObject* e = PyTuple_GET_ITEM(shape, i);
    if (e == Py_None) continue;
    const int64_t want = PyLong_AsLongLong(e);
    if (want == -1 && PyErr_Occurred()) return nullptr;
    if (h.size[i] != want) Py_RETURN_NONE;
  }
  PyObject* out = PyTuple_New(2);
  if (!out) return nullptr;
  PyObject* p = PyLong_FromVoidPtr(h.p);
  PyObject* st = PyLong_FromLongLong(h.stride);
  PyTuple_SET_ITEM(out, 0, p);
  PyTuple_SET_ITEM(out, 1, st);
  if (!p || !st) {
    Py_DECREF(out);
    return nullptr;
  }
  return out;
}

// ---- whole calls ----

// An operand that is not what it should be ends a call with None.
struct Other {};

// The arguments of a call in order, each checked as it is taken; operands lie on
// the device of the first.
struct Args {
  PyObject* const* at;
  Py_ssize_t left;
  at::Device dev = at::Device(at::kCPU);

  Args(PyObject* const* args, Py_ssize_t n) : at(args), left(n) {}
  PyObject* next() {
    if (left-- <= 0) throw Other();
    return *at++;
  }
  void* fn() { return PyLong_AsVoidPtr(next()); }
  int64_t integer() {
    const int64_t v = PyLong_AsLongLong(next());
    if (v == -1 && PyErr_Occurred()) throw Other();
    return v;
  }
  int64_t integer(int64_t none) {
    if (left > 0 && *at == Py_None) return next(), none;
    return integer();
  }
  int32_t small() {
    const int64_t v = integer();
    if (v != (int32_t)v) throw Other();
    return (int32_t)v;
  }
  float real(double none) {
    PyObject* o = next();
    const double v = o == Py_None ? none : PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Other();
    return (float)v;
  }
  // [batch, n, heads, head_dim]; the first of a call says the device
  Heads heads(at::ScalarType type, bool first = false) {
    PyObject* o = next();
    Heads h;
    if (!heads_of(o, &h)) throw Other();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (first) dev = t.device();
    if (t.scalar_type() != type || t.device() != dev) throw Other();
    return h;
  }
  // contiguous, of this shape; null for None where it may be left out
  void* flat(at::ScalarType type, at::IntArrayRef shape, bool may_miss = false) {
    PyObject* o = next();
    if (may_miss && o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) throw Other();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!plain(t) || t.scalar_type() != type || t.device() != dev || !t.is_contiguous() ||
        t.sizes() != shape)
      throw Other();
    return t.data_ptr();
  }
  // a buffer of any type: its address and bytes
  void* buffer(size_t* bytes) {
    PyObject* o = next();
    if (!THPVariable_CheckExact(o)) throw Other();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!plain(t) || t.device() != dev || !t.is_contiguous()) throw Other();
    *bytes = t.nbytes();
    return t.data_ptr();
  }
  at::Tensor made(at::IntArrayRef shape, at::ScalarType type) const {
    return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
  }
  // the caller's tensor, checked by the binding's rules for outputs, or a new one
  at::Tensor result(at::ScalarType type, at::IntArrayRef shape) {
    if (left > 0 && *at == Py_None) return next(), made(shape, type);
    PyObject* o = *at;
    flat(type, shape);
    return THPVariable_Unpack(o);
  }
};

bool equal(const Heads& h, int64_t b, int64_t n, int64_t c, int64_t d) {
  return h.size[0] == b && h.size[1] == n && h.size[2] == c && h.size[3] == d;
}

// The status as an int, or the results.
PyObject* answer(int32_t status, std::initializer_list<at::Tensor> results) {
  if (status) return PyLong_FromLong(status);
  if (results.size() == 1) return THPVariable_Wrap(*results.begin());
  PyObject* out = PyTuple_New((Py_ssize_t)results.size());
  if (!out) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor& t : results) PyTuple_SET_ITEM(out, i++, THPVariable_Wrap(t));
  return out;
}

constexpr auto BF = at::kBFloat16;
constexpr auto F32 = at::kFloat;
constexpr auto I32 = at::kInt;

// (fn, x, freqs, positions, layout, inverse, scale, out, stream)
PyObject* rotary(Args a) {
  const auto fn = (decltype(&hcmix_rotary))a.fn();
  if (a.left < 1 || !THPVariable_CheckExact(*a.at)) throw Other();
  const auto type = THPVariable_Unpack(*a.at).scalar_type();
  if (type != BF && type != F32) throw Other();
  const Heads x = a.heads(type, true);
  if (a.left < 1 || !THPVariable_CheckExact(*a.at)) throw Other();
  const int64_t pairs = THPVariable_Unpack(*a.at).numel();
  if (pairs > 1 << 20) throw Other();
  const double* freqs = (const double*)a.flat(at::kDouble, {pairs});
  const int32_t* pos = (const int32_t*)a.flat(I32, {x.size[0], x.size[1]}, true);
  const int32_t layout = a.small(), inverse = a.small();
  const float scale = a.real(1.0);
  at::Tensor out;
  Heads y;
  if (a.left > 0 && *a.at != Py_None) {
    PyObject* o = *a.at;
    y = a.heads(type);
    if (!equal(y, x.size[0], x.size[1], x.size[2], x.size[3])) throw Other();
    out = THPVariable_Unpack(o);
  } else {
    a.next();
    out = a.made(x.size, type);
    y.p = out.data_ptr();
    y.stride = x.size[2] * x.size[3];
  }
  if (x.size[2] > INT32_MAX || x.size[3] > INT32_MAX) throw Other();
  return answer(fn(x.size[0] * x.size[1], (int32_t)x.size[2], (int32_t)x.size[3],
                   (int32_t)(2 * pairs), layout, inverse, type == BF ? HCMIX_BF16 : HCMIX_F32, x.p,
                   x.stride, pos, x.size[1], freqs, scale, y.p, y.stride, a.fn()),
                {out});
}

struct Grouped {
  Heads q, k, v;
  int64_t b, n_q, n_k;
  int32_t heads, kv, d;
  Grouped(Args& a) : q(a.heads(BF, true)), k(a.heads(BF)), v(a.heads(BF)) {
    b = q.size[0], n_q = q.size[1], n_k = k.size[1];
    if (!equal(k, b, n_k, k.size[2], q.size[3]) || !equal(v, b, n_k, k.size[2], q.size[3]) ||
        q.size[2] > INT32_MAX || k.size[2] > INT32_MAX || q.size[3] > INT32_MAX)
      throw Other();
    heads = (int32_t)q.size[2], kv = (int32_t)k.size[2], d = (int32_t)q.size[3];
  }
};

// (fn, q, k, v, causal, lengths, scale, out, lse, stream)
PyObject* grouped_forward(Args a) {
  const auto fn = (decltype(&hcmix_grouped_attention_forward))a.fn();
  const Grouped g(a);
  const int32_t causal = a.small();
  const int32_t* lengths = (const int32_t*)a.flat(I32, {g.b}, true);
  const float scale = a.real(1.0 / std::sqrt((double)g.d));
  const at::Tensor out = a.result(BF, {g.b, g.n_q, g.heads, g.d});
  const at::Tensor lse = a.result(F32, {g.b, g.heads, g.n_q});
  return answer(fn(g.b, g.n_q, g.n_k, g.heads, g.kv, g.d, causal, scale, lengths, g.q.p, g.q.stride,
                   g.k.p, g.k.stride, g.v.p, g.v.stride, out.data_ptr(), (float*)lse.data_ptr(), a.fn()),
                {out, lse});
}

// (fn, workspace query, q, k, v, out, lse, dout, causal, lengths, scale, dq, dk, dv, stream):
// dq, dk and dv all given or all None, the workspace made here
PyObject* grouped_backward(Args a) {
  const auto fn = (decltype(&hcmix_grouped_attention_backward))a.fn();
  const auto query = (decltype(&hcmix_grouped_attention_backward_workspace_bytes))a.fn();
  const Grouped g(a);
  const void* out = a.flat(BF, {g.b, g.n_q, g.heads, g.d});
  const float* lse = (const float*)a.flat(F32, {g.b, g.heads, g.n_q});
  const void* dout = a.flat(BF, {g.b, g.n_q, g.heads, g.d});
  const int32_t causal = a.small();
  const int32_t* lengths = (const int32_t*)a.flat(I32, {g.b}, true);
  const float scale = a.real(1.0 / std::sqrt((double)g.d));
  at::Tensor t[3];
  Heads grad[3];
  for (int i = 0; i < 3; i++) {
    const Heads& like = i == 0 ? g.q : g.k;
    if (a.left > 0 && *a.at != Py_None) {
      PyObject* o = *a.at;
      grad[i] = a.heads(BF);
      if (!equal(grad[i], like.size[0], like.size[1], like.size[2], like.size[3])) throw Other();
      t[i] = THPVariable_Unpack(o);
    } else {
      a.next();
      t[i] = a.made(like.size, BF);
      grad[i].p = t[i].data_ptr();
      grad[i].stride = like.size[2] * like.size[3];
    }
  }
  const size_t bytes = query(g.b, g.n_q, g.n_k, g.heads, g.kv, g.d);
  if (!bytes) throw Other();
  const at::Tensor ws = a.made({(int64_t)bytes}, at::kByte);
  return answer(fn(g.b, g.n_q, g.n_k, g.heads, g.kv, g.d, causal, scale, lengths, g.q.p, g.q.stride,
                   g.k.p, g.k.stride, g.v.p, g.v.stride, out, lse, dout, grad[0].p, grad[0].stride,
                   grad[1].p, grad[1].stride, grad[2].p, grad[2].stride, ws.data_ptr(), bytes, a.fn()),
                {t[0], t[1], t[2]});
}

// (fn, k, v, positions, counts, cache, capacity, stream) -> the cache
PyObject* cache_append(Args a) {
  const auto fn = (decltype(&hcmix_kv_cache_append))a.fn();
  const Heads k = a.heads(BF, true), v = a.heads(BF);
  if (!equal(v, k.size[0], k.size[1], k.size[2], k.size[3]) || k.size[2] > INT32_MAX ||
      k.size[3] > INT32_MAX)
    throw Other();
  const int32_t* positions = (const int32_t*)a.flat(I32, {k.size[0]});
  const int32_t* counts = (const int32_t*)a.flat(I32, {k.size[0]}, true);
  size_t bytes = 0;
  if (a.left < 1) throw Other();
  PyObject* cache = *a.at;
  void* c = a.buffer(&bytes);
  const int64_t capacity = a.integer();
  return answer(fn(k.size[0], capacity, (int32_t)k.size[2], (int32_t)k.size[3], k.size[1], k.p,
                   k.stride, v.p, v.stride, positions, counts, c, bytes, a.fn()),
                {THPVariable_Unpack(cache)});
}

// (fn, first, lengths, cache, capacity, kv heads, head_dim, tokens, k, v, stream) -> k, v
PyObject* cache_read(Args a) {
  const auto fn = (decltype(&hcmix_kv_cache_read))a.fn();
  if (a.left < 1 || !THPVariable_CheckExact(*a.at)) throw Other();
  const at::Tensor& f = THPVariable_Unpack(*a.at);
  if (!plain(f) || f.dim() != 1) throw Other();
  a.dev = f.device();
  const int64_t b = f.size(0);
  const int32_t* first = (const int32_t*)a.flat(I32, {b});
  const int32_t* lengths = (const int32_t*)a.flat(I32, {b});
  size_t bytes = 0;
  const void* c = a.buffer(&bytes);
  const int64_t capacity = a.integer();
  const int32_t kv = a.small(), d = a.small();
  const int64_t tokens = a.integer();
  if (kv < 1 || d < 1 || tokens < 1) throw Other();
  const at::Tensor k = a.result(BF, {b, tokens, kv, d}), v = a.result(BF, {b, tokens, kv, d});
  return answer(fn(b, capacity, kv, d, tokens, first, lengths, c, bytes, k.data_ptr(), v.data_ptr(),
                   a.fn()),
                {k, v});
}

// (fn, workspace query, q, lengths, cache, capacity, kv heads, scale, max_length, out, stream),
// the workspace made here
PyObject* cache_attention(Args a) {
  const auto fn = (decltype(&hcmix_kv_cache_attention))a.fn();
  const auto query = (decltype(&hcmix_kv_cache_attention_workspace_bytes))a.fn();
  const Heads q = a.heads(BF, true);
  if (q.size[2] > INT32_MAX || q.size[3] > INT32_MAX) throw Other();
  const int64_t b = q.size[0], tokens = q.size[1];
  const int32_t heads = (int32_t)q.size[2], d = (int32_t)q.size[3];
  const int32_t* lengths = (const int32_t*)a.flat(I32, {b});
  size_t bytes = 0;
  const void* c = a.buffer(&bytes);
  const int64_t capacity = a.integer();
  const int32_t kv = a.small();
  const float scale = a.real(1.0 / std::sqrt((double)d));
  const int64_t longest = a.integer(capacity);
  const at::Tensor out = a.result(BF, {b, tokens, heads, d});
  const size_t need = query(b, capacity, heads, kv, d, tokens, longest);
  at::Tensor ws;
  if (need) ws = a.made({(int64_t)need}, at::kByte);
  return answer(fn(b, capacity, heads, kv, d, tokens, scale, q.p, q.stride, lengths, longest, c,
                   bytes, out.data_ptr(), need ? ws.data_ptr() : nullptr, need, a.fn()),
                {out});
}

// No C++ exception passes: an operand of another kind, or one torch has no answer
// for, leaves the call to the binding's own checks.
template <PyObject* (*F)(Args)>
PyObject* guarded_call(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  try {
    return F(Args(args, nargs));
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
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
#define HCMIX_CALL(name)                                                                         \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(guarded_call<name>)),            \
   METH_FASTCALL, "the binding's call, from checked operands to the library"}
    HCMIX_CALL(rotary), HCMIX_CALL(grouped_forward), HCMIX_CALL(grouped_backward),
    HCMIX_CALL(cache_append), HCMIX_CALL(cache_read), HCMIX_CALL(cache_attention),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
