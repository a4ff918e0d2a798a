// The sequence operators' binding for ordinary calls: torch tensors in, the
// argument struct of mg3m_seq.h out, the entry point called.
//
// The smallest calls take 2 to 5 us on the device and 3 for their launch; the
// same steps in Python took 3 (a convolution) to 6 us (a scan) more, here
// about one.  What is not ordinary is left to mg3m.py, which has the whole
// contract and its refusals: every function returns None, with nothing done,
// for other tensor types, devices, strides or shapes than it takes; else the
// result, or the entry point's status if that refused.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

#include "mg3m_seq.h"

namespace {

// Addresses of the library's entry points, as mg3m.py loaded it.
int (*conv1d_fwd)(const mg3m_conv1d*, void*);
int (*conv1d_step)(const mg3m_conv1d*, void*);
int (*scan_fwd)(const mg3m_scan*, void*);
int (*scan_step)(const mg3m_scan*, void*);
int (*scan_space)(int, int, int, int, int, size_t*);
int (*w4_fwd)(const mg3m_w4*, void*);

// A call's device and type, from its first tensor; `ok` falls with the first
// argument that is left to mg3m.py.
struct Call {
  bool ok = false;
  int dev = -1, dtype = 0;
  at::ScalarType type{};
  at::TensorOptions options;

  const at::Tensor* tensor(PyObject* o, at::ScalarType t) {
    if (!ok || !THPVariable_CheckExact(o)) return fail();
    const at::Tensor& v = THPVariable_Unpack(o);
    if (!v.is_cuda() || v.layout() != at::kStrided || v.get_device() != dev || v.scalar_type() != t) return fail();
    return &v;
  }
  const at::Tensor* fail() {
    ok = false;
    return nullptr;
  }

  explicit Call(PyObject* first) {
    if (!THPVariable_CheckExact(first)) return;
    const at::Tensor& v = THPVariable_Unpack(first);
    if (!v.is_cuda() || v.layout() != at::kStrided) return;
    dev = v.get_device();
    type = v.scalar_type();
    if (type == at::kFloat) dtype = MG3M_F32;
    else if (type == at::kBFloat16) dtype = MG3M_BF16;
    else if (type == at::kHalf) dtype = MG3M_F16;
    else return;
    options = v.options();
    ok = dev == c10::hip::current_device();
  }

  // A dense tensor of this shape, or None.
  void* dense(PyObject* o, at::IntArrayRef shape, at::ScalarType t) {
    if (o == Py_None) return nullptr;
    const at::Tensor* v = tensor(o, t);
    if (v == nullptr || v->sizes() != shape || !v->is_contiguous()) {
      ok = false;
      return nullptr;
    }
    return v->data_ptr();
  }
  // A tensor of rows of this shape, the last `tail` sizes a row: dense, or
  // rows of one or two leading sizes at one distance.
  void* rows(PyObject* o, at::IntArrayRef shape, int tail, long long* ld) {
    const at::Tensor* v = tensor(o, type);
    if (v == nullptr || v->sizes() != shape) {
      ok = false;
      return nullptr;
    }
    const int lead = (int)shape.size() - tail;
    if (v->is_contiguous()) {
      *ld = tail == 1 ? shape.back() : shape.back() * shape[shape.size() - 2];
    } else if (v->stride(-1) != 1 || (tail == 2 && v->stride(-2) != shape.back())) {
      ok = false;
    } else if (lead == 1 && shape[0] > 1) {
      *ld = v->stride(0);
    } else if (lead == 2 && shape[0] > 1 && shape[1] > 1 && v->stride(0) == v->stride(1) * shape[1]) {
      *ld = v->stride(1);
    } else {
      ok = false;
    }
    return v->data_ptr();
  }
  // The sequences of rows shaped (T, channels) or (N, L, channels).
  void sequences(at::IntArrayRef shape, bool step, PyObject* offsets, PyObject* begin, PyObject* end, long long* T,
                 long long* N, const int** b, const int** e) {
    if ((shape.size() != 2 && shape.size() != 3) || (step && shape.size() != 2)) {
      ok = false;
      return;
    }
    *T = shape.size() == 2 ? shape[0] : shape[0] * shape[1];
    *N = step || shape.size() == 3 ? shape[0] : 1;
    if (offsets != Py_None) {
      const at::Tensor* v = tensor(offsets, at::kInt);
      if (v == nullptr || begin != Py_None || end != Py_None || v->dim() != 1 || v->size(0) < 1 || !v->is_contiguous()) {
        ok = false;
        return;
      }
      *N = v->size(0) - 1;
      *b = static_cast<const int*>(v->data_ptr());
      *e = *b + 1;
    } else if (begin != Py_None || end != Py_None) {
      const at::Tensor* v = tensor(begin, at::kInt);
      if (v == nullptr || v->dim() != 1 || end == Py_None) {
        ok = false;
        return;
      }
      *N = v->size(0);
      *b = static_cast<const int*>(dense(begin, {*N}, at::kInt));
      *e = static_cast<const int*>(dense(end, {*N}, at::kInt));
    }
  }
  // The result: `given`, or a new tensor of this shape.
  void* result(PyObject* given, at::IntArrayRef shape, at::Tensor* made, long long* ld) {
    if (given != Py_None) return rows(given, shape, 1, ld);
    if (!ok) return nullptr;
    *made = at::empty(shape, options);
    *ld = shape.back();
    return made->data_ptr();
  }
  bool ints(std::initializer_list<long long> vs) {
    for (const long long v : vs)
      if (v > INT_MAX) ok = false;
    return ok;
  }

  template <typename A>
  PyObject* run(int (*f)(const A*, void*), const A& a, PyObject* given, at::Tensor& made) const {
    if (PyErr_Occurred()) return nullptr;        // a flag without a truth value
    void* stream = c10::hip::getCurrentHIPStream(dev).stream();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = f(&a, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) return PyLong_FromLong(rc);
    if (given != Py_None) {
      Py_INCREF(given);
      return given;
    }
    return THPVariable_Wrap(std::move(made));
  }
};

bool truth(PyObject* o) { return PyObject_IsTrue(o) == 1; }

// (step, x, w, bias, silu, state, load, offsets, begin, end, out)
PyObject* conv1d(PyObject*, PyObject* const* v, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 11 || conv1d_fwd == nullptr) Py_RETURN_NONE;
  const bool step = truth(v[0]);
  Call c(v[1]);
  if (!c.ok) Py_RETURN_NONE;
  const at::IntArrayRef shape = THPVariable_Unpack(v[1]).sizes();
  mg3m_conv1d a{};
  long long T = 0, N = 0;
  c.sequences(shape, step, v[7], v[8], v[9], &T, &N, &a.begin, &a.end);
  const at::Tensor* w = c.tensor(v[2], c.type);
  if (w == nullptr || w->dim() != 2) Py_RETURN_NONE;
  const long long R = w->size(0), C = shape.back();
  a.x = c.rows(v[1], shape, 1, &a.ldx);
  a.w = c.dense(v[2], {R, C}, c.type);
  a.bias = c.dense(v[3], {C}, c.type);
  a.state = c.dense(v[5], {N, R - 1, C}, c.type);
  if (!c.ints({T, N, R, C})) Py_RETURN_NONE;
  at::Tensor made;
  a.y = c.result(v[10], shape, &made, &a.ldy);
  if (!c.ok) Py_RETURN_NONE;
  a.T = (int)T;
  a.C = (int)C;
  a.R = (int)R;
  a.N = (int)N;
  a.load_state = truth(v[6]);
  a.silu = truth(v[4]);
  a.dtype = c.dtype;
  return c.run(step ? conv1d_step : conv1d_fwd, a, v[10], made);
  END_HANDLE_TH_ERRORS
}

// (step, u, dt, A, B, C, D, z, dt_bias, softplus, state, load, offsets, begin, end, out)
PyObject* scan(PyObject*, PyObject* const* v, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 16 || scan_fwd == nullptr) Py_RETURN_NONE;
  const bool step = truth(v[0]);
  Call c(v[1]);
  if (!c.ok) Py_RETURN_NONE;
  const at::IntArrayRef shape = THPVariable_Unpack(v[1]).sizes();
  mg3m_scan a{};
  long long T = 0, N = 0;
  c.sequences(shape, step, v[12], v[13], v[14], &T, &N, &a.begin, &a.end);
  const at::Tensor* B = c.tensor(v[4], c.type);
  if (B == nullptr) Py_RETURN_NONE;
  const at::IntArrayRef bshape = B->sizes();
  const int tail = (int)bshape.size() - (int)shape.size() + 1;
  if ((tail != 1 && tail != 2) || bshape.slice(0, shape.size() - 1) != shape.slice(0, shape.size() - 1)) Py_RETURN_NONE;
  const long long D = shape.back(), S = bshape.back(), G = tail == 2 ? bshape[bshape.size() - 2] : 1;
  a.u = c.rows(v[1], shape, 1, &a.ldu);
  a.dt = c.rows(v[2], shape, 1, &a.lddt);
  a.A = static_cast<const float*>(c.dense(v[3], {D, S}, at::kFloat));
  a.B = c.rows(v[4], bshape, tail, &a.ldb);
  a.C = c.rows(v[5], bshape, tail, &a.ldc);
  a.D_skip = static_cast<const float*>(c.dense(v[6], {D}, at::kFloat));
  a.ldz = D;
  if (v[7] != Py_None) a.z = c.rows(v[7], shape, 1, &a.ldz);
  a.dt_bias = static_cast<const float*>(c.dense(v[8], {D}, at::kFloat));
  a.state = static_cast<float*>(c.dense(v[10], {N, D, S}, at::kFloat));
  if (!c.ints({T, N, D, S, G})) Py_RETURN_NONE;
  at::Tensor made, space;
  a.y = c.result(v[15], shape, &made, &a.ldy);
  if (!c.ok) Py_RETURN_NONE;
  if (!step) {
    // From torch's allocator, in the order of its current stream, and in the
    // pool of a graph that is being captured.
    size_t bytes = 0;
    if (const int rc = scan_space((int)T, (int)D, (int)G, (int)S, (int)N, &bytes)) return PyLong_FromLong(rc);
    if (bytes > 0) {
      space = at::empty({(long long)bytes}, c.options.dtype(at::kByte));
      a.workspace = space.data_ptr();
      a.workspace_bytes = bytes;
    }
  }
  a.T = (int)T;
  a.D = (int)D;
  a.G = (int)G;
  a.S = (int)S;
  a.N = (int)N;
  a.load_state = truth(v[11]);
  a.softplus = truth(v[9]);
  a.dtype = c.dtype;
  return c.run(step ? scan_step : scan_fwd, a, v[15], made);
  END_HANDLE_TH_ERRORS
}

// (x, q, scale, zero, out)
PyObject* w4(PyObject*, PyObject* const* v, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 5 || w4_fwd == nullptr) Py_RETURN_NONE;
  Call c(v[0]);
  if (!c.ok) Py_RETURN_NONE;
  const at::IntArrayRef shape = THPVariable_Unpack(v[0]).sizes();
  const at::Tensor *q = c.tensor(v[1], at::kByte), *scale = c.tensor(v[2], c.type);
  if (q == nullptr || scale == nullptr || shape.size() != 2 || q->dim() != 2 || scale->dim() != 2) Py_RETURN_NONE;
  const long long M = shape[0], C = shape[1], K = q->size(0), groups = scale->size(1);
  if (groups < 1 || C % groups != 0) Py_RETURN_NONE;
  mg3m_w4 a{};
  a.x = c.rows(v[0], shape, 1, &a.ldx);
  a.q = static_cast<const unsigned char*>(c.dense(v[1], {K, C / 2}, at::kByte));
  a.scale = c.dense(v[2], {K, groups}, c.type);
  a.zero = static_cast<const unsigned char*>(c.dense(v[3], {K, groups}, at::kByte));
  if (!c.ints({M, C, K})) Py_RETURN_NONE;
  at::Tensor made;
  a.y = c.result(v[4], {M, K}, &made, &a.ldy);
  if (!c.ok) Py_RETURN_NONE;
  a.M = (int)M;
  a.C = (int)C;
  a.K = (int)K;
  a.group = (int)(C / groups);
  a.dtype = c.dtype;
  return c.run(w4_fwd, a, v[4], made);
  END_HANDLE_TH_ERRORS
}

template <typename F>
bool take(PyObject* o, F* f) {
  *f = reinterpret_cast<F>(PyLong_AsVoidPtr(o));
  return *f != nullptr;
}

// The entry points' addresses: conv1d_causal_fwd, conv1d_causal_step,
// selective_scan_fwd, selective_scan_step, selective_scan_workspace_bytes,
// matvec_w4_fwd.
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 6 || !take(v[0], &conv1d_fwd) || !take(v[1], &conv1d_step) || !take(v[2], &scan_fwd) ||
      !take(v[3], &scan_step) || !take(v[4], &scan_space) || !take(v[5], &w4_fwd)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "six addresses");
    return nullptr;
  }
  Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<bind>("bind"), method<conv1d>("conv1d"), method<scan>("scan"), method<w4>("w4"), {}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_seq_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__seq_torch() { return PyModule_Create(&module); }
