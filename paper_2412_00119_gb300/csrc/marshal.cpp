// marshal.cpp -- argument marshalling of the microscaled 4-bit front end for torch tensors, natively:
// the attributes of a dozen tensors cost the interpreter 4 us a call, more than the shortest kernels
// take.
//
// Each function takes the arguments of the Python function of its name (bmlp.py) that are tensors, and makes the
// call of the library where everything about them is as it should be: torch tensors on the current
// device, of the right types, shapes and strides, on the current stream.  In every other case it
// does nothing and returns kSlow, and the Python function goes on, with its own checks and errors.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "bmlp.h"

namespace {

constexpr long kSlow = 1000;

// The library's functions (set by init: the library is loaded by its path).
decltype(&bmlp_mx4_quantize) f_quantize = nullptr;
decltype(&bmlp_mx4_norm_quantize) f_norm = nullptr;
decltype(&bmlp_mx4_dequantize) f_dequantize = nullptr;
decltype(&bmlp_mx4_matmul) f_matmul = nullptr;
decltype(&bmlp_mx4_matmul_grouped) f_grouped = nullptr;

struct Arg {
  char* p = nullptr;
  int64_t ld = 0, group = 0;
};

struct Call {
  int device = -1;
  bool ok = true;
  Call() { device = c10::cuda::current_device(); }
  // The tensor if it is one of that type and that many dimensions on the current device.
  const at::Tensor* tensor(PyObject* o, int64_t dims) {
    if (!ok || !THPVariable_CheckExact(o)) return ok = false, nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.get_device() != device || t.dim() != dims || t.layout() != at::kStrided || !t.has_storage())
      return ok = false, nullptr;
    return &t;
  }
  Arg arg(const at::Tensor& t) { return {static_cast<char*>(t.data_ptr()), t.dim() > 1 ? t.stride(0) : 0, 0}; }
  Arg rows(PyObject* o, at::ScalarType type, int64_t n, int64_t K) {
    const at::Tensor* t = tensor(o, 2);
    if (!t) return {};
    if (t->scalar_type() != type || t->size(0) != n || t->size(1) != K || (K > 1 && t->stride(1) != 1)) return ok = false, Arg{};
    return arg(*t);
  }
  Arg optional_rows(PyObject* o, at::ScalarType type, int64_t n, int64_t K) { return o == Py_None ? Arg{} : rows(o, type, n, K); }
  Arg groups(PyObject* o, at::ScalarType type, int64_t E, int64_t n, int64_t K) {
    const at::Tensor* t = tensor(o, 3);
    if (!t) return {};
    if (t->scalar_type() != type || t->size(0) != E || t->size(1) != n || t->size(2) != K || (K > 1 && t->stride(2) != 1))
      return ok = false, Arg{};
    return {static_cast<char*>(t->data_ptr()), t->stride(1), t->stride(0)};
  }
  char* vector(PyObject* o, at::ScalarType type, int64_t n) {
    if (o == Py_None) return nullptr;
    const at::Tensor* t = tensor(o, 1);
    if (!t) return nullptr;
    if (t->scalar_type() != type || t->size(0) != n || (n > 1 && t->stride(0) != 1)) return ok = false, nullptr;
    return static_cast<char*>(t->data_ptr());
  }
  // A tensor's size, and its type as the library numbers them.
  bool shape(PyObject* o, int64_t& n, int64_t& K, at::ScalarType& type) {
    const at::Tensor* t = tensor(o, 2);
    if (!t) return false;
    n = t->size(0);
    K = t->size(1);
    type = t->scalar_type();
    return true;
  }
  int real(at::ScalarType type) {
    if (type == at::kFloat) return BMLP_F32;
    if (type == at::kHalf) return BMLP_F16;
    if (type == at::kBFloat16) return BMLP_BF16;
    ok = false;
    return -1;
  }
  void fits(int64_t K, int64_t N = 1) { ok = ok && K < (1ll << 31) && N < (1ll << 31); }
  void* stream() { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
};

template <typename F>
PyObject* answer(F f) {
  long rc = kSlow;
  try {
    rc = f();
  } catch (...) {
    rc = kSlow;
  }
  return PyLong_FromLong(rc);
}
// The library's call, without the interpreter's lock, as ctypes makes it.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }   // (also where the call throws)
};
template <typename F>
long unlocked(F f) {
  Unlocked here;
  return f();
}
bool wrong(Py_ssize_t given, Py_ssize_t wanted) {
  if (given == wanted) return false;
  PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
  return true;
}

constexpr at::ScalarType U8 = at::kByte, F32 = at::kFloat;

PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // x, q, scale
  if (wrong(n_args, 3)) return nullptr;
  return answer([&]() -> long {
    Call c;
    int64_t n = 0, K = 0;
    at::ScalarType type;
    if (!f_quantize || !c.shape(a[0], n, K, type)) return kSlow;
    const Arg x = c.rows(a[0], type, n, K), q = c.rows(a[1], U8, n, (K + 1) / 2), s = c.rows(a[2], U8, n, (K + 31) / 32);
    const int code = c.real(type);
    c.fits(K);
    if (!c.ok) return kSlow;
    void* st = c.stream();
    return unlocked([&] { return f_quantize(x.p, code, x.ld, n, (int32_t)K, (uint8_t*)q.p, q.ld, (uint8_t*)s.p, s.ld, st); });
  });
}

PyObject* norm_quantize(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // x, gain, q, scale, row_scale, res, sum_out, eps
  if (wrong(n_args, 8)) return nullptr;
  const double eps = PyFloat_AsDouble(a[7]);
  if (eps == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    return PyLong_FromLong(kSlow);
  }
  return answer([&]() -> long {
    Call c;
    int64_t n = 0, K = 0;
    at::ScalarType type;
    if (!f_norm || a[4] == Py_None || !c.shape(a[0], n, K, type)) return kSlow;
    const Arg x = c.rows(a[0], type, n, K), q = c.rows(a[2], U8, n, (K + 1) / 2), s = c.rows(a[3], U8, n, (K + 31) / 32);
    const Arg res = c.optional_rows(a[5], type, n, K), sum = c.optional_rows(a[6], type, n, K);
    char* gain = c.vector(a[1], type, K);
    char* by = c.vector(a[4], F32, n);
    const int code = c.real(type);
    c.fits(K);
    if (!c.ok) return kSlow;
    void* st = c.stream();
    return unlocked([&] {
      return f_norm(x.p, x.ld, res.p, res.ld, gain, code, n, (int32_t)K, (float)eps, sum.p, sum.ld, (uint8_t*)q.p, q.ld, (uint8_t*)s.p,
                    s.ld, (float*)by, st);
    });
  });
}

PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // q, scale, out, row_scale
  if (wrong(n_args, 4)) return nullptr;
  return answer([&]() -> long {
    Call c;
    int64_t n = 0, K = 0;
    at::ScalarType type;
    if (!f_dequantize || !c.shape(a[2], n, K, type)) return kSlow;
    const Arg out = c.rows(a[2], type, n, K), q = c.rows(a[0], U8, n, (K + 1) / 2), s = c.rows(a[1], U8, n, (K + 31) / 32);
    char* by = c.vector(a[3], F32, n);
    const int code = c.real(type);
    c.fits(K);
    if (!c.ok) return kSlow;
    void* st = c.stream();
    return unlocked([&] {
      return f_dequantize((const uint8_t*)q.p, q.ld, (const uint8_t*)s.p, s.ld, (const float*)by, n, (int32_t)K, out.p, code, out.ld, st);
    });
  });
}

PyObject* matmul(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // a, a_scale, w, w_scale, out, row_scale, bias
  if (wrong(n_args, 7)) return nullptr;
  return answer([&]() -> long {
    Call c;
    int64_t n = 0, half = 0, N = 0, out_N = 0;
    at::ScalarType type;
    if (!f_matmul || !c.shape(a[0], n, half, type) || !c.shape(a[2], N, out_N, type) || !c.shape(a[4], out_N, out_N, type)) return kSlow;
    const int64_t K = 2 * half;
    const Arg x = c.rows(a[0], U8, n, half), xs = c.rows(a[1], U8, n, (K + 31) / 32), w = c.rows(a[2], U8, N, half),
              ws = c.rows(a[3], U8, N, (K + 31) / 32), out = c.rows(a[4], type, n, N);
    char* by = c.vector(a[5], F32, n);
    char* bias = c.vector(a[6], F32, N);
    const int code = c.real(type);
    c.fits(K, N);
    if (!c.ok) return kSlow;
    void* st = c.stream();
    return unlocked([&] {
      return f_matmul((const uint8_t*)x.p, x.ld, (const uint8_t*)xs.p, xs.ld, (const float*)by, (const uint8_t*)w.p, w.ld,
                      (const uint8_t*)ws.p, ws.ld, (const float*)bias, n, (int32_t)K, (int32_t)N, out.p, code, out.ld, st);
    });
  });
}

PyObject* matmul_grouped(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // a, a_scale, w, w_scale, offsets, out, row_scale, bias
  if (wrong(n_args, 8)) return nullptr;
  return answer([&]() -> long {
    Call c;
    int64_t n = 0, half = 0, out_n = 0, out_N = 0;
    at::ScalarType type;
    const at::Tensor* wt = nullptr;
    if (!f_grouped || a[4] == Py_None || !c.shape(a[0], n, half, type) || !(wt = c.tensor(a[2], 3)) || !c.shape(a[5], out_n, out_N, type))
      return kSlow;
    const int64_t K = 2 * half, E = wt->size(0), N = wt->size(1);
    const Arg x = c.rows(a[0], U8, n, half), xs = c.rows(a[1], U8, n, (K + 31) / 32), w = c.groups(a[2], U8, E, N, half),
              ws = c.groups(a[3], U8, E, N, (K + 31) / 32), out = c.rows(a[5], type, n, N), bias = c.optional_rows(a[7], F32, E, N);
    char* at = c.vector(a[4], at::kInt, E + 1);
    char* by = c.vector(a[6], F32, n);
    const int code = c.real(type);
    c.fits(K, N);
    if (!c.ok || E >= (1ll << 31)) return kSlow;
    void* st = c.stream();
    return unlocked([&] {
      return f_grouped((const uint8_t*)x.p, x.ld, (const uint8_t*)xs.p, xs.ld, (const float*)by, (const uint8_t*)w.p, w.ld, w.group,
                       (const uint8_t*)ws.p, ws.ld, ws.group, (const float*)bias.p, bias.ld, (const int32_t*)at, (int32_t)E, n,
                       (int32_t)K, (int32_t)N, out.p, code, out.ld, st);
    });
  });
}

// init(addresses of the five functions, in their order above)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (wrong(n_args, 5)) return nullptr;
  void* p[5];
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  f_quantize = reinterpret_cast<decltype(f_quantize)>(p[0]);
  f_norm = reinterpret_cast<decltype(f_norm)>(p[1]);
  f_dequantize = reinterpret_cast<decltype(f_dequantize)>(p[2]);
  f_matmul = reinterpret_cast<decltype(f_matmul)>(p[3]);
  f_grouped = reinterpret_cast<decltype(f_grouped)>(p[4]);
  Py_RETURN_NONE;
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(init), FAST(quantize), FAST(norm_quantize), FAST(dequantize), FAST(matmul), FAST(matmul_grouped),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddIntConstant(m, "SLOW", kSlow) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
