// The serving calls from Python: tensors are described, checked and handed to libkurtail.so here.  A single token's call
// takes the GPU 3 to 11 us; reading six tensors and filling the structures took 5 us in Python, 0.6 us here.  The library's
// entry points are given as addresses (bind), so this module is not linked with it.  KT_BUILT_FOR names the Python and the
// torch whose headers it was built with.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <exception>

#include "../../include/kurtail.h"

namespace {

decltype(&kt_rmsnorm_quant) g_rmsnorm_quant = nullptr;
decltype(&kt_kv_append) g_kv_append = nullptr;
decltype(&kt_kv_attend) g_kv_attend = nullptr;

struct Refused {};  // (the Python error is set)

[[noreturn]] void refuse(const char* format, ...) {
  va_list args;
  va_start(args, format);
  PyErr_FormatV(PyExc_ValueError, format, args);
  va_end(args);
  throw Refused();
}
long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  return v;
}
int32_t integer32(PyObject* o, const char* what) {
  const long long v = integer(o);
  if (v != static_cast<int32_t>(v)) refuse("%s does not fit 32 bits", what);
  return static_cast<int32_t>(v);
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused();
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Refused();
  return v != 0;
}
template <typename T>
T* address(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (p == nullptr && PyErr_Occurred()) throw Refused();
  return static_cast<T*>(p);
}
const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) refuse("%s must be a tensor", what);
  return THPVariable_Unpack(o);
}
// A row-major matrix on the context's device.  (A stride along a dimension of one entry says nothing: a transposed column is
// a row as good as any.)
kt_mat matrix(PyObject* o, int device, const char* what) {
  const at::Tensor& t = tensor(o, what);
  if (t.dim() != 2 || (t.stride(1) != 1 && t.size(1) != 1) || t.get_device() != device)
    refuse("%s must be 2-D with unit column stride, on the context's device", what);
  kt_mat m = {};
  if (t.scalar_type() == at::kBFloat16) m.dtype = KT_BF16;
  else if (t.scalar_type() == at::kFloat) m.dtype = KT_F32;
  else refuse("%s must be bfloat16 or float32", what);
  m.data = t.data_ptr();
  m.rows = t.size(0);
  m.cols = t.size(1);
  m.ld = m.rows == 1 ? m.cols : t.stride(0);
  return m;
}
struct MatrixOrNone {
  kt_mat m = {};
  const kt_mat* ref = nullptr;
  MatrixOrNone(PyObject* o, int device, const char* what) {
    if (o != Py_None) m = matrix(o, device, what), ref = &m;
  }
};
// A dense tensor of the given type and sizes on the context's device; null for None.
void* dense(PyObject* o, int device, at::ScalarType type, at::IntArrayRef sizes, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  if (t.scalar_type() != type || t.sizes() != sizes || !t.is_contiguous() || t.get_device() != device)
    refuse("%s must be dense %s of %zu dimensions on the context's device, sized as the other arguments say", what,
           c10::toString(type), sizes.size());
  return t.data_ptr();
}

// No exception leaves this module.
template <int N, typename F>
PyObject* guarded(Py_ssize_t given, F&& f) {
  if (given != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments needed, %zd given", N, given);
    return nullptr;
  }
  try {
    return PyLong_FromLong(f());
  } catch (const Refused&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  }
  return nullptr;
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<3>(n, [&] {
    g_rmsnorm_quant = reinterpret_cast<decltype(g_rmsnorm_quant)>(address<void>(a[0]));
    g_kv_append = reinterpret_cast<decltype(g_kv_append)>(address<void>(a[1]));
    g_kv_attend = reinterpret_cast<decltype(g_kv_attend)>(address<void>(a[2]));
    return 0;
  });
}

template <typename F>
F bound(F f) {
  if (f == nullptr) refuse("the library is not loaded (kurtail.lib() binds its entry points)");
  return f;
}

// ctx, device, x, residual, residual_out, gain, eps, bits, clip, codes, scales, values -> status
PyObject* rmsnorm_quant(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<12>(n, [&] {
    const auto call = bound(g_rmsnorm_quant);
    const int dev = integer32(a[1], "device");
    const kt_mat x = matrix(a[2], dev, "x");
    const MatrixOrNone residual(a[3], dev, "residual"), sum(a[4], dev, "residual_out"), values(a[11], dev, "values");
    const float* gain = static_cast<const float*>(dense(a[5], dev, at::kFloat, {x.cols}, "gain"));
    const double eps = number(a[6]);
    kt_quant_spec spec = {};
    if (a[7] != Py_None) {
      spec.bits = integer32(a[7], "bits");
      spec.clip = static_cast<float>(number(a[8]));
    }
    int8_t* codes = static_cast<int8_t*>(dense(a[9], dev, at::kChar, {x.rows, x.cols}, "codes"));
    float* scales = static_cast<float*>(dense(a[10], dev, at::kFloat, {x.rows}, "scales"));
    kt_ctx* ctx = address<kt_ctx>(a[0]);
    kt_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call(ctx, x, residual.ref, sum.ref, gain, eps, a[7] != Py_None ? &spec : nullptr, codes, scales, values.ref);
    Py_END_ALLOW_THREADS
    return st;
  });
}

// ctx, device, cache, batch, q, k, v, rope, hadamard, asymmetric, clip, q_out, k_values, v_values -> status
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<14>(n, [&] {
    const auto call = bound(g_kv_append);
    const int dev = integer32(a[1], "device");
    const kt_kv_cache* cache = address<kt_kv_cache>(a[2]);
    const kt_kv_batch* batch = address<kt_kv_batch>(a[3]);
    const MatrixOrNone q(a[4], dev, "q"), q_out(a[11], dev, "q_out"), k_values(a[12], dev, "k_values"),
        v_values(a[13], dev, "v_values");
    const kt_mat k = matrix(a[5], dev, "k"), v = matrix(a[6], dev, "v");
    const float* rope = nullptr;
    int64_t rope_rows = 0;
    if (a[7] != Py_None) {
      const at::Tensor& t = tensor(a[7], "rope");
      if (t.dim() == 3) rope_rows = t.size(0);
      rope = static_cast<const float*>(dense(a[7], dev, at::kFloat, {rope_rows, cache->head_dim / 2, 2}, "rope"));
    }
    kt_quant_spec spec = {};
    spec.bits = cache->bits;
    spec.asymmetric = truth(a[9]);
    spec.clip = static_cast<float>(number(a[10]));
    const int32_t hadamard = truth(a[8]);
    kt_ctx* ctx = address<kt_ctx>(a[0]);
    kt_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call(ctx, cache, batch, q.ref, k, v, rope, rope_rows, hadamard, &spec, q_out.ref, k_values.ref, v_values.ref);
    Py_END_ALLOW_THREADS
    return st;
  });
}

// ctx, device, cache, batch, q, out, lse, scale, causal, window, scratch, scratch_bytes -> status
PyObject* kv_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded<12>(n, [&] {
    const auto call = bound(g_kv_attend);
    const int dev = integer32(a[1], "device");
    const kt_kv_cache* cache = address<kt_kv_cache>(a[2]);
    const kt_mat q = matrix(a[4], dev, "q"), out = matrix(a[5], dev, "out");
    float* lse = static_cast<float*>(dense(a[6], dev, at::kFloat, {q.rows, q.cols / cache->head_dim}, "lse"));
    const float scale = static_cast<float>(number(a[7]));
    const int32_t causal = truth(a[8]), window = integer32(a[9], "window");
    void* scratch = address<void>(a[10]);
    const size_t bytes = static_cast<size_t>(integer(a[11]));
    const kt_kv_batch* batch = address<kt_kv_batch>(a[3]);
    kt_ctx* ctx = address<kt_ctx>(a[0]);
    kt_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call(ctx, cache, batch, q, out, lse, scale, causal, window, scratch, bytes);
    Py_END_ALLOW_THREADS
    return st;
  });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name, const char* doc) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, doc};
}
PyMethodDef g_methods[] = {
    method<bind>("bind", "addresses of kt_rmsnorm_quant, kt_kv_append, kt_kv_attend"),
    method<rmsnorm_quant>("rmsnorm_quant", "kt_rmsnorm_quant on tensors; returns the status"),
    method<kv_append>("kv_append", "kt_kv_append on tensors; returns the status"),
    method<kv_attend>("kv_attend", "kt_kv_attend on tensors; returns the status"),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_serving", "the serving calls of libkurtail.so on tensors", -1, g_methods};

}  // namespace

PyMODINIT_FUNC PyInit__serving() {
  PyObject* m = PyModule_Create(&g_module);
  if (m != nullptr && PyModule_AddStringConstant(m, "built_for", KT_BUILT_FOR) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
