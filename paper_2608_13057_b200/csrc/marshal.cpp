// Python module _marshal: argument marshalling of the calls whose kernels take a few microseconds (the norms, the router,
// the few-token layer).  It checks tensors and calls the C entry points, nothing else; the Python wrappers in binding.py
// document the arguments.  The addresses of the C functions and the exception class come from binding.py at import, so the
// library that is called is the one it loaded.
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>

#include "tempo.h"

namespace {

PyObject* g_error = nullptr;
decltype(&tempo_norm_in) g_norm_in = nullptr;
decltype(&tempo_norm_out) g_norm_out = nullptr;
decltype(&tempo_route) g_route = nullptr;
decltype(&tempo_few_ffn) g_few[2] = {nullptr, nullptr};               // fp8, bf16 weights
decltype(&tempo_few_workspace_bytes) g_few_bytes = nullptr;
decltype(&tempo_packed_weight_bytes) g_packed_bytes[2] = {nullptr, nullptr};

struct Refused : std::runtime_error { using std::runtime_error::runtime_error; };

// Text without iostreams: a number written to a stream crashed in the process of a GPU run, where more than one
// library brings a C++ runtime of its own.
std::string text(const char* v) { return v; }
std::string text(int64_t v) { return std::to_string(v); }
std::string text(int32_t v) { return std::to_string(v); }
std::string text(at::ScalarType v) { return c10::toString(v); }
std::string text(at::IntArrayRef v) {
  std::string r = "[";
  for (size_t i = 0; i < v.size(); ++i) r += (i ? ", " : "") + std::to_string(v[i]);
  return r + "]";
}
template <typename... A>
[[noreturn]] void refuse(const A&... a) {
  throw Refused((text(a) + ...));
}

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) refuse(what, ": expected a tensor, got ", Py_TYPE(o)->tp_name);
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda()) refuse("expected a CUDA tensor (the library has no CPU path)");
  return t;
}

// The current stream, for operands (the tensors among a call's arguments) that are all on the current device.
void* current_stream(PyObject* const* v, Py_ssize_t n) {
  int dev = -1;
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (v[i] == Py_None || PyLong_Check(v[i]) || PyFloat_Check(v[i]) || !THPVariable_Check(v[i])) continue;
    const at::Tensor& t = THPVariable_Unpack(v[i]);
    if (!t.is_cuda()) refuse("expected a CUDA tensor (the library has no CPU path)");
    const int d = t.get_device();
    if (dev >= 0 && d != dev) refuse("operands on cuda:", dev, " and cuda:", d);
    dev = d;
  }
  const int current = c10::cuda::current_device();
  if (dev >= 0 && dev != current) refuse("operands on cuda:", dev, ", but the current device is cuda:", current);
  return c10::cuda::getCurrentCUDAStream(current).stream();
}

// Elements that the C entry reads or writes by the sizes it is given.
void holds(PyObject* o, int64_t want, const char* what) {
  if (o != Py_None && THPVariable_Unpack(o).numel() < want) refuse(what, ": expected at least ", want, " elements");
}

// Address of a contiguous tensor of the given type; None is a NULL pointer.
void* addr(PyObject* o, at::ScalarType dtype, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  if (!t.is_contiguous()) refuse(what, ": expected a contiguous tensor");
  if (t.scalar_type() != dtype) refuse(what, ": expected dtype ", dtype, ", got ", t.scalar_type());
  return t.data_ptr();
}
// Address of a device word: n_valid, status.  An empty tensor has none, and NULL would mean that no count is given.
void* word(PyObject* o, const char* what) {
  void* p = addr(o, at::kInt, what);
  holds(o, 1, what);
  return p;
}

bool is_f32(const at::Tensor& t, const char* what) {
  if (t.scalar_type() == at::kFloat) return true;
  if (t.scalar_type() != at::kBFloat16) refuse(what, ": expected bf16 or f32, got ", t.scalar_type());
  return false;
}

// Address and row pitch of a [T, d] tensor whose rows are contiguous (the rows themselves may be strided).
void* rows(PyObject* o, at::ScalarType dtype, const char* what, int64_t T, int64_t d, int64_t& pitch) {
  const at::Tensor& t = tensor(o, what);
  if (t.scalar_type() != dtype) refuse(what, ": expected dtype ", dtype, ", got ", t.scalar_type());
  if (t.dim() != 2 || t.size(0) != T || t.size(1) != d) refuse(what, ": expected shape [", T, ", ", d, "], got ", t.sizes());
  if (d > 1 && t.stride(1) != 1) refuse(what, ": expected contiguous rows");
  pitch = t.stride(0);
  if (pitch < d) {
    if (T > 1) refuse(what, ": rows overlap");
    pitch = d;
  }
  return t.data_ptr();
}

// Address of a weight or bias [d]; the first given one sets the call's parameter type.
const void* param(PyObject* o, const char* what, int64_t d, int& f32) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  const int is = is_f32(t, what) ? 1 : 0;
  if (f32 >= 0 && f32 != is) refuse(what, ": weights and biases must have one dtype");
  f32 = is;
  if (t.dim() != 1 || t.size(0) != d) refuse(what, ": expected shape [", d, "], got ", t.sizes());
  if (!t.is_contiguous()) refuse(what, ": expected a contiguous tensor");
  return t.data_ptr();
}

void stream_shape(PyObject* o, tempo_norm& a) {
  const at::Tensor& t = tensor(o, "r");
  if (t.dim() != 2) refuse("r: expected 2 dimensions, got ", t.dim());
  if (t.size(0) > INT32_MAX || t.size(1) > INT32_MAX) refuse("r: shape ", t.sizes(), " is too large");
  a.stream_f32 = is_f32(t, "r") ? 1 : 0;
  a.T = static_cast<int32_t>(t.size(0));
  a.d = static_cast<int32_t>(t.size(1));
}

// Numbers and flags are converted before a tensor is looked at: the conversion may run Python code and may fail.
float number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused("");
  return static_cast<float>(v);
}
int32_t integer(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused("");
  if (v < INT32_MIN || v > INT32_MAX) refuse("expected a 32-bit integer, got ", static_cast<int64_t>(v));
  return static_cast<int32_t>(v);
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Refused("");
  return v != 0;
}

template <typename F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t want, F f) {
  if (got != want) return PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
  try {
    return PyLong_FromLong(f());
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(g_error != nullptr ? g_error : PyExc_RuntimeError, e.what());
  } catch (...) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

// (r, w, x_out, b, kind, eps, n_valid)
PyObject* norm_in(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> int {
    tempo_norm a{};
    a.kind = integer(v[4]);
    a.eps = number(v[5]);
    void* stream = current_stream(v, n);
    stream_shape(v[0], a);
    int f32 = -1;
    void* r = rows(v[0], a.stream_f32 ? at::kFloat : at::kBFloat16, "r", a.T, a.d, a.ld_r);
    const void* w = param(v[1], "w", a.d, f32);
    void* x = rows(v[2], at::kBFloat16, "x_out", a.T, a.d, a.ld_x);
    const void* b = param(v[3], "b", a.d, f32);
    a.param_f32 = f32 > 0;
    return g_norm_in(&a, r, w, b, static_cast<const int32_t*>(word(v[6], "n_valid")), x, stream);
  });
}

// (y, r, r_out, post_w, post_b, gate, next_w, next_b, x_out, kind, eps, r_scale, y_scale, n_valid)
PyObject* norm_out(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 14, [&]() -> int {
    tempo_norm a{};
    a.kind = integer(v[9]);
    a.eps = number(v[10]);
    a.r_scale = number(v[11]);
    a.y_scale = number(v[12]);
    void* stream = current_stream(v, n);
    stream_shape(v[1], a);
    const at::ScalarType dtype = a.stream_f32 ? at::kFloat : at::kBFloat16;
    int f32 = -1;
    void* y = rows(v[0], at::kBFloat16, "y", a.T, a.d, a.ld_y);
    void* r = rows(v[1], dtype, "r", a.T, a.d, a.ld_r);
    void* r_out = rows(v[2], dtype, "r_out", a.T, a.d, a.ld_r_out);
    const void* post_w = param(v[3], "post_w", a.d, f32);
    const void* post_b = param(v[4], "post_b", a.d, f32);
    const void* gate = nullptr;
    if (v[5] != Py_None) {                              // any shape that broadcasts to [T, d]
      const at::Tensor& g = tensor(v[5], "gate");
      a.gate_f32 = is_f32(g, "gate") ? 1 : 0;
      const int64_t dims = g.dim(), rows_g = dims > 1 ? g.size(-2) : 1, cols_g = dims > 0 ? g.size(-1) : 1;
      if (dims > 2 || (rows_g != 1 && rows_g != a.T) || (cols_g != 1 && cols_g != a.d))
        refuse("gate: shape ", g.sizes(), " does not broadcast to [", a.T, ", ", a.d, "]");
      a.gate_row = rows_g == 1 ? 0 : g.stride(-2);
      a.gate_col = cols_g == 1 ? 0 : g.stride(-1);
      gate = g.data_ptr();
    }
    const void* next_w = param(v[6], "next_w", a.d, f32);
    const void* next_b = param(v[7], "next_b", a.d, f32);
    void* x = v[8] == Py_None ? nullptr : rows(v[8], at::kBFloat16, "x_out", a.T, a.d, a.ld_x);
    a.param_f32 = f32 > 0;
    return g_norm_out(&a, y, r, post_w, post_b, gate, next_w, next_b,
                      static_cast<const int32_t*>(word(v[13], "n_valid")), r_out, x, stream);
  });
}

const tempo_shape* shape_at(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (p == nullptr && PyErr_Occurred()) throw Refused("");
  return static_cast<const tempo_shape*>(p);
}

// (shape address, x, w_router, bias, n_valid, topk_ids, topk_w, status, score, renormalise, scale)
PyObject* route(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> int {
    const tempo_shape* s = shape_at(v[0]);
    const int32_t score = integer(v[8]);
    const bool renormalise = truth(v[9]);
    const float scale = number(v[10]);
    void* stream = current_stream(v, n);
    void* x = addr(v[1], at::kBFloat16, "x");
    void* wr = addr(v[2], at::kBFloat16, "w_router");
    void* bias = addr(v[3], at::kFloat, "bias");
    void* nv = word(v[4], "n_valid");
    void* ids = addr(v[5], at::kInt, "topk_ids");
    void* w = addr(v[6], at::kFloat, "topk_w");
    void* status = word(v[7], "status");
    if (s != nullptr && s->T > 0 && s->d > 0 && s->E > 0 && s->k > 0) {
      const int64_t T = s->T;
      holds(v[1], T * s->d, "x");
      holds(v[2], static_cast<int64_t>(s->E) * s->d, "w_router");
      holds(v[3], s->E, "bias");
      holds(v[5], T * s->k, "topk_ids");
      holds(v[6], T * s->k, "topk_w");
    }
    return g_route(s, score, renormalise, scale, x, wr,
                   static_cast<const float*>(bias), static_cast<const int32_t*>(nv), static_cast<int32_t*>(ids),
                   static_cast<float*>(w), static_cast<uint32_t*>(status), stream);
  });
}

// (bf16, shape address, x, topk_ids, topk_w, n_valid, replica_map, packed, out, status, workspace)
PyObject* few(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> int {
    const bool bf16 = truth(v[0]);
    const tempo_shape* s = shape_at(v[1]);
    void* stream = current_stream(v, n);
    void* x = addr(v[2], at::kBFloat16, "x");
    void* ids = addr(v[3], at::kInt, "topk_ids");
    void* w = addr(v[4], at::kFloat, "topk_w");
    void* nv = word(v[5], "n_valid");
    void* map = addr(v[6], at::kInt, "replica_map");
    void* packed = addr(v[7], at::kByte, "packed");
    void* out = addr(v[8], at::kBFloat16, "out");
    void* status = word(v[9], "status");
    void* workspace = addr(v[10], at::kByte, "workspace");
    if (s != nullptr && s->T > 0 && s->d > 0 && s->E > 0 && s->k > 0 && s->R_max > 0) {
      const int64_t T = s->T;
      holds(v[2], T * s->d, "x");
      holds(v[3], T * s->k, "topk_ids");
      holds(v[4], T * s->k, "topk_w");
      holds(v[6], static_cast<int64_t>(s->E) * s->R_max, "replica_map");
      holds(v[8], T * s->d, "out");
    }
    size_t bytes = 0;                                   // a shape that these refuse, the call refuses too
    if (g_few_bytes(s, &bytes) == TEMPO_OK) holds(v[10], static_cast<int64_t>(bytes), "workspace");
    if (g_packed_bytes[bf16](s, &bytes) == TEMPO_OK) holds(v[7], static_cast<int64_t>(bytes), "packed");
    return g_few[bf16](s, x, static_cast<const int32_t*>(ids), static_cast<const float*>(w),
                       static_cast<const int32_t*>(nv), static_cast<const int32_t*>(map), packed, out,
                       static_cast<uint32_t*>(status), workspace, stream);
  });
}

// (exception class, address of each C function below)
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n) {
  void** const at[] = {reinterpret_cast<void**>(&g_norm_in), reinterpret_cast<void**>(&g_norm_out), reinterpret_cast<void**>(&g_route),
                       reinterpret_cast<void**>(&g_few[0]), reinterpret_cast<void**>(&g_few[1]),
                       reinterpret_cast<void**>(&g_few_bytes), reinterpret_cast<void**>(&g_packed_bytes[0]),
                       reinterpret_cast<void**>(&g_packed_bytes[1])};
  constexpr Py_ssize_t want = 1 + sizeof(at) / sizeof(at[0]);
  if (n != want) return PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  for (Py_ssize_t i = 1; i < want; ++i) {
    void* f = PyLong_AsVoidPtr(v[i]);
    if (f == nullptr) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "address %zd is NULL", i);
    *at[i - 1] = f;
  }
  Py_INCREF(v[0]);
  Py_XSETREF(g_error, v[0]);
  Py_RETURN_NONE;
}

#define TEMPO_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {TEMPO_METHOD(bind), TEMPO_METHOD(norm_in), TEMPO_METHOD(norm_out), TEMPO_METHOD(route), TEMPO_METHOD(few),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of the few-microsecond calls (built for " TEMPO_BUILT_FOR ").", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
