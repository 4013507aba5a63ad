// The calls of the 8-bit operators from Python: argument checks, output tensors and the current stream, then
// the C entry point - what binding.py does for the other calls with ctypes, here in native code because these
// are called once per layer and token: a call's arguments cost 1-2 us instead of 10-25 us in the
// interpreter, as much as the kernels themselves take at that size.  No operator is computed here.
//
// The entry points are those of the library that binding.load() has opened (their addresses are handed
// over once), so the checking build is served as well.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <exception>
#include <optional>
#include <string>
#include <utility>

#include "luq.h"

namespace {

struct Entry {
  decltype(&luq_layer_norm) layer_norm;
  decltype(&luq_layer_norm_bwd) layer_norm_bwd;
  decltype(&luq_layer_norm_int8) layer_norm_int8;
  decltype(&luq_quant_int8_rows) quant_int8_rows;
  decltype(&luq_gemm_int8) gemm_int8;
  decltype(&luq_gemm_int8_grouped) gemm_int8_grouped;
  decltype(&luq_quant_int8_gemm) quant_int8_gemm;
  decltype(&luq_layer_norm_int8_gemm) layer_norm_int8_gemm;
  decltype(&luq_quant_int8_gemm_grouped) quant_int8_gemm_grouped;
  decltype(&luq_set_allocator) set_allocator;
} lib{};
PyObject* error_class = nullptr;   // binding.LuqError(code, what)

// A Python exception that is already set, or is made from a message.
struct Raised {};
[[noreturn]] void type_error(const std::string& what) {
  PyErr_SetString(PyExc_TypeError, what.c_str());
  throw Raised{};
}
// What the workspace's allocation threw: it must not pass the library's C entry points, and leaves here.
thread_local std::exception_ptr thrown;

void check(int rc, const char* what) {
  if (rc == LUQ_OK) return;
  if (thrown) std::rethrow_exception(std::exchange(thrown, nullptr));
  PyObject* e = PyObject_CallFunction(error_class, "is", rc, what);
  if (e) {
    PyErr_SetObject(error_class, e);
    Py_DECREF(e);
  }
  throw Raised{};
}

// The arguments of one call, taken in order.
struct Args {
  PyObject* const* at;
  luq_ctx* ctx;
  int64_t device;
  Args(PyObject* const* args, Py_ssize_t given, Py_ssize_t wanted) : at(args) {
    if (given != wanted) type_error("wrong number of arguments");
    ctx = static_cast<luq_ctx*>(PyLong_AsVoidPtr(*at++));
    if (PyErr_Occurred()) throw Raised{};
    thrown = nullptr;
    if (!ctx) check(LUQ_ERR_ARG, "the context is closed");
    device = integer();
  }
  int64_t integer() {
    const int64_t v = PyLong_AsLongLong(*at++);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
  }
  float real() {
    const double v = PyFloat_AsDouble(*at++);
    if (v == -1.0 && PyErr_Occurred()) throw Raised{};
    return static_cast<float>(v);
  }
  const at::Tensor* optional(const char* what) {
    PyObject* o = *at++;
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) type_error(std::string(what) + ": tensor expected");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device)
      type_error(std::string(what) + ": tensor on cuda:" + std::to_string(device) + " expected, got " + t.device().str());
    return &t;
  }
  const at::Tensor& tensor(const char* what) {
    const at::Tensor* t = optional(what);
    if (!t) type_error(std::string(what) + ": tensor expected");
    return *t;
  }
};

int dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return LUQ_F32;
  if (t.scalar_type() == at::kBFloat16) return LUQ_BF16;
  type_error("float32 or bfloat16 tensor expected");
}
at::ScalarType dtype_of(int64_t code) { return code == LUQ_BF16 ? at::kBFloat16 : at::kFloat; }

// Tokens: rows of a 2-D tensor with contiguous rows.  Leading dimensions are flattened; other layouts and
// broadcast rows are copied.
struct Rows {
  at::Tensor t;
  int dtype;
  int64_t rows, cols, ld;
};
bool rows_fit(const at::Tensor& t) {
  const int64_t rows = t.size(0), cols = t.size(1);
  return (cols <= 1 || t.stride(1) == 1) && (rows <= 1 || t.stride(0) >= cols);
}
Rows rows_of(const at::Tensor& given, const char* what) {
  Rows r;
  r.dtype = dtype_code(given);
  if (given.dim() == 0) type_error(std::string(what) + ": at least one dimension expected");
  r.t = given;
  if (given.dim() != 2) {
    int64_t rows = 1;
    for (int64_t i = 0; i + 1 < given.dim(); ++i) rows *= given.size(i);
    r.t = given.reshape({rows, given.size(-1)});
  }
  if (!rows_fit(r.t)) r.t = r.t.contiguous();
  r.rows = r.t.size(0);
  r.cols = r.t.size(1);
  r.ld = r.rows > 1 ? r.t.stride(0) : r.cols;
  return r;
}
float* floats(const at::Tensor* t, int64_t numel, const char* what) {
  if (!t) return nullptr;
  if (t->scalar_type() != at::kFloat || t->numel() != numel || !t->is_contiguous())
    type_error(std::string(what) + ": contiguous float32 tensor of " + std::to_string(numel) + " elements expected");
  return static_cast<float*>(t->data_ptr());
}
// row stride of int8 codes [.., rows, cols] after checking them
int64_t codes_ld(const at::Tensor& t, const char* what) {
  const int64_t rows = t.size(-2), cols = t.size(-1);
  const int64_t ld = rows > 1 ? t.stride(-2) : (cols + 15) / 16 * 16;
  if (t.scalar_type() != at::kChar) type_error(std::string(what) + ": int8 tensor expected");
  if ((cols > 1 && t.stride(-1) != 1) || ld % 16 || ld < cols || (reinterpret_cast<uintptr_t>(t.data_ptr()) & 15u))
    type_error(std::string(what) + ": rows have to start at multiples of 16 bytes (see new_codes)");
  return ld;
}
struct Weights {
  const int8_t* codes;
  int64_t groups, N, ld, stride;
};
Weights weights_of(const at::Tensor& t, int64_t K, bool grouped) {
  if (t.dim() != (grouped ? 3 : 2) || t.size(-1) != K)
    type_error(std::string("weight codes: ") + (grouped ? "[groups, N, K]" : "[N, K]") + " with K = " + std::to_string(K) + " expected");
  Weights w;
  w.groups = grouped ? t.size(0) : 1;
  w.N = t.size(-2);
  w.ld = codes_ld(t, "weight codes");
  w.stride = grouped && w.groups > 1 ? t.stride(0) : w.N * w.ld;
  w.codes = static_cast<const int8_t*>(t.data_ptr());
  return w;
}
const int32_t* offsets_of(const at::Tensor& t, int64_t groups) {
  if (t.scalar_type() != at::kInt || t.numel() != groups + 1 || !t.is_contiguous())
    type_error("offsets: contiguous int32 tensor of " + std::to_string(groups + 1) + " elements expected");
  return static_cast<const int32_t*>(t.data_ptr());
}

// (past the dispatcher: it costs as much as the workspace's allocation)
at::Tensor make(at::IntArrayRef size, at::ScalarType type, int64_t device) {
  return at::detail::empty_cuda(size, type, at::Device(at::kCUDA, static_cast<at::DeviceIndex>(device)), std::nullopt);
}
// the caller's output (checked), or a new one of type `code`
at::Tensor output(const at::Tensor* out, int64_t rows, int64_t cols, int64_t code, int64_t device) {
  if (!out) return make({rows, cols}, dtype_of(code), device);
  dtype_code(*out);
  if (out->dim() != 2 || out->size(0) != rows || out->size(1) != cols || !rows_fit(*out))
    type_error("output: " + std::to_string(rows) + " x " + std::to_string(cols) + " tensor with contiguous rows expected");
  return *out;
}
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
void* stream_of(int64_t device) { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream(); }
PyObject* wrap(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None); }
PyObject* wrap(const at::Tensor& a, const at::Tensor& b) { return Py_BuildValue("(NN)", wrap(a), wrap(b)); }
PyObject* wrap(const at::Tensor& a, const at::Tensor& b, const at::Tensor& c) { return Py_BuildValue("(NNN)", wrap(a), wrap(b), wrap(c)); }
at::Tensor like(const at::Tensor& result, const at::Tensor& given) { return given.dim() == 2 ? result : result.reshape(given.sizes()); }

using Body = PyObject* (*)(PyObject* const*, Py_ssize_t);
template <Body body>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    // outputs carry no gradient: nothing here is recorded
    at::AutoDispatchBelowADInplaceOrView below;
    return body(args, n);
  } catch (const Raised&) {
    return nullptr;
  } catch (const c10::OutOfMemoryError& e) {
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* cls = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    if (cls) PyErr_SetString(cls, e.what_without_backtrace());
    Py_XDECREF(cls);
    Py_XDECREF(torch);
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// layer_norm(ctx, device, x, weight, bias, eps, out) -> y, mean, rstd
PyObject* layer_norm(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 7);
  const at::Tensor& given = a.tensor("x");
  const Rows x = rows_of(given, "x");
  const float* w = floats(a.optional("weight"), x.cols, "weight");
  const float* b = floats(a.optional("bias"), x.cols, "bias");
  const float eps = a.real();
  const at::Tensor* out = a.optional("out");
  const at::Tensor y = output(out, x.rows, x.cols, x.dtype, a.device);
  if (dtype_code(y) != x.dtype) type_error("layer norm's result has the type of its input");
  const at::Tensor mean = make({x.rows}, at::kFloat, a.device), rstd = make({x.rows}, at::kFloat, a.device);
  check(lib.layer_norm(a.ctx, x.t.data_ptr(), x.dtype, x.rows, x.cols, x.ld, w, b, eps, y.data_ptr(), row_stride(y),
                       static_cast<float*>(mean.data_ptr()), static_cast<float*>(rstd.data_ptr()), stream_of(a.device)),
        "luq_layer_norm");
  return wrap(out ? y : like(y, given), mean, rstd);
}

// layer_norm_bwd(ctx, device, dy, x, mean, rstd, weight, need_dx, need_dweight, need_dbias) -> dx, dweight, dbias
PyObject* layer_norm_bwd(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 10);
  const at::Tensor &dy_given = a.tensor("dy"), &given = a.tensor("x");
  if (dy_given.sizes() != given.sizes() || dy_given.scalar_type() != given.scalar_type())
    type_error("dy has the shape and type of x");
  const Rows x = rows_of(given, "x"), dy = rows_of(dy_given, "dy");
  const float* mean = floats(&a.tensor("mean"), x.rows, "mean");
  const float* rstd = floats(&a.tensor("rstd"), x.rows, "rstd");
  const float* w = floats(a.optional("weight"), x.cols, "weight");
  at::Tensor dx, dw, db;
  if (a.integer()) dx = make({x.rows, x.cols}, given.scalar_type(), a.device);
  if (a.integer()) dw = make({x.cols}, at::kFloat, a.device);
  if (a.integer()) db = make({x.cols}, at::kFloat, a.device);
  check(lib.layer_norm_bwd(a.ctx, dy.t.data_ptr(), dy.ld, x.t.data_ptr(), x.ld, x.dtype, x.rows, x.cols, w, mean, rstd,
                           dx.defined() ? dx.data_ptr() : nullptr, x.cols,
                           dw.defined() ? static_cast<float*>(dw.data_ptr()) : nullptr,
                           db.defined() ? static_cast<float*>(db.data_ptr()) : nullptr, stream_of(a.device)),
        "luq_layer_norm_bwd");
  return wrap(dx.defined() ? like(dx, given) : dx, dw, db);
}

at::Tensor new_codes(const Rows& x, int64_t device) {
  const int64_t ld = (x.cols + 15) / 16 * 16;
  const at::Tensor q = make({x.rows, ld}, at::kChar, device);
  return ld == x.cols ? q : q.narrow(1, 0, x.cols);
}

// layer_norm_int8(ctx, device, x, weight, bias, eps) -> codes, scale
PyObject* layer_norm_int8(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 6);
  const Rows x = rows_of(a.tensor("x"), "x");
  const float* w = floats(a.optional("weight"), x.cols, "weight");
  const float* b = floats(a.optional("bias"), x.cols, "bias");
  const float eps = a.real();
  const at::Tensor q = new_codes(x, a.device), s = make({x.rows}, at::kFloat, a.device);
  check(lib.layer_norm_int8(a.ctx, x.t.data_ptr(), x.dtype, x.rows, x.cols, x.ld, w, b, eps, static_cast<int8_t*>(q.data_ptr()),
                            (x.cols + 15) / 16 * 16, static_cast<float*>(s.data_ptr()), stream_of(a.device)),
        "luq_layer_norm_int8");
  return wrap(q, s);
}

// quant_int8_rows(ctx, device, x) -> codes, scale
PyObject* quant_int8_rows(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 3);
  const Rows x = rows_of(a.tensor("x"), "x");
  const at::Tensor q = new_codes(x, a.device), s = make({x.rows}, at::kFloat, a.device);
  check(lib.quant_int8_rows(a.ctx, x.t.data_ptr(), x.dtype, x.rows, x.cols, x.ld, static_cast<int8_t*>(q.data_ptr()),
                            (x.cols + 15) / 16 * 16, static_cast<float*>(s.data_ptr()), stream_of(a.device)),
        "luq_quant_int8_rows");
  return wrap(q, s);
}

// gemm_int8(ctx, device, codes, scale, w_codes, w_scale, bias, out, out_dtype) -> z; grouped: offsets after scale
template <bool GROUPED>
PyObject* gemm_int8(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, GROUPED ? 10 : 9);
  const at::Tensor& x = a.tensor("token codes");
  if (x.dim() != 2) type_error("token codes: [rows, K] expected");
  const int64_t M = x.size(0), K = x.size(1), ld_x = codes_ld(x, "token codes");
  const float* sx = floats(&a.tensor("scale"), M, "scale");
  const at::Tensor* offsets = GROUPED ? &a.tensor("offsets") : nullptr;
  const Weights w = weights_of(a.tensor("weight codes"), K, GROUPED);
  const float* sw = floats(&a.tensor("w_scale"), w.groups * w.N, "w_scale");
  const float* bias = floats(a.optional("bias"), w.groups * w.N, "bias");
  const at::Tensor* out = a.optional("out");
  const at::Tensor z = output(out, M, w.N, a.integer(), a.device);
  const int8_t* q = static_cast<const int8_t*>(x.data_ptr());
  if constexpr (GROUPED)
    check(lib.gemm_int8_grouped(a.ctx, q, ld_x, sx, offsets_of(*offsets, w.groups), static_cast<int>(w.groups), w.codes, w.ld,
                                w.stride, sw, bias, z.data_ptr(), dtype_code(z), row_stride(z), M, w.N, K, stream_of(a.device)),
          "luq_gemm_int8_grouped");
  else
    check(lib.gemm_int8(a.ctx, q, ld_x, sx, w.codes, w.ld, sw, bias, z.data_ptr(), dtype_code(z), row_stride(z), M, w.N, K,
                        stream_of(a.device)), "luq_gemm_int8");
  return wrap(z);
}

// the type of an output that the caller did not give: `code`, or (negative) that of x
int64_t type_or(int64_t code, const Rows& x) { return code < 0 ? x.dtype : code; }

// quant_int8_gemm(ctx, device, x, w_codes, w_scale, bias, out, out_dtype) -> z; grouped: offsets after x
template <bool GROUPED>
PyObject* quant_int8_gemm(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, GROUPED ? 9 : 8);
  const Rows x = rows_of(a.tensor("x"), "x");
  const at::Tensor* offsets = GROUPED ? &a.tensor("offsets") : nullptr;
  const Weights w = weights_of(a.tensor("weight codes"), x.cols, GROUPED);
  const float* sw = floats(&a.tensor("w_scale"), w.groups * w.N, "w_scale");
  const float* bias = floats(a.optional("bias"), w.groups * w.N, "bias");
  const at::Tensor* out = a.optional("out");
  const at::Tensor z = output(out, x.rows, w.N, type_or(a.integer(), x), a.device);
  if constexpr (GROUPED)
    check(lib.quant_int8_gemm_grouped(a.ctx, x.t.data_ptr(), x.dtype, x.ld, offsets_of(*offsets, w.groups),
                                      static_cast<int>(w.groups), w.codes, w.ld, w.stride, sw, bias, z.data_ptr(), dtype_code(z),
                                      row_stride(z), x.rows, w.N, x.cols, stream_of(a.device)), "luq_quant_int8_gemm_grouped");
  else
    check(lib.quant_int8_gemm(a.ctx, x.t.data_ptr(), x.dtype, x.ld, w.codes, w.ld, sw, bias, z.data_ptr(), dtype_code(z),
                              row_stride(z), x.rows, w.N, x.cols, stream_of(a.device)), "luq_quant_int8_gemm");
  return wrap(z);
}

// layer_norm_int8_gemm(ctx, device, x, weight, bias, eps, w_codes, w_scale, w_bias, out, out_dtype) -> z
PyObject* layer_norm_int8_gemm(PyObject* const* args, Py_ssize_t n) {
  Args a(args, n, 11);
  const Rows x = rows_of(a.tensor("x"), "x");
  const float* gamma = floats(a.optional("weight"), x.cols, "weight");
  const float* beta = floats(a.optional("bias"), x.cols, "bias");
  const float eps = a.real();
  const Weights w = weights_of(a.tensor("weight codes"), x.cols, false);
  const float* sw = floats(&a.tensor("w_scale"), w.N, "w_scale");
  const float* bias = floats(a.optional("w_bias"), w.N, "w_bias");
  const at::Tensor* out = a.optional("out");
  const at::Tensor z = output(out, x.rows, w.N, type_or(a.integer(), x), a.device);
  check(lib.layer_norm_int8_gemm(a.ctx, x.t.data_ptr(), x.dtype, x.ld, gamma, beta, eps, w.codes, w.ld, sw, bias, z.data_ptr(),
                                 dtype_code(z), row_stride(z), x.rows, w.N, x.cols, stream_of(a.device)),
        "luq_layer_norm_int8_gemm");
  return wrap(z);
}

// A call's workspace is torch's memory of the call's stream: calls on several streams, and graphs, each have their own.
void* workspace_alloc(void*, size_t bytes, void* stream) {
  try {
    return c10::cuda::CUDACachingAllocator::raw_alloc_with_stream(bytes, static_cast<cudaStream_t>(stream));
  } catch (...) {
    thrown = std::current_exception();
    return nullptr;
  }
}
void workspace_release(void*, void* ptr, void*) {
  try {
    c10::cuda::CUDACachingAllocator::raw_delete(ptr);
  } catch (...) {                                        // (the memory is lost, the call's results are there)
  }
}
// attach(ctx): a new context takes its workspaces from torch
PyObject* attach(PyObject* const* args, Py_ssize_t n) {
  if (n != 1) type_error("wrong number of arguments");
  luq_ctx* const ctx = static_cast<luq_ctx*>(PyLong_AsVoidPtr(args[0]));
  if (PyErr_Occurred()) throw Raised{};
  thrown = nullptr;
  check(lib.set_allocator(ctx, workspace_alloc, workspace_release, nullptr), "luq_set_allocator");
  return Py_NewRef(Py_None);
}

// bind(error class, addresses of the entry points in the order of Entry)
PyObject* bind(PyObject* const* args, Py_ssize_t n) {
  constexpr Py_ssize_t count = sizeof(Entry) / sizeof(void*);
  if (n != 1 + count) type_error("wrong number of arguments");
  void* at[count];
  for (Py_ssize_t i = 0; i < count; ++i) {
    at[i] = PyLong_AsVoidPtr(args[1 + i]);
    if (PyErr_Occurred()) throw Raised{};
  }
  std::memcpy(&lib, at, sizeof(lib));
  Py_XDECREF(error_class);
  error_class = Py_NewRef(args[0]);
  return Py_NewRef(Py_None);
}

#define CALL(name, body) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<body>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL("bind", bind),
                         CALL("attach", attach),
                         CALL("layer_norm", layer_norm),
                         CALL("layer_norm_bwd", layer_norm_bwd),
                         CALL("layer_norm_int8", layer_norm_int8),
                         CALL("quant_int8_rows", quant_int8_rows),
                         CALL("gemm_int8", gemm_int8<false>),
                         CALL("gemm_int8_grouped", gemm_int8<true>),
                         CALL("quant_int8_gemm", quant_int8_gemm<false>),
                         CALL("quant_int8_gemm_grouped", quant_int8_gemm<true>),
                         CALL("layer_norm_int8_gemm", layer_norm_int8_gemm),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Native argument handling of the 8-bit operators.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
