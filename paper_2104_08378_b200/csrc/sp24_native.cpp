// Native form of the binding's short calls (a Python extension module over torch's C++ API): argument marshalling, the
// allocation of the result, and the call of the C ABI.  For a small product the marshalling in Python costs more than the
// kernel takes (f16 256 x 256 x 512: 9.9 us of host time a call for 3.2 us on the device; 2.9 of it the allocation through
// torch's Python layer, 3 the marshalling, 1 ctypes, 3.1 the launch); here the call takes 4.5 us, 2.8 with the result given.
//
// Every function takes what the Python one has been given and returns None if anything about it is out of the ordinary
// (another type than a plain CUDA tensor, an active torch-function mode, a type or shape that the Python form rejects, no
// workspace yet, an exception from torch): the Python form then deals with the call from the start.  Otherwise it
// returns the result, or the status as an int if the library refused the call.  The interpreter lock is released around
// the allocation and the call, as torch and ctypes do.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "sp24.h"

namespace {

const at::ScalarType kScalar[7] = {at::kHalf, at::kBFloat16, at::kChar, at::kFloat, at::kInt, at::kFloat8_e4m3fn, at::kFloat8_e5m2};
const char* const kName[7] = {"f16", "bf16", "i8", "f32", "i32", "e4m3", "e5m2"};

// sp24_dtype of a torch type, of a type's name (-1: none)
int type_code(at::ScalarType t) {
  for (int i = 0; i < 7; ++i)
    if (kScalar[i] == t) return i;
  return -1;
}
int type_code(PyObject* name) {
  if (!PyUnicode_CheckExact(name)) return -1;
  for (int i = 0; i < 7; ++i)
    if (PyUnicode_CompareWithASCIIString(name, kName[i]) == 0) return i;
  return -1;
}

// A torch.Tensor itself (no subclass, no wrapper of a transform) in CUDA memory with at least `dims` dimensions, else null.
const at::Tensor* plain(PyObject* o, int64_t dims) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  const c10::DispatchKeySet keys = t.key_set();
  if (!t.is_cuda() || t.layout() != at::kStrided || t.dim() < dims || !t.has_storage() || t.is_conj() || t.is_neg() ||
      keys.has(c10::DispatchKey::Functionalize) || keys.has(c10::DispatchKey::Python))
    return nullptr;
  return &t;
}

// data_ptr() of an optional tensor; false: not an ordinary one
bool pointer(PyObject* o, const void** p) {
  if (o == Py_None) {
    *p = nullptr;
    return true;
  }
  const at::Tensor* t = plain(o, 0);
  if (t == nullptr) return false;
  *p = t->data_ptr();
  return true;
}

// an ordinary Python number
bool number(PyObject* o, double* v) {
  if (PyFloat_CheckExact(o)) {
    *v = PyFloat_AS_DOUBLE(o);
    return true;
  }
  return false;
}

struct Stream {
  cudaStream_t handle;
  Stream() : handle(c10::cuda::getCurrentCUDAStream().stream()) {}
};

// The workspace: the caller's, or the one kept for the device and stream.
bool workspace(PyObject* kept, PyObject* ws, const at::Tensor& a, cudaStream_t stream, void** p, size_t* bytes) {
  if (ws == Py_None) {
    PyObject* key = Py_BuildValue("(iN)", (int)a.get_device(), PyLong_FromUnsignedLongLong((unsigned long long)(uintptr_t)stream));
    if (key == nullptr) return false;
    ws = PyDict_GetItemWithError(kept, key);
    Py_DECREF(key);
    if (ws == nullptr) return false;
  }
  const at::Tensor* t = plain(ws, 0);
  if (t == nullptr) return false;
  *p = t->data_ptr();
  *bytes = (size_t)t->numel();
  return true;
}

PyObject* none() {
  PyErr_Clear();
  Py_RETURN_NONE;
}

// What the three products share: A, the result's type and place, C, the orders.
struct Product {
  const at::Tensor* a = nullptr;
  sp24_gemm_desc d = {};
  const void *meta = nullptr, *c = nullptr;
  void* ws = nullptr;
  size_t ws_bytes = 0;
  cudaStream_t stream = nullptr;
  bool cols = false;

  bool init(PyObject* A, PyObject* meta_, int ab, PyObject* cd, PyObject* dense, PyObject* b_rows, PyObject* cd_cols) {
    if (at::impl::torch_function_mode_enabled()) return false;
    a = plain(A, 2);
    if (a == nullptr || !pointer(meta_, &meta)) return false;
    if (ab < 0) ab = type_code(a->scalar_type());
    int out = cd == Py_None ? (ab == SP24_I8 ? SP24_I32 : (ab == SP24_E4M3 || ab == SP24_E5M2 ? SP24_BF16 : ab)) : type_code(cd);
    if (ab < 0 || out < 0) return false;
    cols = cd_cols == Py_True;
    if ((dense != Py_True && dense != Py_False) || (b_rows != Py_True && b_rows != Py_False) || (!cols && cd_cols != Py_False)) return false;
    d.ab_type = (sp24_dtype)ab;
    d.cd_type = (sp24_dtype)out;
    d.a_is_dense = dense == Py_True;
    d.M = a->size(0);
    d.K = d.a_is_dense ? a->size(1) : 2 * a->size(1);
    d.lda = a->stride(0);
    d.order_b = b_rows == Py_True ? SP24_ROW_MAJOR : SP24_COL_MAJOR;
    d.order_c = d.order_d = cols ? SP24_COL_MAJOR : SP24_ROW_MAJOR;
    return true;
  }
  // N and K are set: C, the workspace, and the call with the result's pointer
  template <typename Call>
  PyObject* run(PyObject* kept, PyObject* C, PyObject* out, PyObject* ws_, Call call) {
    d.ldc = cols ? d.M : d.N;
    if (C != Py_None) {
      const at::Tensor* t = plain(C, 1);
      if (t == nullptr) return none();
      d.ldc = t->stride(0);
      c = t->data_ptr();
    }
    stream = Stream().handle;
    if (!workspace(kept, ws_, *a, stream, &ws, &ws_bytes)) return none();
    const void* A = a->data_ptr();
    at::Tensor made;
    void* D = nullptr;
    if (out == Py_None) {
      d.ldd = cols ? d.M : d.N;
    } else {
      const at::Tensor* t = plain(out, 1);
      if (t == nullptr) return none();
      d.ldd = t->stride(0);
      D = t->data_ptr();
    }
    int status;
    {
      pybind11::gil_scoped_release unlocked;
      if (out == Py_None) {
        made = at::empty({cols ? d.N : d.M, cols ? d.M : d.N}, a->options().dtype(kScalar[d.cd_type]));
        if (d.ldd < 1) d.ldd = 1;  // (as torch reports the stride of an empty tensor)
        D = made.data_ptr();
      }
      status = call(*this, A, D);
    }
    if (status != SP24_OK) return PyLong_FromLong(status);
    if (out == Py_None) return THPVariable_Wrap(std::move(made));
    Py_INCREF(out);
    return out;
  }
};

template <typename F>
F function(PyObject* address) {
  return reinterpret_cast<F>(PyLong_AsVoidPtr(address));
}

// gemm(address, workspaces, A, meta, Bt, alpha, beta, C, out, cd, a_is_dense, ws, b_row_major, cd_col_major)
PyObject* gemm(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 14) return none();
  try {
    Product p;
    double alpha, beta;
    if (!p.init(v[2], v[3], -1, v[9], v[10], v[12], v[13])) return none();
    const at::Tensor* b = plain(v[4], 2);
    if (b == nullptr || !number(v[5], &alpha)) return none();
    if (PyLong_CheckExact(v[6]) && p.d.ab_type == SP24_I8) beta = (double)PyLong_AsLong(v[6]);
    else if (!number(v[6], &beta)) return none();
    const bool rows = p.d.order_b == SP24_ROW_MAJOR, whole = p.d.ab_type == SP24_I8;
    if (b->size(rows ? 0 : 1) != p.d.K) return none();
    if (whole && (alpha != 1.0 || (beta != 0.0 && beta != 1.0))) return none();
    p.d.N = b->size(rows ? 1 : 0);
    p.d.ldb = b->stride(0);
    const void* B = b->data_ptr();
    const auto fn = function<decltype(&sp24_gemm)>(v[0]);
    return p.run(v[1], v[7], v[8], v[11], [&](const Product& q, const void* A, void* D) {
      const float fa = (float)alpha, fb = (float)beta;
      const int32_t ia = 1, ib = (int32_t)(whole ? beta : 0.0);
      return (int)fn(&q.d, whole ? (const void*)&ia : &fa, A, q.meta, B, whole ? (const void*)&ib : &fb, q.c, D, q.ws, q.ws_bytes, q.stream);
    });
  } catch (...) {
    return none();
  }
}

// gemm_i8_dequant(address, workspaces, A, meta, Bt, row_scale, bias, relu, out_scale, cd, out, a_is_dense, ws, b_row_major,
// cd_col_major)
PyObject* gemm_i8_dequant(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 15) return none();
  try {
    Product p;
    double out_scale;
    if (v[9] == Py_None || !p.init(v[2], v[3], SP24_I8, v[9], v[11], v[13], v[14])) return none();
    const at::Tensor* b = plain(v[4], 2);
    const void *scale, *bias;
    if (b == nullptr || !pointer(v[5], &scale) || !pointer(v[6], &bias) || !number(v[8], &out_scale)) return none();
    const int relu = PyObject_IsTrue(v[7]);
    if (relu < 0) return none();
    p.d.N = b->size(p.d.order_b == SP24_ROW_MAJOR ? 1 : 0);
    p.d.ldb = b->stride(0);
    const void* B = b->data_ptr();
    const auto fn = function<decltype(&sp24_gemm_i8_dequant)>(v[0]);
    return p.run(v[1], Py_None, v[10], v[12], [&](const Product& q, const void* A, void* D) {
      return (int)fn(&q.d, A, q.meta, B, (const float*)scale, (const float*)bias, relu, (float)out_scale, D, q.ws, q.ws_bytes, q.stream);
    });
  } catch (...) {
    return none();
  }
}

// conv3x3_nhwc(address, workspaces, A, meta, x, alpha, beta, C, out, cd, a_is_dense, ws, nhwc_out)
PyObject* conv3x3_nhwc(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 13) return none();
  try {
    Product p;
    double alpha, beta;
    if (!p.init(v[2], v[3], -1, v[9], v[10], Py_False, v[12])) return none();
    const at::Tensor* x = plain(v[4], 4);
    if (x == nullptr || x->dim() != 4 || p.d.ab_type == SP24_I8 || !number(v[5], &alpha) || !number(v[6], &beta)) return none();
    const int64_t nb = x->size(0), h = x->size(1), w = x->size(2), cin = x->size(3);
    p.d.K = p.d.ldb = 9 * cin;
    p.d.N = nb * h * w;
    const void* X = x->data_ptr();
    const auto fn = function<decltype(&sp24_conv3x3_nhwc)>(v[0]);
    return p.run(v[1], v[7], v[8], v[11], [&](const Product& q, const void* A, void* D) {
      const float fa = (float)alpha, fb = (float)beta;
      return (int)fn(&q.d, nb, h, w, cin, &fa, A, q.meta, X, &fb, q.c, D, q.ws, q.ws_bytes, q.stream);
    });
  } catch (...) {
    return none();
  }
}

// compress(address, address of sp24_meta_bytes, x, layout) -> (vals, meta, None)
PyObject* compress(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 4 || !PyLong_CheckExact(v[3]) || at::impl::torch_function_mode_enabled()) return none();
  try {
    const at::Tensor* x = plain(v[2], 2);
    if (x == nullptr || x->dim() != 2) return none();
    const int dt = type_code(x->scalar_type());
    const long layout = PyLong_AsLong(v[3]);
    if (dt < 0 || (layout != 0 && layout != 1)) return none();
    const int64_t M = x->size(0), K = x->size(1);
    const auto fn = function<decltype(&sp24_compress)>(v[0]);
    const auto bytes = function<decltype(&sp24_meta_bytes)>(v[1]);
    const cudaStream_t stream = Stream().handle;
    const void* X = x->data_ptr();
    at::Tensor vals, meta;
    int status;
    {
      pybind11::gil_scoped_release unlocked;
      vals = at::empty({M, K / 2}, x->options());
      meta = at::empty({(int64_t)bytes((sp24_dtype)dt, M, K, (sp24_meta_layout)layout)}, x->options().dtype(at::kByte));
      status = (int)fn((sp24_dtype)dt, M, K, X, M > 1 ? x->stride(0) : K, vals.data_ptr(), K / 2, meta.data_ptr(),
                       (sp24_meta_layout)layout, nullptr, stream);
    }
    if (status != SP24_OK) return PyLong_FromLong(status);
    return Py_BuildValue("(NNO)", THPVariable_Wrap(std::move(vals)), THPVariable_Wrap(std::move(meta)), Py_None);
  } catch (...) {
    return none();
  }
}

// apply_mask(address, w, meta, layout, out) -> out
PyObject* apply_mask(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 5 || !PyLong_CheckExact(v[3]) || at::impl::torch_function_mode_enabled()) return none();
  try {
    const at::Tensor *w = plain(v[1], 2), *out = plain(v[4], 1);
    const void* meta;
    if (w == nullptr || w->dim() != 2 || out == nullptr || !pointer(v[2], &meta)) return none();
    const int dt = type_code(w->scalar_type());
    const long layout = PyLong_AsLong(v[3]);
    if (dt < 0 || (layout != 0 && layout != 1)) return none();
    const int64_t M = w->size(0), K = w->size(1);
    const auto fn = function<decltype(&sp24_apply_mask)>(v[0]);
    const cudaStream_t stream = Stream().handle;
    const void* W = w->data_ptr();
    void* Y = out->data_ptr();
    const int64_t ldw = M > 1 ? w->stride(0) : K, ldy = M > 1 ? out->stride(0) : K;
    int status;
    {
      pybind11::gil_scoped_release unlocked;
      status = (int)fn((sp24_dtype)dt, M, K, W, ldw, meta, (sp24_meta_layout)layout, Y, ldy, stream);
    }
    if (status != SP24_OK) return PyLong_FromLong(status);
    Py_INCREF(v[4]);
    return v[4];
  } catch (...) {
    return none();
  }
}

// ---- the operators around the products: as the Python forms check and call them -----------------------------------------
// A matrix with contiguous rows on the current device, of the sizes and type given (-1: any); false: not an ordinary one.
struct Matrix {
  const at::Tensor* t = nullptr;
  void* p = nullptr;
  int64_t ld = 0;
  bool init(PyObject* o, int64_t rows, int64_t cols, int type) {
    t = plain(o, 2);
    if (t == nullptr || t->dim() != 2 || t->get_device() != c10::cuda::current_device()) return false;
    if ((rows >= 0 && (t->size(0) != rows || t->size(1) != cols)) || (type >= 0 && t->scalar_type() != kScalar[type])) return false;
    if (t->size(1) > 1 && t->stride(1) != 1) return false;
    ld = t->size(0) > 1 ? t->stride(0) : (t->size(1) > 1 ? t->size(1) : 1);
    p = t->data_ptr();
    return true;
  }
};
// The same for a contiguous vector, or None; *type (if asked for): which of the two types it has.
bool vector(PyObject* o, int64_t n, int type_a, int type_b, const void** p, int* type = nullptr) {
  *p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = plain(o, 1);
  if (t == nullptr || t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1) || t->get_device() != c10::cuda::current_device()) return false;
  const int code = type_code(t->scalar_type());
  if (code != type_a && code != type_b) return false;
  if (type) *type = code;
  *p = t->data_ptr();
  return true;
}
bool float_type(int code) { return code == SP24_F16 || code == SP24_BF16 || code == SP24_F32; }
// 8-bit type of a name, `otherwise` for None, -1: no such type
int quant_code(PyObject* name, int otherwise) {
  if (name == Py_None) return otherwise;
  const int code = type_code(name);
  return code == SP24_I8 || code == SP24_E4M3 || code == SP24_E5M2 ? code : -1;
}
int act_code(PyObject* name) {
  static const char* const names[5] = {nullptr, "relu", "gelu", "silu", "gelu_tanh"};
  if (name == Py_None) return SP24_ACT_NONE;
  if (!PyUnicode_CheckExact(name)) return -1;
  for (int i = 1; i < 5; ++i)
    if (PyUnicode_CompareWithASCIIString(name, names[i]) == 0) return i;
  return -1;
}
// A given result (its checks passed), or the tensor made for it
struct Result {
  PyObject* given;
  at::Tensor made;
  PyObject* object() {
    if (given != Py_None) {
      Py_INCREF(given);
      return given;
    }
    return made.defined() ? THPVariable_Wrap(std::move(made)) : Py_NewRef(Py_None);
  }
};
// (What makes and calls without the interpreter's lock: a Python error is none of its possible outcomes.)
template <typename Call>
int unlocked(Call call) {
  pybind11::gil_scoped_release go;
  return (int)call();
}

// rms_norm(address, x, weight, eps, residual, quant, with_rstd, h_out, out) -> (y, h, scale, rstd)
PyObject* rms_norm(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 9 || at::impl::torch_function_mode_enabled()) return none();
  try {
    Matrix x, r, h, y;
    double eps;
    if (!x.init(v[1], -1, -1, -1) || !number(v[3], &eps) || (v[6] != Py_True && v[6] != Py_False)) return none();
    const int t = type_code(x.t->scalar_type()), out = quant_code(v[5], t);
    const int64_t rows = x.t->size(0), K = x.t->size(1);
    const void* weight;
    int weight_type = SP24_F32;
    if (!float_type(t) || out < 0 || !vector(v[2], K, t, SP24_F32, &weight, &weight_type)) return none();
    if (v[4] != Py_None ? !r.init(v[4], rows, K, t) : v[7] != Py_None) return none();
    if ((v[7] != Py_None && !h.init(v[7], rows, K, t)) || (v[8] != Py_None && !y.init(v[8], rows, K, out))) return none();
    const auto fn = function<decltype(&sp24_rms_norm)>(v[0]);
    const cudaStream_t stream = Stream().handle;
    const int64_t packed = rows > 1 && K > 1 ? K : (K > 1 ? K : 1);
    Result ry{v[8], {}}, rh{v[7], {}};
    at::Tensor scale, rstd;
    const int status = unlocked([&] {
      const auto options = x.t->options();
      if (v[4] != Py_None && v[7] == Py_None) {
        rh.made = at::empty({rows, K}, options);
        h.p = rh.made.data_ptr();
        h.ld = packed;
      }
      if (v[8] == Py_None) {
        ry.made = at::empty({rows, K}, options.dtype(kScalar[out]));
        y.p = ry.made.data_ptr();
        y.ld = packed;
      }
      if (out != t) scale = at::empty({rows}, options.dtype(at::kFloat));
      if (v[6] == Py_True) rstd = at::empty({rows}, options.dtype(at::kFloat));
      return fn((sp24_dtype)t, rows, K, x.p, x.ld, r.p, r.ld, weight, (sp24_dtype)weight_type, (float)eps, h.p, h.ld, (sp24_dtype)out, y.p, y.ld,
                scale.defined() ? (float*)scale.data_ptr() : nullptr, rstd.defined() ? (float*)rstd.data_ptr() : nullptr, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    Result rs{Py_None, std::move(scale)}, rr{Py_None, std::move(rstd)};
    return Py_BuildValue("(NNNN)", ry.object(), rh.object(), rs.object(), rr.object());
  } catch (...) {
    return none();
  }
}

// rms_norm_backward(address, address of the workspace's size, dy, h, weight, rstd, dh, out) -> (dx, dweight)
PyObject* rms_norm_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 8 || v[5] == Py_None || at::impl::torch_function_mode_enabled()) return none();
  try {
    Matrix dy, h, dh, dx;
    if (!dy.init(v[2], -1, -1, -1)) return none();
    const int t = type_code(dy.t->scalar_type());
    const int64_t rows = dy.t->size(0), K = dy.t->size(1);
    const void *weight, *rstd;
    int weight_type = SP24_F32;
    if (!float_type(t) || !h.init(v[3], rows, K, t) || !vector(v[4], K, t, SP24_F32, &weight, &weight_type) ||
        !vector(v[5], rows, SP24_F32, SP24_F32, &rstd))
      return none();
    if ((v[6] != Py_None && !dh.init(v[6], rows, K, t)) || (v[7] != Py_None && !dx.init(v[7], rows, K, t))) return none();
    const auto fn = function<decltype(&sp24_rms_norm_backward)>(v[0]);
    const auto size = function<decltype(&sp24_rms_norm_backward_workspace_bytes)>(v[1]);
    const cudaStream_t stream = Stream().handle;
    Result rdx{v[7], {}}, rdw{Py_None, {}};
    const int status = unlocked([&] {
      const auto options = dy.t->options();
      if (v[7] == Py_None) {
        rdx.made = at::empty({rows, K}, options);
        dx.p = rdx.made.data_ptr();
        dx.ld = K > 1 ? K : 1;
      }
      at::Tensor ws;
      size_t bytes = 0;
      if (v[4] != Py_None) {
        rdw.made = at::empty({K}, options.dtype(at::kFloat));
        bytes = size(rows, K);
        ws = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
      }
      return fn((sp24_dtype)t, rows, K, dy.p, dy.ld, h.p, h.ld, weight, (sp24_dtype)weight_type, (const float*)rstd, dh.p, dh.ld, dx.p, dx.ld,
                rdw.made.defined() ? (float*)rdw.made.data_ptr() : nullptr, ws.defined() ? ws.data_ptr() : nullptr, bytes, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return Py_BuildValue("(NN)", rdx.object(), rdw.object());
  } catch (...) {
    return none();
  }
}

// gated_act(address, g, u, act, quant, out) -> (y, scale)
PyObject* gated_act(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 6 || at::impl::torch_function_mode_enabled()) return none();
  try {
    Matrix g, u, y;
    if (!g.init(v[1], -1, -1, -1)) return none();
    const int t = type_code(g.t->scalar_type()), act = act_code(v[3]), out = quant_code(v[4], t);
    const int64_t rows = g.t->size(0), F = g.t->size(1);
    if (!float_type(t) || act < 0 || out < 0 || (v[2] != Py_None && !u.init(v[2], rows, F, t)) || (v[5] != Py_None && !y.init(v[5], rows, F, out)))
      return none();
    const auto fn = function<decltype(&sp24_gated_act)>(v[0]);
    const cudaStream_t stream = Stream().handle;
    Result ry{v[5], {}}, rs{Py_None, {}};
    const int status = unlocked([&] {
      const auto options = g.t->options();
      if (v[5] == Py_None) {
        ry.made = at::empty({rows, F}, options.dtype(kScalar[out]));
        y.p = ry.made.data_ptr();
        y.ld = F > 1 ? F : 1;
      }
      if (out != t) rs.made = at::empty({rows}, options.dtype(at::kFloat));
      return fn((sp24_dtype)t, (sp24_act)act, rows, F, g.p, g.ld, u.p, u.ld, (sp24_dtype)out, y.p, y.ld,
                rs.made.defined() ? (float*)rs.made.data_ptr() : nullptr, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return Py_BuildValue("(NN)", ry.object(), rs.object());
  } catch (...) {
    return none();
  }
}

// gated_act_backward(address, dy, g, u, act, dg, du) -> (dg, du)
PyObject* gated_act_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 7 || at::impl::torch_function_mode_enabled()) return none();
  try {
    Matrix dy, g, u, dg, du;
    if (!dy.init(v[1], -1, -1, -1)) return none();
    const int t = type_code(dy.t->scalar_type()), act = act_code(v[4]);
    const int64_t rows = dy.t->size(0), F = dy.t->size(1);
    if (!float_type(t) || act < 0 || !g.init(v[2], rows, F, t) || (v[3] != Py_None ? !u.init(v[3], rows, F, t) : v[6] != Py_None)) return none();
    if ((v[5] != Py_None && !dg.init(v[5], rows, F, t)) || (v[6] != Py_None && !du.init(v[6], rows, F, t))) return none();
    const auto fn = function<decltype(&sp24_gated_act_backward)>(v[0]);
    const cudaStream_t stream = Stream().handle;
    Result rdg{v[5], {}}, rdu{v[6], {}};
    const int status = unlocked([&] {
      auto make = [&](Result& r, Matrix& m) {
        r.made = at::empty({rows, F}, dy.t->options());
        m.p = r.made.data_ptr();
        m.ld = F > 1 ? F : 1;
      };
      if (v[5] == Py_None) make(rdg, dg);
      if (v[3] != Py_None && v[6] == Py_None) make(rdu, du);
      return fn((sp24_dtype)t, (sp24_act)act, rows, F, dy.p, dy.ld, g.p, g.ld, u.p, u.ld, dg.p, dg.ld, du.p, du.ld, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return Py_BuildValue("(NN)", rdg.object(), rdu.object());
  } catch (...) {
    return none();
  }
}

// act_backward(address, address of the workspace's size, dy, pre, act, cd_col_major, transposed, bias, out) -> (dz, dzt, dbias)
PyObject* act_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 9 || at::impl::torch_function_mode_enabled()) return none();
  try {
    for (int i = 5; i < 8; ++i)
      if (v[i] != Py_True && v[i] != Py_False) return none();
    Matrix dy, z, dz;
    const int act = act_code(v[4]);
    if (act < 0 || !dy.init(v[2], -1, -1, -1)) return none();
    const int t = type_code(dy.t->scalar_type());
    const int64_t rows = dy.t->size(0), cols = dy.t->size(1);
    if (!float_type(t)) return none();
    if ((act != SP24_ACT_NONE && !z.init(v[3], rows, cols, t)) || (v[8] != Py_None && !dz.init(v[8], rows, cols, t))) return none();
    const int over_rows = v[5] == Py_True;
    const auto fn = function<decltype(&sp24_act_backward)>(v[0]);
    const auto size = function<decltype(&sp24_act_backward_workspace_bytes)>(v[1]);
    const cudaStream_t stream = Stream().handle;
    Result rdz{act == SP24_ACT_NONE && v[8] == Py_None ? v[2] : v[8], {}}, rdzt{Py_None, {}}, rdb{Py_None, {}};
    const int status = unlocked([&] {
      const auto options = dy.t->options();
      if (act != SP24_ACT_NONE && v[8] == Py_None) {
        rdz.made = at::empty({rows, cols}, options);
        dz.p = rdz.made.data_ptr();
        dz.ld = cols > 1 ? cols : 1;
      }
      if (v[6] == Py_True) rdzt.made = at::empty({cols, rows}, options);
      at::Tensor ws;
      size_t bytes = 0;
      if (v[7] == Py_True) {
        rdb.made = at::empty({over_rows ? cols : rows}, options.dtype(at::kFloat));
        bytes = size(rows, cols, over_rows);
        ws = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
      }
      return fn((sp24_dtype)t, (sp24_act)act, rows, cols, dy.p, dy.ld, z.p, z.ld, dz.p, dz.ld, rdzt.made.defined() ? rdzt.made.data_ptr() : nullptr,
                rows > 1 ? rows : 1, rdb.made.defined() ? (float*)rdb.made.data_ptr() : nullptr, over_rows, ws.defined() ? ws.data_ptr() : nullptr, bytes, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return Py_BuildValue("(NNN)", rdz.object(), rdzt.object(), rdb.object());
  } catch (...) {
    return none();
  }
}

// linear(address, workspaces, address of sp24_meta_bytes, A, meta, Bt, bias, act, residual, row_scale, col_scale, pre, out, cd, a_is_dense, b_row_major,
// cd_col_major, ws) -> D or (D, pre)
PyObject* linear(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 18) return none();
  try {
    Product p;
    Matrix a, b, r, z, d;
    if (!a.init(v[3], -1, -1, -1)) return none();
    const int ab = type_code(a.t->scalar_type()), act = act_code(v[7]);
    PyObject* bf16 = nullptr;  // (Product takes INT32 results of int8 operands where none is named)
    if (v[13] == Py_None && ab == SP24_I8 && (bf16 = PyUnicode_FromString("bf16")) == nullptr) return none();
    const bool ok = ab >= 0 && ab != SP24_I32 && act >= 0 && p.init(v[3], v[4], -1, bf16 ? bf16 : v[13], v[14], v[15], v[16]);
    Py_XDECREF(bf16);
    if (!ok || !b.init(v[5], -1, -1, ab)) return none();
    p.d.lda = a.ld;
    p.d.ldb = b.ld;
    const bool b_rows = p.d.order_b == SP24_ROW_MAJOR;
    if (b.t->size(b_rows ? 0 : 1) != p.d.K) return none();
    p.d.N = b.t->size(b_rows ? 1 : 0);
    const auto bytes = function<decltype(&sp24_meta_bytes)>(v[2]);
    const void* meta = nullptr;
    if (!p.d.a_is_dense) {
      const at::Tensor* m = plain(v[4], 1);
      if (m == nullptr || m->dim() != 1 || m->scalar_type() != at::kByte || (m->size(0) > 1 && m->stride(0) != 1) ||
          m->get_device() != c10::cuda::current_device() || (size_t)m->size(0) != bytes((sp24_dtype)ab, p.d.M, p.d.K, SP24_META_TCGEN05))
        return none();
      meta = m->data_ptr();
    }
    const int64_t rows = p.cols ? p.d.N : p.d.M, cols = p.cols ? p.d.M : p.d.N;
    const int cd = (int)p.d.cd_type;
    sp24_linear_epilogue e = {};
    e.act = (sp24_act)act;
    if (!vector(v[6], p.d.M, SP24_F32, SP24_F32, (const void**)&e.bias) || !vector(v[9], p.d.M, SP24_F32, SP24_F32, (const void**)&e.row_scale) ||
        !vector(v[10], p.d.N, SP24_F32, SP24_F32, (const void**)&e.col_scale))
      return none();
    if (v[8] != Py_None && !r.init(v[8], rows, cols, cd)) return none();
    const bool make_pre = v[11] == Py_True, no_pre = v[11] == Py_False || v[11] == Py_None;
    if (!make_pre && !no_pre && !z.init(v[11], rows, cols, cd)) return none();
    if (v[12] != Py_None && !d.init(v[12], rows, cols, cd)) return none();
    p.stream = Stream().handle;
    if (!workspace(v[1], v[17], *a.t, p.stream, &p.ws, &p.ws_bytes)) return none();
    const auto fn = function<decltype(&sp24_linear)>(v[0]);
    Result rd{v[12], {}}, rz{make_pre || no_pre ? Py_None : v[11], {}};
    const int status = unlocked([&] {
      auto make = [&](Result& to, Matrix& m) {
        to.made = at::empty({rows, cols}, a.t->options().dtype(kScalar[cd]));
        m.p = to.made.data_ptr();
        m.ld = cols > 1 ? cols : 1;
      };
      if (v[12] == Py_None) make(rd, d);
      if (make_pre) make(rz, z);
      p.d.ldd = d.ld;
      p.d.ldc = r.p || v[8] != Py_None ? r.ld : d.ld;
      e.residual = r.p;
      e.pre = z.p;
      e.ld_pre = z.ld;
      return fn(&p.d, &e, a.p, meta, b.p, d.p, p.ws, p.ws_bytes, p.stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    if (no_pre) return rd.object();
    return Py_BuildValue("(NN)", rd.object(), rz.object());
  } catch (...) {
    return none();
  }
}

// linear_backward(addresses of sp24_act_backward, of its workspace's size, of sp24_gemm, of sp24_meta_bytes, of sp24_apply_mask, workspaces, dy, pre, Bt, W, act,
// meta, b_row_major, cd_col_major, ws) -> (dBt, dW, dbias)
PyObject* linear_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 15 || at::impl::torch_function_mode_enabled()) return none();
  try {
    for (int i = 12; i < 14; ++i)
      if (v[i] != Py_True && v[i] != Py_False) return none();
    Matrix dy, z, b, w;
    const int act = act_code(v[10]);
    if (act < 0 || !dy.init(v[6], -1, -1, -1)) return none();
    const int t = type_code(dy.t->scalar_type());
    if (!float_type(t) || !w.init(v[9], -1, -1, t) || !b.init(v[8], -1, -1, t)) return none();
    const bool b_rows = v[12] == Py_True, cols_out = v[13] == Py_True;
    const int64_t M = w.t->size(0), K = w.t->size(1), N = b.t->size(b_rows ? 1 : 0);
    const int64_t rows = dy.t->size(0), cols = dy.t->size(1);
    if (b.t->size(b_rows ? 0 : 1) != K || rows != (cols_out ? N : M) || cols != (cols_out ? M : N) || M % 16 || N % 16 || K % 16 || M == 0 || N == 0 || K == 0)
      return none();
    if (act != SP24_ACT_NONE && !z.init(v[7], rows, cols, t)) return none();
    const void* meta = nullptr;
    if (v[11] != Py_None) {
      const at::Tensor* m = plain(v[11], 1);
      if (t == SP24_F32 || m == nullptr || m->dim() != 1 || m->scalar_type() != at::kByte || (m->size(0) > 1 && m->stride(0) != 1) ||
          m->get_device() != c10::cuda::current_device() ||
          (size_t)m->size(0) != function<decltype(&sp24_meta_bytes)>(v[3])((sp24_dtype)t, M, K, SP24_META_TCGEN05))
        return none();
      meta = m->data_ptr();
    }
    const cudaStream_t stream = Stream().handle;
    void* ws;
    size_t ws_bytes;
    if (!workspace(v[5], v[14], *dy.t, stream, &ws, &ws_bytes)) return none();
    const auto act_fn = function<decltype(&sp24_act_backward)>(v[0]);
    const auto act_bytes = function<decltype(&sp24_act_backward_workspace_bytes)>(v[1]);
    const auto gemm_fn = function<decltype(&sp24_gemm)>(v[2]);
    const auto mask_fn = function<decltype(&sp24_apply_mask)>(v[4]);
    Result rx{Py_None, {}}, rw{Py_None, {}}, rb{Py_None, {}};
    const int status = unlocked([&]() -> int {
      const auto options = dy.t->options();
      // dz (without an activation dy itself, where a product can take it), its transpose and the partial sums of the bias's gradient, in one allocation
      const bool makes_dz = act != SP24_ACT_NONE || (uintptr_t)dy.p % 16 != 0 || dy.ld * dy.t->element_size() % 16 != 0;
      const size_t bytes = act_bytes(rows, cols, cols_out), matrix = ((size_t)rows * cols * dy.t->element_size() + 255) / 256 * 256;
      const at::Tensor scratch = at::empty({(int64_t)(matrix * (makes_dz ? 2 : 1) + bytes)}, options.dtype(at::kByte));
      char* const pdzt = (char*)scratch.data_ptr();
      void* const sums = pdzt + matrix * (makes_dz ? 2 : 1);
      void* const pdz = makes_dz ? pdzt + matrix : dy.p;
      const int64_t lddz = makes_dz ? cols : dy.ld;
      rb.made = at::empty({M}, options.dtype(at::kFloat));
      int st = act_fn((sp24_dtype)t, (sp24_act)act, rows, cols, dy.p, dy.ld, z.p, z.ld, makes_dz ? pdz : nullptr, lddz, pdzt, rows,
                      (float*)rb.made.data_ptr(), cols_out, sums, bytes, stream);
      if (st != SP24_OK) return st;
      rx.made = at::empty({b.t->size(0), b.t->size(1)}, options);
      rw.made = at::empty({M, K}, options);
      const float one = 1.f, zero = 0.f;
      // D = A B of dense A (rows_ x inner), B by rows if `by_rows`
      auto product = [&](const void* A, int64_t lda, int64_t m, int64_t n_, int64_t inner, const void* B, int64_t ldb, bool by_rows, void* D, bool cols_) {
        const sp24_order order = cols_ ? SP24_COL_MAJOR : SP24_ROW_MAJOR;
        const int64_t ldd = cols_ ? m : n_;
        const sp24_gemm_desc d = {(sp24_dtype)t, (sp24_dtype)t, m, n_, inner, lda, ldb, ldd, ldd, by_rows ? SP24_ROW_MAJOR : SP24_COL_MAJOR, order, order, 1};
        return (int)gemm_fn(&d, &one, A, nullptr, B, &zero, nullptr, D, ws, ws_bytes, stream);
      };
      const void *tokens = cols_out ? pdz : pdzt, *features = cols_out ? pdzt : pdz;  // N x M, M x N
      const int64_t ld_tokens = cols_out ? lddz : rows, ld_features = cols_out ? rows : lddz;
      st = product(tokens, ld_tokens, N, K, M, w.p, w.ld, true, rx.made.data_ptr(), b_rows);
      if (st != SP24_OK) return st;
      st = product(features, ld_features, M, K, N, b.p, b.ld, !b_rows, rw.made.data_ptr(), false);
      if (st != SP24_OK || meta == nullptr) return st;
      return (int)mask_fn((sp24_dtype)t, M, K, rw.made.data_ptr(), K, meta, SP24_META_TCGEN05, rw.made.data_ptr(), K, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return Py_BuildValue("(NNN)", rx.object(), rw.object(), rb.object());
  } catch (...) {
    return none();
  }
}

// ---- experts ------------------------------------------------------------------------------------------------------------
// A contiguous [T, k] of the type on the current device (T or k < 0: any)
struct Slots {
  const at::Tensor* t = nullptr;
  void* p = nullptr;
  int64_t T = 0, k = 0;
  bool init(PyObject* o, int64_t rows, int64_t cols, at::ScalarType type) {
    t = plain(o, 2);
    if (t == nullptr || t->dim() != 2 || t->scalar_type() != type || t->get_device() != c10::cuda::current_device() || !t->is_contiguous()) return false;
    T = t->size(0);
    k = t->size(1);
    if ((rows >= 0 && T != rows) || (cols >= 0 && k != cols)) return false;
    p = t->data_ptr();
    return true;
  }
};
bool whole(PyObject* o, int64_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  *v = PyLong_AsLongLongAndOverflow(o, &over);
  return over == 0;
}
bool truth(PyObject* o, int* v) {
  *v = o == Py_True;
  return o == Py_True || o == Py_False;
}
int one_of(PyObject* name, const char* zero, const char* one) {
  if (!PyUnicode_CheckExact(name)) return -1;
  return PyUnicode_CompareWithASCIIString(name, zero) == 0 ? 0 : PyUnicode_CompareWithASCIIString(name, one) == 0 ? 1 : -1;
}
// [E, M, columns]: matrices with contiguous rows one after the other
struct Stack {
  const at::Tensor* t = nullptr;
  void* p = nullptr;
  int64_t E = 0, M = 0, n = 0, ld = 0;
  bool init(PyObject* o, int type) {
    t = plain(o, 3);
    if (t == nullptr || t->dim() != 3 || t->get_device() != c10::cuda::current_device() || (type >= 0 && t->scalar_type() != kScalar[type])) return false;
    E = t->size(0);
    M = t->size(1);
    n = t->size(2);
    if (E < 1 || M < 2 || n < 2 || t->stride(2) != 1 || (E > 1 && t->stride(0) != M * t->stride(1))) return false;
    ld = t->stride(1);
    p = t->data_ptr();
    return true;
  }
};

// route(address, logits, k, score, bias, groups, top_groups, group_score, renorm, scale) -> (weights, experts)
PyObject* route(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 10 || at::impl::torch_function_mode_enabled()) return none();
  try {
    Matrix x;
    int64_t k, groups, top;
    int renorm;
    double scale;
    if (!x.init(v[1], -1, -1, -1) || !whole(v[2], &k) || !whole(v[5], &groups) || !truth(v[8], &renorm) || !number(v[9], &scale)) return none();
    if (v[6] == Py_None) top = groups;
    else if (!whole(v[6], &top)) return none();
    const int t = type_code(x.t->scalar_type()), score = one_of(v[3], "softmax", "sigmoid"), by = one_of(v[7], "max", "top2");
    const int64_t T = x.t->size(0), E = x.t->size(1);
    const void* bias;
    if (!float_type(t) || score < 0 || by < 0 || !vector(v[4], E, SP24_F32, SP24_F32, &bias) || k < 1 || k > E || groups < 1 || groups > E || top < 1 || top > groups)
      return none();
    const auto fn = function<decltype(&sp24_route)>(v[0]);
    const cudaStream_t stream = Stream().handle;
    at::Tensor weights, experts;
    const int status = unlocked([&] {
      weights = at::empty({T, k}, x.t->options().dtype(at::kFloat));
      experts = at::empty({T, k}, x.t->options().dtype(at::kInt));
      return fn((sp24_dtype)t, T, E, x.p, x.ld, (sp24_score)score, (const float*)bias, (int)groups, (int)top, (sp24_group_score)by, (int)k, renorm, (float)scale,
                (float*)weights.data_ptr(), (int32_t*)experts.data_ptr(), stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(weights)), THPVariable_Wrap(std::move(experts)));
  } catch (...) {
    return none();
  }
}

// route_backward(address, dweights, logits, experts, score, renorm, scale, out) -> dlogits
PyObject* route_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 8 || at::impl::torch_function_mode_enabled()) return none();
  try {
    Matrix x, d;
    Slots g, e;
    int renorm;
    double scale;
    if (!x.init(v[2], -1, -1, -1) || !truth(v[5], &renorm) || !number(v[6], &scale)) return none();
    const int t = type_code(x.t->scalar_type()), score = one_of(v[4], "softmax", "sigmoid");
    const int64_t T = x.t->size(0), E = x.t->size(1);
    if (!float_type(t) || score < 0 || !e.init(v[3], T, -1, at::kInt) || !g.init(v[1], T, e.k, at::kFloat) || (v[7] != Py_None && !d.init(v[7], T, E, t)))
      return none();
    const auto fn = function<decltype(&sp24_route_backward)>(v[0]);
    const cudaStream_t stream = Stream().handle;
    Result rd{v[7], {}};
    const int status = unlocked([&] {
      if (v[7] == Py_None) {
        rd.made = at::empty({T, E}, x.t->options());
        d.p = rd.made.data_ptr();
        d.ld = E > 1 ? E : 1;
      }
      return fn((sp24_dtype)t, T, E, (const float*)g.p, x.p, x.ld, (const int32_t*)e.p, (int)e.k, (sp24_score)score, renorm, (float)scale, d.p, d.ld, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return rd.object();
  } catch (...) {
    return none();
  }
}

// expert_order(addresses of sp24_expert_order, of sp24_expert_rows, of the workspace's size, experts, E, align) -> (offsets, position, source)
PyObject* expert_order(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 6 || at::impl::torch_function_mode_enabled()) return none();
  try {
    Slots x;
    int64_t E, align;
    if (!x.init(v[3], -1, -1, at::kInt) || !whole(v[4], &E) || !whole(v[5], &align) || E < 1 || E > 1024 || align < 1 || align > 256) return none();
    const int64_t slots = x.T * x.k;
    if (slots >= int64_t(1) << 31) return none();
    const auto fn = function<decltype(&sp24_expert_order)>(v[0]);
    const int64_t rows = function<decltype(&sp24_expert_rows)>(v[1])(slots, E, align);
    const size_t bytes = function<decltype(&sp24_expert_order_workspace_bytes)>(v[2])(slots, E);
    const cudaStream_t stream = Stream().handle;
    at::Tensor offsets, position, source, ws;
    const int status = unlocked([&] {
      const auto options = x.t->options();
      offsets = at::empty({E + 1}, options);
      position = at::empty({x.T, x.k}, options);
      source = at::empty({rows}, options);
      if (bytes) ws = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
      return fn(slots, E, align, (const int32_t*)x.p, (int32_t*)offsets.data_ptr(), (int32_t*)position.data_ptr(), (int32_t*)source.data_ptr(),
                bytes ? ws.data_ptr() : nullptr, bytes, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return Py_BuildValue("(NNN)", THPVariable_Wrap(std::move(offsets)), THPVariable_Wrap(std::move(position)), THPVariable_Wrap(std::move(source)));
  } catch (...) {
    return none();
  }
}

// expert_gather(address, x, position, source, scale, out) -> (rows, their scales)
PyObject* expert_gather(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 6 || at::impl::torch_function_mode_enabled()) return none();
  try {
    Matrix x, y;
    Slots at_;
    if (!x.init(v[1], -1, -1, -1)) return none();
    const int t = type_code(x.t->scalar_type());
    const int64_t T = x.t->size(0), K = x.t->size(1);
    const at::Tensor* s = plain(v[3], 1);
    if (t < 0 || s == nullptr || s->dim() != 1 || !at_.init(v[2], T, -1, at::kInt)) return none();
    const int64_t rows = s->size(0);
    const void *source, *scale;
    if (!vector(v[3], rows, SP24_I32, SP24_I32, &source) || !vector(v[4], T, SP24_F32, SP24_F32, &scale) || (v[5] != Py_None && !y.init(v[5], rows, K, t))) return none();
    const auto fn = function<decltype(&sp24_expert_gather)>(v[0]);
    const cudaStream_t stream = Stream().handle;
    Result ry{v[5], {}}, rs{Py_None, {}};
    const int status = unlocked([&] {
      if (v[5] == Py_None) {
        ry.made = at::empty({rows, K}, x.t->options());
        y.p = ry.made.data_ptr();
        y.ld = K > 1 ? K : 1;
      }
      if (v[4] != Py_None) rs.made = at::empty({rows}, x.t->options().dtype(at::kFloat));
      return fn((sp24_dtype)t, T, K, x.p, x.ld, (const float*)scale, (int)at_.k, (const int32_t*)at_.p, rows, (const int32_t*)source, y.p, y.ld,
                rs.made.defined() ? (float*)rs.made.data_ptr() : nullptr, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return Py_BuildValue("(NN)", ry.object(), rs.object());
  } catch (...) {
    return none();
  }
}

// expert_combine(address, y, position, source, weights, residual, out) -> out
PyObject* expert_combine(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 7 || at::impl::torch_function_mode_enabled()) return none();
  try {
    Matrix y, r, o;
    Slots at_, w;
    if (!y.init(v[1], -1, -1, -1) || !at_.init(v[2], -1, -1, at::kInt)) return none();
    const int t = type_code(y.t->scalar_type());
    const int64_t rows = y.t->size(0), K = y.t->size(1), T = at_.T;
    const void* source;
    if (!float_type(t) || v[3] == Py_None || !vector(v[3], rows, SP24_I32, SP24_I32, &source) || (v[4] != Py_None && !w.init(v[4], T, at_.k, at::kFloat)) ||
        (v[5] != Py_None && !r.init(v[5], T, K, t)) || (v[6] != Py_None && !o.init(v[6], T, K, t)))
      return none();
    const auto fn = function<decltype(&sp24_expert_combine)>(v[0]);
    const cudaStream_t stream = Stream().handle;
    Result ro{v[6], {}};
    const int status = unlocked([&] {
      if (v[6] == Py_None) {
        ro.made = at::empty({T, K}, y.t->options());
        o.p = ro.made.data_ptr();
        o.ld = K > 1 ? K : 1;
      }
      return fn((sp24_dtype)t, T, K, rows, y.p, y.ld, (int)at_.k, (const int32_t*)at_.p, (const float*)w.p, r.p, r.ld, o.p, o.ld, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return ro.object();
  } catch (...) {
    return none();
  }
}

// expert_combine_backward(address, dout, y, position, source, weights, out) -> (dy, dweights)
PyObject* expert_combine_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 7 || at::impl::torch_function_mode_enabled()) return none();
  try {
    Matrix g, y, dy;
    Slots at_, w;
    if (!g.init(v[1], -1, -1, -1) || !y.init(v[2], -1, -1, -1)) return none();
    const int t = type_code(g.t->scalar_type());
    const int64_t T = g.t->size(0), K = g.t->size(1), rows = y.t->size(0);
    const void* source;
    if (!float_type(t) || y.t->scalar_type() != g.t->scalar_type() || y.t->size(1) != K || !at_.init(v[3], T, -1, at::kInt) || v[4] == Py_None ||
        !vector(v[4], rows, SP24_I32, SP24_I32, &source) || !w.init(v[5], T, at_.k, at::kFloat) || (v[6] != Py_None && !dy.init(v[6], rows, K, t)))
      return none();
    const auto fn = function<decltype(&sp24_expert_combine_backward)>(v[0]);
    const cudaStream_t stream = Stream().handle;
    Result rdy{v[6], {}}, rdw{Py_None, {}};
    const int status = unlocked([&] {
      if (v[6] == Py_None) {
        rdy.made = at::empty({rows, K}, g.t->options());
        dy.p = rdy.made.data_ptr();
        dy.ld = K > 1 ? K : 1;
      }
      rdw.made = at::empty({T, at_.k}, w.t->options());
      return fn((sp24_dtype)t, T, K, rows, g.p, g.ld, y.p, y.ld, (int)at_.k, (const int32_t*)at_.p, (const int32_t*)source, (const float*)w.p, dy.p, dy.ld,
                (float*)rdw.made.data_ptr(), stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return Py_BuildValue("(NN)", rdy.object(), rdw.object());
  } catch (...) {
    return none();
  }
}

// the experts' metadata: [E, bytes], contiguous
bool expert_meta(PyObject* o, PyObject* bytes_of, int type, int64_t E, int64_t M, int64_t K, const void** meta) {
  Slots m;
  const size_t bytes = function<decltype(&sp24_meta_bytes)>(bytes_of)((sp24_dtype)type, M, K, SP24_META_TCGEN05);
  if (!m.init(o, E, (int64_t)bytes, at::kByte)) return false;
  *meta = m.p;
  return true;
}

// expert_linear(address, workspaces, address of sp24_meta_bytes, A, meta, X, offsets, bias, act, residual, row_scale, col_scale, pre, out, cd, a_is_dense, ws)
PyObject* expert_linear(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 17 || at::impl::torch_function_mode_enabled()) return none();
  try {
    Stack a;
    Matrix x, r, z, o;
    Slots bias, scale;
    int dense;
    if (!a.init(v[3], -1) || !truth(v[15], &dense)) return none();
    const int ab = type_code(a.t->scalar_type()), act = act_code(v[8]);
    if (ab < 0 || ab == SP24_I32 || ab == SP24_F32 || act < 0 || !x.init(v[5], -1, -1, ab)) return none();
    const bool one_byte = ab == SP24_I8 || ab == SP24_E4M3 || ab == SP24_E5M2;
    const int cd = v[14] == Py_None ? (one_byte ? (int)SP24_BF16 : ab) : type_code(v[14]);
    const int64_t E = a.E, M = a.M, K = dense ? a.n : 2 * a.n, rows = x.t->size(0);
    const void *meta = nullptr, *offsets, *col_scale;
    if (cd < 0 || x.t->size(1) != K || v[6] == Py_None || !vector(v[6], E + 1, SP24_I32, SP24_I32, &offsets)) return none();
    if (!dense && !expert_meta(v[4], v[2], ab, E, M, K, &meta)) return none();
    if ((v[7] != Py_None && !bias.init(v[7], E, M, at::kFloat)) || (v[10] != Py_None && !scale.init(v[10], E, M, at::kFloat)) ||
        !vector(v[11], rows, SP24_F32, SP24_F32, &col_scale) || (v[9] != Py_None && !r.init(v[9], rows, M, cd)))
      return none();
    const bool make_pre = v[12] == Py_True, no_pre = v[12] == Py_False || v[12] == Py_None;
    if ((!make_pre && !no_pre && !z.init(v[12], rows, M, cd)) || (v[13] != Py_None && !o.init(v[13], rows, M, cd))) return none();
    const cudaStream_t stream = Stream().handle;
    void* ws;
    size_t ws_bytes;
    if (!workspace(v[1], v[16], *a.t, stream, &ws, &ws_bytes)) return none();
    const auto fn = function<decltype(&sp24_expert_linear)>(v[0]);
    Result ro{v[13], {}}, rz{make_pre || no_pre ? Py_None : v[12], {}};
    const int status = unlocked([&] {
      auto make = [&](Result& to, Matrix& m) {
        to.made = at::empty({rows, M}, a.t->options().dtype(kScalar[cd]));
        m.p = to.made.data_ptr();
        m.ld = M;
      };
      if (v[13] == Py_None) make(ro, o);
      if (make_pre) make(rz, z);
      const sp24_expert_desc d = {(sp24_dtype)ab, (sp24_dtype)cd, E, M, K, rows, a.ld, x.ld, o.ld, r.ld, z.ld, dense};
      const sp24_expert_epilogue e = {(const float*)scale.p, (const float*)col_scale, (const float*)bias.p, (sp24_act)act, r.p, z.p};
      return fn(&d, &e, a.p, meta, x.p, (const int32_t*)offsets, o.p, ws, ws_bytes, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    if (no_pre) return ro.object();
    return Py_BuildValue("(NN)", ro.object(), rz.object());
  } catch (...) {
    return none();
  }
}

// expert_linear_backward(addresses of sp24_expert_act_backward, of its workspace's size, of sp24_expert_linear_dx, of sp24_expert_linear_dw, of sp24_meta_bytes,
// workspaces, dy, pre, X, W, offsets, act, meta, bias, ws) -> (dX, dW, dbias)
PyObject* expert_linear_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
  if (n != 15 || at::impl::torch_function_mode_enabled()) return none();
  try {
    Matrix dy, z, x;
    Stack w;
    int with_bias;
    const int act = act_code(v[11]);
    if (act < 0 || !truth(v[13], &with_bias) || !dy.init(v[6], -1, -1, -1)) return none();
    const int t = type_code(dy.t->scalar_type());
    if ((t != SP24_F16 && t != SP24_BF16) || !w.init(v[9], t)) return none();
    const int64_t rows = dy.t->size(0), E = w.E, M = w.M, K = w.n;
    const void *offsets, *meta = nullptr;
    if (rows < 1 || dy.t->size(1) != M || M % 16 != 0 || K % 16 != 0 || !x.init(v[8], rows, K, t) || v[10] == Py_None || !vector(v[10], E + 1, SP24_I32, SP24_I32, &offsets) ||
        (act != SP24_ACT_NONE && !z.init(v[7], rows, M, t)) || (v[12] != Py_None && !expert_meta(v[12], v[4], t, E, M, K, &meta)))
      return none();
    const cudaStream_t stream = Stream().handle;
    void* ws;
    size_t ws_bytes;
    if (!workspace(v[5], v[14], *dy.t, stream, &ws, &ws_bytes)) return none();
    const auto act_fn = function<decltype(&sp24_expert_act_backward)>(v[0]);
    const auto act_bytes = function<decltype(&sp24_expert_act_backward_workspace_bytes)>(v[1]);
    const auto dx_fn = function<decltype(&sp24_expert_linear_dx)>(v[2]);
    const auto dw_fn = function<decltype(&sp24_expert_linear_dw)>(v[3]);
    Result rx{Py_None, {}}, rw{Py_None, {}}, rb{Py_None, {}};
    const int status = unlocked([&]() -> int {
      const auto options = dy.t->options();
      // dz (without an activation dy itself, where a product can take it) and the partial sums of the bias's gradient, in one allocation
      const bool makes_dz = act != SP24_ACT_NONE || (uintptr_t)dy.p % 16 != 0 || dy.ld * 2 % 16 != 0;
      const int64_t lddz = makes_dz ? M : dy.ld;
      const size_t bytes = with_bias ? act_bytes(E, M, rows) : 0, matrix = makes_dz ? ((size_t)rows * M * 2 + 255) / 256 * 256 : 0;
      at::Tensor scratch;
      char* room = nullptr;
      if (matrix + bytes) {
        scratch = at::empty({(int64_t)(matrix + bytes)}, options.dtype(at::kByte));
        room = (char*)scratch.data_ptr();
      }
      void* const pdz = makes_dz ? room : dy.p;
      if (with_bias) rb.made = at::empty({E, M}, options.dtype(at::kFloat));
      int st = act_fn((sp24_dtype)t, (sp24_act)act, E, M, rows, dy.p, dy.ld, z.p, z.ld, (const int32_t*)offsets, makes_dz ? pdz : nullptr, lddz,
                      with_bias ? (float*)rb.made.data_ptr() : nullptr, with_bias ? room + matrix : nullptr, bytes, stream);
      if (st != SP24_OK) return st;
      rx.made = at::empty({rows, K}, options);
      rw.made = at::empty({E, M, K}, options);
      sp24_expert_desc d = {(sp24_dtype)t, (sp24_dtype)t, E, M, K, rows, w.ld, K, lddz, 0, 0, 1};
      st = dx_fn(&d, pdz, w.p, (const int32_t*)offsets, rx.made.data_ptr(), ws, ws_bytes, stream);
      if (st != SP24_OK) return st;
      d.lda = K;
      d.ldx = x.ld;
      return dw_fn(&d, pdz, x.p, (const int32_t*)offsets, meta, rw.made.data_ptr(), ws, ws_bytes, stream);
    });
    if (status != SP24_OK) return PyLong_FromLong(status);
    return Py_BuildValue("(NNN)", rx.object(), rw.object(), rb.object());
  } catch (...) {
    return none();
  }
}

#define SP24_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SP24_METHOD(gemm), SP24_METHOD(gemm_i8_dequant), SP24_METHOD(conv3x3_nhwc), SP24_METHOD(compress),
                         SP24_METHOD(apply_mask), SP24_METHOD(rms_norm), SP24_METHOD(rms_norm_backward), SP24_METHOD(gated_act),
                         SP24_METHOD(gated_act_backward), SP24_METHOD(act_backward), SP24_METHOD(linear),
                         SP24_METHOD(linear_backward), SP24_METHOD(route), SP24_METHOD(route_backward), SP24_METHOD(expert_order),
                         SP24_METHOD(expert_gather), SP24_METHOD(expert_combine), SP24_METHOD(expert_combine_backward),
                         SP24_METHOD(expert_linear), SP24_METHOD(expert_linear_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
