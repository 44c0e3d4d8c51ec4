// Python calls of the 8-bit training operators without the interpreter's share: checks the
// tensors of a call against its descriptor and calls the library.  A small layer's call is bound by
// the host; marshalling it in Python takes 4 to 6 us, here about half a microsecond.
//
// Every function takes the descriptor (an object with the buffer protocol: the ctypes structure),
// the tensors in the library's order (None: not given) and the stream (None: the current one), and
// returns the library's status, or -1 where an argument is not what the descriptor says in the
// plainest way; train8.py then goes through the arguments one by one and raises, or calls.
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/maxdnn.h"

namespace {

decltype(&maxdnn_quant8) f_quant8;
decltype(&maxdnn_dequant8) f_dequant8;
decltype(&maxdnn_gemm8) f_gemm8;
decltype(&maxdnn_layer_norm_fprop) f_layer_norm_fprop;
decltype(&maxdnn_layer_norm_bprop) f_layer_norm_bprop;
decltype(&maxdnn_act8_fprop) f_act8_fprop;
decltype(&maxdnn_act8_bprop) f_act8_bprop;

int64_t blocks(int64_t n) { return (n + 127) / 128; }

bool type_ok(at::ScalarType t, int dtype) {
  switch (dtype) {
    case MAXDNN_F32: return t == at::kFloat;
    case MAXDNN_BF16: return t == at::kBFloat16;
    case MAXDNN_F16: return t == at::kHalf;
    case MAXDNN_E4M3: return t == at::kFloat8_e4m3fn || t == at::kByte;
    case MAXDNN_E5M2: return t == at::kFloat8_e5m2 || t == at::kByte;
    case MAXDNN_E8M0: return t == at::kFloat8_e8m0fnu || t == at::kByte;
  }
  return false;
}

// The arguments of one call; `ok` turns false at the first that is not plain.
struct Call {
  PyObject* const* args;
  Py_ssize_t n;
  bool ok = true;
  int device = -1;
  Py_buffer desc = {};
  bool have_desc = false;

  Call(PyObject* const* a, Py_ssize_t count, Py_ssize_t want, size_t desc_bytes) : args(a), n(count) {
    if (n != want || PyObject_GetBuffer(args[0], &desc, PyBUF_SIMPLE) != 0) {
      PyErr_Clear();
      ok = false;
      return;
    }
    have_desc = true;
    if ((size_t)desc.len != desc_bytes) ok = false;
    else device = c10::cuda::current_device();
  }
  ~Call() { if (have_desc) PyBuffer_Release(&desc); }

  template <class D> const D& as() const { return *static_cast<const D*>(desc.buf); }

  const at::Tensor* tensor(int i) {
    if (!THPVariable_Check(args[i])) { ok = false; return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(args[i]);
    if (!t.is_cuda() || t.get_device() != device) { ok = false; return nullptr; }
    return &t;
  }
  // [rows][cols] with row pitch ld
  void* mat(int i, int dtype, int64_t rows, int64_t cols, int64_t ld, bool optional = false) {
    if (!ok || args[i] == Py_None) { ok = ok && optional; return nullptr; }
    const at::Tensor* t = tensor(i);
    if (!t) return nullptr;
    if (!type_ok(t->scalar_type(), dtype) || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols ||
        t->stride(1) != 1 || t->stride(0) != ld) {
      ok = false;
      return nullptr;
    }
    return t->data_ptr();
  }
  void* vec(int i, int dtype, int64_t count, bool optional = false) {
    if (!ok || args[i] == Py_None) { ok = ok && optional; return nullptr; }
    const at::Tensor* t = tensor(i);
    if (!t) return nullptr;
    if (!type_ok(t->scalar_type(), dtype) || t->numel() != count || !t->is_contiguous()) {
      ok = false;
      return nullptr;
    }
    return t->data_ptr();
  }
  void* stream(int i) {
    if (!ok) return nullptr;
    if (args[i] == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    const long long v = PyLong_AsLongLong(args[i]);
    if (v == -1 && PyErr_Occurred()) {
      PyErr_Clear();
      ok = false;
    }
    return reinterpret_cast<void*>(v);
  }
  // values and scales of a packed matrix: both or neither
  void pair(int i, int dtype, int64_t rows, int64_t cols, int64_t ld, int64_t n_scales, void** q, void** s) {
    *q = mat(i, dtype, rows, cols, ld, true);
    *s = vec(i + 1, MAXDNN_E8M0, n_scales, true);
    if ((*q == nullptr) != (*s == nullptr)) ok = false;
  }
};

PyObject* not_plain() { return PyLong_FromLong(-1); }

// The library's call with the interpreter's lock released: a launch may wait (a full queue, a device's first
// call), and other threads run meanwhile.  (The descriptor was copied before: it is a Python object's memory.)
template <class F> PyObject* unlocked(F call) {
  maxdnn_status st;
  Py_BEGIN_ALLOW_THREADS
  st = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

#define MAXDNN_TRY try {
#define MAXDNN_CATCH } catch (...) { PyErr_Clear(); return not_plain(); }

PyObject* quant8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MAXDNN_TRY
  Call c(a, n, 10, sizeof(maxdnn_quant8_desc));
  if (!c.ok) return not_plain();
  const auto d = c.as<maxdnn_quant8_desc>();
  const int64_t r = d.rows, k = d.cols, rs = blocks(k) * r;
  void* x = c.mat(1, d.x_type, r, k, d.ldx);
  void* xs = d.x_type >= MAXDNN_E4M3 ? c.vec(2, MAXDNN_E8M0, rs) : nullptr;
  void *q[3], *s[3];
  c.pair(3, d.q_type, r, k, d.ldq, rs, &q[0], &s[0]);
  c.pair(5, d.q_type, r, k, d.ldq, blocks(r) * k, &q[1], &s[1]);
  c.pair(7, d.q_type, r, k, d.ldq, blocks(r) * blocks(k), &q[2], &s[2]);
  void* stream = c.stream(9);
  if (!c.ok) return not_plain();
  return unlocked([&] { return f_quant8(&d, x, xs, q[0], s[0], q[1], s[1], q[2], s[2], stream); });
  MAXDNN_CATCH
}

PyObject* dequant8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MAXDNN_TRY
  Call c(a, n, 6, sizeof(maxdnn_quant8_desc));
  if (!c.ok) return not_plain();
  const auto d = c.as<maxdnn_quant8_desc>();
  const long block = PyLong_AsLong(a[1]);
  if (PyErr_Occurred() || block < 0 || block > 2) { PyErr_Clear(); return not_plain(); }
  const int64_t r = d.rows, k = d.cols;
  void* q = c.mat(2, d.q_type, r, k, d.ldq);
  void* s = c.vec(3, MAXDNN_E8M0, block == 0 ? blocks(k) * r : block == 1 ? blocks(r) * k : blocks(r) * blocks(k));
  void* x = c.mat(4, d.x_type, r, k, d.ldx);
  void* stream = c.stream(5);
  if (!c.ok) return not_plain();
  return unlocked([&] { return f_dequant8(&d, (maxdnn_block)block, q, s, x, stream); });
  MAXDNN_CATCH
}

PyObject* gemm8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MAXDNN_TRY
  Call c(a, n, 7, sizeof(maxdnn_gemm8_desc));
  if (!c.ok) return not_plain();
  const auto d = c.as<maxdnn_gemm8_desc>();
  auto side = [&](int i, int type, int major, int block, int scale_type, int64_t mn, int64_t ld, void** q, void** s) {
    const int64_t rows = major == MAXDNN_MAJOR_K ? mn : d.K, cols = major == MAXDNN_MAJOR_K ? d.K : mn;
    *q = c.mat(i, type, rows, cols, ld);
    *s = c.vec(i + 1, scale_type, block == MAXDNN_BLOCK_ROW ? blocks(cols) * rows
                                  : block == MAXDNN_BLOCK_COL ? blocks(rows) * cols : blocks(rows) * blocks(cols));
  };
  void *qa, *sa, *qb, *sb;
  side(1, d.a_type, d.a_major, d.a_block, d.a_scale_type, d.M, d.lda, &qa, &sa);
  side(3, d.b_type, d.b_major, d.b_block, d.b_scale_type, d.N, d.ldb, &qb, &sb);
  void* out = c.mat(5, d.c_type, d.M, d.N, d.ldc);
  void* stream = c.stream(6);
  if (!c.ok) return not_plain();
  return unlocked([&] { return f_gemm8(&d, qa, sa, qb, sb, out, stream); });
  MAXDNN_CATCH
}

PyObject* layer_norm_fprop(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MAXDNN_TRY
  Call c(a, n, 12, sizeof(maxdnn_layer_norm_desc));
  if (!c.ok) return not_plain();
  const auto d = c.as<maxdnn_layer_norm_desc>();
  const int64_t r = d.rows, k = d.cols, rs = blocks(k) * r;
  void* x = c.mat(1, d.x_type, r, k, d.ldx);
  void* gamma = c.vec(2, d.w_type, k, true);
  void* beta = c.vec(3, d.w_type, k, true);
  void* y = c.mat(4, d.y_type, r, k, d.ldy, true);
  void* mean = c.vec(5, MAXDNN_F32, r, true);
  void* rstd = c.vec(6, MAXDNN_F32, r, true);
  void *q, *s, *ck, *sc;
  c.pair(7, d.q_type, r, k, d.ldq, rs, &q, &s);
  c.pair(9, d.q_type, r, k, d.ldq, rs, &ck, &sc);
  void* stream = c.stream(11);
  if (!c.ok) return not_plain();
  return unlocked([&] { return f_layer_norm_fprop(&d, x, gamma, beta, y, (float*)mean, (float*)rstd, q, s, ck, sc, stream); });
  MAXDNN_CATCH
}

PyObject* layer_norm_bprop(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MAXDNN_TRY
  Call c(a, n, 12, sizeof(maxdnn_layer_norm_desc));
  if (!c.ok) return not_plain();
  const auto d = c.as<maxdnn_layer_norm_desc>();
  const int64_t r = d.rows, k = d.cols;
  void* dy = c.mat(1, d.y_type, r, k, d.ldy);
  void* x = c.mat(2, d.x_type, r, k, d.ldx);
  void* xs = d.x_type >= MAXDNN_E4M3 ? c.vec(3, MAXDNN_E8M0, blocks(k) * r) : nullptr;
  void* gamma = c.vec(4, d.w_type, k, true);
  void* mean = c.vec(5, MAXDNN_F32, r);
  void* rstd = c.vec(6, MAXDNN_F32, r);
  void* dx = c.mat(7, d.y_type, r, k, d.ldy);
  void* dg = c.vec(8, MAXDNN_F32, k, true);
  void* db = c.vec(9, MAXDNN_F32, k, true);
  void* ws = nullptr;
  size_t ws_bytes = 0;
  if (c.ok && a[10] != Py_None) {
    const at::Tensor* t = c.tensor(10);
    if (t && t->is_contiguous()) {
      ws = t->data_ptr();
      ws_bytes = t->nbytes();
    } else {
      c.ok = false;
    }
  }
  void* stream = c.stream(11);
  if (!c.ok) return not_plain();
  return unlocked([&] { return f_layer_norm_bprop(&d, dy, x, xs, gamma, (float*)mean, (float*)rstd, dx, (float*)dg, (float*)db,
                                            ws, ws_bytes, stream); });
  MAXDNN_CATCH
}

PyObject* act8_fprop(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MAXDNN_TRY
  Call c(a, n, 8, sizeof(maxdnn_act8_desc));
  if (!c.ok) return not_plain();
  const auto d = c.as<maxdnn_act8_desc>();
  const int64_t r = d.rows, k = d.cols, many = 1 + d.gated, rs = blocks(k) * r;
  void* h = c.mat(1, d.x_type, r, many * k, d.ldh);
  void* out = c.mat(2, d.x_type, r, k, d.lda, true);
  void *q, *s, *ck, *sc;
  c.pair(3, d.q_type, r, k, d.ldq, rs, &q, &s);
  c.pair(5, d.q_type, r, many * k, d.ldc, many * rs, &ck, &sc);
  void* stream = c.stream(7);
  if (!c.ok) return not_plain();
  return unlocked([&] { return f_act8_fprop(&d, h, out, q, s, ck, sc, stream); });
  MAXDNN_CATCH
}

PyObject* act8_bprop(PyObject*, PyObject* const* a, Py_ssize_t n) {
  MAXDNN_TRY
  Call c(a, n, 6, sizeof(maxdnn_act8_desc));
  if (!c.ok) return not_plain();
  const auto d = c.as<maxdnn_act8_desc>();
  const int64_t r = d.rows, k = d.cols, many = 1 + d.gated;
  const bool packed = d.h_type >= MAXDNN_E4M3;
  void* da = c.mat(1, d.x_type, r, k, d.lda);
  void* h = c.mat(2, d.h_type, r, many * k, packed ? d.ldc : d.ldh);
  void* hs = packed ? c.vec(3, MAXDNN_E8M0, many * blocks(k) * r) : nullptr;
  void* dh = c.mat(4, d.x_type, r, many * k, d.ldh);
  void* stream = c.stream(5);
  if (!c.ok) return not_plain();
  return unlocked([&] { return f_act8_bprop(&d, da, h, hs, dh, stream); });
  MAXDNN_CATCH
}

// bind(addresses): where the loaded library has the seven functions, in the order below.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* p[7];
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "bind takes seven addresses");
    return nullptr;
  }
  for (int i = 0; i < 7; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
      return nullptr;
    }
  }
  f_quant8 = reinterpret_cast<decltype(f_quant8)>(p[0]);
  f_dequant8 = reinterpret_cast<decltype(f_dequant8)>(p[1]);
  f_gemm8 = reinterpret_cast<decltype(f_gemm8)>(p[2]);
  f_layer_norm_fprop = reinterpret_cast<decltype(f_layer_norm_fprop)>(p[3]);
  f_layer_norm_bprop = reinterpret_cast<decltype(f_layer_norm_bprop)>(p[4]);
  f_act8_fprop = reinterpret_cast<decltype(f_act8_fprop)>(p[5]);
  f_act8_bprop = reinterpret_cast<decltype(f_act8_bprop)>(p[6]);
  Py_RETURN_NONE;
}

template <class F> PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {
    {"bind", fast(bind), METH_FASTCALL, nullptr},
    {"quant8", fast(quant8), METH_FASTCALL, nullptr},
    {"dequant8", fast(dequant8), METH_FASTCALL, nullptr},
    {"gemm8", fast(gemm8), METH_FASTCALL, nullptr},
    {"layer_norm_fprop", fast(layer_norm_fprop), METH_FASTCALL, nullptr},
    {"layer_norm_bprop", fast(layer_norm_bprop), METH_FASTCALL, nullptr},
    {"act8_fprop", fast(act8_fprop), METH_FASTCALL, nullptr},
    {"act8_bprop", fast(act8_bprop), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_train8", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The torch whose headers this was compiled with, after a fixed prefix (build.py looks for it).
PyMODINIT_FUNC PyInit__train8() {
  static const char built_for[] = MAXDNN_BUILT_FOR;
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", built_for + sizeof("built for torch ") - 1) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
