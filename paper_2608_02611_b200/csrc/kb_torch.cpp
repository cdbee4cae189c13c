// The model operators' Python calls, natively: checks tensors, makes the outputs and calls the C
// entry points (include/kb_ops.h).  Marshalling only, like binding.py, whose Context methods are
// thin wrappers around these functions.  Through ctypes such a call spends 13 to 18 us in Python and
// the kernels of a single token take 3 to 15 us; from here it spends about half of that.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/kb_ops.h"

namespace {

PyObject* g_error = nullptr;   // binding.KbError
// The entry points, from the library that binding.py has loaded
struct {
  decltype(&::kb_quantize_blocks) quantize_blocks;
  decltype(&::kb_layernorm) layernorm;
  decltype(&::kb_layernorm_backward) layernorm_backward;
  decltype(&::kb_matmul_blocks) matmul_blocks;
  decltype(&::kb_last_error) last_error;
} g_lib;

struct Refused {};             // a Python exception is set

[[noreturn]] void refuse(const char* where, const std::string& text, int status = KB_ERR_INVALID_ARG) {
  PyObject* e = g_error ? PyObject_CallFunction(g_error, "iss", status, where, text.c_str()) : nullptr;
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, text.c_str());
  }
  throw Refused{};
}

// A call's context: the C handle and its device
struct Call {
  const char* where;
  kb_ctx* ctx;
  at::Device device;
  void* stream;
  // Runs an entry point without Python's lock (as ctypes would): a launch can wait for room in the stream's
  // queue and a workspace can grow, and other threads go on meanwhile.  The tensors stay alive: the
  // caller holds them.
  template <class F>
  void run(F entry) const {
    PyThreadState* held = PyEval_SaveThread();
    const kb_status rc = entry();
    PyEval_RestoreThread(held);
    if (rc != KB_OK) refuse(where, g_lib.last_error(ctx), rc);
  }
  at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type) const {
    return at::empty(sizes, at::TensorOptions().dtype(type).device(device));
  }
  at::Tensor codes(int64_t rows, int64_t cols, at::ScalarType type) const {   // rows on 16-byte boundaries
    if (cols % 16 == 0) return empty({rows, cols}, type);
    return empty({rows, (cols + 15) / 16 * 16}, type).narrow(1, 0, cols);
  }
};

Call open_call(const char* where, PyObject* handle, PyObject* index) {
  void* h = handle == Py_None ? nullptr : PyLong_AsVoidPtr(handle);
  const long dev = PyLong_AsLong(index);
  if (PyErr_Occurred()) throw Refused{};
  if (!h || !g_lib.last_error) refuse(where, h ? "the library is not loaded" : "the context is closed");
  return {where, static_cast<kb_ctx*>(h), at::Device(at::kCUDA, (c10::DeviceIndex)dev),
          c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream()};
}

const at::Tensor& tensor(const Call& c, PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(c.where, std::string(name) + " must be a tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.device() != c.device) refuse(c.where, std::string(name) + " must be on " + c.device.str());
  return t;
}

// Python's truth value and whole numbers; what raises there raises here, before any launch
bool truth(PyObject* o) {
  const int t = PyObject_IsTrue(o);
  if (t < 0) throw Refused{};
  return t != 0;
}
long whole(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{};
  return v;
}

int code_of(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return KB_F32;
    case at::kHalf: return KB_F16;
    case at::kBFloat16: return KB_BF16;
    case at::kFloat8_e4m3fn: return KB_F8E4M3;
    case at::kFloat8_e5m2: return KB_F8E5M2;
    default: return -1;   // the C call refuses it
  }
}
// The reverse, for outputs: an unknown code is given room as bytes and refused by the C call.
at::ScalarType type_of(long code) {
  switch (code) {
    case KB_F32: return at::kFloat;
    case KB_F16: return at::kHalf;
    case KB_BF16: return at::kBFloat16;
    case KB_F8E4M3: return at::kFloat8_e4m3fn;
    case KB_F8E5M2: return at::kFloat8_e5m2;
    default: return at::kDouble;
  }
}

// A tensor as a matrix [rows, columns] with adjacent columns, without copying: 2-D with any row
// stride, or of any rank if it is contiguous.
struct Rows {
  int64_t rows, cols;
  uint64_t ld;
  void* p;
};
Rows rows_of(const Call& c, const at::Tensor& t, const char* name) {
  int64_t rows, cols, stride;
  if (t.dim() == 2) {
    rows = t.size(0);
    cols = t.size(1);
    stride = t.stride(0);
    if ((cols > 1 && rows > 0 && t.stride(1) != 1) || (rows > 1 && stride < cols))
      refuse(c.where, std::string("the columns of ") + name + " must be adjacent and its rows must not overlap");
  } else {
    if (t.dim() == 0 || !(t.is_contiguous() || t.numel() == 0))
      refuse(c.where, std::string(name) + " must be 2-D or contiguous");
    cols = t.size(-1);
    rows = cols ? t.numel() / cols : 0;
    stride = cols;
  }
  // the stride of a single row is free (torch may report anything)
  const int64_t ld = rows > 1 ? std::max(stride, cols) : (cols + 15) / 16 * 16;
  return {rows, cols, (uint64_t)ld, t.data_ptr()};
}

// Address of a contiguous vector of n elements of one of two types
void* vector_of(const Call& c, const at::Tensor& t, int64_t n, const char* name, at::ScalarType a, at::ScalarType b) {
  if (t.numel() != n || (t.scalar_type() != a && t.scalar_type() != b) || !t.is_contiguous())
    refuse(c.where, std::string(name) + " must be a contiguous tensor of " + std::to_string(n) + " elements of " +
                        c10::toString(a) + (a == b ? std::string() : std::string(" or ") + c10::toString(b)));
  return t.data_ptr();
}

PyObject* wrap(const at::Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
template <size_t N>
PyObject* wrap_tuple(const at::Tensor (&t)[N]) {
  PyObject* r = PyTuple_New(N);
  if (!r) throw Refused{};
  for (size_t i = 0; i < N; ++i) {
    PyObject* o = wrap(t[i]);
    if (!o) {
      Py_DECREF(r);
      throw Refused{};
    }
    PyTuple_SET_ITEM(r, i, o);
  }
  return r;
}
int64_t blocks(int64_t n) { return (n + KB_BLOCK - 1) / KB_BLOCK; }

// Runs a body that may throw and turns what it throws into a Python exception.
template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F body) {
  if (n != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return body();
  } catch (const Refused&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

// (handle, device, x, code, tiles, transpose) -> (q, scale)
PyObject* quantize_blocks(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const Call c = open_call("kb_quantize_blocks", a[0], a[1]);
    const at::Tensor& x = tensor(c, a[2], "x");
    const long code = whole(a[3]);
    const bool tiles = truth(a[4]), transpose = truth(a[5]);
    const Rows m = rows_of(c, x, "x");
    const int64_t R = transpose ? m.cols : m.rows, C = transpose ? m.rows : m.cols;
    const at::Tensor q = c.codes(R, C, type_of(code));
    const at::Tensor scale = c.empty({blocks(C), tiles ? blocks(R) : R}, at::kFloat);
    void* qp = q.data_ptr();
    float* sp = scale.data_ptr<float>();
    const kb_dtype type = (kb_dtype)code_of(x.scalar_type());
    c.run([&] {
      return g_lib.quantize_blocks(c.ctx, m.p, m.rows, m.cols, m.ld, type, transpose, tiles ? KB_SCALE_TILES : KB_SCALE_ROWS,
                                   qp, (C + 15) / 16 * 16, (kb_dtype)code, sp, c.stream);
    });
    return wrap_tuple({q, scale});
  });
}

// (handle, device, x, weight, bias, eps, want_y, want_stats, code or None) -> (y, mean, rstd, q, scale)
PyObject* layernorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject* {
    const Call c = open_call("kb_layernorm", a[0], a[1]);
    const at::Tensor& x = tensor(c, a[2], "x");
    const Rows m = rows_of(c, x, "x");
    const at::ScalarType type = x.scalar_type();
    at::ScalarType params = type;
    void *w = nullptr, *b = nullptr;
    if (a[3] != Py_None) {
      const at::Tensor& t = tensor(c, a[3], "weight");
      w = vector_of(c, t, m.cols, "weight", type, at::kFloat);
      params = t.scalar_type();
    }
    if (a[4] != Py_None) {
      const at::Tensor& t = tensor(c, a[4], "bias");
      b = vector_of(c, t, m.cols, "bias", type, at::kFloat);
      if (w && t.scalar_type() != params) refuse(c.where, "weight and bias must have the same type");
      params = t.scalar_type();
    }
    const double eps = PyFloat_AsDouble(a[5]);
    if (eps == -1.0 && PyErr_Occurred()) throw Refused{};
    const bool want_y = truth(a[6]), want_stats = truth(a[7]), want_q = a[8] != Py_None;
    const long code = want_q ? whole(a[8]) : KB_F8E4M3;
    at::Tensor y, mean, rstd, q, scale;
    if (want_y) y = c.empty(x.sizes(), type);
    if (want_stats) {
      mean = c.empty({m.rows}, at::kFloat);
      rstd = c.empty({m.rows}, at::kFloat);
    }
    if (want_q) {
      q = c.codes(m.rows, m.cols, type_of(code));
      scale = c.empty({blocks(m.cols), m.rows}, at::kFloat);
    }
    // the addresses of empty tensors are null, which would mean "not wanted": with no row the call checks
    // its arguments and writes nothing, so any address does
    alignas(16) static float no_row[4];
    auto out = [&](bool want, const at::Tensor& t) -> void* { return !want ? nullptr : m.rows ? t.data_ptr() : no_row; };
    void *yp = out(want_y, y), *mp = out(want_stats, mean), *rp = out(want_stats, rstd), *qp = out(want_q, q), *sp = out(want_q, scale);
    c.run([&] {
      return g_lib.layernorm(c.ctx, m.p, m.rows, m.cols, m.ld, (kb_dtype)code_of(type), w, b, (kb_dtype)code_of(params),
                             (float)eps, yp, m.cols, static_cast<float*>(mp), static_cast<float*>(rp), qp,
                             (m.cols + 15) / 16 * 16, (kb_dtype)code, static_cast<float*>(sp), c.stream);
    });
    return wrap_tuple({y, mean, rstd, q, scale});
  });
}

// (handle, device, dy, x, weight, mean, rstd, want_bias) -> (dx, dweight, dbias)
PyObject* layernorm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const Call c = open_call("kb_layernorm_backward", a[0], a[1]);
    const at::Tensor &dy = tensor(c, a[2], "dy"), &x = tensor(c, a[3], "x");
    const Rows mg = rows_of(c, dy, "dy"), m = rows_of(c, x, "x");
    const at::ScalarType type = x.scalar_type();
    if (mg.rows != m.rows || mg.cols != m.cols || dy.scalar_type() != type)
      refuse(c.where, "dy must have the shape and type of x");
    at::ScalarType params = at::kFloat;
    void* w = nullptr;
    if (a[4] != Py_None) {
      const at::Tensor& t = tensor(c, a[4], "weight");
      w = vector_of(c, t, m.cols, "weight", type, at::kFloat);
      params = t.scalar_type();
    }
    void* mean = vector_of(c, tensor(c, a[5], "mean"), m.rows, "mean", at::kFloat, at::kFloat);
    void* rstd = vector_of(c, tensor(c, a[6], "rstd"), m.rows, "rstd", at::kFloat, at::kFloat);
    const bool want_bias = truth(a[7]);
    const at::Tensor dx = c.empty(x.sizes(), type), dweight = c.empty({m.cols}, params);
    at::Tensor dbias;
    if (want_bias) dbias = c.empty({m.cols}, params);
    void *dxp = dx.data_ptr(), *dwp = dweight.data_ptr(), *dbp = want_bias ? dbias.data_ptr() : nullptr;
    c.run([&] {
      return g_lib.layernorm_backward(c.ctx, mg.p, mg.ld, m.p, m.ld, m.rows, m.cols, (kb_dtype)code_of(type), w,
                                      (kb_dtype)code_of(params), static_cast<float*>(mean), static_cast<float*>(rstd), dxp,
                                      m.cols, dwp, dbp, c.stream);
    });
    return wrap_tuple({dx, dweight, dbias});
  });
}

// (handle, device, a, a_scale, b, b_scale, code, out or None) -> D
PyObject* matmul_blocks(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const Call c = open_call("kb_matmul_blocks", a[0], a[1]);
    const at::Tensor &A = tensor(c, a[2], "a"), &SA = tensor(c, a[3], "a_scale");
    const at::Tensor &B = tensor(c, a[4], "b"), &SB = tensor(c, a[5], "b_scale");
    const Rows ma = rows_of(c, A, "a"), mb = rows_of(c, B, "b");
    const int64_t M = ma.rows, N = mb.rows, K = ma.cols, kb = blocks(K);
    if (mb.cols != K) refuse(c.where, "a has " + std::to_string(K) + " columns, b " + std::to_string(mb.cols));
    const bool shaped = SA.dim() == 2 && SB.dim() == 2 && SA.size(0) == kb && SA.size(1) == M && SB.size(0) == kb;
    const bool tiles = shaped && SB.size(1) != N;
    if (!shaped || (tiles && SB.size(1) != blocks(N)))
      refuse(c.where, "scales are laid out [ceil(K/128), rows] or [ceil(K/128), ceil(rows/128)]");
    void* sa = vector_of(c, SA, SA.numel(), "a_scale", at::kFloat, at::kFloat);
    void* sb = vector_of(c, SB, SB.numel(), "b_scale", at::kFloat, at::kFloat);
    at::Tensor D;
    if (a[7] == Py_None) {
      D = c.empty({M, N}, type_of(whole(a[6])));
    } else {
      D = tensor(c, a[7], "out");
      if (D.dim() != 2 || D.size(0) != M || D.size(1) != N)
        refuse(c.where, "out must be a matrix [" + std::to_string(M) + ", " + std::to_string(N) + "]");
    }
    const Rows md = rows_of(c, D, "out");
    const kb_dtype ta = (kb_dtype)code_of(A.scalar_type()), tb = (kb_dtype)code_of(B.scalar_type());
    const kb_dtype td = (kb_dtype)code_of(D.scalar_type());
    c.run([&] {
      return g_lib.matmul_blocks(c.ctx, ma.p, ma.ld, ta, static_cast<float*>(sa), mb.p, mb.ld, tb, static_cast<float*>(sb),
                                 tiles ? KB_SCALE_TILES : KB_SCALE_ROWS, M, N, K, md.p, md.ld, td, c.stream);
    });
    return wrap(D);
  });
}

// (error class, addresses of the five entry points in the order above)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    void* p[5];
    for (int i = 0; i < 5; ++i) {
      p[i] = PyLong_AsVoidPtr(a[1 + i]);
      if (!p[i]) throw Refused{};
    }
    g_lib = {reinterpret_cast<decltype(g_lib.quantize_blocks)>(p[0]), reinterpret_cast<decltype(g_lib.layernorm)>(p[1]),
             reinterpret_cast<decltype(g_lib.layernorm_backward)>(p[2]),
             reinterpret_cast<decltype(g_lib.matmul_blocks)>(p[3]), reinterpret_cast<decltype(g_lib.last_error)>(p[4])};
    Py_INCREF(a[0]);
    Py_XSETREF(g_error, a[0]);
    Py_RETURN_NONE;
  });
}

#define KB_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {KB_FAST(quantize_blocks),
                         KB_FAST(layernorm),
                         KB_FAST(layernorm_backward),
                         KB_FAST(matmul_blocks),
                         KB_FAST(bind),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kb_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kb_torch() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", KB_BUILT_FOR) < 0) Py_CLEAR(m);
  return m;
}
