// The model operators' Python calls, natively: checks tensors, makes the outputs and calls the C
// entry points (include/kb_ops.h, include/kb_attention.h).  Marshalling only, like binding.py, whose Context methods are
// thin wrappers around these functions.  Through ctypes such a call spends 13 to 18 us in Python and
// the kernels of a single token take 3 to 15 us; from here it spends about half of that.
#include <Python.h>

#include <cmath>
#include <cstring>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/kb_attention.h"

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
struct {
  decltype(&::kb_qk_norm_rope) qk_norm_rope;
  decltype(&::kb_attention) attention;
  decltype(&::kb_attention_paged) attention_paged;
} g_attention;

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

// ---- attention (include/kb_attention.h) ----------------------------------------------------------

// A tensor as heads [tokens][heads][dim] with adjacent elements, any other strides.  The stride of an axis of
// one element is free (torch may report anything) and becomes one that suits the kernels.
struct Heads {
  int64_t tokens, heads, dim;
  uint64_t row, head;
  void* p;
};
uint64_t stride_of(const Call& c, const at::Tensor& t, int64_t axis, int64_t dim, const char* name) {
  if (t.size(axis) <= 1) return (uint64_t)((dim + 7) / 8 * 8);
  if (t.stride(axis) < 0) refuse(c.where, std::string(name) + " has a negative stride");
  return (uint64_t)t.stride(axis);
}
Heads heads_of(const Call& c, const at::Tensor& t, const char* name) {
  if (t.dim() != 3) refuse(c.where, std::string(name) + " must be [tokens, heads, dim]");
  const int64_t dim = t.size(2);
  if (t.size(1) > 0x7FFFFFFF || dim > 0x7FFFFFFF) refuse(c.where, std::string(name) + " has more than 2^31 - 1 heads, or elements of one");
  if (dim > 1 && t.numel() && t.stride(2) != 1) refuse(c.where, std::string("the elements of the heads of ") + name + " must be adjacent");
  Heads h{t.size(0), t.size(1), dim, 0, 0, t.data_ptr()};
  h.head = stride_of(c, t, 1, dim, name);
  h.row = t.size(0) <= 1 ? (uint64_t)std::max<int64_t>(1, t.size(1)) * std::max<uint64_t>(h.head, (uint64_t)((dim + 7) / 8 * 8)) : stride_of(c, t, 0, dim, name);
  if (t.size(1) <= 1 && t.size(0) > 1) h.head = (uint64_t)((dim + 7) / 8 * 8);
  return h;
}
void same_type(const Call& c, const at::Tensor& t, at::ScalarType type, const char* name) {
  if (t.scalar_type() != type) refuse(c.where, std::string(name) + " must be of type " + c10::toString(type));
}
kb_paged_cache cache_of(const Call& c, const at::Tensor& k, const at::Tensor& v, int64_t heads, int64_t dim, at::ScalarType type) {
  const char* names[2] = {"k_cache", "v_cache"};
  const at::Tensor* both[2] = {&k, &v};
  for (int i = 0; i < 2; ++i) {
    const at::Tensor& t = *both[i];
    if (t.dim() != 4 || t.size(2) != heads || t.size(3) != dim || (dim > 1 && t.numel() && t.stride(3) != 1))
      refuse(c.where, std::string(names[i]) + " must be [pages, page size, " + std::to_string(heads) + ", " + std::to_string(dim) +
                          "] with adjacent elements");
    same_type(c, t, type, names[i]);
  }
  if (k.size(0) != v.size(0) || k.size(1) != v.size(1)) refuse(c.where, "k_cache and v_cache differ in pages or their size");
  if (k.size(1) < 1 || k.size(1) > 0x7FFFFFFF) refuse(c.where, "pages of no slot, or of more than 2^31 - 1");
  kb_paged_cache r;
  r.d_k = k.data_ptr();
  r.d_v = v.data_ptr();
  r.k_page = stride_of(c, k, 0, dim, "k_cache");
  r.k_row = stride_of(c, k, 1, dim, "k_cache");
  r.k_head = stride_of(c, k, 2, dim, "k_cache");
  r.v_page = stride_of(c, v, 0, dim, "v_cache");
  r.v_row = stride_of(c, v, 1, dim, "v_cache");
  r.v_head = stride_of(c, v, 2, dim, "v_cache");
  r.pages = (uint64_t)k.size(0);
  r.page_size = (uint32_t)k.size(1);
  return r;
}
const at::Tensor& given(const Call& c, PyObject* o, const at::Tensor& like, int64_t heads, const char* name) {
  const at::Tensor& t = tensor(c, o, name);
  if (t.dim() != 3 || t.size(0) != like.size(0) || t.size(1) != heads || t.size(2) != like.size(2))
    refuse(c.where, std::string(name) + " must be [" + std::to_string(like.size(0)) + ", " + std::to_string(heads) + ", " +
                        std::to_string(like.size(2)) + "]");
  same_type(c, t, like.scalar_type(), name);
  return t;
}
uint32_t count32(const Call& c, int64_t n, const char* what) {
  if (n > 0x7FFFFFFF) refuse(c.where, std::string(what) + " beyond 2^31 - 1");
  return (uint32_t)n;
}
// the addresses of empty tensors are null, which would mean "not given": with nothing to do any address will do
alignas(16) float g_nothing[4];
template <class T>
T* some(T* p) {
  return p ? p : reinterpret_cast<T*>(g_nothing);
}

// (handle, device, q, k, positions, inv_freq, q_weight, k_weight, eps, norm, interleaved, want_q, want_k, v, k_cache, v_cache,
//  slots, q_out, k_out) -> (q_out, k_out)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 19, [&]() -> PyObject* {
    const Call c = open_call("kb_qk_norm_rope", a[0], a[1]);
    const at::Tensor &q = tensor(c, a[2], "q"), &k = tensor(c, a[3], "k");
    const Heads hq = heads_of(c, q, "q"), hk = heads_of(c, k, "k");
    const at::ScalarType type = q.scalar_type();
    if (hk.tokens != hq.tokens || hk.dim != hq.dim) refuse(c.where, "k must have the tokens and the dim of q");
    same_type(c, k, type, "k");
    const double eps = PyFloat_AsDouble(a[8]);
    if (eps == -1.0 && PyErr_Occurred()) throw Refused{};
    const bool norm = truth(a[9]), interleaved = truth(a[10]), want_q = truth(a[11]), want_k = truth(a[12]);
    uint32_t rotary = 0;
    const int64_t* positions = nullptr;
    const double* inv_freq = nullptr;
    if (a[5] != Py_None) {
      const at::Tensor &f = tensor(c, a[5], "inv_freq"), &t = tensor(c, a[4], "positions");
      inv_freq = static_cast<const double*>(vector_of(c, f, f.numel(), "inv_freq", at::kDouble, at::kDouble));
      positions = static_cast<const int64_t*>(vector_of(c, t, hq.tokens, "positions", at::kLong, at::kLong));
      if (f.numel() > KB_ROPE_MAX_DIM) refuse(c.where, "inv_freq has more elements than a head has pairs");
      rotary = (uint32_t)(2 * f.numel());
    }
    at::ScalarType params = type;
    void *wq = nullptr, *wk = nullptr;
    if (a[6] != Py_None) {
      const at::Tensor& t = tensor(c, a[6], "q_weight");
      wq = vector_of(c, t, hq.dim, "q_weight", type, at::kFloat);
      params = t.scalar_type();
    }
    if (a[7] != Py_None) {
      const at::Tensor& t = tensor(c, a[7], "k_weight");
      wk = vector_of(c, t, hq.dim, "k_weight", type, at::kFloat);
      if (wq && t.scalar_type() != params) refuse(c.where, "q_weight and k_weight must have the same type");
      params = t.scalar_type();
    }
    const bool cached = a[14] != Py_None || a[15] != Py_None;
    kb_paged_cache cache = {};
    Heads hv = {};
    const int64_t* slots = nullptr;
    if (cached) {
      const at::Tensor& v = tensor(c, a[13], "v");
      hv = heads_of(c, v, "v");
      if (hv.tokens != hk.tokens || hv.heads != hk.heads || hv.dim != hk.dim) refuse(c.where, "v must have the shape of k");
      same_type(c, v, type, "v");
      cache = cache_of(c, tensor(c, a[14], "k_cache"), tensor(c, a[15], "v_cache"), hk.heads, hk.dim, type);
      slots = static_cast<const int64_t*>(vector_of(c, tensor(c, a[16], "slots"), hq.tokens, "slots", at::kLong, at::kLong));
    } else if (a[13] != Py_None || a[16] != Py_None) {
      refuse(c.where, "v and slots belong to a cache");
    }
    at::Tensor qo, ko;
    if (a[17] != Py_None)
      qo = given(c, a[17], q, hq.heads, "q_out");
    else if (want_q)
      qo = c.empty({hq.tokens, hq.heads, hq.dim}, type);
    if (a[18] != Py_None)
      ko = given(c, a[18], k, hk.heads, "k_out");
    else if (want_k)
      ko = c.empty({hk.tokens, hk.heads, hk.dim}, type);
    Heads oq = {}, ok = {};
    if (qo.defined()) oq = heads_of(c, qo, "q_out");
    if (ko.defined()) ok = heads_of(c, ko, "k_out");
    c.run([&] {
      return g_attention.qk_norm_rope(c.ctx, hq.p, hq.row, hq.head, (uint32_t)hq.heads, hk.p, hk.row, hk.head, (uint32_t)hk.heads,
                                hq.tokens, (uint32_t)hq.dim, (kb_dtype)code_of(type), norm, wq, wk, (kb_dtype)code_of(params),
                                (float)eps, positions, inv_freq, rotary, interleaved, oq.p, oq.row, oq.head, ok.p, ok.row,
                                ok.head, hv.p, hv.row, hv.head, cached ? &cache : nullptr, slots, c.stream);
    });
    return wrap_tuple({qo, ko});
  });
}

double scale_of(PyObject* o, int64_t dim) {
  if (o == Py_None) return 1.0 / std::sqrt((double)std::max<int64_t>(1, dim));
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{};
  return v;
}

// (handle, device, q, k, v, q_offsets or None, k_offsets or None, causal, scale or None, want_lse, out or None) -> (out, lse)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    const Call c = open_call("kb_attention", a[0], a[1]);
    const at::Tensor &q = tensor(c, a[2], "q"), &k = tensor(c, a[3], "k"), &v = tensor(c, a[4], "v");
    const Heads hq = heads_of(c, q, "q"), hk = heads_of(c, k, "k"), hv = heads_of(c, v, "v");
    const at::ScalarType type = q.scalar_type();
    same_type(c, k, type, "k");
    same_type(c, v, type, "v");
    if (hk.dim != hq.dim) refuse(c.where, "k must have the dim of q");
    if (hv.tokens != hk.tokens || hv.heads != hk.heads || hv.dim != hk.dim) refuse(c.where, "v must have the shape of k");
    int64_t sequences = 1;
    const int32_t *qo = nullptr, *ko = nullptr;
    if (a[5] != Py_None) {
      const at::Tensor& t = tensor(c, a[5], "q_offsets");
      sequences = t.numel() - 1;
      if (sequences < 0) refuse(c.where, "q_offsets must have an element more than there are sequences");
      qo = ko = static_cast<const int32_t*>(vector_of(c, t, t.numel(), "q_offsets", at::kInt, at::kInt));
      if (a[6] != Py_None) ko = static_cast<const int32_t*>(vector_of(c, tensor(c, a[6], "k_offsets"), sequences + 1, "k_offsets", at::kInt, at::kInt));
      else if (hk.tokens != hq.tokens) refuse(c.where, "without k_offsets k must have the tokens of q");
    } else if (a[6] != Py_None) {
      refuse(c.where, "k_offsets without q_offsets");
    }
    const bool causal = truth(a[7]), want_lse = truth(a[9]);
    const double scale = scale_of(a[8], hq.dim);
    const at::Tensor out = a[10] == Py_None ? c.empty({hq.tokens, hq.heads, hq.dim}, type) : given(c, a[10], q, hq.heads, "out");
    const Heads ho = heads_of(c, out, "out");
    at::Tensor lse;
    if (want_lse) lse = c.empty({hq.tokens, hq.heads}, at::kFloat);
    float* lp = want_lse ? lse.data_ptr<float>() : nullptr;
    const uint32_t count = count32(c, sequences, "sequences");
    c.run([&] {
      return g_attention.attention(c.ctx, hq.p, hq.row, hq.head, (uint32_t)hq.heads, hq.tokens, hk.p, hk.row, hk.head, hv.p, hv.row,
                             hv.head, (uint32_t)hk.heads, hk.tokens, (uint32_t)hq.dim, (kb_dtype)code_of(type), qo, ko, count,
                             causal, (float)scale, ho.p, ho.row, ho.head, lp, c.stream);
    });
    return wrap_tuple({out, lse});
  });
}

// (handle, device, q, k_cache, v_cache, table, lengths, scale or None, want_lse, out or None) -> (out, lse)
PyObject* attention_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const Call c = open_call("kb_attention_paged", a[0], a[1]);
    const at::Tensor &q = tensor(c, a[2], "q"), &k = tensor(c, a[3], "k_cache"), &v = tensor(c, a[4], "v_cache");
    const at::Tensor &table = tensor(c, a[5], "table"), &lengths = tensor(c, a[6], "lengths");
    const Heads hq = heads_of(c, q, "q");
    const at::ScalarType type = q.scalar_type();
    if (k.dim() != 4) refuse(c.where, "k_cache must be [pages, page size, heads, dim]");
    const int64_t hkv = k.size(2);
    const kb_paged_cache cache = cache_of(c, k, v, hkv, hq.dim, type);
    if (table.dim() != 2 || table.size(0) != hq.tokens || table.scalar_type() != at::kInt || (table.size(1) > 1 && table.numel() && table.stride(1) != 1))
      refuse(c.where, "table must be an int32 matrix [" + std::to_string(hq.tokens) + ", pages] with adjacent columns");
    const uint64_t table_row = hq.tokens > 1 ? (uint64_t)std::max<int64_t>(0, table.stride(0)) : (uint64_t)table.size(1);
    const int32_t* lens = static_cast<const int32_t*>(vector_of(c, lengths, hq.tokens, "lengths", at::kInt, at::kInt));
    const double scale = scale_of(a[7], hq.dim);
    const bool want_lse = truth(a[8]);
    const at::Tensor out = a[9] == Py_None ? c.empty({hq.tokens, hq.heads, hq.dim}, type) : given(c, a[9], q, hq.heads, "out");
    const Heads ho = heads_of(c, out, "out");
    at::Tensor lse;
    if (want_lse) lse = c.empty({hq.tokens, hq.heads}, at::kFloat);
    float* lp = want_lse ? lse.data_ptr<float>() : nullptr;
    const uint32_t most = count32(c, table.size(1), "pages of a sequence"), sequences = count32(c, hq.tokens, "sequences");
    const int32_t* tp = table.data_ptr<int32_t>();
    kb_paged_cache held = cache;
    if (held.pages == 0) held.d_k = some(held.d_k), held.d_v = some(held.d_v);
    c.run([&] {
      return g_attention.attention_paged(c.ctx, hq.p, hq.row, hq.head, (uint32_t)hq.heads, &held, (uint32_t)hkv, (uint32_t)hq.dim,
                                   (kb_dtype)code_of(type), tp, table_row, most, lens, sequences, (float)scale, ho.p, ho.row,
                                   ho.head, lp, c.stream);
    });
    return wrap_tuple({out, lse});
  });
}

// Sets the entry points of `table` to the addresses a[0], a[1], ..
template <typename Table>
void set_entries(Table& table, PyObject* const* a) {
  void* p[sizeof table / sizeof(void*)];
  for (size_t i = 0; i < sizeof p / sizeof *p; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) throw Refused{};
  }
  static_assert(sizeof p == sizeof table, "one address per entry point");
  std::memcpy(&table, p, sizeof p);
}
// (error class, addresses of the entry points in the order of g_lib)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 1 + sizeof g_lib / sizeof(void*), [&]() -> PyObject* {
    set_entries(g_lib, a + 1);
    Py_INCREF(a[0]);
    Py_XSETREF(g_error, a[0]);
    Py_RETURN_NONE;
  });
}
// (addresses of the entry points in the order of g_attention)
PyObject* bind_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, sizeof g_attention / sizeof(void*), [&]() -> PyObject* {
    set_entries(g_attention, a);
    Py_RETURN_NONE;
  });
}

#define KB_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {KB_FAST(quantize_blocks),
                         KB_FAST(layernorm),
                         KB_FAST(layernorm_backward),
                         KB_FAST(matmul_blocks),
                         KB_FAST(qk_norm_rope),
                         KB_FAST(attention),
                         KB_FAST(attention_paged),
                         KB_FAST(bind),
                         KB_FAST(bind_attention),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kb_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kb_torch() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", KB_BUILT_FOR) < 0) Py_CLEAR(m);
  return m;
}
