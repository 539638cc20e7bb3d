// Python module of the operators that need no handle: argument checks, output
// allocation and the call, on torch tensors. It computes nothing. Calls of a few
// microseconds on the GPU come from here and not from ctypes, because the host's
// share was most of their time (balance loss of 256 tokens: 30 us a call with
// ctypes, 8.5 us on the GPU).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <string>
#include <vector>

#include "../../include/unif_moe.h"

namespace {

PyObject* g_error = nullptr;   // UnifMoeError
PyObject* g_memory = nullptr;  // torch's error for a failed allocation

// A Python exception is set.
struct Raised {};

[[noreturn]] void value_error(const std::string& what) {
  PyErr_SetString(PyExc_ValueError, what.c_str());
  throw Raised();
}

void check(int rc) {
  if (rc == UNIF_MOE_OK) return;
  PyObject* e = PyObject_CallFunction(g_error, "is", rc, unif_moe_last_error());
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw Raised();
}

using at::Tensor;

// The tensor of an argument; an undefined one for None.
Tensor tensor(PyObject* o, const char* name) {
  if (o == Py_None) return Tensor();
  if (!THPVariable_Check(o)) value_error(std::string(name) + ": need a tensor");
  return THPVariable_Unpack(o);
}

std::string shown(const Tensor& t) {
  std::string s = "[";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + "] of " + std::string(c10::toString(t.scalar_type())) + " on " + t.device().str();
}

int code(at::ScalarType t) {
  return t == at::kFloat ? UNIF_MOE_F32 : t == at::kBFloat16 ? UNIF_MOE_BF16 : -1;
}
at::ScalarType type_of(long c, const char* name) {
  if (c != UNIF_MOE_F32 && c != UNIF_MOE_BF16) value_error(std::string(name) + ": bad dtype");
  return c == UNIF_MOE_F32 ? at::kFloat : at::kBFloat16;
}

// The device that all tensors of a call are on and the call's stream, both current while
// the call runs: memory taken for outputs and workspaces then belongs to the stream
// that uses it, and is not given to another before that stream is done with it.
struct Place {
  c10::Device dev;
  c10::cuda::CUDAGuard guard;
  c10::cuda::OptionalCUDAStreamGuard on_stream;
  static c10::Device of(const Tensor& t, const char* name) {
    if (!t.defined() || !t.is_cuda()) value_error(std::string(name) + ": need a CUDA tensor");
    return t.device();
  }
  Place(const Tensor& t, const char* name, PyObject* s) : dev(of(t, name)), guard(dev) {
    if (s == Py_None) return;
    PyObject* h = PyObject_HasAttrString(s, "cuda_stream") ? PyObject_GetAttrString(s, "cuda_stream")
                                                           : Py_NewRef(s);
    if (!h) throw Raised();
    void* p = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    if (PyErr_Occurred()) throw Raised();
    on_stream.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(p), dev.index()));
  }
  void on(const Tensor& t, const char* name) const {
    if (t.device() != dev)
      value_error(std::string(name) + ": on " + t.device().str() + ", need " + dev.str());
  }
  void* stream() const { return c10::cuda::getCurrentCUDAStream(dev.index()).stream(); }
  Tensor empty(at::IntArrayRef size, at::ScalarType t) const {
    return Tensor(at::detail::empty_cuda(size, t, dev, std::nullopt));
  }
};

struct Rows {
  void* p = nullptr;
  int64_t ld = 0;
};

// [rows][width] with dense rows; NULL for an undefined tensor.
Rows rows_of(const Place& at, const Tensor& t, const char* name, int64_t rows, int64_t width,
             at::ScalarType type) {
  Rows r;
  if (!t.defined()) return r;
  if (t.scalar_type() != type || t.dim() != 2 || t.size(0) != rows || t.size(1) != width ||
      !t.is_cuda() || (width > 1 && t.stride(1) != 1))
    value_error(std::string(name) + ": need a CUDA tensor [" + std::to_string(rows) + "][" +
                std::to_string(width) + "] of " + c10::toString(type) + " with dense rows, got " +
                shown(t));
  at.on(t, name);
  r.p = t.data_ptr();
  r.ld = rows > 1 ? t.stride(0) : std::max<int64_t>(t.stride(0), width);
  return r;
}

// A contiguous tensor of `count` elements; NULL for an undefined tensor.
void* dense(const Place& at, const Tensor& t, const char* name, int64_t count, at::ScalarType type) {
  if (!t.defined()) return nullptr;
  if (t.scalar_type() != type || t.numel() != count || !t.is_cuda() || !t.is_contiguous())
    value_error(std::string(name) + ": need a contiguous CUDA tensor of " + std::to_string(count) +
                " elements of " + c10::toString(type) + ", got " + shown(t));
  at.on(t, name);
  return t.data_ptr();
}

const uint8_t* mask_of(const Place& at, const Tensor& t, int64_t T) {
  if (!t.defined()) return nullptr;
  return static_cast<const uint8_t*>(
      dense(at, t, "mask", T, t.scalar_type() == at::kBool ? at::kBool : at::kByte));
}

void put(PyObject* d, const char* key, const Tensor& t) {
  PyObject* o = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
  if (!o) throw Raised();
  const int rc = PyDict_SetItemString(d, key, o);
  Py_DECREF(o);
  if (rc) throw Raised();
}

long as_long(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}
int as_int(PyObject* o) {
  const long v = as_long(o);
  if (v != (int)v) value_error(std::to_string(v) + " does not fit in 32 bits");
  return (int)v;
}
bool as_bool(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised();
  return v != 0;
}
double as_double(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return v;
}

// C++ exceptions end here: Raised has its Python exception set, others become one.
template <typename F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t want, F f) {
  if (got != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, need %zd", got, want);
    return nullptr;
  }
  try {
    return f();
  } catch (const Raised&) {
    return nullptr;
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(g_memory, e.what_without_backtrace());
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// (tokens), then BlockNorm's (width, stream, branch, post, pre, gate_rows, scale, eps)
unif_moe_block_norm desc_of(PyObject* t, int64_t T) {
  if (!PyTuple_Check(t) || PyTuple_GET_SIZE(t) != 8) value_error("bad description");
  unif_moe_block_norm d;
  if (T > 0x7fffffff) value_error("more than 2^31 - 1 tokens");
  d.tokens = (int)T;
  int* ints[6] = {&d.width, &d.stream_dtype, &d.branch_dtype, &d.post_norm, &d.pre_norm, &d.gate_rows};
  for (int i = 0; i < 6; ++i) *ints[i] = as_int(PyTuple_GET_ITEM(t, i));
  d.res_scale = (float)as_double(PyTuple_GET_ITEM(t, 6));
  d.eps = (float)as_double(PyTuple_GET_ITEM(t, 7));
  return d;
}

struct NormParams {
  void *w_post, *b_post, *gate, *w_pre;
  int64_t gate_rows;
};
NormParams norm_params(const Place& at, const unif_moe_block_norm& d, PyObject* const* a) {
  const at::ScalarType tb = type_of(d.branch_dtype, "branch_dtype");
  const int64_t w = d.width;
  NormParams p;
  p.gate_rows = d.gate_rows == 0 ? 1 : ((int64_t)d.tokens + d.gate_rows - 1) / d.gate_rows;
  p.w_post = dense(at, tensor(a[0], "post_weight"), "post_weight", w, tb);
  p.b_post = dense(at, tensor(a[1], "post_bias"), "post_bias", w, tb);
  const Tensor gate = tensor(a[2], "gate");
  p.gate = dense(at, gate, "gate", p.gate_rows * w, tb);
  p.w_pre = dense(at, tensor(a[3], "pre_weight"), "pre_weight", w, tb);
  return p;
}

// desc, x, y, post_weight, post_bias, gate, pre_weight, pre_bias, mask, out, u, stats, stream
PyObject* norm_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 13, [&]() -> PyObject* {
    const Tensor x = tensor(a[1], "x"), y = tensor(a[2], "y");
    const Place at(x, "x", a[12]);
    if (x.dim() != 2) value_error("x: need two dimensions");
    const int64_t T = x.size(0);
    const unif_moe_block_norm d = desc_of(a[0], T);
    const at::ScalarType ts = type_of(d.stream_dtype, "stream_dtype"),
                         tb = type_of(d.branch_dtype, "branch_dtype");
    const Rows px = rows_of(at, x, "x", T, d.width, ts), py = rows_of(at, y, "y", T, d.width, tb);
    const NormParams p = norm_params(at, d, a + 3);
    const void* b_pre = dense(at, tensor(a[7], "pre_bias"), "pre_bias", d.width, tb);
    const uint8_t* mask = mask_of(at, tensor(a[8], "mask"), T);
    Tensor out = tensor(a[9], "out"), u = tensor(a[10], "u"), st[4];
    if (y.defined() && !out.defined()) out = at.empty({T, d.width}, ts);
    if (d.pre_norm && !u.defined()) u = at.empty({T, d.width}, tb);
    const Rows po = rows_of(at, out, "out", T, d.width, ts), pu = rows_of(at, u, "u", T, d.width, tb);
    float* sp[4] = {nullptr, nullptr, nullptr, nullptr};
    const bool stats = as_bool(a[11]);
    const bool there[2] = {y.defined() && d.post_norm != 0, d.pre_norm != 0};
    for (int i = 0; i < 4; ++i)  // of the norms that there are: nothing writes the others
      if (stats && there[i / 2]) {
        st[i] = at.empty({T}, at::kFloat);
        sp[i] = st[i].data_ptr<float>();
      }
    check(unif_moe_block_norm_forward(&d, px.p, px.ld, py.p, py.ld, mask, p.w_post, p.b_post, p.gate,
                                      p.w_pre, b_pre, po.p, po.ld, pu.p, pu.ld, sp[0], sp[1], sp[2],
                                      sp[3], at.stream()));
    PyObject* r = PyDict_New();
    if (!r) throw Raised();
    try {
      put(r, "out", y.defined() ? out : x);
      put(r, "u", d.pre_norm ? u : Tensor());
      static const char* names[4] = {"post_mean", "post_rstd", "pre_mean", "pre_rstd"};
      if (stats)
        for (int i = 0; i < 4; ++i) put(r, names[i], st[i]);
    } catch (...) {
      Py_DECREF(r);
      throw;
    }
    return r;
  });
}

// desc, out, y, (post_mean, post_rstd, pre_mean, pre_rstd), dout, du, post_weight, post_bias,
// gate, pre_weight, mask, stream
PyObject* norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 15, [&]() -> PyObject* {
    const Tensor out = tensor(a[1], "out"), y = tensor(a[2], "y"), dout = tensor(a[7], "dout"),
                 du = tensor(a[8], "du");
    const Tensor& ref = dout.defined() ? dout : du;
    if (!ref.defined()) value_error("dout and du are both None");
    const Place at(ref, dout.defined() ? "dout" : "du", a[14]);
    if (ref.dim() != 2) value_error("dout and du: need two dimensions");
    const int64_t T = ref.size(0);
    const unif_moe_block_norm d = desc_of(a[0], T);
    const at::ScalarType ts = type_of(d.stream_dtype, "stream_dtype"),
                         tb = type_of(d.branch_dtype, "branch_dtype");
    const int64_t w = d.width;
    Rows po;
    if (d.pre_norm) po = rows_of(at, out, "out", T, w, ts);
    const Rows py = rows_of(at, y, "y", T, w, tb), pdo = rows_of(at, dout, "dout", T, w, ts),
               pdu = rows_of(at, du, "du", T, w, tb);
    static const char* names[4] = {"post_mean", "post_rstd", "pre_mean", "pre_rstd"};
    float* st[4];
    for (int i = 0; i < 4; ++i)
      st[i] = static_cast<float*>(dense(at, tensor(a[3 + i], names[i]), names[i], T, at::kFloat));
    const NormParams p = norm_params(at, d, a + 9);
    const uint8_t* mask = mask_of(at, tensor(a[13], "mask"), T);
    const int64_t need = unif_moe_block_norm_workspace(&d, p.gate != nullptr);
    if (need < 0) check(UNIF_MOE_ERR_ARG);
    const Tensor dx = at.empty({T, w}, ts), ws = at.empty({need}, at::kByte);
    Tensor dy, g[5];
    if (y.defined()) dy = at.empty({T, w}, tb);
    float* gp[5] = {nullptr, nullptr, nullptr, nullptr, nullptr};
    const bool want[5] = {d.post_norm != 0, d.post_norm != 0, p.gate != nullptr, d.pre_norm != 0,
                          d.pre_norm != 0};
    for (int i = 0; i < 5; ++i)
      if (want[i]) {
        g[i] = i == 2 ? at.empty({p.gate_rows, w}, at::kFloat) : at.empty({w}, at::kFloat);
        gp[i] = g[i].data_ptr<float>();
      }
    check(unif_moe_block_norm_backward(
        &d, po.p, po.ld, py.p, py.ld, mask, p.w_post, p.b_post, p.gate, p.w_pre, st[0], st[1], st[2],
        st[3], pdo.p, pdo.ld, pdu.p, pdu.ld, dx.data_ptr(), w, y.defined() ? dy.data_ptr() : nullptr, w,
        gp[0], gp[1], gp[2], gp[3], gp[4], ws.data_ptr(), need, at.stream()));
    PyObject* r = PyDict_New();
    if (!r) throw Raised();
    try {
      put(r, "dx", dx);
      put(r, "dy", dy);
      static const char* keys[5] = {"d_post_weight", "d_post_bias", "d_gate", "d_pre_weight",
                                    "d_pre_bias"};
      for (int i = 0; i < 5; ++i)
        if (want[i]) put(r, keys[i], g[i]);
    } catch (...) {
      Py_DECREF(r);
      throw;
    }
    return r;
  });
}

// logits, q, k, mask, balance_weight, z_weight, grad, stream
PyObject* balance(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const Tensor z = tensor(a[0], "logits"), q = tensor(a[1], "q");
    const Place at(z, "logits", a[7]);
    const int type = code(z.scalar_type());
    if (type < 0 || z.dim() != 2) value_error("logits: need [T][K] of fp32 or bf16, got " + shown(z));
    const int64_t T = z.size(0), K = z.size(1);
    if (T > 0x7fffffff || K > 0x7fffffff) value_error("logits: too large");
    if (!q.defined() || q.dim() != 2) value_error("q: need two dimensions");
    const int64_t n_q = q.size(1);
    const Rows pz = rows_of(at, z, "logits", T, K, z.scalar_type()), pq = rows_of(at, q, "q", T, n_q, at::kInt);
    const void* k = dense(at, tensor(a[2], "k"), "k", T, at::kInt);
    const uint8_t* mask = mask_of(at, tensor(a[3], "mask"), T);
    const int64_t need = unif_moe_balance_workspace((int)T, (int)K);
    if (need < 0) check(K > UNIF_MOE_BALANCE_MAX_EXPERTS ? UNIF_MOE_ERR_SHAPE : UNIF_MOE_ERR_ARG);
    Tensor ws;
    if (need) ws = at.empty({need}, at::kByte);
    const Tensor loss = at.empty({3}, at::kFloat), counts = at.empty({K}, at::kInt), prob = at.empty({K}, at::kFloat);
    Tensor d;
    if (as_bool(a[6])) d = at.empty({T, K}, at::kFloat);
    check(unif_moe_balance_loss(
        (int)T, (int)K, pz.p, (unif_moe_dtype)type, pz.ld, static_cast<const int32_t*>(pq.p), (int)n_q,
        pq.ld, static_cast<const int32_t*>(k), mask, (float)as_double(a[4]), (float)as_double(a[5]),
        loss.data_ptr<float>(), counts.data_ptr<int32_t>(), prob.data_ptr<float>(),
        d.defined() ? d.data_ptr<float>() : nullptr, need ? ws.data_ptr() : nullptr, need,
        at.stream()));
    PyObject* r = PyDict_New();
    if (!r) throw Raised();
    try {
      put(r, "loss", loss);
      put(r, "counts", counts);
      put(r, "prob", prob);
      put(r, "dlogits", d);
    } catch (...) {
      Py_DECREF(r);
      throw;
    }
    return r;
  });
}

struct Fp4 {
  const uint8_t *codes = nullptr, *scales = nullptr;
  int64_t rows = 0;
};
int64_t code_bytes(int64_t cols) { return (cols + 31) / 32 * 16; }
int64_t scale_bytes(int64_t cols) { return (cols + 255) / 256 * 8; }
int64_t cols_of(PyObject* o, const char* name) {
  const long c = as_long(o);
  if (c < 1 || c > UNIF_MOE_MXFP4_MAX_COLS)
    value_error(std::string(name) + ": " + std::to_string(c) + " columns");
  return c;
}

// Rows in 4 bits: codes [...][code_bytes], scales of as many rows.
Fp4 fp4_of(const Place& at, const Tensor& codes, const Tensor& scales, int64_t cols, const char* name) {
  const std::string n(name);
  if (codes.dim() < 1 || codes.size(-1) != code_bytes(cols))
    value_error(n + ": codes of " + std::to_string(cols) + " columns are " +
                std::to_string(code_bytes(cols)) + " bytes a row, got " + shown(codes));
  if (!scales.defined()) value_error(n + ".scales: need a tensor");
  Fp4 r;
  r.rows = codes.numel() / code_bytes(cols);
  r.codes = static_cast<const uint8_t*>(dense(at, codes, (n + ".codes").c_str(), codes.numel(), at::kByte));
  r.scales = static_cast<const uint8_t*>(
      dense(at, scales, (n + ".scales").c_str(), r.rows * scale_bytes(cols), at::kByte));
  return r;
}

// x, out codes, out scales, out cols (or None), stream
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> PyObject* {
    const Tensor x = tensor(a[0], "x");
    const Place at(x, "x", a[4]);
    const int type = code(x.scalar_type());
    if (type < 0 || x.dim() < 1) value_error("x: need rows of fp32 or bf16, got " + shown(x));
    const int64_t cols = x.size(-1);
    if (cols < 1 || cols > UNIF_MOE_MXFP4_MAX_COLS) value_error("x: " + std::to_string(cols) + " columns");
    const int64_t rows = x.numel() / cols;
    Rows px;
    if (x.dim() == 2) {
      px = rows_of(at, x, "x", rows, cols, x.scalar_type());
    } else {
      px.p = dense(at, x, "x", rows * cols, x.scalar_type());
      px.ld = cols;
    }
    Tensor codes = tensor(a[1], "out.codes"), scales = tensor(a[2], "out.scales");
    if (codes.defined()) {
      if (as_long(a[3]) != cols || fp4_of(at, codes, scales, cols, "out").rows != rows)
        value_error("out: need " + std::to_string(rows) + " rows of " + std::to_string(cols) + " columns");
    } else {
      std::vector<int64_t> size(x.sizes().begin(), x.sizes().end());
      size.back() = code_bytes(cols);
      codes = at.empty(size, at::kByte);
      size.back() = scale_bytes(cols);
      scales = at.empty(size, at::kByte);
    }
    check(unif_moe_mxfp4_quantize(px.p, (unif_moe_dtype)type, rows, (int)cols, px.ld,
                                  static_cast<uint8_t*>(codes.data_ptr()),
                                  static_cast<uint8_t*>(scales.data_ptr()), at.stream()));
    return Py_BuildValue("(NNL)", THPVariable_Wrap(codes), THPVariable_Wrap(scales), (long long)cols);
  });
}

// codes, scales, cols, dtype code, out, stream
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const Tensor codes = tensor(a[0], "q.codes"), scales = tensor(a[1], "q.scales");
    const Place at(codes, "q.codes", a[5]);
    const int64_t cols = cols_of(a[2], "q");
    const Fp4 q = fp4_of(at, codes, scales, cols, "q");
    const long type = as_long(a[3]);
    const at::ScalarType t = type_of(type, "dtype");
    Tensor out = tensor(a[4], "out");
    Rows po;
    if (out.defined()) {
      po = rows_of(at, out, "out", q.rows, cols, t);
    } else {
      std::vector<int64_t> size(codes.sizes().begin(), codes.sizes().end());
      size.back() = cols;
      out = at.empty(size, t);
      po.p = out.data_ptr();
      po.ld = cols;
    }
    check(unif_moe_mxfp4_dequantize(q.codes, q.scales, q.rows, (int)cols, po.p, (unif_moe_dtype)type,
                                    po.ld, at.stream()));
    return THPVariable_Wrap(out);
  });
}

// a codes, a scales, a cols, w codes, w scales, w cols, offsets, activation, dtype code, out,
// status, stream
PyObject* product(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const Tensor ac = tensor(a[0], "a.codes"), wc = tensor(a[3], "w.codes");
    const Place at(ac, "a.codes", a[11]);
    const int64_t cols = cols_of(a[2], "a");
    if (as_long(a[5]) != cols) value_error("a and w have different numbers of columns");
    const Fp4 x = fp4_of(at, ac, tensor(a[1], "a.scales"), cols, "a");
    if (!wc.defined()) value_error("w.codes: need a tensor");
    const Fp4 w = fp4_of(at, wc, tensor(a[4], "w.scales"), cols, "w");
    const int64_t N = wc.dim() > 1 ? wc.size(-2) : 1, groups = N ? w.rows / N : 0;
    const Tensor offsets = tensor(a[6], "offsets");
    if (!offsets.defined() && groups != 1)
      value_error("offsets: needed with " + std::to_string(groups) + " groups");
    const long type = as_long(a[8]);
    const at::ScalarType t = type_of(type, "dtype");
    if (x.rows > 0x7fffffff || w.rows > 0x7fffffff) value_error("more than 2^31 - 1 rows");
    Tensor out = tensor(a[9], "out");
    if (!out.defined()) out = at.empty({x.rows, N}, t);
    const Rows po = rows_of(at, out, "out", x.rows, N, t);
    check(unif_moe_mxfp4_product(
        x.codes, x.scales, x.rows, (int)cols, w.codes, w.scales, (int)N, (int)groups,
        static_cast<const int32_t*>(dense(at, offsets, "offsets", groups + 1, at::kInt)),
        as_int(a[7]), po.p, (unif_moe_dtype)type, po.ld,
        static_cast<int32_t*>(dense(at, tensor(a[10], "status"), "status", 1, at::kInt)),
        at.stream()));
    return THPVariable_Wrap(out);
  });
}

// The classes that failed calls and failed allocations raise; before any other call.
PyObject* set_errors(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 2, [&]() -> PyObject* {
    Py_XSETREF(g_error, Py_NewRef(a[0]));
    Py_XSETREF(g_memory, Py_NewRef(a[1]));
    Py_RETURN_NONE;
  });
}

#define UNIF_FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {UNIF_FAST(norm_forward), UNIF_FAST(norm_backward), UNIF_FAST(balance),
                         UNIF_FAST(quantize), UNIF_FAST(dequantize), UNIF_FAST(product),
                         UNIF_FAST(set_errors), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
