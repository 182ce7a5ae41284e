// Marshalling of the entry points that a program calls per layer or per batch: torch tensors to raw pointers, the current
// stream, one call of the C ABI without the interpreter lock.  The same checks, errors and results as the ctypes layer in
// binding.py, which holds the declarations and everything that is called rarely; a call through ctypes costs its eleven
// conversions (q8_conv2d of the smallest layer 7.0 us of host time, detection output with six sources 52 us).
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>
#include <ATen/cuda/EmptyTensor.h>

#include <cstdint>
#include <vector>

#include "q8.h"

namespace {

// C ABI entry points, by the addresses the ctypes layer has loaded (one copy of the library, one set of error strings).
struct Entry {
  decltype(&q8_conv2d) conv2d;
  decltype(&q8_conv2d_then_1x1) then_1x1;
  decltype(&q8_calibrate_maxabs) maxabs;
  decltype(&q8_quantize) quantize;
  decltype(&q8_dequantize) dequantize;
  decltype(&q8_detection_output_workspace_bytes) det_bytes;
  decltype(&q8_detection_output) detect;
  decltype(&q8_quantize_tokens) quantize_tokens;
  decltype(&q8_dequantize_tokens) dequantize_tokens;
  decltype(&q8_linear_workspace_bytes) linear_bytes;
  decltype(&q8_linear) linear;
  decltype(&q8_moe_workspace_bytes) moe_bytes;
  decltype(&q8_moe) moe;
} g_q8;

void* current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// Address of a contiguous CUDA tensor or of nothing (None); on anything else a TypeError is set and false returned.
bool dev(PyObject* o, const char* what, void** p) {
  *p = nullptr;
  if (o == Py_None) return true;
  if (THPVariable_Check(o)) {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.is_cuda() && t.is_contiguous()) {
      *p = t.numel() ? t.data_ptr() : nullptr;
      return true;
    }
  }
  PyErr_Format(PyExc_TypeError, "%s: expected a contiguous CUDA tensor", what);
  return false;
}

PyObject* g_desc_type = nullptr;  // the binding's ctypes structure

// The bytes of a descriptor, an instance of that structure or of a class derived from it.
struct Bytes {
  Py_buffer b{};
  bool ok = false;
  explicit Bytes(PyObject* o) { ok = PyObject_IsInstance(o, g_desc_type) == 1 && PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) == 0; }
  ~Bytes() { if (ok) PyBuffer_Release(&b); }
  const q8_conv_desc* desc() const {
    if (ok && (size_t)b.len >= sizeof(q8_conv_desc)) return static_cast<const q8_conv_desc*>(b.buf);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "expected a q8_conv_desc");
    return nullptr;
  }
};

template <typename F>
PyObject* call(F f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

// The same for a call whose status the caller goes on with.
template <typename F>
int unlocked(F f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return rc;
}

bool number(PyObject* o, float* v) {
  const double d = PyFloat_AsDouble(o);
  if (d == -1.0 && PyErr_Occurred()) return false;
  *v = (float)d;
  return true;
}
bool number(PyObject* o, int* v) {
  const long l = PyLong_AsLong(o);
  if (l == -1 && PyErr_Occurred()) return false;
  *v = (int)l;
  return true;
}

bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments", want);
  return false;
}

// (desc, x, w, bias, scale, residual, residual_scale, y, workspace) -> status
PyObject* py_conv2d(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 9)) return nullptr;
  HANDLE_TH_ERRORS
  Bytes d(a[0]);
  const q8_conv_desc* desc = d.desc();
  void *x, *w, *bias, *scale, *res, *y, *ws;
  float rs;
  if (!desc || !dev(a[1], "x", &x) || !dev(a[2], "w", &w) || !dev(a[3], "bias", &bias) || !dev(a[4], "scale", &scale) ||
      !dev(a[5], "residual", &res) || !number(a[6], &rs) || !dev(a[7], "y", &y) || !dev(a[8], "workspace", &ws))
    return nullptr;
  const size_t bytes = a[8] == Py_None ? 0 : THPVariable_Unpack(a[8]).nbytes();
  void* s = current_stream();
  return call([&] {
    return g_q8.conv2d(desc, x, static_cast<const int8_t*>(w), static_cast<const int32_t*>(bias), static_cast<const float*>(scale), res, rs,
                       y, ws, bytes, s);
  });
  END_HANDLE_TH_ERRORS
}

// (d1, d2, x, w1, bias1, scale1, w2, bias2, scale2, residual, residual_scale, y) -> status
PyObject* py_then_1x1(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 12)) return nullptr;
  HANDLE_TH_ERRORS
  Bytes b1(a[0]), b2(a[1]);
  const q8_conv_desc* d1 = b1.desc();
  const q8_conv_desc* d2 = d1 ? b2.desc() : nullptr;
  void *x, *w1, *bias1, *scale1, *w2, *bias2, *scale2, *res, *y;
  float rs;
  if (!d1 || !d2 || !dev(a[2], "x", &x) || !dev(a[3], "w1", &w1) || !dev(a[4], "bias1", &bias1) || !dev(a[5], "scale1", &scale1) ||
      !dev(a[6], "w2", &w2) || !dev(a[7], "bias2", &bias2) || !dev(a[8], "scale2", &scale2) || !dev(a[9], "residual", &res) ||
      !number(a[10], &rs) || !dev(a[11], "y", &y))
    return nullptr;
  void* s = current_stream();
  return call([&] {
    return g_q8.then_1x1(d1, d2, x, static_cast<const int8_t*>(w1), static_cast<const int32_t*>(bias1), static_cast<const float*>(scale1),
                         static_cast<const int8_t*>(w2), static_cast<const int32_t*>(bias2), static_cast<const float*>(scale2), res, rs, y, s);
  });
  END_HANDLE_TH_ERRORS
}

// The elements of a tensor; anything else has the error of its attribute (dev() has let nothing but None through).
bool numel(PyObject* o, size_t* n) {
  if (THPVariable_Check(o)) {
    *n = (size_t)THPVariable_Unpack(o).numel();
    return true;
  }
  THPObjectPtr attr(PyObject_GetAttrString(o, "numel"));
  if (attr) PyErr_SetString(PyExc_TypeError, "expected a tensor");
  return false;
}

// (x, running_max) -> status
PyObject* py_maxabs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 2)) return nullptr;
  HANDLE_TH_ERRORS
  void *x, *m;
  size_t k;
  if (!dev(a[0], "x", &x) || !dev(a[1], "running_max", &m) || !numel(a[0], &k)) return nullptr;
  void* s = current_stream();
  return call([&] { return g_q8.maxabs(static_cast<const float*>(x), k, static_cast<float*>(m), s); });
  END_HANDLE_TH_ERRORS
}

// (x, q, type, out) -> status
PyObject* py_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 4)) return nullptr;
  HANDLE_TH_ERRORS
  void *x, *out;
  float q;
  int type;
  size_t k;
  if (!dev(a[0], "x", &x) || !number(a[1], &q) || !number(a[2], &type) || !dev(a[3], "out", &out) || !numel(a[0], &k)) return nullptr;
  void* s = current_stream();
  return call([&] { return g_q8.quantize(static_cast<const float*>(x), k, q, type, out, s); });
  END_HANDLE_TH_ERRORS
}

// (z, type, q, out) -> status
PyObject* py_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 4)) return nullptr;
  HANDLE_TH_ERRORS
  void *z, *out;
  float q;
  int type;
  size_t k;
  if (!dev(a[0], "z", &z) || !number(a[1], &type) || !number(a[2], &q) || !dev(a[3], "out", &out) || !numel(a[0], &k)) return nullptr;
  void* s = current_stream();
  return call([&] { return g_q8.dequantize(z, type, k, q, static_cast<float*>(out), s); });
  END_HANDLE_TH_ERRORS
}

// Address, cell stride in floats and cells per image of a CUDA fp32 tensor [N, cells..., values] whose cells lie a fixed
// stride apart (a contiguous tensor, or a slice of the last dimension of one).
bool cell_view(PyObject* o, const char* what, const float** p, int* stride, int* cells, int64_t* images) {
  const at::Tensor* t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
  if (!t || !t->is_cuda() || t->scalar_type() != at::kFloat || t->dim() < 2 || t->stride(-1) != 1) {
    PyErr_Format(PyExc_TypeError, "%s: expected a CUDA fp32 tensor with unit stride in its last dimension", what);
    return false;
  }
  *p = static_cast<const float*>(t->numel() ? t->data_ptr() : nullptr);
  *images = t->size(0);
  const int64_t d = t->dim();
  if (d == 2) {
    *stride = (int)t->stride(0);
    *cells = 1;
    return true;
  }
  *stride = (int)t->stride(-2);
  int64_t c = 1;
  for (int64_t i = 0; i < d - 2; ++i)
    if (t->size(i) > 1 && t->stride(i) != t->stride(i + 1) * t->size(i + 1)) {
      PyErr_Format(PyExc_TypeError, "%s: cells are not a fixed stride apart", what);
      return false;
    }
  for (int64_t i = 1; i < d - 1; ++i) c *= t->size(i);
  *cells = (int)c;
  return true;
}

// The sources of a detection output, a sequence of (loc, conf, boxes per cell); what int() takes counts boxes.
struct Sources {
  std::vector<const float*> loc, conf;
  std::vector<int> ls, cs, cells, boxes;
  int64_t images = 0;
  long long P = 0;   // boxes per image

  bool parse(PyObject* sources) {
    THPObjectPtr seq(PySequence_Fast(sources, "sources: expected a sequence"));
    if (!seq) return false;
    const Py_ssize_t k = PySequence_Fast_GET_SIZE(seq.get());
    loc.resize(k); conf.resize(k);
    ls.resize(k); cs.resize(k); cells.resize(k); boxes.resize(k);
    for (Py_ssize_t i = 0; i < k; ++i) {
      THPObjectPtr item(PySequence_Fast(PySequence_Fast_GET_ITEM(seq.get(), i), "sources: expected (loc, conf, boxes per cell)"));
      if (!item) return false;
      if (PySequence_Fast_GET_SIZE(item.get()) != 3) { PyErr_SetString(PyExc_ValueError, "sources: expected (loc, conf, boxes per cell)"); return false; }
      PyObject** e = PySequence_Fast_ITEMS(item.get());
      int ccells;
      int64_t ni, nc;
      if (!cell_view(e[0], "loc", &loc[i], &ls[i], &cells[i], &ni) || !cell_view(e[1], "conf", &conf[i], &cs[i], &ccells, &nc)) return false;
      if (i == 0) images = ni;
      if (ccells != cells[i] || nc != images || ni != images) {
        PyErr_SetString(PyExc_ValueError, "loc and conf of a source must cover the same cells of the same images");
        return false;
      }
      THPObjectPtr count(PyNumber_Long(e[2]));
      if (!count || !number(count.get(), &boxes[i])) return false;
      P += (long long)cells[i] * boxes[i];
    }
    return true;
  }
  int boxes_per_image() const { return (int)(P > 0x7fffffff ? 0x7fffffff : P); }
};

// (sources) -> (images, boxes per image)
PyObject* py_detect_size(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 1)) return nullptr;
  HANDLE_TH_ERRORS
  Sources src;
  if (!src.parse(a[0])) return nullptr;
  return Py_BuildValue("Li", (long long)src.images, src.boxes_per_image());
  END_HANDLE_TH_ERRORS
}

// Up to four numbers, what float() takes; those not given are zero.
bool variances(PyObject* o, float (&var)[4]) {
  THPObjectPtr vars(PySequence_Fast(o, "variances: expected a sequence"));
  if (!vars) return false;
  const Py_ssize_t k = PySequence_Fast_GET_SIZE(vars.get());
  if (k > 4) { PyErr_SetString(PyExc_IndexError, "variances: more than four values"); return false; }
  for (Py_ssize_t i = 0; i < 4; ++i) {
    var[i] = 0.0f;
    if (i >= k) continue;
    THPObjectPtr v(PyNumber_Float(PySequence_Fast_GET_ITEM(vars.get(), i)));
    if (!v || !number(v.get(), &var[i])) return false;
  }
  return true;
}

// (sources, priors, variances, classes, background, conf_thresh, nms_thresh, nms_top_k, keep_top_k, workspace, out, counts)
// -> status.  workspace, out and counts are given.
PyObject* py_detect(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 12)) return nullptr;
  HANDLE_TH_ERRORS
  Sources src;
  float var[4];
  if (!src.parse(a[0]) || !variances(a[2], var)) return nullptr;
  void *priors, *ws, *out, *counts;
  int classes, background, top, keep;
  float ct, nt;
  if (!dev(a[1], "priors", &priors) || !number(a[3], &classes) || !number(a[4], &background) || !number(a[5], &ct) || !number(a[6], &nt) ||
      !number(a[7], &top) || !number(a[8], &keep) || !dev(a[9], "workspace", &ws) || !dev(a[10], "out", &out) || !dev(a[11], "counts", &counts))
    return nullptr;
  size_t ws_bytes;
  if (!numel(a[9], &ws_bytes)) return nullptr;
  void* s = current_stream();
  return call([&] {
    size_t need;
    const int rc = g_q8.det_bytes((int)src.images, src.boxes_per_image(), classes, background, top, keep, &need);
    if (rc != Q8_OK) return rc;
    return g_q8.detect((int)src.loc.size(), src.loc.data(), src.ls.data(), src.conf.data(), src.cs.data(), src.cells.data(), src.boxes.data(),
                       static_cast<const float*>(priors), var, (int)src.images, classes, background, ct, nt, top, keep, ws, ws_bytes,
                       static_cast<float*>(out), static_cast<int32_t*>(counts), s);
  });
  END_HANDLE_TH_ERRORS
}

// ---- token operators: tensors of rows a fixed stride apart, outputs made here where none are given

int float_type(at::ScalarType t) { return t == at::kFloat ? Q8_F32 : (t == at::kHalf ? Q8_F16 : (t == at::kBFloat16 ? Q8_BF16 : -1)); }
bool scalar_of(int type, at::ScalarType* t) {
  switch (type) {
    case Q8_F32: *t = at::kFloat; return true;
    case Q8_F16: *t = at::kHalf; return true;
    case Q8_BF16: *t = at::kBFloat16; return true;
    default: return false;
  }
}

enum Kinds { kFloats = 1, kCodes = 2 };

// A CUDA tensor [..., C] on the current device whose rows lie a fixed stride apart (contiguous, or a slice of the last dimension
// of a wider tensor).  type: Q8_S8 or a floating-point type.
struct Rows {
  void* p = nullptr;
  int64_t rows = 0, C = 0, ld = 0;
  int type = -1;
  const at::Tensor* t = nullptr;

  bool parse(PyObject* o, const char* what, int kinds) {
    t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
    if (t && t->is_cuda()) {
      type = t->scalar_type() == at::kChar ? (int)Q8_S8 : float_type(t->scalar_type());
      if (!(type == Q8_S8 ? kinds & kCodes : kinds & kFloats)) type = -1;
    }
    if (!t || type < 0 || t->dim() < 1) {
      PyErr_Format(PyExc_TypeError, "%s: expected a CUDA tensor of %s with at least one dimension", what,
                   kinds == kCodes ? "int8" : (kinds == kFloats ? "fp32, fp16 or bf16" : "int8, fp32, fp16 or bf16"));
      return false;
    }
    if (t->device().index() != c10::cuda::current_device()) { PyErr_Format(PyExc_TypeError, "%s: expected a tensor on the current device", what); return false; }
    const int64_t d = t->dim();
    C = ld = t->size(d - 1);
    if (t->numel() == 0) return true;
    if (C > 1 && t->stride(d - 1) != 1) { PyErr_Format(PyExc_TypeError, "%s: expected unit stride in the last dimension", what); return false; }
    rows = 1;
    for (int64_t i = d - 2; i >= 0; --i) {
      if (t->size(i) == 1) continue;
      if (rows == 1) {
        ld = t->stride(i);
      } else if (t->stride(i) != ld * rows) {
        PyErr_Format(PyExc_TypeError, "%s: rows are not a fixed stride apart", what);
        return false;
      }
      rows *= t->size(i);
    }
    if (rows > 1 && ld < C) { PyErr_Format(PyExc_TypeError, "%s: rows overlap", what); return false; }
    p = t->data_ptr();
    return true;
  }
};

// Address of a contiguous CUDA tensor of n values of type `st` on the current device; None: null where that is allowed.
bool values(PyObject* o, const char* what, int64_t n, at::ScalarType st, const char* st_name, bool optional, void** p) {
  *p = nullptr;
  if (optional && o == Py_None) return true;
  const at::Tensor* t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
  if (!t || !t->is_cuda() || t->scalar_type() != st || !t->is_contiguous() || t->numel() != n || t->device().index() != c10::cuda::current_device()) {
    PyErr_Format(PyExc_TypeError, "%s: expected a contiguous CUDA tensor of %lld %s values on the current device", what, (long long)n, st_name);
    return false;
  }
  *p = n ? t->data_ptr() : nullptr;
  return true;
}
// ... of the shape given.
bool dense(PyObject* o, const char* what, at::IntArrayRef shape, at::ScalarType st, const char* st_name, void** p) {
  const at::Tensor* t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
  if (!t || t->sizes() != shape) {
    PyErr_Format(PyExc_TypeError, "%s: expected another shape", what);
    return false;
  }
  return values(o, what, t->numel(), st, st_name, false, p);
}

// A new tensor where `like` is, past the dispatcher (a fifth of the time of at::empty less, which an eager call of a small kernel
// feels: codes and factors of one token 5.1 -> 4.8 us on the host).
at::Tensor fresh(at::IntArrayRef sizes, const at::Tensor& like, at::ScalarType st) {
  return at::Tensor(at::detail::empty_cuda(sizes, st, like.device(), std::nullopt));
}
// ... with the sizes of `like` but for the last, and without it.
at::Tensor made(const at::Tensor& like, int64_t last, at::ScalarType st) {
  auto sizes = like.sizes().vec();
  sizes.back() = last;
  return fresh(sizes, like, st);
}
at::Tensor made_scalar_per_row(const at::Tensor& like, at::ScalarType st) {
  return fresh(like.sizes().slice(0, like.dim() - 1), like, st);
}

// The interpreter's status for a call that has written `result` (stolen): (status, result).
PyObject* answer(int rc, PyObject* result) {
  if (!result) return nullptr;
  PyObject* t = Py_BuildValue("(iN)", rc, result);
  return t;
}

// (x, out, scale) -> (status, (out, scale))
PyObject* py_quantize_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 3)) return nullptr;
  HANDLE_TH_ERRORS
  Rows x, z;
  if (!x.parse(a[0], "x", kFloats)) return nullptr;
  THPObjectPtr out, scale;
  if (a[1] == Py_None) {
    const at::Tensor wide = made(*x.t, (x.C + 15) / 16 * 16, at::kChar);
    out = THPVariable_Wrap(x.C % 16 ? wide.narrow(-1, 0, x.C) : wide);
  } else {
    out = Py_NewRef(a[1]);
  }
  scale = a[2] == Py_None ? THPVariable_Wrap(made_scalar_per_row(*x.t, at::kFloat)) : Py_NewRef(a[2]);
  if (!out || !scale) return nullptr;
  void* s;
  if (!z.parse(out.get(), "out", kCodes)) return nullptr;
  if (z.rows != x.rows || z.C != x.C) { PyErr_SetString(PyExc_TypeError, "out: expected the shape of x"); return nullptr; }
  if (!values(scale.get(), "scale", x.rows, at::kFloat, "fp32", false, &s)) return nullptr;
  void* stream = current_stream();
  const int rc = unlocked([&] {
    return g_q8.quantize_tokens(x.p, x.type, (size_t)x.rows, (size_t)x.C, (size_t)x.ld, static_cast<int8_t*>(z.p), (size_t)z.ld, static_cast<float*>(s), stream);
  });
  return answer(rc, PyTuple_Pack(2, out.get(), scale.get()));
  END_HANDLE_TH_ERRORS
}

// (z, scale, out_type, out) -> (status, out)
PyObject* py_dequantize_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 4)) return nullptr;
  HANDLE_TH_ERRORS
  Rows z, r;
  int type;
  void* s;
  if (!z.parse(a[0], "z", kCodes) || !number(a[2], &type) || !values(a[1], "scale", z.rows, at::kFloat, "fp32", false, &s)) return nullptr;
  THPObjectPtr out;
  if (a[3] == Py_None) {
    at::ScalarType st;
    if (!scalar_of(type, &st)) { PyErr_SetString(PyExc_ValueError, "out_type must be Q8_F32, Q8_F16 or Q8_BF16"); return nullptr; }
    out = THPVariable_Wrap(made(*z.t, z.C, st));
  } else {
    out = Py_NewRef(a[3]);
  }
  if (!out || !r.parse(out.get(), "out", kFloats)) return nullptr;
  if (r.rows != z.rows || r.C != z.C) { PyErr_SetString(PyExc_TypeError, "out: expected the shape of z"); return nullptr; }
  void* stream = current_stream();
  const int rc = unlocked([&] {
    return g_q8.dequantize_tokens(static_cast<const int8_t*>(z.p), (size_t)z.rows, (size_t)z.C, (size_t)z.ld, static_cast<const float*>(s), r.p, r.type,
                                  (size_t)r.ld, stream);
  });
  return answer(rc, out.release());
  END_HANDLE_TH_ERRORS
}

bool fits_int(int64_t v, const char* what) {
  if (v <= 0x7fffffff) return true;
  PyErr_Format(PyExc_ValueError, "%s: too large", what);
  return false;
}

// A workspace of `need` bytes: the tensor given, or one made here (held by *own until the call is enqueued).
bool workspace_of(PyObject* o, size_t need, const at::Tensor& like, at::Tensor* own, void** p, size_t* bytes) {
  if (o == Py_None) {
    *p = nullptr;
    *bytes = need;
    if (need) {
      *own = fresh({(int64_t)need}, like, at::kByte);
      *p = own->data_ptr();
    }
    return true;
  }
  if (!THPVariable_Check(o)) { PyErr_SetString(PyExc_TypeError, "workspace: expected a tensor"); return false; }
  *bytes = (size_t)THPVariable_Unpack(o).numel();
  return values(o, "workspace", (int64_t)*bytes, at::kByte, "uint8", false, p);
}

// (x, w, w_scale, x_scale, bias, out_type, out, workspace) -> (status, out)
PyObject* py_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 8)) return nullptr;
  HANDLE_TH_ERRORS
  Rows x, w, y;
  int type;
  void *ws, *xs, *bias, *space;
  if (!x.parse(a[0], "x", kFloats | kCodes) || !w.parse(a[1], "w", kCodes) || !number(a[5], &type)) return nullptr;
  if (w.t->dim() != 2 || w.C != x.C) { PyErr_SetString(PyExc_TypeError, "w: expected [K, C]"); return nullptr; }
  const int64_t K = w.t->size(0);
  if (!values(a[2], "w_scale", K, at::kFloat, "fp32", false, &ws) || !values(a[3], "x_scale", x.rows, at::kFloat, "fp32", true, &xs) ||
      !values(a[4], "bias", K, at::kFloat, "fp32", true, &bias) || !fits_int(x.rows, "x") || !fits_int(K, "w") || !fits_int(x.C, "x"))
    return nullptr;
  THPObjectPtr out;
  if (a[6] == Py_None) {
    at::ScalarType st;
    if (!scalar_of(type, &st)) { PyErr_SetString(PyExc_ValueError, "out_type must be Q8_F32, Q8_F16 or Q8_BF16"); return nullptr; }
    out = THPVariable_Wrap(made(*x.t, K, st));
  } else {
    out = Py_NewRef(a[6]);
  }
  if (!out || !y.parse(out.get(), "out", kFloats)) return nullptr;
  if (y.rows != x.rows || y.C != K) { PyErr_SetString(PyExc_TypeError, "out: expected [..., K]"); return nullptr; }
  const q8_linear_desc d{x.ld, w.ld, y.ld, (int32_t)x.rows, (int32_t)x.C, (int32_t)K, x.type, y.type, 0};
  size_t need = 0, bytes = 0;
  at::Tensor own;
  q8_linear_desc asked = d;  // rows that begin off the 16-byte grid need what those with a pitch off it do
  if (reinterpret_cast<uintptr_t>(x.p) % 16) asked.ldx |= 1;
  if (reinterpret_cast<uintptr_t>(w.p) % 16) asked.ldw |= 1;
  int rc = a[7] == Py_None ? g_q8.linear_bytes(&asked, &need) : Q8_OK;
  if (rc == Q8_OK) {
    if (!workspace_of(a[7], need, *x.t, &own, &space, &bytes)) return nullptr;
    void* stream = current_stream();
    rc = unlocked([&] {
      return g_q8.linear(&d, x.p, static_cast<const float*>(xs), static_cast<const int8_t*>(w.p), static_cast<const float*>(ws), static_cast<const float*>(bias),
                         y.p, space, bytes, stream);
    });
  }
  return answer(rc, out.release());
  END_HANDLE_TH_ERRORS
}

// (x, router, w_gate_up, s_gate_up, w_down, s_down, top_k, renormalize, out, ids, probs, workspace) -> (status, (out, ids, probs))
PyObject* py_moe(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 12)) return nullptr;
  HANDLE_TH_ERRORS
  Rows x, y;
  int top_k, renorm = PyObject_IsTrue(a[7]);
  if (renorm < 0 || !x.parse(a[0], "x", kFloats) || !number(a[6], &top_k)) return nullptr;
  const at::Tensor* wd = THPVariable_Check(a[4]) ? &THPVariable_Unpack(a[4]) : nullptr;
  if (!wd || wd->dim() != 3) { PyErr_SetString(PyExc_TypeError, "w_down: expected [E, C, I]"); return nullptr; }
  const int64_t E = wd->size(0), I = wd->size(2), C = x.C;
  void *router, *wgu, *sgu, *wdp, *sd, *ids, *probs, *space;
  if (!dense(a[1], "router", {E, C}, at::kFloat, "fp32", &router) || !dense(a[2], "w_gate_up", {E, 2 * I, C}, at::kChar, "int8", &wgu) ||
      !dense(a[3], "s_gate_up", {E, 2 * I}, at::kFloat, "fp32", &sgu) || !dense(a[4], "w_down", {E, C, I}, at::kChar, "int8", &wdp) ||
      !dense(a[5], "s_down", {E, C}, at::kFloat, "fp32", &sd) || !fits_int(x.rows, "x") || !fits_int(E, "router") || !fits_int(C, "x") || !fits_int(I, "w_down"))
    return nullptr;
  q8_moe_desc d{x.ld, 0, (int32_t)x.rows, (int32_t)C, (int32_t)I, (int32_t)E, top_k, x.type, renorm, 0};
  size_t need = 0, bytes = 0;
  int rc = g_q8.moe_bytes(&d, &need);
  if (rc != Q8_OK) return answer(rc, Py_NewRef(Py_None));
  THPObjectPtr out, o_ids, o_probs;
  out = a[8] == Py_None ? THPVariable_Wrap(made(*x.t, C, x.t->scalar_type())) : Py_NewRef(a[8]);
  o_ids = a[9] == Py_None ? THPVariable_Wrap(made(*x.t, top_k, at::kInt)) : Py_NewRef(a[9]);
  o_probs = a[10] == Py_None ? THPVariable_Wrap(made(*x.t, top_k, at::kFloat)) : Py_NewRef(a[10]);
  if (!out || !o_ids || !o_probs || !y.parse(out.get(), "out", kFloats)) return nullptr;
  if (y.rows != x.rows || y.C != C || y.type != x.type) { PyErr_SetString(PyExc_TypeError, "out: expected the shape and type of x"); return nullptr; }
  if (!values(o_ids.get(), "ids", x.rows * top_k, at::kInt, "int32", false, &ids) || !values(o_probs.get(), "probs", x.rows * top_k, at::kFloat, "fp32", false, &probs))
    return nullptr;
  d.ldy = y.ld;
  at::Tensor own;
  if (!workspace_of(a[11], need, *x.t, &own, &space, &bytes)) return nullptr;
  void* stream = current_stream();
  rc = unlocked([&] {
    return g_q8.moe(&d, x.p, static_cast<const float*>(router), static_cast<const int8_t*>(wgu), static_cast<const float*>(sgu), static_cast<const int8_t*>(wdp),
                    static_cast<const float*>(sd), y.p, static_cast<int32_t*>(ids), static_cast<float*>(probs), space, bytes, stream);
  });
  return answer(rc, PyTuple_Pack(3, out.get(), o_ids.get(), o_probs.get()));
  END_HANDLE_TH_ERRORS
}

// (addresses of the entry points, in the order of Entry, the descriptors' class)
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!count(n, 14)) return nullptr;
  void* p[13];
  for (int i = 0; i < 13; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) return nullptr;
  }
  PyObject* old = g_desc_type;
  Py_INCREF(a[13]);
  g_desc_type = a[13];
  Py_XDECREF(old);
  g_q8.conv2d = reinterpret_cast<decltype(g_q8.conv2d)>(p[0]);
  g_q8.then_1x1 = reinterpret_cast<decltype(g_q8.then_1x1)>(p[1]);
  g_q8.maxabs = reinterpret_cast<decltype(g_q8.maxabs)>(p[2]);
  g_q8.quantize = reinterpret_cast<decltype(g_q8.quantize)>(p[3]);
  g_q8.dequantize = reinterpret_cast<decltype(g_q8.dequantize)>(p[4]);
  g_q8.det_bytes = reinterpret_cast<decltype(g_q8.det_bytes)>(p[5]);
  g_q8.detect = reinterpret_cast<decltype(g_q8.detect)>(p[6]);
  g_q8.quantize_tokens = reinterpret_cast<decltype(g_q8.quantize_tokens)>(p[7]);
  g_q8.dequantize_tokens = reinterpret_cast<decltype(g_q8.dequantize_tokens)>(p[8]);
  g_q8.linear_bytes = reinterpret_cast<decltype(g_q8.linear_bytes)>(p[9]);
  g_q8.linear = reinterpret_cast<decltype(g_q8.linear)>(p[10]);
  g_q8.moe_bytes = reinterpret_cast<decltype(g_q8.moe_bytes)>(p[11]);
  g_q8.moe = reinterpret_cast<decltype(g_q8.moe)>(p[12]);
  Py_RETURN_NONE;
}

#define Q8_METHOD(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {Q8_METHOD("bind", py_bind),         Q8_METHOD("conv2d", py_conv2d),     Q8_METHOD("then_1x1", py_then_1x1),
                         Q8_METHOD("maxabs", py_maxabs),     Q8_METHOD("quantize", py_quantize), Q8_METHOD("dequantize", py_dequantize),
                         Q8_METHOD("detect", py_detect),     Q8_METHOD("detect_size", py_detect_size),
                         Q8_METHOD("quantize_tokens", py_quantize_tokens), Q8_METHOD("dequantize_tokens", py_dequantize_tokens),
                         Q8_METHOD("linear", py_linear),     Q8_METHOD("moe", py_moe),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_q8native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__q8native(void) { return PyModule_Create(&module); }
