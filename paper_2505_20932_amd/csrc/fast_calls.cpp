// The binding's most frequent calls without ctypes: a Python extension module that reads the tensors' pointers, sizes
// and strides directly, takes the current stream and calls the C entry point.
//
// Why: a call through ctypes takes 9 to 10 us of host time (a dozen tensor attributes and argument conversions through
// Python objects), the launch itself about 3.5; where kernels are shorter than that - a decoding step, one image -
// the host sets the pace.
//
// Every function returns True when the call was made and returned CWAC_OK, and False otherwise: an argument that is
// not exactly what the call documents, or an error status (nothing was launched then).  The caller goes on with
// the ctypes form, which makes the checks again and raises.  So nothing is refused or accepted here that was not before.
// CWAC_E_LAUNCH alone is raised from here: the runtime's error is taken with the status, and a second call could pass.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/TensorBase.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "cwac.h"

namespace {

// The entry points of the library that the ctypes binding loaded (`bind`), and its structure type for parameters.
struct Entries {
  decltype(&::cwac_quantize_act) quantize_act;
  decltype(&::cwac_quantize_rows_sym) quantize_rows_sym;
  decltype(&::qlinear_cwac_forward) forward;
  decltype(&::qlinear_cwac_forward_table) forward_table;
  decltype(&::qlinear_cwac_forward_fixed_point) forward_fixed_point;
  decltype(&::qconv2d_cwac_forward) conv2d;
  decltype(&::qlinear_w4a16_cwac_forward) w4a16;
  decltype(&::cwac_mx4_quantize) mx4_quantize;
  decltype(&::cwac_mx4_dequantize) mx4_dequantize;
  decltype(&::qlinear_mx4_cwac_forward) mx4_forward;
  decltype(&::llm_kv_assign_pages) kv_assign;
  decltype(&::llm_kv_append) kv_append;
  decltype(&::llm_paged_attention) paged_attention;
} g;
PyObject *g_qparams_type = nullptr, *g_check = nullptr;  // the binding's structure type and its check of a status

// What a call is given, checked one by one; `ok` stays true while everything is what the call documents.
struct Args {
  bool ok = true;

  // a plain tensor on the device
  const at::TensorBase *tensor(PyObject *o) {
    if (!ok || !THPVariable_CheckExact(o)) return fail();
    const at::TensorBase &t = THPVariable_Unpack(o);
    return t.is_cuda() ? &t : fail();
  }
  const at::TensorBase *typed(PyObject *o, at::ScalarType type) {
    const at::TensorBase *t = tensor(o);
    return t && t->scalar_type() == type ? t : fail();
  }
  // ... of two dimensions whose rows are contiguous
  const at::TensorBase *matrix(PyObject *o, at::ScalarType type) {
    const at::TensorBase *t = typed(o, type);
    return t && t->dim() == 2 && t->stride(1) == 1 ? t : fail();
  }
  // pointer of a tensor, NULL for None (elements are not looked at, as in the ctypes form)
  void *pointer(PyObject *o) {
    if (o == Py_None) return nullptr;
    const at::TensorBase *t = tensor(o);
    return t ? t->data_ptr() : nullptr;
  }
  long long integer(PyObject *o) {
    if (!PyLong_CheckExact(o)) return ok = false, 0;
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow || v > INT32_MAX || v < INT32_MIN) ok = false;
    return v;
  }
  float number(PyObject *o) {
    if (!PyFloat_CheckExact(o)) return ok = false, 0.0f;
    return (float)PyFloat_AS_DOUBLE(o);
  }
  // the caller's ctypes structure, read in place (the call copies it)
  const cwac_qparams *qparams(PyObject *o, bool nullable) {
    if (nullable && o == Py_None) return nullptr;
    Py_buffer view;
    if (!ok || (PyObject *)Py_TYPE(o) != g_qparams_type || PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) return fail_qp();
    if (view.len == (Py_ssize_t)sizeof(cwac_qparams))
      memcpy(&qp, view.buf, sizeof qp);
    else
      ok = false;
    PyBuffer_Release(&view);
    return &qp;
  }
  // None: the current stream of the current device
  void *stream(PyObject *o) {
    if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
    PyObject *v = PyObject_GetAttrString(o, "cuda_stream");
    void *s = v && PyLong_Check(v) ? PyLong_AsVoidPtr(v) : (ok = false, nullptr);
    Py_XDECREF(v);
    return s;
  }

 private:
  cwac_qparams qp;
  const at::TensorBase *fail() { return ok = false, nullptr; }
  const cwac_qparams *fail_qp() { return ok = false, nullptr; }
};

// A matrix of one row counts as one with the smallest pitch that holds it.
int64_t pitch(const at::TensorBase &t) {
  return t.size(0) > 1 ? t.stride(0) : (t.stride(0) > t.size(1) ? t.stride(0) : t.size(1));
}
bool same_shape(const at::TensorBase &a, const at::TensorBase &b) { return a.size(0) == b.size(0) && a.size(1) == b.size(1); }

// `f` for the entry point `name`: its result, False for tensors without storage (torch throws), an exception
// for a launch that failed.
struct LaunchFailed {};
template <typename F>
PyObject *guarded(const char *name, F &&f) {
  bool done = false;
  try {
    done = f();
  } catch (const LaunchFailed &) {
    PyErr_Clear();
    return PyObject_CallFunction(g_check, "is", (int)CWAC_E_LAUNCH, name);  // raises
  } catch (...) {
    done = false;
  }
  if (PyErr_Occurred()) PyErr_Clear();
  return PyBool_FromLong(done);
}

// Runs `call` with Python's lock released.
struct Unlock {
  PyThreadState *state = PyEval_SaveThread();
  ~Unlock() { PyEval_RestoreThread(state); }
};
template <typename F>
bool unlocked(F &&call) {
  const cwac_status st = [&] {
    Unlock u;
    return call();
  }();
  if (st == CWAC_E_LAUNCH) throw LaunchFailed();
  return st == CWAC_OK;
}

constexpr auto kI8 = at::kChar;
constexpr auto kF32 = at::kFloat;

// (x, s, z, q, stream)
PyObject *py_quantize_act(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("cwac_quantize_act", [&] {
    Args v;
    if (n != 5) return false;
    const at::TensorBase *x = v.matrix(a[0], kF32), *q = v.matrix(a[3], kI8);
    const float s = v.number(a[1]);
    const int32_t z = (int32_t)v.integer(a[2]);
    if (!v.ok || !same_shape(*x, *q)) return false;
    void *st = v.stream(a[4]);
    const float *xp = static_cast<const float *>(x->data_ptr());
    int8_t *qp = static_cast<int8_t *>(q->data_ptr());
    const int64_t rows = x->size(0), k = x->size(1), lx = pitch(*x), lq = pitch(*q);
    if (!v.ok || k > INT32_MAX) return false;
    return unlocked([&] { return g.quantize_act(xp, lx, rows, (int32_t)k, s, z, qp, lq, st); });
  });
}

// (x, scale, q, stream)
PyObject *py_quantize_rows_sym(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("cwac_quantize_rows_sym", [&] {
    Args v;
    if (n != 4) return false;
    const at::TensorBase *x = v.matrix(a[0], kF32), *scale = v.typed(a[1], kF32), *q = v.matrix(a[2], kI8);
    if (!v.ok || !same_shape(*x, *q) || scale->numel() != x->size(0)) return false;
    void *st = v.stream(a[3]);
    const float *xp = static_cast<const float *>(x->data_ptr());
    float *sp = static_cast<float *>(scale->data_ptr());
    int8_t *qp = static_cast<int8_t *>(q->data_ptr());
    const int64_t rows = x->size(0), k = x->size(1), lx = pitch(*x), lq = pitch(*q);
    if (!v.ok || k > INT32_MAX) return false;
    return unlocked([&] { return g.quantize_rows_sym(xp, lx, rows, (int32_t)k, sp, qp, lq, st); });
  });
}

// x_q [m, k] and w_q [n, k] of a linear layer and its output [m, n] of the given type
struct Linear {
  const int8_t *x, *w;
  void *out;
  int64_t m, ldx, ldw, ldo;
  int32_t n, k;
  bool take(Args &v, PyObject *xo, PyObject *wo, PyObject *oo, at::ScalarType type) {
    const at::TensorBase *xt = v.matrix(xo, kI8), *wt = v.matrix(wo, kI8), *ot = v.matrix(oo, type);
    if (!v.ok || xt->size(1) != wt->size(1) || ot->size(0) != xt->size(0) || ot->size(1) != wt->size(0) ||
        wt->size(0) > INT32_MAX || xt->size(1) > INT32_MAX)
      return false;
    x = static_cast<const int8_t *>(xt->data_ptr());
    w = static_cast<const int8_t *>(wt->data_ptr());
    out = ot->data_ptr();
    m = xt->size(0), n = (int32_t)wt->size(0), k = (int32_t)xt->size(1);
    ldx = pitch(*xt), ldw = pitch(*wt), ldo = pitch(*ot);
    return true;
  }
};

at::ScalarType out_type(long long kind) {
  return kind == CWAC_OUT_INT8 ? at::kChar : kind == CWAC_OUT_FP32 ? at::kFloat : kind == CWAC_OUT_INT32 ? at::kInt : at::kDouble;
}

// (x_q, w_q, qp, mult, offset, fbias, s_x_row, out_kind, out, stream)
PyObject *py_forward(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("qlinear_cwac_forward", [&] {
    Args v;
    if (n != 10) return false;
    const int32_t kind = (int32_t)v.integer(a[7]);
    Linear l;
    if (!v.ok || out_type(kind) == at::kDouble || !l.take(v, a[0], a[1], a[8], out_type(kind))) return false;
    const cwac_qparams *qp = v.qparams(a[2], true);
    const float *mult = static_cast<const float *>(v.pointer(a[3])), *fbias = static_cast<const float *>(v.pointer(a[5])),
                *rows = static_cast<const float *>(v.pointer(a[6]));
    const int32_t *offset = static_cast<const int32_t *>(v.pointer(a[4]));
    void *st = v.stream(a[9]);
    if (!v.ok) return false;
    return unlocked([&] {
      return g.forward(l.x, l.ldx, l.w, l.ldw, l.m, l.n, l.k, qp, mult, offset, fbias, rows, kind, l.out, l.ldo, st);
    });
  });
}

// (x_q, w_q, qp, mult, offset, table, out, stream)
PyObject *py_forward_table(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("qlinear_cwac_forward_table", [&] {
    Args v;
    Linear l;
    if (n != 8 || !l.take(v, a[0], a[1], a[6], kI8)) return false;
    const cwac_qparams *qp = v.qparams(a[2], false);
    const float *mult = static_cast<const float *>(v.pointer(a[3]));
    const int32_t *offset = static_cast<const int32_t *>(v.pointer(a[4]));
    const at::TensorBase *table = v.typed(a[5], kI8);
    if (!v.ok || table->numel() != 256) return false;
    const int8_t *tp = static_cast<const int8_t *>(table->data_ptr());
    void *st = v.stream(a[7]);
    if (!v.ok) return false;
    return unlocked([&] {
      return g.forward_table(l.x, l.ldx, l.w, l.ldw, l.m, l.n, l.k, qp, mult, offset, tp, static_cast<int8_t *>(l.out), l.ldo, st);
    });
  });
}

// (x_q, w_q, qp, m0, shift, offset, out, stream)
PyObject *py_forward_fixed_point(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("qlinear_cwac_forward_fixed_point", [&] {
    Args v;
    Linear l;
    if (n != 8 || !l.take(v, a[0], a[1], a[6], kI8)) return false;
    const cwac_qparams *qp = v.qparams(a[2], false);
    const at::TensorBase *m0 = v.typed(a[3], at::kInt), *shift = v.typed(a[4], at::kInt);
    const int32_t *offset = static_cast<const int32_t *>(v.pointer(a[5]));
    void *st = v.stream(a[7]);
    if (!v.ok) return false;
    const int32_t *mp = static_cast<const int32_t *>(m0->data_ptr()), *sp = static_cast<const int32_t *>(shift->data_ptr());
    return unlocked([&] {
      return g.forward_fixed_point(l.x, l.ldx, l.w, l.ldw, l.m, l.n, l.k, qp, mp, sp, offset, static_cast<int8_t *>(l.out), l.ldo,
                                   st);
    });
  });
}

// (x_q, w_q, stride, pad, qp, mult, offset, fbias, out_kind, out, stream)
PyObject *py_conv2d(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("qconv2d_cwac_forward", [&] {
    Args v;
    if (n != 11) return false;
    const at::TensorBase *x = v.typed(a[0], kI8), *w = v.typed(a[1], kI8);
    const int32_t stride = (int32_t)v.integer(a[2]), pad = (int32_t)v.integer(a[3]), kind = (int32_t)v.integer(a[8]);
    if (!v.ok || out_type(kind) == at::kDouble || x->dim() != 4 || w->dim() != 4 || !x->is_contiguous() || !w->is_contiguous() ||
        x->size(3) != w->size(3))
      return false;
    const at::TensorBase *out = v.matrix(a[9], out_type(kind));
    if (!v.ok || out->size(1) != w->size(0)) return false;
    int32_t d[7];  // batch, h, w, c_in; c_out, kh, kw
    for (int i = 0; i < 7; ++i) {
      const int64_t s = i < 4 ? x->size(i) : w->size(i - 4);
      if (s > INT32_MAX) return false;
      d[i] = (int32_t)s;
    }
    const cwac_qparams *qp = v.qparams(a[4], false);
    const float *mult = static_cast<const float *>(v.pointer(a[5])), *fbias = static_cast<const float *>(v.pointer(a[7]));
    const int32_t *offset = static_cast<const int32_t *>(v.pointer(a[6]));
    void *st = v.stream(a[10]);
    if (!v.ok) return false;
    const int8_t *xp = static_cast<const int8_t *>(x->data_ptr()), *wp = static_cast<const int8_t *>(w->data_ptr());
    void *op = out->data_ptr();
    const int64_t ldo = pitch(*out);
    return unlocked([&] {
      return g.conv2d(xp, wp, d[0], d[1], d[2], d[3], d[4], d[5], d[6], stride, pad, qp, mult, offset, fbias, kind, op, ldo, st);
    });
  });
}

// (x, packed_w, packed_sz, n, mult, fbias, out, stream)
PyObject *py_w4a16(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("qlinear_w4a16_cwac_forward", [&] {
    Args v;
    if (n != 8) return false;
    const at::TensorBase *x = v.matrix(a[0], at::kHalf), *out = v.tensor(a[6]);
    const long long channels = v.integer(a[3]);
    if (!v.ok || (out->scalar_type() != at::kHalf && out->scalar_type() != kF32)) return false;
    out = v.matrix(a[6], out->scalar_type());
    if (!v.ok || out->size(0) != x->size(0) || out->size(1) != channels || x->size(1) > INT32_MAX) return false;
    const void *pw = v.pointer(a[1]);
    const uint32_t *sz = static_cast<const uint32_t *>(v.pointer(a[2]));
    const float *mult = static_cast<const float *>(v.pointer(a[4])), *fbias = static_cast<const float *>(v.pointer(a[5]));
    void *st = v.stream(a[7]);
    if (!v.ok) return false;
    const int32_t kind = out->scalar_type() == at::kHalf ? CWAC_OUT_FP16 : CWAC_OUT_FP32;
    const uint16_t *xp = static_cast<const uint16_t *>(x->data_ptr());
    void *op = out->data_ptr();
    const int64_t m = x->size(0), k = x->size(1), ldx = pitch(*x), ldo = pitch(*out);
    return unlocked([&] {
      return g.w4a16(xp, ldx, pw, sz, m, (int32_t)channels, (int32_t)k, mult, fbias, kind, op, ldo, st);
    });
  });
}

// ---- microscaled 4-bit format and paged cache: all tensors on the current device (the ctypes form serves another one)
constexpr auto kU8 = at::kByte;
constexpr auto kI32 = at::kInt;
constexpr auto kI64 = at::kLong;

int32_t kind_of(at::ScalarType t) {
  return t == at::kFloat ? CWAC_OUT_FP32 : t == at::kHalf ? CWAC_OUT_FP16 : t == at::kBFloat16 ? CWAC_OUT_BF16 : t == at::kChar ? CWAC_OUT_INT8 : -1;
}

struct HereArgs : Args {
  const c10::DeviceIndex device = c10::hip::current_device();
  const at::TensorBase *here(PyObject *o) {
    const at::TensorBase *t = tensor(o);
    if (t && t->device().index() != device) ok = false;
    return ok ? t : nullptr;
  }
  // contiguous, of a type, with `n` elements (-1: any number); NULL without one
  template <typename T>
  T *flat(PyObject *o, at::ScalarType type, int64_t n) {
    const at::TensorBase *t = here(o);
    if (!t || t->scalar_type() != type || !t->is_contiguous() || t->dim() != 1 || (n >= 0 && t->numel() != n)) return ok = false, nullptr;
    return static_cast<T *>(t->data_ptr());
  }
  template <typename T>
  T *flat_or_none(PyObject *o, at::ScalarType type, int64_t n) {
    return o == Py_None ? nullptr : flat<T>(o, type, n);
  }
  // a matrix with contiguous rows, any type
  const at::TensorBase *rows(PyObject *o) {
    const at::TensorBase *t = here(o);
    if (t && (t->dim() != 2 || t->stride(1) != 1 || t->size(1) > INT32_MAX)) ok = false;
    return ok ? t : nullptr;
  }
  // codes and scales of a [rows, k] matrix in the microscaled format
  bool mx4(PyObject *co, PyObject *so, int64_t m, int64_t k, uint8_t **codes, int64_t *ld, uint8_t **scales) {
    const at::TensorBase *c = rows(co), *s = here(so);
    if (!ok || c->scalar_type() != kU8 || c->size(0) != m || 2 * c->size(1) != k || s->scalar_type() != kU8 || !s->is_contiguous() ||
        s->dim() != 3 || s->size(0) != (k + CWAC_MX4_PANEL - 1) / CWAC_MX4_PANEL || s->size(1) != m || s->size(2) != 8)
      return ok = false;
    *codes = static_cast<uint8_t *>(c->data_ptr());
    *ld = pitch(*c);
    *scales = static_cast<uint8_t *>(s->data_ptr());
    return true;
  }
  // rows of heads [rows, heads, d], a row's heads side by side
  const at::TensorBase *heads(PyObject *o, int64_t *ld) {
    const at::TensorBase *t = here(o);
    if (!t || t->dim() != 3 || t->stride(2) != 1 || (t->size(1) > 1 && t->stride(1) != t->size(2)) || t->size(1) > 65536 || t->size(2) > 65536)
      return ok = false, nullptr;
    const int64_t width = t->size(1) * t->size(2);
    *ld = t->size(0) > 1 || t->stride(0) > width ? t->stride(0) : width;
    return t;
  }
  struct Cache {
    void *k, *v;
    float *ks, *vs;
    int32_t type, pages, page;
    int64_t heads, d;
  };
  bool cache(PyObject *ko, PyObject *vo, PyObject *kso, PyObject *vso, Cache *c) {
    const at::TensorBase *k = here(ko), *v = here(vo);
    if (!ok || k->dim() != 4 || v->dim() != 4 || k->scalar_type() != v->scalar_type() || !k->is_contiguous() || !v->is_contiguous())
      return ok = false;
    for (int i = 0; i < 4; ++i)
      if (k->size(i) != v->size(i) || k->size(i) > INT32_MAX) return ok = false;
    c->k = k->data_ptr(), c->v = v->data_ptr(), c->type = kind_of(k->scalar_type());
    c->pages = (int32_t)k->size(0), c->heads = k->size(1), c->page = (int32_t)k->size(2), c->d = k->size(3);
    c->ks = c->vs = nullptr;
    PyObject *so[2] = {kso, vso};
    float **sp[2] = {&c->ks, &c->vs};
    for (int i = 0; i < 2; ++i) {
      if (so[i] == Py_None) continue;  // the entry point refuses an 8-bit cache without them
      const at::TensorBase *t = here(so[i]);
      if (!ok || c->type != CWAC_OUT_INT8 || t->scalar_type() != kF32 || !t->is_contiguous() || t->dim() != 3 || t->size(0) != c->pages ||
          t->size(1) != c->heads || t->size(2) != c->page)
        return ok = false;
      *sp[i] = static_cast<float *>(t->data_ptr());
    }
    return true;
  }
};

// (x, codes, scales, stream)
PyObject *py_mx4_quantize(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("cwac_mx4_quantize", [&] {
    HereArgs v;
    uint8_t *c, *s;
    int64_t ldc;
    if (n != 4 || !g.mx4_quantize) return false;
    const at::TensorBase *x = v.rows(a[0]);
    if (!v.ok || kind_of(x->scalar_type()) < 0 || !v.mx4(a[1], a[2], x->size(0), x->size(1), &c, &ldc, &s)) return false;
    void *st = v.stream(a[3]);
    const void *xp = x->data_ptr();
    const int32_t kind = kind_of(x->scalar_type());
    const int64_t m = x->size(0), k = x->size(1), ldx = pitch(*x);
    if (!v.ok) return false;
    return unlocked([&] { return g.mx4_quantize(xp, kind, ldx, m, (int32_t)k, c, ldc, s, st); });
  });
}

// (codes, scales, out, stream)
PyObject *py_mx4_dequantize(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("cwac_mx4_dequantize", [&] {
    HereArgs v;
    uint8_t *c, *s;
    int64_t ldc;
    if (n != 4 || !g.mx4_dequantize) return false;
    const at::TensorBase *o = v.rows(a[2]);
    if (!v.ok || kind_of(o->scalar_type()) < 0 || !v.mx4(a[0], a[1], o->size(0), o->size(1), &c, &ldc, &s)) return false;
    void *st = v.stream(a[3]), *op = o->data_ptr();
    const int32_t kind = kind_of(o->scalar_type());
    const int64_t m = o->size(0), k = o->size(1), ldo = pitch(*o);
    if (!v.ok) return false;
    return unlocked([&] { return g.mx4_dequantize(c, ldc, s, m, (int32_t)k, op, kind, ldo, st); });
  });
}

// (x_codes, x_scales, w_codes, w_scales, mult, fbias, out, stream)
PyObject *py_mx4_forward(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("qlinear_mx4_cwac_forward", [&] {
    HereArgs v;
    uint8_t *x, *xs, *w, *ws;
    int64_t ldx, ldw;
    if (n != 8 || !g.mx4_forward) return false;
    const at::TensorBase *o = v.rows(a[6]), *xc = v.rows(a[0]);
    if (!v.ok || kind_of(o->scalar_type()) < 0) return false;
    const int64_t m = o->size(0), nn = o->size(1), k = 2 * xc->size(1), ldo = pitch(*o);
    if (k > INT32_MAX || !v.mx4(a[0], a[1], m, k, &x, &ldx, &xs) || !v.mx4(a[2], a[3], nn, k, &w, &ldw, &ws)) return false;
    const float *mult = v.flat_or_none<float>(a[4], kF32, nn), *fb = v.flat_or_none<float>(a[5], kF32, nn);
    void *st = v.stream(a[7]), *op = o->data_ptr();
    const int32_t kind = kind_of(o->scalar_type());
    if (!v.ok) return false;
    return unlocked([&] { return g.mx4_forward(x, ldx, xs, w, ldw, ws, m, (int32_t)nn, (int32_t)k, mult, fb, kind, op, ldo, st); });
  });
}

// (old_lens, new_lens, page, free_pages, n_free, table, slots, token_start, seq_lens, n_left, stream)
PyObject *py_kv_assign(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("llm_kv_assign_pages", [&] {
    HereArgs v;
    if (n != 11 || !g.kv_assign) return false;
    const at::TensorBase *old = v.here(a[0]), *fr = v.here(a[3]), *table = v.rows(a[5]), *sl = v.here(a[6]);
    const int32_t page = (int32_t)v.integer(a[2]);
    if (!v.ok) return false;
    const int64_t batch = old->numel(), ldt = pitch(*table), cols = table->size(1), n_free = fr->numel(), n_slots = sl->numel();
    if (batch > INT32_MAX - 1 || n_free > INT32_MAX || table->scalar_type() != kI32 || table->size(0) != batch) return false;
    const int32_t *op = v.flat<int32_t>(a[0], kI32, batch), *np = v.flat<int32_t>(a[1], kI32, batch), *fp = v.flat<int32_t>(a[3], kI32, -1),
                  *nf = v.flat<int32_t>(a[4], kI32, 1);
    int64_t *sp = v.flat<int64_t>(a[6], kI64, -1);
    int32_t *ts = v.flat<int32_t>(a[7], kI32, batch + 1), *sq = v.flat<int32_t>(a[8], kI32, batch), *nl = v.flat<int32_t>(a[9], kI32, 1);
    int32_t *tp = static_cast<int32_t *>(table->data_ptr());
    void *st = v.stream(a[10]);
    if (!v.ok) return false;
    return unlocked([&] {
      return g.kv_assign(op, np, (int32_t)batch, page, fp, (int32_t)n_free, nf, tp, ldt, (int32_t)cols, sp, n_slots, ts, sq, nl, st);
    });
  });
}

// (k, v, slots, k_cache, v_cache, k_scales, v_scales, stream)
PyObject *py_kv_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("llm_kv_append", [&] {
    HereArgs v;
    HereArgs::Cache c;
    int64_t ldk, ldv;
    if (n != 8 || !g.kv_append) return false;
    const at::TensorBase *k = v.heads(a[0], &ldk), *w = v.heads(a[1], &ldv);
    if (!v.ok || !v.cache(a[3], a[4], a[5], a[6], &c) || k->scalar_type() != w->scalar_type()) return false;
    const int64_t tokens = k->size(0);
    if (w->size(0) != tokens || k->size(1) != c.heads || w->size(1) != c.heads || k->size(2) != c.d || w->size(2) != c.d) return false;
    const int64_t *sl = v.flat<int64_t>(a[2], kI64, tokens);
    const int32_t type = kind_of(k->scalar_type());
    const void *kp = k->data_ptr(), *vp = w->data_ptr();
    void *st = v.stream(a[7]);
    if (!v.ok) return false;
    return unlocked([&] {
      return g.kv_append(kp, ldk, vp, ldv, type, sl, tokens, (int32_t)c.heads, (int32_t)c.d, c.k, c.v, c.type, c.ks, c.vs, c.pages, c.page, st);
    });
  });
}

// (q, k_cache, v_cache, k_scales, v_scales, table, lens, scale, window, out, workspace, stream)
PyObject *py_paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded("llm_paged_attention", [&] {
    HereArgs v;
    HereArgs::Cache c;
    int64_t ldq, ldo;
    if (n != 12 || !g.paged_attention) return false;
    const at::TensorBase *q = v.heads(a[0], &ldq), *o = v.heads(a[9], &ldo), *table = v.rows(a[5]);
    const float scale = v.number(a[7]);
    const int32_t window = (int32_t)v.integer(a[8]);
    if (!v.ok || !v.cache(a[1], a[2], a[3], a[4], &c) || o->scalar_type() != q->scalar_type()) return false;
    const int64_t batch = q->size(0), ldt = pitch(*table), cols = table->size(1);
    for (int i = 0; i < 3; ++i)
      if (o->size(i) != q->size(i)) return false;
    if (batch > INT32_MAX || q->size(2) != c.d || table->scalar_type() != kI32 || table->size(0) != batch) return false;
    const int32_t *lens = v.flat<int32_t>(a[6], kI32, batch);
    void *ws = nullptr;
    size_t bytes = 0;
    if (a[10] != Py_None) {
      const at::TensorBase *t = v.here(a[10]);
      if (!v.ok) return false;
      ws = t->data_ptr(), bytes = t->numel() * t->element_size();
    }
    const int32_t type = kind_of(q->scalar_type());
    const int32_t *tp = static_cast<const int32_t *>(table->data_ptr());
    const void *qp = q->data_ptr();
    void *op = o->data_ptr(), *st = v.stream(a[11]);
    if (!v.ok) return false;
    return unlocked([&] {
      return g.paged_attention(qp, ldq, type, c.k, c.v, c.type, c.ks, c.vs, c.pages, c.page, tp, ldt, (int32_t)cols, lens, (int32_t)batch,
                               (int32_t)q->size(1), (int32_t)c.heads, (int32_t)c.d, scale, window, op, ldo, ws, bytes, st);
    });
  });
}

// (the type of cwac_qparams, {entry point: address}, the check of a status)
PyObject *py_bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
  if (n != 3 || !PyDict_Check(a[1])) return PyErr_Format(PyExc_TypeError, "bind(type, addresses, check)");
  const struct {
    const char *name;
    void **slot;
  } slots[] = {{"cwac_quantize_act", (void **)&g.quantize_act},
               {"cwac_quantize_rows_sym", (void **)&g.quantize_rows_sym},
               {"qlinear_cwac_forward", (void **)&g.forward},
               {"qlinear_cwac_forward_table", (void **)&g.forward_table},
               {"qlinear_cwac_forward_fixed_point", (void **)&g.forward_fixed_point},
               {"qconv2d_cwac_forward", (void **)&g.conv2d},
               {"qlinear_w4a16_cwac_forward", (void **)&g.w4a16}};
  for (const auto &s : slots) {
    PyObject *v = PyDict_GetItemString(a[1], s.name);
    if (!v || !PyLong_Check(v)) return PyErr_Format(PyExc_KeyError, "%s", s.name);
    *s.slot = PyLong_AsVoidPtr(v);
  }
  // these keep their address where the caller names none; without one the call is declined
  const struct {
    const char *name;
    void **slot;
  } optional[] = {{"cwac_mx4_quantize", (void **)&g.mx4_quantize},
                  {"cwac_mx4_dequantize", (void **)&g.mx4_dequantize},
                  {"qlinear_mx4_cwac_forward", (void **)&g.mx4_forward},
                  {"llm_kv_assign_pages", (void **)&g.kv_assign},
                  {"llm_kv_append", (void **)&g.kv_append},
                  {"llm_paged_attention", (void **)&g.paged_attention}};
  for (const auto &s : optional) {
    PyObject *v = PyDict_GetItemString(a[1], s.name);
    if (v && PyLong_Check(v)) *s.slot = PyLong_AsVoidPtr(v);
  }
  Py_INCREF(a[0]);
  Py_XSETREF(g_qparams_type, a[0]);
  Py_INCREF(a[2]);
  Py_XSETREF(g_check, a[2]);
  Py_RETURN_NONE;
}

#define CWAC_METHOD(name) \
  { #name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, nullptr }
PyMethodDef methods[] = {CWAC_METHOD(bind),    CWAC_METHOD(quantize_act),  CWAC_METHOD(quantize_rows_sym),
                         CWAC_METHOD(forward), CWAC_METHOD(forward_table), CWAC_METHOD(forward_fixed_point),
                         CWAC_METHOD(conv2d),  CWAC_METHOD(w4a16),         CWAC_METHOD(mx4_quantize),
                         CWAC_METHOD(mx4_dequantize), CWAC_METHOD(mx4_forward), CWAC_METHOD(kv_assign),
                         CWAC_METHOD(kv_append), CWAC_METHOD(paged_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fast_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fast_calls() { return PyModule_Create(&module); }
