// The way from torch tensors to the library for calls whose kernels take a few microseconds: checks, outputs and the C call in one
// step, where the same in Python takes as long as several such kernels (8 rows of 256, norm with residual and 8-bit output: 17.3 us
// through ctypes, 3 us of them the launch).
//
// A launch can wait for room in the device's queue, and an allocation for the device, so both run without the interpreter's lock, as a call through
// ctypes does: other threads go on meanwhile, those among them that the queue waits for.
//
// Each function serves the plain case of its wrapper in binding.py and nothing else: tensors of one device, which is the current one, of
// the right types, on the current stream, with outputs and workspaces made here.  It answers None for any other, and the wrapper
// goes its own way, with its own errors; a status other than PSRL_OK is answered as it is.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>

#include "../../include/psrl.h"

namespace {

using at::Tensor;

// A call's tensors: `ok` turns false for whatever this file does not serve.
struct Call {
  bool ok = true;
  int dev = -1;
  at::ScalarType type = at::kFloat;

  // NULL for None
  const Tensor* get(PyObject* o) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) {
      ok = false;
      return nullptr;
    }
    return &THPVariable_Unpack(o);
  }
  // the tensor that the others are measured by
  const Tensor* first(PyObject* o) {
    const Tensor* t = get(o);
    if (!t || !t->is_cuda() || t->layout() != at::kStrided || t->get_device() != c10::cuda::current_device()) {
      ok = false;
      return nullptr;
    }
    dev = t->get_device();
    type = t->scalar_type();
    return t;
  }
  const Tensor* like(PyObject* o, at::ScalarType want) {
    const Tensor* t = get(o);
    if (t && (!t->is_cuda() || t->layout() != at::kStrided || t->get_device() != dev || t->scalar_type() != want)) ok = false;
    return ok ? t : nullptr;
  }
  // [rows, cols], the elements of a row contiguous: its pitch
  int64_t matrix(const Tensor* t, int64_t rows, int64_t cols) {
    if (!t || !ok) return 0;
    if (t->dim() != 2 || t->size(0) != rows || t->size(1) != cols || (t->stride(1) != 1 && cols != 1)) {
      ok = false;
      return 0;
    }
    return rows > 1 ? t->stride(0) : (cols + 15) / 16 * 16;
  }
  // [rows, heads, dim] or, with heads == 1, also [rows, dim]: the heads of a row contiguous
  int64_t rows(const Tensor* t, int64_t n, int64_t heads, int64_t dim, int dims) {
    if (!t || !ok) return 0;
    if (t->dim() != dims) ok = false;
    else if (dims == 2) return matrix(t, n, dim);
    else if (t->size(0) != n || t->size(1) != heads || t->size(2) != dim || (t->stride(2) != 1 && dim != 1) || (t->stride(1) != dim && heads != 1)) ok = false;
    return ok ? (n > 1 ? t->stride(0) : heads * dim) : 0;
  }
  const void* vector(const Tensor* t, int64_t n) {
    if (!t || !ok) return nullptr;
    if (t->dim() != 1 || t->size(0) != n || !t->is_contiguous()) ok = false;
    return ok ? t->data_ptr() : nullptr;
  }

  Tensor make(at::IntArrayRef shape, at::ScalarType t) const {
    return at::detail::empty_cuda(shape, t, at::Device(at::kCUDA, static_cast<c10::DeviceIndex>(dev)), std::nullopt);
  }
  // [rows, cols] with rows that are whole 16-byte vectors apart
  Tensor make_matrix(int64_t rows, int64_t cols, at::ScalarType t, int64_t& pitch) const {
    pitch = (cols + 7) / 8 * 8;
    Tensor m = make({rows, pitch}, t);
    return pitch == cols ? m : m.narrow(1, 0, cols);
  }
  void* stream() const { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(dev)).stream(); }
};

// f() without the interpreter's lock, which is taken again whichever way f ends.
template <class F>
psrl_status_t unlocked(F f) {
  struct Lock {
    PyThreadState* state = PyEval_SaveThread();
    ~Lock() { PyEval_RestoreThread(state); }
  } lock;
  return f();
}

const void* at_of(const Tensor* t) { return t ? t->data_ptr() : nullptr; }
PyObject* none() { Py_RETURN_NONE; }
PyObject* wrap(const Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : none(); }

template <class... T>
PyObject* answer(psrl_status_t st, const T&... out) {
  if (st != PSRL_OK) return PyLong_FromLong(st);
  PyObject* r = PyTuple_New(sizeof...(out));
  if (!r) return nullptr;
  Py_ssize_t i = 0;
  bool all = true;
  auto put = [&](const Tensor& t) {
    PyObject* o = wrap(t);
    if (!o) all = false;
    PyTuple_SET_ITEM(r, i++, o);
  };
  (put(out), ...);
  if (all) return r;
  Py_DECREF(r);
  return nullptr;
}

int code_of(at::ScalarType t) { return t == at::kFloat ? PSRL_F32 : t == at::kBFloat16 ? PSRL_BF16 : t == at::kFloat8_e4m3fn ? PSRL_E4M3 : -1; }

// No C++ exception leaves a function: they turn into torch's own Python errors (memory that is out among them).
template <class F>
PyObject* guarded(F f) {
  HANDLE_TH_ERRORS
  return f();
  END_HANDLE_TH_ERRORS
}

bool int_of(PyObject* o, int64_t& v) {
  v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return true;
}
bool double_of(PyObject* o, double& v) {
  v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return true;
}
// what has no truth value is the wrapper's to refuse
bool truth(Call& c, PyObject* o) {
  const int t = PyObject_IsTrue(o);
  if (t >= 0) return t == 1;
  PyErr_Clear();
  c.ok = false;
  return false;
}

// The sizes of a norm: x [rows, dim] or [rows, heads, dim], f32 or bf16; weight [dim] or None.
struct Norm {
  int64_t rows = 0, heads = 1, dim = 0;
  int dims = 0;
  const void* weight = nullptr;
  Norm(Call& c, const Tensor* x, PyObject* w) {
    if (!c.ok || !(c.type == at::kFloat || c.type == at::kBFloat16) || x->dim() < 2 || x->dim() > 3) {
      c.ok = false;
      return;
    }
    dims = int(x->dim());
    rows = x->size(0);
    if (dims == 3) heads = x->size(1);
    dim = x->size(dims - 1);
    if (heads > 65535 || dim > INT32_MAX) c.ok = false;
    weight = c.vector(c.like(w, c.type), dim);
  }
};

// x, weight, eps, residual, want_y, want_codes -> (y, summed, codes, scales)
PyObject* rms_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    double eps;
    if (n != 6 || !double_of(a[2], eps)) return none();
    Call c;
    const Tensor* x = c.first(a[0]);
    Norm m(c, x, a[1]);
    const Tensor* res = c.like(a[3], c.type);
    const int64_t px = c.rows(x, m.rows, m.heads, m.dim, m.dims), pr = c.rows(res, m.rows, m.heads, m.dim, m.dims), least = m.heads * m.dim;
    const bool want_y = truth(c, a[4]), want_codes = truth(c, a[5]);
    if (!c.ok || (want_codes && least % 16)) return none();
    Tensor y, summed, codes, scales;
    const psrl_status_t st = unlocked([&] {
      if (want_y) y = c.make(x->sizes(), c.type);
      if (res) summed = c.make(x->sizes(), c.type);
      if (want_codes) {
        codes = c.make(x->sizes(), at::kFloat8_e4m3fn);
        scales = c.make(x->sizes().slice(0, m.dims - 1), at::kFloat);
      }
      return psrl_rms_norm_fwd(psrl_dtype_t(code_of(c.type)), m.rows, int32_t(m.heads), int32_t(m.dim), x->data_ptr(), px, at_of(res), pr, m.weight, float(eps),
                               res ? summed.data_ptr() : nullptr, least, want_y ? y.data_ptr() : nullptr, least, want_codes ? codes.data_ptr() : nullptr, least,
                               want_codes ? static_cast<float*>(scales.data_ptr()) : nullptr, c.stream());
    });
    return answer(st, y, summed, codes, scales);
  });
}

// summed, weight, d_y, eps, d_summed, want_x, want_weight -> (d_x, d_weight)
PyObject* rms_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    double eps;
    if (n != 7 || !double_of(a[3], eps)) return none();
    Call c;
    const Tensor* h = c.first(a[0]);
    Norm m(c, h, a[1]);
    const Tensor *dy = c.like(a[2], c.type), *ds = c.like(a[4], c.type);
    const int64_t ph = c.rows(h, m.rows, m.heads, m.dim, m.dims), pd = c.rows(dy, m.rows, m.heads, m.dim, m.dims), ps = c.rows(ds, m.rows, m.heads, m.dim, m.dims);
    const bool want_x = truth(c, a[5]), want_w = truth(c, a[6]) && m.weight;
    if (!c.ok || !dy) return none();
    const psrl_dtype_t t = psrl_dtype_t(code_of(c.type));
    Tensor dx, dw, ws;
    const psrl_status_t st = unlocked([&] {
      size_t bytes = 0;
      if (want_x) dx = c.make(h->sizes(), c.type);
      if (want_w) {
        dw = c.make({m.dim}, c.type);
        bytes = psrl_rms_norm_workspace_bytes(t, m.rows, int32_t(m.heads), int32_t(m.dim));
        ws = c.make({int64_t(bytes)}, at::kByte);
      }
      return psrl_rms_norm_bwd(t, m.rows, int32_t(m.heads), int32_t(m.dim), h->data_ptr(), ph, m.weight, float(eps), dy->data_ptr(), pd, at_of(ds), ps,
                               want_x ? dx.data_ptr() : nullptr, m.heads * m.dim, want_w ? dw.data_ptr() : nullptr, want_w ? ws.data_ptr() : nullptr, bytes, c.stream());
    });
    return answer(st, dx, dw);
  });
}

// The sizes of a product and the type of what is beside its operands.
struct Product {
  const Tensor *x = nullptr, *w = nullptr;
  int64_t m = 0, k = 0, n = 0, px = 0, pw = 0;
  at::ScalarType out = at::kBFloat16;
  Product(Call& c, PyObject* ax, PyObject* aw) {
    x = c.first(ax);
    if (!c.ok || code_of(c.type) < 0 || x->dim() != 2) {
      c.ok = false;
      return;
    }
    w = c.like(aw, c.type);
    if (!w || w->dim() != 2) {
      c.ok = false;
      return;
    }
    m = x->size(0); k = x->size(1); n = w->size(0);
    if (k > INT32_MAX || n > INT32_MAX) c.ok = false;
    if (c.type != at::kFloat8_e4m3fn) out = c.type;
    px = c.matrix(x, m, k);
    pw = c.matrix(w, n, k);
  }
};

// x, weight, bias, activation (number), mul, residual, x_scale, weight_scale, want_z -> (y, z)
PyObject* linear_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int64_t act;
    if (n != 9 || !int_of(a[3], act)) return none();
    Call c;
    Product p(c, a[0], a[1]);
    if (!c.ok) return none();
    const bool codes = c.type == at::kFloat8_e4m3fn;
    const Tensor *mul = c.like(a[4], p.out), *res = c.like(a[5], p.out);
    const void* bias = c.vector(c.like(a[2], p.out), p.n);
    const void *sx = c.vector(c.like(a[6], at::kFloat), p.m), *sw = c.vector(c.like(a[7], at::kFloat), p.n);
    const int64_t pm = c.matrix(mul, p.m, p.n), pr = c.matrix(res, p.m, p.n);
    const bool want_z = truth(c, a[8]);
    if (!c.ok || codes != (a[6] != Py_None) || codes != (a[7] != Py_None)) return none();
    const psrl_dtype_t t = psrl_dtype_t(code_of(c.type));
    Tensor y, z, ws;
    const psrl_status_t st = unlocked([&] {
      int64_t py, pz = 0;
      y = c.make_matrix(p.m, p.n, p.out, py);
      if (want_z) z = c.make_matrix(p.m, p.n, p.out, pz);
      size_t bytes = 0;
      if (t == PSRL_F32) {
        bytes = psrl_linear_workspace_bytes(t, p.m, int32_t(p.k), int32_t(p.n), 0);
        ws = c.make({int64_t(bytes)}, at::kByte);
      }
      return psrl_linear_fwd(t, p.m, int32_t(p.k), int32_t(p.n), p.x->data_ptr(), p.px, static_cast<const float*>(sx), p.w->data_ptr(), p.pw,
                             static_cast<const float*>(sw), bias, psrl_activation_t(act), at_of(mul), pm, at_of(res), pr, y.data_ptr(), py,
                             z.defined() ? z.data_ptr() : nullptr, pz, bytes ? ws.data_ptr() : nullptr, bytes, c.stream());
    });
    return answer(st, y, z);
  });
}

// x, weight, d_y, z, activation (number), mul, want_x, want_weight, want_bias, want_mul -> (d_x, d_weight, d_bias, d_mul)
PyObject* linear_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int64_t act;
    if (n != 10 || !int_of(a[4], act)) return none();
    Call c;
    Product p(c, a[0], a[1]);
    if (!c.ok || c.type == at::kFloat8_e4m3fn) return none();
    const Tensor *dy = c.like(a[2], c.type), *z = c.like(a[3], c.type), *mul = c.like(a[5], c.type);
    const int64_t pd = c.matrix(dy, p.m, p.n), pz = c.matrix(z, p.m, p.n), pm = c.matrix(mul, p.m, p.n);
    const bool want_x = truth(c, a[6]), want_w = truth(c, a[7]), want_b = truth(c, a[8]), want_m = truth(c, a[9]);
    if (!c.ok || !dy) return none();
    const psrl_dtype_t t = psrl_dtype_t(code_of(c.type));
    Tensor dx, dw, db, dm, ws;
    const psrl_status_t st = unlocked([&] {
      int64_t px = 0, pw = 0, pq = 0;
      if (want_x) dx = c.make_matrix(p.m, p.k, c.type, px);
      if (want_w) dw = c.make_matrix(p.n, p.k, c.type, pw);
      if (want_b) db = c.make({p.n}, c.type);
      if (want_m) dm = c.make_matrix(p.m, p.n, c.type, pq);
      size_t bytes = 0;
      if (act != PSRL_ACT_NONE || mul || want_b || t == PSRL_F32) {
        bytes = psrl_linear_workspace_bytes(t, p.m, int32_t(p.k), int32_t(p.n), 1);
        ws = c.make({int64_t(bytes)}, at::kByte);
      }
      auto at_or = [](const Tensor& v) { return v.defined() ? v.data_ptr() : nullptr; };
      return psrl_linear_bwd(t, p.m, int32_t(p.k), int32_t(p.n), p.x->data_ptr(), p.px, p.w->data_ptr(), p.pw, at_of(z), pz, psrl_activation_t(act), at_of(mul), pm,
                             dy->data_ptr(), pd, at_or(dx), px, at_or(dw), pw, at_or(db), at_or(dm), pq, at_or(ws), bytes, c.stream());
    });
    return answer(st, dx, dw, db, dm);
  });
}

// Handles and sizes of a plan and a rope, as the wrapper keeps them.
struct Tree {
  const psrl_plan_t* plan = nullptr;
  const psrl_rope_t* rope = nullptr;
  int64_t axes = 0, type = 0, rows = 0, hq = 0, hkv = 0, d = 0;
  bool ok;
  Tree(PyObject* const* a) {
    int64_t h = 0, r = 0;
    ok = int_of(a[0], h) && int_of(a[1], r) && int_of(a[2], axes) && int_of(a[3], type) && int_of(a[4], rows) && int_of(a[5], hq) && int_of(a[6], hkv) &&
         int_of(a[7], d) && h && r;
    plan = reinterpret_cast<const psrl_plan_t*>(h);
    rope = reinterpret_cast<const psrl_rope_t*>(r);
  }
};
constexpr int kTreeArgs = 8;

// [axes, rows], the rows of an axis contiguous: the elements from one axis to the next.  One row may be a slice as well as many: its axes
// are then as far apart as those of the matrix that it was cut from.
int64_t positions_of(Call& c, const Tensor* p, int64_t axes, int64_t rows) {
  if (!p || !c.ok) {
    c.ok = false;
    return 0;
  }
  if (p->dim() != 2 || p->size(0) != axes || p->size(1) != rows || (rows > 1 && p->stride(1) != 1)) c.ok = false;
  return axes > 1 && !p->is_contiguous() ? p->stride(0) : rows;
}

// plan, rope, axes, type, T_q, Hq, Hkv, d, positions, q, k, v, k_pool, v_pool, q_out -> (q_out,)
PyObject* rope_axes_qkv_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != kTreeArgs + 7) return none();
    Tree t(a);
    a += kTreeArgs;
    Call c;
    const Tensor* q = c.first(a[1]);
    if (!t.ok || !c.ok || code_of(c.type) != t.type) return none();
    const Tensor *k = c.like(a[2], c.type), *v = c.like(a[3], c.type), *kp = c.like(a[4], c.type), *vp = c.like(a[5], c.type), *out = c.like(a[6], c.type);
    const Tensor* pos = c.like(a[0], at::kInt);
    if (!c.ok || !k || !v || !kp || !vp || kp->dim() != 3 || kp->size(0) != t.hkv || kp->size(2) != t.d || vp->sizes() != kp->sizes() || !kp->is_contiguous() ||
        !vp->is_contiguous() || (out && (!out->is_contiguous() || out->sizes() != q->sizes())))
      return none();
    const int64_t pq = c.rows(q, t.rows, t.hq, t.d, 3), pk = c.rows(k, t.rows, t.hkv, t.d, 3), pv = c.rows(v, t.rows, t.hkv, t.d, 3), pa = positions_of(c, pos, t.axes, t.rows);
    if (!c.ok) return none();
    Tensor made;
    const psrl_status_t st = unlocked([&] {
      if (!out) made = c.make({t.rows, t.hq, t.d}, c.type);
      return psrl_rope_axes_qkv_fwd(t.plan, t.rope, static_cast<const int32_t*>(pos->data_ptr()), pa, q->data_ptr(), pq, k->data_ptr(), pk, v->data_ptr(), pv,
                                    out ? out->data_ptr() : made.data_ptr(), kp->data_ptr(), vp->data_ptr(), kp->size(1), c.stream());
    });
    return answer(st, out ? *out : made);
  });
}

// plan, rope, axes, type, T_q, Hq, Hkv, d, positions, d_q, dk_pool, dv_pool, dq_out, dk_out, dv_out -> the three outputs
PyObject* rope_axes_qkv_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != kTreeArgs + 7) return none();
    Tree t(a);
    a += kTreeArgs;
    Call c;
    const Tensor* q = c.first(a[1]);
    if (!t.ok || !c.ok || code_of(c.type) != t.type) return none();
    const Tensor *kp = c.like(a[2], c.type), *vp = c.like(a[3], c.type), *pos = c.like(a[0], at::kInt);
    const Tensor* given[3] = {c.like(a[4], c.type), c.like(a[5], c.type), c.like(a[6], c.type)};
    if (!c.ok || !kp || !vp || kp->dim() != 3 || kp->size(0) != t.hkv || kp->size(2) != t.d || vp->sizes() != kp->sizes() || !kp->is_contiguous() || !vp->is_contiguous() ||
        !q->is_contiguous())
      return none();
    c.rows(q, t.rows, t.hq, t.d, 3);
    const int64_t pa = positions_of(c, pos, t.axes, t.rows);
    if (!c.ok) return none();
    Tensor out[3];
    int64_t pitch[3];
    for (int i = 0; i < 3; ++i) {
      const int64_t heads = i == 0 ? t.hq : t.hkv;
      pitch[i] = given[i] ? c.rows(given[i], t.rows, heads, t.d, 3) : heads * t.d;
    }
    if (!c.ok) return none();
    const psrl_status_t st = unlocked([&] {
      for (int i = 0; i < 3; ++i) {
        if (given[i]) out[i] = *given[i];
        else out[i] = c.make({t.rows, i == 0 ? t.hq : t.hkv, t.d}, c.type);
      }
      return psrl_rope_axes_qkv_bwd(t.plan, t.rope, static_cast<const int32_t*>(pos->data_ptr()), pa, q->data_ptr(), kp->data_ptr(), vp->data_ptr(), kp->size(1),
                                    out[0].data_ptr(), pitch[0], out[1].data_ptr(), pitch[1], out[2].data_ptr(), pitch[2], c.stream());
    });
    return answer(st, out[0], out[1], out[2]);
  });
}

// rope, axes, d, x, positions, inverse -> (y,)
PyObject* rope_axes_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    int64_t r, axes, d;
    if (n != 6 || !int_of(a[0], r) || !int_of(a[1], axes) || !int_of(a[2], d) || !r) return none();
    Call c;
    const Tensor* x = c.first(a[3]);
    if (!c.ok || !(c.type == at::kFloat || c.type == at::kBFloat16) || x->dim() != 3) return none();
    const int64_t rows = x->size(0), heads = x->size(1);
    const Tensor* pos = c.like(a[4], at::kInt);
    const int64_t px = c.rows(x, rows, heads, d, 3), pa = positions_of(c, pos, axes, rows);
    const bool inverse = truth(c, a[5]);
    if (!c.ok || heads > INT32_MAX) return none();
    Tensor y;
    const psrl_status_t st = unlocked([&] {
      y = c.make(x->sizes(), c.type);
      return psrl_rope_axes_rows(reinterpret_cast<const psrl_rope_t*>(r), psrl_dtype_t(code_of(c.type)), x->data_ptr(), px, static_cast<const int32_t*>(pos->data_ptr()), pa,
                                 rows, int32_t(heads), y.data_ptr(), heads * d, inverse ? 1 : 0, c.stream());
    });
    return answer(st, y);
  });
}

PyMethodDef kMethods[] = {
    {"rms_norm_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rms_norm_fwd)), METH_FASTCALL, nullptr},
    {"rms_norm_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rms_norm_bwd)), METH_FASTCALL, nullptr},
    {"linear_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(linear_fwd)), METH_FASTCALL, nullptr},
    {"linear_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(linear_bwd)), METH_FASTCALL, nullptr},
    {"rope_axes_qkv_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rope_axes_qkv_fwd)), METH_FASTCALL, nullptr},
    {"rope_axes_qkv_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rope_axes_qkv_bwd)), METH_FASTCALL, nullptr},
    {"rope_axes_rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rope_axes_rows)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls(void) { return PyModule_Create(&kModule); }
