// Native argument marshalling of the Python binding: torch tensors -> the C
// ABI's structs -> the call. The same checks and errors as api.py documents;
// a call's 15 segments took 45 to 80 us through ctypes (shape, strides, type
// and address of every tensor, each an interpreted call), longer than many of
// the kernels they describe; here 1 to 2 us.
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdio>
#include <cstring>
#include <vector>

#include "refadapt.h"

namespace {

// A Python error is set; unwinds to the entry point, which returns NULL.
struct Raised {};

[[noreturn]] void raise(PyObject* type, const char* msg) {
  PyErr_SetString(type, msg);
  throw Raised{};
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "expected a tensor, got %R", o);
    throw Raised{};
  }
  return THPVariable_Unpack(o);
}

// Device address of a tensor, NULL for None.
void* address(PyObject* o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }

long long integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}
int32_t integer32(PyObject* o) { return int32_t(integer(o)); }
// int(o): any number, or its text.
int32_t as_int32(PyObject* o) {
  PyObject* v = PyNumber_Long(o);
  if (!v) throw Raised{};
  const long long x = PyLong_AsLongLong(v);
  Py_DECREF(v);
  if (x == -1 && PyErr_Occurred()) throw Raised{};
  return int32_t(x);
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return v;
}

PyObject* shape_of(PyObject* o) {
  PyObject* s = PyObject_GetAttrString(o, "shape");
  PyObject* t = s ? PySequence_Tuple(s) : nullptr;
  Py_XDECREF(s);
  if (!t) throw Raised{};
  return t;
}

// ra_seg of a [B, H, n, d] bf16 CUDA tensor; None: absent, n query rows.
ra_seg seg(PyObject* o, int64_t n = 0) {
  if (o == Py_None) return ra_seg{nullptr, 0, 0, 0, int32_t(n), 0};
  const at::Tensor& t = tensor(o);
  if (t.dim() != 4 || t.scalar_type() != at::kBFloat16 || !t.is_cuda() || (t.size(3) > 1 && t.stride(3) != 1)) {
    PyObject* shape = shape_of(o);
    PyObject* dtype = PyObject_GetAttrString(o, "dtype");
    PyObject* device = PyObject_GetAttrString(o, "device");
    if (dtype && device)
      PyErr_Format(PyExc_ValueError,
                   "expected a [B, H, n, d] bf16 CUDA tensor with contiguous last axis, got %S %S %S", shape, dtype,
                   device);
    Py_DECREF(shape);
    Py_XDECREF(dtype);
    Py_XDECREF(device);
    throw Raised{};
  }
  return ra_seg{t.numel() > 0 ? t.data_ptr() : nullptr, t.stride(0), t.stride(1), t.stride(2), int32_t(t.size(2)), 0};
}

struct Rows {
  void* ptr;
  int64_t stride_s, stride_r, rows, samples;
};
// A [B, rows, F] CUDA tensor with contiguous last axis.
Rows rows_of(PyObject* o, const char* what) {
  const at::Tensor& t = tensor(o);
  if (t.dim() != 3 || !t.is_cuda() || (t.size(2) > 1 && t.stride(2) != 1)) {
    PyObject* shape = shape_of(o);
    PyErr_Format(PyExc_ValueError, "%s: expected a [B, rows, F] CUDA tensor with contiguous last axis, got %S", what,
                 shape);
    Py_DECREF(shape);
    throw Raised{};
  }
  return Rows{t.numel() > 0 ? t.data_ptr() : nullptr, t.stride(0), t.stride(1), t.size(1), t.size(0)};
}

// B, H and d of a [B, H, n, d] tensor.
struct Dims {
  int32_t B, H, d;
};
Dims dims_of(PyObject* o) {
  const at::Tensor& t = tensor(o);
  if (t.dim() != 4) raise(PyExc_ValueError, "expected a tensor of four dimensions [B, H, n, d]");
  return Dims{int32_t(t.size(0)), int32_t(t.size(1)), int32_t(t.size(3))};
}
int64_t rows4(PyObject* o) {
  const at::Tensor& t = tensor(o);
  if (t.dim() < 3) raise(PyExc_IndexError, "tuple index out of range");
  return t.size(2);
}

// Items of a sequence of at least `want` entries.
struct Seq {
  PyObject* fast;
  Seq(PyObject* o, Py_ssize_t want) : fast(PySequence_Fast(o, "expected a sequence")) {
    if (!fast) throw Raised{};
    if (size() < want) {
      Py_DECREF(fast);
      raise(PyExc_IndexError, "tuple index out of range");
    }
  }
  Seq(const Seq&) = delete;
  ~Seq() { Py_DECREF(fast); }
  Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(fast); }
  PyObject* operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(fast, i); }
};

// A segment's dict (any mapping): need() raises KeyError, get() gives None.
struct Map {
  PyObject* dict;
  explicit Map(PyObject* o) : dict(nullptr) {
    if (PyDict_Check(o)) {
      dict = o;
      Py_INCREF(dict);
      return;
    }
    dict = PyDict_New();
    if (!dict || PyDict_Update(dict, o) != 0) {
      Py_XDECREF(dict);
      throw Raised{};
    }
  }
  Map(const Map&) = delete;
  ~Map() { Py_DECREF(dict); }
  PyObject* get(PyObject* key) const {
    PyObject* v = PyDict_GetItemWithError(dict, key);
    if (!v && PyErr_Occurred()) throw Raised{};
    return v ? v : Py_None;
  }
  bool has(PyObject* key) const {
    const int v = PyDict_Contains(dict, key);
    if (v < 0) throw Raised{};
    return v != 0;
  }
  PyObject* need(PyObject* key) const {
    PyObject* v = PyDict_GetItemWithError(dict, key);
    if (!v) {
      if (!PyErr_Occurred()) PyErr_SetObject(PyExc_KeyError, key);
      throw Raised{};
    }
    return v;
  }
};

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v != 0;
}

// Interned names of the segments' entries.
struct Names {
  PyObject *h, *x, *shift, *scale, *gated, *a, *w, *bias, *out, *resid, *gate, *q, *k, *v, *q_norm, *k_norm, *pos_offset;
  PyObject *y, *h_out, *post_w, *pre_w, *dx, *dh_out, *dh, *dy, *dgate, *dscale, *dshift, *dpost_w, *dpre_w;
  PyObject *w_gate, *w_up, *pre_gate, *pre_up;
  PyObject *codes, *scales, *codes_t, *scales_t, *exponent, *a_scales, *w_scales, *a_exponent, *w_exponent;
  PyObject *p, *g, *m, *m_scale, *v_scale;
} N;

// Stream argument: None is the calling thread's current stream.
void* stream_of(PyObject* o) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
  return reinterpret_cast<void*>(uintptr_t(integer(o)));
}

template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return nullptr;
  }
  try {
    return PyLong_FromLong(long(f()));
  } catch (const Raised&) {
    return nullptr;
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

template <class F>
ra_status released(F f) {
  ra_status s;
  Py_BEGIN_ALLOW_THREADS;
  s = f();
  Py_END_ALLOW_THREADS;
  return s;
}

// joint_attn(q, k, v, o, mass_partial, mode, softmax_scale, ref_logit_bias, mass_rows, err_word, mass_row_stride,
//            ref_fresh, a_b, step, stream)
PyObject* joint_attn(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 15, [&] {
    const Seq q(g[0], 3), k(g[1], 3), v(g[2], 3), o(g[3], 3);
    ra_attn_args a;
    std::memset(&a, 0, sizeof(a));
    const Dims dm = dims_of(k[2]);
    a.B = dm.B, a.H = dm.H, a.d = dm.d;
    for (int r = 0; r < 3; ++r) {
      const int64_t n_q = rows4(q[r] != Py_None ? q[r] : k[r]);
      a.q[r] = seg(q[r], n_q);
      a.k[r] = seg(k[r]);
      a.v[r] = seg(v[r]);
      a.o[r] = seg(o[r], n_q);
    }
    a.mass_partial = static_cast<float*>(address(g[4]));
    a.mode = static_cast<const int32_t*>(address(g[5]));
    a.softmax_scale = float(real(g[6]));
    a.ref_logit_bias = static_cast<const float*>(address(g[7]));
    a.mass_rows = integer32(g[8]);
    a.err_word = static_cast<int32_t*>(address(g[9]));
    a.mass_row_stride = integer32(g[10]);
    if (g[11] != Py_None) {
      const Seq f(g[11], 0);
      if (f.size() != 3) raise(PyExc_ValueError, "ref_fresh: expected (q, k, v)");
      a.ref_fresh_q = seg(f[0]);
      a.ref_fresh_k = seg(f[1]);
      a.ref_fresh_v = seg(f[2]);
      a.a_b = static_cast<int32_t*>(address(g[12]));
      a.step = integer32(g[13]);
    }
    void* st = stream_of(g[14]);
    return released([&] { return refadapt_joint_attn(&a, st); });
  });
}

size_t bytes_of(PyObject* o) {
  const at::Tensor& t = tensor(o);
  return size_t(t.numel()) * size_t(t.element_size());
}

// q_delta(q_cur, q_prev, d_out, workspace, eps, stream)
PyObject* q_delta(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 6, [&] {
    const Dims dm = dims_of(g[0]);
    const ra_seg c = seg(g[0]), p = seg(g[1]);
    float* d_out = static_cast<float*>(address(g[2]));
    void* ws = address(g[3]);
    const size_t ws_bytes = bytes_of(g[3]);
    const float eps = float(real(g[4]));
    void* st = stream_of(g[5]);
    return released([&] { return refadapt_q_delta(&c, &p, dm.B, dm.H, dm.d, eps, d_out, ws, ws_bytes, st); });
  });
}

// head: t, b, state, mode_out, theta, delta_max; tail: mass_partial_prev, mass_row_count, forced_boundary, gbar_out,
// m_out, cue
ra_gate_args gate_args(PyObject* const* head, int32_t B, int32_t H, PyObject* q_delta, PyObject* const* tail) {
  ra_gate_args a;
  std::memset(&a, 0, sizeof(a));
  a.t = integer32(head[0]);
  a.b = integer32(head[1]);
  a.state = static_cast<ra_state*>(address(head[2]));
  a.mode_out = static_cast<int32_t*>(address(head[3]));
  a.theta = real(head[4]);
  a.delta_max = integer32(head[5]);
  a.B = B;
  a.H = H;
  a.q_delta = static_cast<const float*>(address(q_delta));
  a.mass_partial_prev = static_cast<const float*>(address(tail[0]));
  if (tail[0] != Py_None) {
    const at::Tensor& m = tensor(tail[0]);
    if (m.dim() < 1) raise(PyExc_IndexError, "tuple index out of range");
    a.mass_partial_len = int32_t(m.size(-1));
  }
  a.mass_row_count = integer32(tail[1]);
  a.forced_boundary = integer32(tail[2]);
  a.gbar_out = static_cast<float*>(address(tail[3]));
  a.m_out = static_cast<float*>(address(tail[4]));
  a.cue = integer32(tail[5]);
  return a;
}

// gate(<head>, B, H, q_delta, <tail>, stream)
PyObject* gate(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 16, [&] {
    const ra_gate_args a = gate_args(g, integer32(g[6]), integer32(g[7]), g[8], g + 9);
    void* st = stream_of(g[15]);
    return released([&] { return refadapt_gate(&a, st); });
  });
}

// q_delta_gate(q_cur, q_prev, d_out, workspace, eps, stream, <head>, <tail>)
PyObject* q_delta_gate(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 18, [&] {
    const Dims dm = dims_of(g[0]);
    const ra_seg c = seg(g[0]), p = seg(g[1]);
    float* d_out = static_cast<float*>(address(g[2]));
    void* ws = address(g[3]);
    const size_t ws_bytes = bytes_of(g[3]);
    const float eps = float(real(g[4]));
    const ra_gate_args a = gate_args(g + 6, dm.B, dm.H, g[2], g + 12);
    void* st = stream_of(g[5]);
    return released([&] { return refadapt_q_delta_gate(&c, &p, dm.B, dm.H, dm.d, eps, d_out, ws, ws_bytes, &a, st); });
  });
}

[[noreturn]] void too_many_segments() { raise(PyExc_IndexError, "invalid index"); }

// ln_modulate(segs, C, eps, mode, stream)
PyObject* ln_modulate(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const Seq segs(g[0], 0);
    ra_lnmod_args a;
    std::memset(&a, 0, sizeof(a));
    for (Py_ssize_t i = 0; i < segs.size(); ++i) {
      if (i >= 3) too_many_segments();
      const Map sd(segs[i]);
      ra_lnmod_seg& s = a.seg[i];
      const Rows h = rows_of(sd.need(N.h), "h"), x = rows_of(sd.need(N.x), "x");
      if (h.rows != x.rows) raise(PyExc_ValueError, "h and x rows differ");
      a.B = int32_t(h.samples);
      s.h = h.ptr, s.h_stride_s = h.stride_s, s.h_stride_r = h.stride_r;
      s.x = x.ptr, s.x_stride_s = x.stride_s, s.x_stride_r = x.stride_r;
      const at::Tensor &shift = tensor(sd.need(N.shift)), &scale = tensor(sd.need(N.scale));
      s.shift = static_cast<const float*>(shift.data_ptr());
      s.scale = static_cast<const float*>(scale.data_ptr());
      s.mod_stride_s = shift.stride(0);
      if (scale.stride(0) != s.mod_stride_s) raise(PyExc_ValueError, "shift and scale must share a row stride");
      s.rows = int32_t(h.rows);
      s.gated = truth(sd.get(N.gated));
    }
    if (segs.size() == 0) raise(PyExc_TypeError, "refadapt_ln_modulate: no segments");
    a.n_seg = int32_t(segs.size());
    a.C = integer32(g[1]);
    a.eps = float(real(g[2]));
    a.mode = static_cast<const int32_t*>(address(g[3]));
    void* st = stream_of(g[4]);
    return released([&] { return refadapt_ln_modulate(&a, st); });
  });
}

// gemm(segs, N, K, epilogue, mode, rope, H, d, norm_eps, err_word, tile_mode, stream)
PyObject* gemm(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 12, [&] {
    const Seq segs(g[0], 0);
    ra_gemm_args a;
    std::memset(&a, 0, sizeof(a));
    a.N = integer32(g[1]);
    a.K = integer32(g[2]);
    a.epilogue = integer32(g[3]);
    for (Py_ssize_t i = 0; i < segs.size(); ++i) {
      if (i >= 3) too_many_segments();
      const Map sd(segs[i]);
      ra_gemm_seg& s = a.seg[i];
      const Rows ar = rows_of(sd.need(N.a), "a");
      a.B = int32_t(ar.samples);
      s.a = ar.ptr, s.a_stride_s = ar.stride_s, s.a_stride_r = ar.stride_r, s.rows = int32_t(ar.rows);
      s.gated = truth(sd.get(N.gated));
      PyObject* wo = sd.need(N.w);
      const at::Tensor& w = tensor(wo);
      if (w.dim() != 2 || w.size(0) != a.N || w.size(1) != a.K || !w.is_contiguous() ||
          w.scalar_type() != at::kBFloat16) {
        PyObject* shape = shape_of(wo);
        PyErr_Format(PyExc_ValueError, "w: expected a contiguous [N, K] = [%d, %d] bf16 tensor, got %S", int(a.N),
                     int(a.K), shape);
        Py_DECREF(shape);
        throw Raised{};
      }
      s.w = w.data_ptr();
      s.bias = static_cast<const float*>(address(sd.get(N.bias)));
      if (PyObject* out = sd.get(N.out); out != Py_None) {
        const Rows r = rows_of(out, "out");
        s.out = r.ptr, s.out_stride_s = r.stride_s, s.out_stride_r = r.stride_r;
      }
      if (PyObject* res = sd.get(N.resid); res != Py_None) {
        const Rows r = rows_of(res, "resid");
        s.resid = r.ptr, s.resid_stride_s = r.stride_s, s.resid_stride_r = r.stride_r;
      }
      if (PyObject* gt = sd.get(N.gate); gt != Py_None) {
        const at::Tensor& t = tensor(gt);
        s.gate = static_cast<const float*>(t.data_ptr());
        s.gate_stride_s = t.stride(0);
      }
      if (a.epilogue == RA_EPI_QKV) {
        s.q_out = seg(sd.need(N.q));
        s.k_out = seg(sd.need(N.k));
        s.v_out = seg(sd.need(N.v));
        s.q_norm = static_cast<const float*>(address(sd.need(N.q_norm)));
        s.k_norm = static_cast<const float*>(address(sd.need(N.k_norm)));
        s.pos_offset = sd.has(N.pos_offset) ? as_int32(sd.need(N.pos_offset)) : 0;
      }
    }
    if (segs.size() == 0) raise(PyExc_TypeError, "refadapt_gemm: no segments");
    a.n_seg = int32_t(segs.size());
    a.mode = static_cast<const int32_t*>(address(g[4]));
    a.rope = static_cast<const float*>(address(g[5]));
    a.rope_len = g[5] != Py_None ? int32_t(tensor(g[5]).size(0)) : 0;
    a.H = integer32(g[6]);
    a.d = integer32(g[7]);
    a.norm_eps = float(real(g[8]));
    a.err_word = static_cast<int32_t*>(address(g[9]));
    a.tile_mode = integer32(g[10]);
    void* st = stream_of(g[11]);
    return released([&] { return refadapt_gemm(&a, st); });
  });
}

[[noreturn]] void bad_tensor(PyObject* o, const char* what, const char* want) {
  PyObject* shape = shape_of(o);
  PyObject* dtype = PyObject_GetAttrString(o, "dtype");
  PyObject* device = PyObject_GetAttrString(o, "device");
  if (dtype && device) PyErr_Format(PyExc_ValueError, "%s: expected %s, got %S %S %S", what, want, shape, dtype, device);
  Py_DECREF(shape);
  Py_XDECREF(dtype);
  Py_XDECREF(device);
  throw Raised{};
}

// Rows of a layer call: [B, rows, F] bf16 CUDA, contiguous features; all of one
// call's rows agree in B and rows, which the first fixes.
struct RowShape {
  int64_t B = -1, rows = -1;
  Rows take(PyObject* o, const char* what, int64_t F) {
    if (o == Py_None) return Rows{nullptr, 0, 0, 0, 0};
    const at::Tensor& t = tensor(o);
    if (t.dim() != 3 || t.scalar_type() != at::kBFloat16 || !t.is_cuda() || t.size(2) != F ||
        (F > 1 && t.numel() > 0 && t.stride(2) != 1) || (B >= 0 && (t.size(0) != B || t.size(1) != rows))) {
      char want[160];
      if (B >= 0)
        snprintf(want, sizeof(want), "a [%lld, %lld, %lld] bf16 CUDA tensor with contiguous last axis", (long long)B,
                 (long long)rows, (long long)F);
      else
        snprintf(want, sizeof(want), "a [B, rows, %lld] bf16 CUDA tensor with contiguous last axis", (long long)F);
      bad_tensor(o, what, want);
    }
    B = t.size(0), rows = t.size(1);
    if (B > INT32_MAX || rows > INT32_MAX) raise(PyExc_ValueError, "too many samples or rows");
    // the stride of an axis with one entry says nothing
    return Rows{t.numel() > 0 ? t.data_ptr() : nullptr, B > 1 ? t.stride(0) : 0, rows > 1 ? t.stride(1) : (F + 7) / 8 * 8,
                rows, B};
  }
};

struct Vecs {
  float* ptr;
  int64_t stride;
};
// [B, C] fp32 CUDA (None: absent), contiguous last axis.
Vecs vecs_of(PyObject* o, const char* what, int64_t B, int64_t C, bool contiguous = false) {
  if (o == Py_None) return Vecs{nullptr, 0};
  const at::Tensor& t = tensor(o);
  if (t.dim() != 2 || t.scalar_type() != at::kFloat || !t.is_cuda() || t.size(0) != B || t.size(1) != C ||
      (C > 1 && t.stride(1) != 1) || (contiguous && !t.is_contiguous())) {
    char want[128];
    snprintf(want, sizeof(want), "a %s[%lld, %lld] fp32 CUDA tensor", contiguous ? "contiguous " : "", (long long)B,
             (long long)C);
    bad_tensor(o, what, want);
  }
  return Vecs{static_cast<float*>(t.data_ptr()), B > 1 ? t.stride(0) : 0};
}
// [C] fp32 CUDA (None: absent), contiguous.
float* vec_of(PyObject* o, const char* what, int64_t C) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.dim() != 1 || t.scalar_type() != at::kFloat || !t.is_cuda() || t.size(0) != C || !t.is_contiguous()) {
    char want[96];
    snprintf(want, sizeof(want), "a contiguous [%lld] fp32 CUDA tensor", (long long)C);
    bad_tensor(o, what, want);
  }
  return static_cast<float*>(t.data_ptr());
}
struct Scratch {
  void* ptr;
  size_t bytes;
};
Scratch scratch_of(PyObject* o) {
  const at::Tensor& t = tensor(o);
  if (!t.is_cuda() || !t.is_contiguous()) bad_tensor(o, "workspace", "a contiguous CUDA tensor");
  return Scratch{t.data_ptr(), bytes_of(o)};
}
// [B] int32 CUDA modes (None: absent).
const int32_t* modes_of(PyObject* o, int64_t B) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != at::kInt || !t.is_cuda() || t.dim() != 1 || t.size(0) != B || !t.is_contiguous())
    bad_tensor(o, "mode", "a contiguous [B] int32 CUDA tensor");
  return static_cast<const int32_t*>(t.data_ptr());
}

// rope_axes(tensors, pos, axes, base, inverse, stream)
PyObject* rope_axes(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 6, [&] {
    const Seq ts(g[0], 1), axes(g[2], 1);
    ra_rope_args a;
    std::memset(&a, 0, sizeof(a));
    if (ts.size() > 2) raise(PyExc_ValueError, "refadapt_rope_axes: at most two tensors");
    if (axes.size() > 4) raise(PyExc_ValueError, "refadapt_rope_axes: at most four axes");
    a.n_tensors = int32_t(ts.size());
    a.n_axes = int32_t(axes.size());
    for (Py_ssize_t i = 0; i < axes.size(); ++i) a.axis_dim[i] = integer32(axes[i]);
    for (Py_ssize_t i = 0; i < ts.size(); ++i) {
      const Seq pair(ts[i], 2);
      a.t[i].x = seg(pair[0]);
      a.t[i].out = seg(pair[1]);
      const at::Tensor &x = tensor(pair[0]), &o = tensor(pair[1]);
      if (x.sizes() != o.sizes() || x.size(0) != tensor(Seq(ts[0], 2)[0]).size(0) || x.size(2) != a.t[0].x.n ||
          x.size(3) != tensor(Seq(ts[0], 2)[0]).size(3))
        raise(PyExc_ValueError, "refadapt_rope_axes: a tensor and its output, and the tensors but for their heads, have "
                                "one shape");
      a.t[i].heads = int32_t(x.size(1));
      a.B = int32_t(x.size(0));
      a.n = int32_t(x.size(2));
      a.d = int32_t(x.size(3));
    }
    const at::Tensor& pos = tensor(g[1]);
    const bool per_sample = pos.dim() == 3;
    if (!pos.is_cuda() || pos.scalar_type() != at::kFloat || (pos.dim() != 2 && !per_sample) ||
        pos.size(-1) != a.n_axes || pos.size(-2) != a.n || (per_sample && pos.size(0) != a.B && pos.size(0) != 1) ||
        (a.n > 1 && pos.stride(-2) != a.n_axes) || (a.n_axes > 1 && pos.stride(-1) != 1))
      bad_tensor(g[1], "pos", "an [n, axes] or [B, n, axes] fp32 CUDA tensor with contiguous rows");
    a.pos = static_cast<const float*>(pos.data_ptr());
    a.pos_stride_s = per_sample && pos.size(0) > 1 ? pos.stride(0) : 0;
    a.base = real(g[3]);
    a.inverse = truth(g[4]);
    void* st = stream_of(g[5]);
    return released([&] { return refadapt_rope_axes(&a, st); });
  });
}

// residual_norm(segs, C, post, pre, eps, alpha, mode, stream)
PyObject* residual_norm(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    const Seq segs(g[0], 0);
    ra_resnorm_args a;
    std::memset(&a, 0, sizeof(a));
    a.C = integer32(g[1]);
    for (Py_ssize_t i = 0; i < segs.size(); ++i) {
      if (i >= 3) too_many_segments();
      const Map sd(segs[i]);
      ra_resnorm_seg& s = a.seg[i];
      RowShape shape;
      const Rows h = shape.take(sd.need(N.h), "h", a.C), y = shape.take(sd.get(N.y), "y", a.C),
                 o = shape.take(sd.get(N.h_out), "h_out", a.C), x = shape.take(sd.get(N.x), "x", a.C);
      if (shape.B < 0) raise(PyExc_ValueError, "h: expected a tensor");
      if (i > 0 && a.B != shape.B) raise(PyExc_ValueError, "refadapt_residual_norm: segments of one batch size needed");
      a.B = int32_t(shape.B);
      s.h = h.ptr, s.h_stride_s = h.stride_s, s.h_stride_r = h.stride_r;
      s.y = y.ptr, s.y_stride_s = y.stride_s, s.y_stride_r = y.stride_r;
      s.h_out = o.ptr, s.h_out_stride_s = o.stride_s, s.h_out_stride_r = o.stride_r;
      s.x = x.ptr, s.x_stride_s = x.stride_s, s.x_stride_r = x.stride_r;
      const Vecs gate = vecs_of(sd.get(N.gate), "gate", a.B, a.C), scale = vecs_of(sd.get(N.scale), "scale", a.B, a.C),
                 shift = vecs_of(sd.get(N.shift), "shift", a.B, a.C);
      if (scale.ptr && shift.ptr && scale.stride != shift.stride)
        raise(PyExc_ValueError, "shift and scale must share a row stride");
      s.gate = gate.ptr, s.gate_stride_s = gate.stride;
      s.scale = scale.ptr, s.shift = shift.ptr, s.mod_stride_s = scale.ptr ? scale.stride : shift.stride;
      s.post_w = vec_of(sd.get(N.post_w), "post_w", a.C);
      s.pre_w = vec_of(sd.get(N.pre_w), "pre_w", a.C);
      s.rows = int32_t(shape.rows);
      s.gated = truth(sd.get(N.gated));
    }
    if (segs.size() == 0) raise(PyExc_TypeError, "refadapt_residual_norm: no segments");
    a.n_seg = int32_t(segs.size());
    a.post = integer32(g[2]);
    a.pre = integer32(g[3]);
    a.eps = float(real(g[4]));
    a.alpha = float(real(g[5]));
    a.mode = modes_of(g[6], a.B);
    void* st = stream_of(g[7]);
    return released([&] { return refadapt_residual_norm(&a, st); });
  });
}

// residual_norm_backward(seg, C, post, pre, workspace, eps, alpha, err_word, stream)
PyObject* residual_norm_backward(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    const Map sd(g[0]);
    ra_resnorm_grad_args a;
    std::memset(&a, 0, sizeof(a));
    a.C = integer32(g[1]);
    RowShape shape;
    const Rows h = shape.take(sd.need(N.h), "h", a.C), y = shape.take(sd.get(N.y), "y", a.C),
               dx = shape.take(sd.get(N.dx), "dx", a.C), dho = shape.take(sd.get(N.dh_out), "dh_out", a.C),
               dh = shape.take(sd.get(N.dh), "dh", a.C), dy = shape.take(sd.get(N.dy), "dy", a.C);
    if (shape.B < 0) raise(PyExc_ValueError, "h: expected a tensor");
    a.B = int32_t(shape.B), a.rows = int32_t(shape.rows);
    a.h = h.ptr, a.h_stride_s = h.stride_s, a.h_stride_r = h.stride_r;
    a.y = y.ptr, a.y_stride_s = y.stride_s, a.y_stride_r = y.stride_r;
    a.dx = dx.ptr, a.dx_stride_s = dx.stride_s, a.dx_stride_r = dx.stride_r;
    a.dh_out = dho.ptr, a.dh_out_stride_s = dho.stride_s, a.dh_out_stride_r = dho.stride_r;
    a.dh = dh.ptr, a.dh_stride_s = dh.stride_s, a.dh_stride_r = dh.stride_r;
    a.dy = dy.ptr, a.dy_stride_s = dy.stride_s, a.dy_stride_r = dy.stride_r;
    const Vecs gate = vecs_of(sd.get(N.gate), "gate", a.B, a.C), scale = vecs_of(sd.get(N.scale), "scale", a.B, a.C);
    a.gate = gate.ptr, a.gate_stride_s = gate.stride;
    a.scale = scale.ptr, a.mod_stride_s = scale.stride;
    a.post_w = vec_of(sd.get(N.post_w), "post_w", a.C);
    a.pre_w = vec_of(sd.get(N.pre_w), "pre_w", a.C);
    a.dgate = vecs_of(sd.get(N.dgate), "dgate", a.B, a.C, true).ptr;
    a.dscale = vecs_of(sd.get(N.dscale), "dscale", a.B, a.C, true).ptr;
    a.dshift = vecs_of(sd.get(N.dshift), "dshift", a.B, a.C, true).ptr;
    a.dpost_w = vec_of(sd.get(N.dpost_w), "dpost_w", a.C);
    a.dpre_w = vec_of(sd.get(N.dpre_w), "dpre_w", a.C);
    a.post = integer32(g[2]);
    a.pre = integer32(g[3]);
    const Scratch ws = scratch_of(g[4]);
    a.workspace = ws.ptr, a.workspace_bytes = ws.bytes;
    a.eps = float(real(g[5]));
    a.alpha = float(real(g[6]));
    a.err_word = static_cast<int32_t*>(address(g[7]));
    void* st = stream_of(g[8]);
    return released([&] { return refadapt_residual_norm_backward(&a, st); });
  });
}

// [rows, cols] bf16 CUDA weight (None: absent), contiguous.
void* weight_of(PyObject* o, const char* what, int64_t rows, int64_t cols) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.dim() != 2 || t.scalar_type() != at::kBFloat16 || !t.is_cuda() || t.size(0) != rows || t.size(1) != cols ||
      !t.is_contiguous()) {
    char want[128];
    snprintf(want, sizeof(want), "a contiguous [%lld, %lld] bf16 CUDA tensor", (long long)rows, (long long)cols);
    bad_tensor(o, what, want);
  }
  return t.data_ptr();
}

// glu(segs, F, C, act, mode, err_word, stream)
PyObject* glu(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    const Seq segs(g[0], 0);
    ra_glu_args a;
    std::memset(&a, 0, sizeof(a));
    a.F = integer32(g[1]);
    a.C = integer32(g[2]);
    a.act = integer32(g[3]);
    for (Py_ssize_t i = 0; i < segs.size(); ++i) {
      if (i >= 3) too_many_segments();
      const Map sd(segs[i]);
      ra_glu_seg& s = a.seg[i];
      RowShape shape;
      const Rows x = shape.take(sd.need(N.x), "x", a.C), o = shape.take(sd.need(N.out), "out", a.F),
                 pg = shape.take(sd.get(N.pre_gate), "pre_gate", a.F), pu = shape.take(sd.get(N.pre_up), "pre_up", a.F);
      if (shape.B < 0) raise(PyExc_ValueError, "x: expected a tensor");
      if (i > 0 && a.B != shape.B) raise(PyExc_ValueError, "refadapt_glu: segments of one batch size needed");
      a.B = int32_t(shape.B);
      s.x = x.ptr, s.x_stride_s = x.stride_s, s.x_stride_r = x.stride_r;
      s.out = o.ptr, s.out_stride_s = o.stride_s, s.out_stride_r = o.stride_r;
      s.pre_gate = pg.ptr, s.pre_gate_stride_s = pg.stride_s, s.pre_gate_stride_r = pg.stride_r;
      s.pre_up = pu.ptr, s.pre_up_stride_s = pu.stride_s, s.pre_up_stride_r = pu.stride_r;
      s.w_gate = weight_of(sd.need(N.w_gate), "w_gate", a.F, a.C);
      s.w_up = weight_of(sd.need(N.w_up), "w_up", a.F, a.C);
      s.rows = int32_t(shape.rows);
      s.gated = truth(sd.get(N.gated));
    }
    if (segs.size() == 0) raise(PyExc_TypeError, "refadapt_glu: no segments");
    a.n_seg = int32_t(segs.size());
    a.mode = modes_of(g[4], a.B);
    a.err_word = static_cast<int32_t*>(address(g[5]));
    void* st = stream_of(g[6]);
    return released([&] { return refadapt_glu(&a, st); });
  });
}

// glu_backward(dy, x, w_gate, w_up, w_down, pre_gate, pre_up, hidden, act, workspace, dx, dw_gate, dw_up, dw_down,
//              err_word, stream)
PyObject* glu_backward(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 16, [&] {
    ra_glu_grad_args a;
    std::memset(&a, 0, sizeof(a));
    const at::Tensor &dy = tensor(g[0]), &wg = tensor(g[2]);
    if (dy.dim() != 3) bad_tensor(g[0], "dy", "a [B, rows, O] bf16 CUDA tensor");
    if (wg.dim() != 2) bad_tensor(g[2], "w_gate", "a contiguous [F, C] bf16 CUDA tensor");
    if (dy.size(2) > INT32_MAX || wg.size(0) > INT32_MAX || wg.size(1) > INT32_MAX)
      raise(PyExc_ValueError, "refadapt_glu_backward: too many features");
    a.O = int32_t(dy.size(2)), a.F = int32_t(wg.size(0)), a.C = int32_t(wg.size(1));
    RowShape shape;
    const Rows d = shape.take(g[0], "dy", a.O), x = shape.take(g[1], "x", a.C), pg = shape.take(g[5], "pre_gate", a.F),
               pu = shape.take(g[6], "pre_up", a.F), h = shape.take(g[7], "hidden", a.F), dx = shape.take(g[10], "dx", a.C);
    a.B = int32_t(shape.B), a.rows = int32_t(shape.rows);
    a.dy = d.ptr, a.dy_stride_s = d.stride_s, a.dy_stride_r = d.stride_r;
    a.x = x.ptr, a.x_stride_s = x.stride_s, a.x_stride_r = x.stride_r;
    a.pre_gate = pg.ptr, a.pre_gate_stride_s = pg.stride_s, a.pre_gate_stride_r = pg.stride_r;
    a.pre_up = pu.ptr, a.pre_up_stride_s = pu.stride_s, a.pre_up_stride_r = pu.stride_r;
    a.hidden = h.ptr, a.hidden_stride_s = h.stride_s, a.hidden_stride_r = h.stride_r;
    a.dx = dx.ptr, a.dx_stride_s = dx.stride_s, a.dx_stride_r = dx.stride_r;
    a.w_gate = weight_of(g[2], "w_gate", a.F, a.C);
    a.w_up = weight_of(g[3], "w_up", a.F, a.C);
    a.w_down = weight_of(g[4], "w_down", a.O, a.F);
    a.act = integer32(g[8]);
    const Scratch ws = scratch_of(g[9]);
    a.workspace = ws.ptr, a.workspace_bytes = ws.bytes;
    a.dw_gate = weight_of(g[11], "dw_gate", a.F, a.C);
    a.dw_up = weight_of(g[12], "dw_up", a.F, a.C);
    a.dw_down = weight_of(g[13], "dw_down", a.O, a.F);
    a.err_word = static_cast<int32_t*>(address(g[14]));
    void* st = stream_of(g[15]);
    // without rows there is nothing in dx, and its address says nothing
    if (a.rows == 0 && g[10] != Py_None && !a.dw_gate && !a.dw_up && !a.dw_down) return RA_OK;
    return released([&] { return refadapt_glu_backward(&a, st); });
  });
}

// Bytes of a 4-bit matrix's codes or scales (None: absent): uint8 CUDA.
struct Bytes {
  void* ptr;
  int64_t stride_s, stride_r;
};
// Codes [B, rows, width], contiguous last axis.
Bytes codes_of(PyObject* o, const char* what, int64_t B, int64_t rows, int64_t width) {
  if (o == Py_None) return Bytes{nullptr, 0, 0};
  const at::Tensor& t = tensor(o);
  if (t.dim() != 3 || t.scalar_type() != at::kByte || !t.is_cuda() || t.size(0) != B || t.size(1) != rows ||
      t.size(2) != width || (width > 1 && t.stride(2) != 1)) {
    char want[160];
    snprintf(want, sizeof(want), "a [%lld, %lld, %lld] uint8 CUDA tensor with contiguous last axis", (long long)B,
             (long long)rows, (long long)width);
    bad_tensor(o, what, want);
  }
  return Bytes{t.numel() > 0 ? t.data_ptr() : nullptr, B > 1 ? t.stride(0) : 0,
               rows > 1 ? t.stride(1) : (width + 15) / 16 * 16};
}
// Scales of `matrices` matrices of rows x cols: any contiguous shape of that many bytes.
void* scales_of(PyObject* o, const char* what, int64_t matrices, int64_t rows, int64_t cols, int32_t format) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  const int64_t bytes = matrices * int64_t(refadapt_quant4_scales_size(int32_t(rows), int32_t(cols), format));
  if (t.scalar_type() != at::kByte || !t.is_cuda() || !t.is_contiguous() || t.numel() != bytes) {
    char want[96];
    snprintf(want, sizeof(want), "a contiguous uint8 CUDA tensor of %lld bytes", (long long)bytes);
    bad_tensor(o, what, want);
  }
  return bytes > 0 ? t.data_ptr() : nullptr;
}
int32_t optional_int(PyObject* o) { return o == Py_None ? 0 : as_int32(o); }

// quant4(segs, C, format, mode, stream)
PyObject* quant4(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const Seq segs(g[0], 0);
    ra_quant4_args a;
    std::memset(&a, 0, sizeof(a));
    a.C = integer32(g[1]);
    a.format = integer32(g[2]);
    for (Py_ssize_t i = 0; i < segs.size(); ++i) {
      if (i >= 3) too_many_segments();
      const Map sd(segs[i]);
      ra_quant4_seg& s = a.seg[i];
      RowShape shape;
      const Rows x = shape.take(sd.need(N.x), "x", a.C);
      if (shape.B < 0) raise(PyExc_ValueError, "x: expected a tensor");
      if (i > 0 && a.B != shape.B) raise(PyExc_ValueError, "refadapt_quant4: segments of one batch size needed");
      a.B = int32_t(shape.B);
      if (shape.B * shape.rows >= (int64_t(1) << 30)) raise(PyExc_ValueError, "too many samples or rows");
      s.x = x.ptr, s.x_stride_s = x.stride_s, s.x_stride_r = x.stride_r;
      const Bytes c = codes_of(sd.get(N.codes), "codes", shape.B, shape.rows, a.C / 2);
      s.codes = c.ptr, s.codes_stride_s = c.stride_s, s.codes_stride_r = c.stride_r;
      s.scales = scales_of(sd.get(N.scales), "scales", shape.B, shape.rows, a.C, a.format);
      const int64_t padded = (shape.B * shape.rows + 63) / 64 * 64;
      if (PyObject* o = sd.get(N.codes_t); o != Py_None) {
        const at::Tensor& t = tensor(o);
        if (t.dim() != 2 || t.scalar_type() != at::kByte || !t.is_cuda() || t.size(0) != a.C ||
            t.size(1) != padded / 2 || (padded > 2 && t.stride(1) != 1)) {
          char want[128];
          snprintf(want, sizeof(want), "a [%d, %lld] uint8 CUDA tensor with contiguous last axis", int(a.C),
                   (long long)(padded / 2));
          bad_tensor(o, "codes_t", want);
        }
        s.codes_t = t.numel() > 0 ? t.data_ptr() : nullptr, s.codes_t_stride = t.stride(0);
      }
      s.scales_t = scales_of(sd.get(N.scales_t), "scales_t", 1, a.C, padded, a.format);
      s.rows = int32_t(shape.rows);
      s.gated = truth(sd.get(N.gated));
      s.exponent = optional_int(sd.get(N.exponent));
    }
    if (segs.size() == 0) raise(PyExc_TypeError, "refadapt_quant4: no segments");
    a.n_seg = int32_t(segs.size());
    a.mode = modes_of(g[3], a.B);
    void* st = stream_of(g[4]);
    return released([&] { return refadapt_quant4(&a, st); });
  });
}

// ra_seg of a [B, H, rows, d] output.
ra_seg heads_of(PyObject* o, const char* what, int64_t B, int64_t H, int64_t rows, int64_t d) {
  const ra_seg s = seg(o);
  const at::Tensor& t = tensor(o);
  if (t.size(0) != B || t.size(1) != H || t.size(2) != rows || t.size(3) != d) {
    char want[128];
    snprintf(want, sizeof(want), "a [%lld, %lld, %lld, %lld] bf16 CUDA tensor", (long long)B, (long long)H,
             (long long)rows, (long long)d);
    bad_tensor(o, what, want);
  }
  return s;
}

// gemm4(segs, N, K, epilogue, format, mode, rope, H, d, norm_eps, err_word, tile_mode, stream)
PyObject* gemm4(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 13, [&] {
    const Seq segs(g[0], 0);
    ra_gemm4_args a;
    std::memset(&a, 0, sizeof(a));
    a.N = integer32(g[1]);
    a.K = integer32(g[2]);
    a.epilogue = integer32(g[3]);
    a.format = integer32(g[4]);
    a.H = integer32(g[7]);
    a.d = integer32(g[8]);
    for (Py_ssize_t i = 0; i < segs.size(); ++i) {
      if (i >= 3) too_many_segments();
      const Map sd(segs[i]);
      ra_gemm4_seg& q = a.seg[i];
      ra_gemm_seg& s = q.lin;
      PyObject* ao = sd.need(N.a);
      const at::Tensor& at = tensor(ao);
      if (at.dim() != 3) bad_tensor(ao, "a", "a [B, rows, K / 2] uint8 CUDA tensor with contiguous last axis");
      const int64_t B = at.size(0), rows = at.size(1);
      if (i > 0 && a.B != B) raise(PyExc_ValueError, "refadapt_gemm4: segments of one batch size needed");
      if (B > INT32_MAX || rows > INT32_MAX) raise(PyExc_ValueError, "too many samples or rows");
      a.B = int32_t(B);
      const Bytes c = codes_of(ao, "a", B, rows, a.K / 2);
      s.a = c.ptr, s.a_stride_s = c.stride_s, s.a_stride_r = c.stride_r, s.rows = int32_t(rows);
      s.gated = truth(sd.get(N.gated));
      PyObject* wo = sd.need(N.w);
      const at::Tensor& w = tensor(wo);
      if (w.dim() != 2 || w.size(0) != a.N || w.size(1) != a.K / 2 || !w.is_contiguous() || !w.is_cuda() ||
          w.scalar_type() != at::kByte)
        bad_tensor(wo, "w", "a contiguous [N, K / 2] uint8 CUDA tensor");
      s.w = w.data_ptr();
      q.a_scales = scales_of(sd.need(N.a_scales), "a_scales", B, rows, a.K, a.format);
      q.w_scales = scales_of(sd.need(N.w_scales), "w_scales", 1, a.N, a.K, a.format);
      q.a_exponent = optional_int(sd.get(N.a_exponent));
      q.w_exponent = optional_int(sd.get(N.w_exponent));
      s.bias = vec_of(sd.get(N.bias), "bias", a.N);
      RowShape shape;
      shape.B = B, shape.rows = rows;
      if (a.epilogue == RA_EPI_QKV) {
        s.q_out = heads_of(sd.need(N.q), "q", B, a.H, rows, a.d);
        s.k_out = heads_of(sd.need(N.k), "k", B, a.H, rows, a.d);
        s.v_out = heads_of(sd.need(N.v), "v", B, a.H, rows, a.d);
        s.q_norm = vec_of(sd.need(N.q_norm), "q_norm", a.d);
        s.k_norm = vec_of(sd.need(N.k_norm), "k_norm", a.d);
        s.pos_offset = optional_int(sd.get(N.pos_offset));
      } else {
        const Rows o = shape.take(sd.need(N.out), "out", a.N), r = shape.take(sd.get(N.resid), "resid", a.N);
        s.out = o.ptr, s.out_stride_s = o.stride_s, s.out_stride_r = o.stride_r;
        s.resid = r.ptr, s.resid_stride_s = r.stride_s, s.resid_stride_r = r.stride_r;
        const Vecs gate = vecs_of(sd.get(N.gate), "gate", B, a.N);
        s.gate = gate.ptr, s.gate_stride_s = gate.stride;
      }
    }
    if (segs.size() == 0) raise(PyExc_TypeError, "refadapt_gemm4: no segments");
    a.n_seg = int32_t(segs.size());
    a.mode = modes_of(g[5], a.B);
    if (g[6] != Py_None) {
      const at::Tensor& r = tensor(g[6]);
      if (r.dim() != 3 || r.scalar_type() != at::kFloat || !r.is_cuda() || !r.is_contiguous() || 2 * r.size(1) != a.d ||
          r.size(2) != 2 || r.size(0) > INT32_MAX)
        bad_tensor(g[6], "rope", "a contiguous [positions, d / 2, 2] fp32 CUDA tensor");
      a.rope = static_cast<const float*>(r.data_ptr());
      a.rope_len = int32_t(r.size(0));
    }
    a.norm_eps = float(real(g[9]));
    a.err_word = static_cast<int32_t*>(address(g[10]));
    a.tile_mode = integer32(g[11]);
    void* st = stream_of(g[12]);
    return released([&] { return refadapt_gemm4(&a, st); });
  });
}

// linear4_backward(dy, x, w, workspace, dx, dw, err_word, stream)
PyObject* linear4_backward(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    ra_linear4_grad_args a;
    std::memset(&a, 0, sizeof(a));
    const at::Tensor &dy = tensor(g[0]), &wide = tensor(g[2] != Py_None ? g[2] : g[1]);
    if (dy.dim() != 3) bad_tensor(g[0], "dy", "a [B, rows, N] bf16 CUDA tensor");
    if (wide.dim() < 1 || dy.size(2) > INT32_MAX || wide.size(-1) > INT32_MAX)
      raise(PyExc_ValueError, "refadapt_linear4_backward: w or x: expected [N, K] or [B, rows, K]");
    a.N = int32_t(dy.size(2)), a.K = int32_t(wide.size(-1));
    RowShape shape;
    const Rows d = shape.take(g[0], "dy", a.N), x = shape.take(g[1], "x", a.K), dx = shape.take(g[4], "dx", a.K);
    a.B = int32_t(shape.B), a.rows = int32_t(shape.rows);
    a.dy = d.ptr, a.dy_stride_s = d.stride_s, a.dy_stride_r = d.stride_r;
    a.x = x.ptr, a.x_stride_s = x.stride_s, a.x_stride_r = x.stride_r;
    a.dx = dx.ptr, a.dx_stride_s = dx.stride_s, a.dx_stride_r = dx.stride_r;
    a.w = weight_of(g[2], "w", a.N, a.K);
    a.dw = weight_of(g[5], "dw", a.N, a.K);
    const Scratch ws = scratch_of(g[3]);
    a.workspace = ws.ptr, a.workspace_bytes = ws.bytes;
    a.err_word = static_cast<int32_t*>(address(g[6]));
    void* st = stream_of(g[7]);
    // without rows there is nothing in dx, and its address says nothing
    if (a.rows == 0 && g[4] != Py_None && !a.dw) return RA_OK;
    return released([&] { return refadapt_linear4_backward(&a, st); });
  });
}

// A contiguous CUDA tensor of n elements (n < 0: any number) of one of two types.
const at::Tensor& flat_of(PyObject* o, const char* what, int64_t n, at::ScalarType a, at::ScalarType b, const char* want) {
  const at::Tensor& t = tensor(o);
  if (!t.is_cuda() || !t.is_contiguous() || (t.scalar_type() != a && t.scalar_type() != b) || (n >= 0 && t.numel() != n))
    bad_tensor(o, what, want);
  return t;
}

// grad_norm(grads, max_norm, out, workspace, stream)
PyObject* grad_norm(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const Seq grads(g[0], 0);
    std::vector<ra_grad> list(size_t(grads.size()));
    for (Py_ssize_t i = 0; i < grads.size(); ++i) {
      const at::Tensor& t =
          flat_of(grads[i], "grads", -1, at::kFloat, at::kBFloat16, "contiguous fp32 or bf16 CUDA tensors");
      list[size_t(i)] = ra_grad{t.data_ptr(), t.numel(), t.scalar_type() == at::kBFloat16 ? RA_BF16 : RA_F32, 0};
    }
    float* out = static_cast<float*>(
        flat_of(g[2], "out", 2, at::kFloat, at::kFloat, "a contiguous [2] fp32 CUDA tensor").data_ptr());
    const Scratch ws = scratch_of(g[3]);
    const float most = float(real(g[1]));
    void* st = stream_of(g[4]);
    if (list.size() > size_t(INT32_MAX)) raise(PyExc_ValueError, "too many tensors");
    return released(
        [&] { return refadapt_grad_norm(list.data(), int32_t(list.size()), most, out, ws.ptr, ws.bytes, st); });
  });
}

// adamw(tensors, lr, step, beta1, beta2, eps, decay, grad_scale, seed, stream); lr and step numbers or device tensors
PyObject* adamw(PyObject*, PyObject* const* g, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    const Seq ts(g[0], 0);
    std::vector<ra_adamw_tensor> list(size_t(ts.size()));
    ra_adamw_args a;
    std::memset(&a, 0, sizeof(a));
    a.bits = 32;
    for (Py_ssize_t i = 0; i < ts.size(); ++i) {
      const Map sd(ts[i]);
      ra_adamw_tensor& d = list[size_t(i)];
      std::memset(&d, 0, sizeof(d));
      const at::Tensor& p = flat_of(sd.need(N.p), "p", -1, at::kFloat, at::kFloat, "a contiguous fp32 CUDA tensor");
      d.n = p.numel();
      d.p = p.data_ptr();
      const at::Tensor& gr =
          flat_of(sd.need(N.g), "g", d.n, at::kFloat, at::kBFloat16, "a contiguous fp32 or bf16 CUDA tensor like p");
      d.g = gr.data_ptr();
      d.g_type = gr.scalar_type() == at::kBFloat16 ? RA_BF16 : RA_F32;
      PyObject *ms = sd.get(N.m_scale), *vs = sd.get(N.v_scale);
      const bool small = ms != Py_None || vs != Py_None;
      if (i == 0) a.bits = small ? 8 : 32;
      if (small != (a.bits == 8)) raise(PyExc_ValueError, "refadapt_adamw: all tensors' moments are in 32 or all in 8 bits");
      const at::ScalarType state = small ? at::kFloat8_e4m3fn : at::kFloat, other = small ? at::kByte : at::kFloat;
      const char* want = small ? "a contiguous float8_e4m3fn or uint8 CUDA tensor like p" : "a contiguous fp32 CUDA tensor like p";
      d.m = flat_of(sd.need(N.m), "m", d.n, state, other, want).data_ptr();
      d.v = flat_of(sd.need(N.v), "v", d.n, state, other, want).data_ptr();
      if (small) {
        const char* s_want = "a contiguous float8_e8m0fnu or uint8 CUDA tensor, one for 32 elements";
        const int64_t blocks = (d.n + 31) / 32;
        if (ms == Py_None || vs == Py_None) raise(PyExc_ValueError, "refadapt_adamw: m_scale and v_scale go together");
        d.m_scale = flat_of(ms, "m_scale", blocks, at::kFloat8_e8m0fnu, at::kByte, s_want).data_ptr();
        d.v_scale = flat_of(vs, "v_scale", blocks, at::kFloat8_e8m0fnu, at::kByte, s_want).data_ptr();
      }
      if (PyObject* w = sd.get(N.w); w != Py_None)
        d.w = flat_of(w, "w", d.n, at::kBFloat16, at::kBFloat16, "a contiguous bf16 CUDA tensor like p").data_ptr();
    }
    if (list.size() > size_t(INT32_MAX)) raise(PyExc_ValueError, "too many tensors");
    a.tensors = list.data();
    a.n_tensors = int32_t(list.size());
    if (THPVariable_Check(g[1]))
      a.lr_dev = static_cast<const float*>(
          flat_of(g[1], "lr", 1, at::kFloat, at::kFloat, "a number or an fp32 CUDA tensor of one").data_ptr());
    else
      a.lr = real(g[1]);
    if (THPVariable_Check(g[2]))
      a.step_dev = static_cast<const int32_t*>(
          flat_of(g[2], "step", 1, at::kInt, at::kInt, "a number or an int32 CUDA tensor of one").data_ptr());
    else
      a.step = integer(g[2]);
    a.beta1 = real(g[3]);
    a.beta2 = real(g[4]);
    a.eps = real(g[5]);
    a.decay = real(g[6]);
    if (g[7] != Py_None)
      a.grad_scale = static_cast<const float*>(
          flat_of(g[7], "grad_scale", 1, at::kFloat, at::kFloat, "an fp32 CUDA tensor of one").data_ptr());
    a.seed = PyLong_AsUnsignedLongLong(g[8]);
    if (PyErr_Occurred()) throw Raised{};
    void* st = stream_of(g[9]);
    return released([&] { return refadapt_adamw(&a, st); });
  });
}

#define RA_METHOD(f) \
  {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {RA_METHOD(joint_attn), RA_METHOD(q_delta), RA_METHOD(gate),   RA_METHOD(q_delta_gate),
                         RA_METHOD(ln_modulate), RA_METHOD(gemm),   RA_METHOD(rope_axes), RA_METHOD(residual_norm),
                         RA_METHOD(residual_norm_backward), RA_METHOD(glu), RA_METHOD(glu_backward),
                         RA_METHOD(quant4), RA_METHOD(gemm4), RA_METHOD(linear4_backward), RA_METHOD(grad_norm),
                         RA_METHOD(adamw), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
  const struct {
    PyObject** slot;
    const char* name;
  } names[] = {{&N.h, "h"},       {&N.x, "x"},         {&N.shift, "shift"},   {&N.scale, "scale"},
               {&N.gated, "gated"}, {&N.a, "a"},         {&N.w, "w"},           {&N.bias, "bias"},
               {&N.out, "out"},   {&N.resid, "resid"}, {&N.gate, "gate"},     {&N.q, "q"},
               {&N.k, "k"},       {&N.v, "v"},         {&N.q_norm, "q_norm"}, {&N.k_norm, "k_norm"},
               {&N.pos_offset, "pos_offset"}, {&N.y, "y"}, {&N.h_out, "h_out"}, {&N.post_w, "post_w"},
               {&N.pre_w, "pre_w"}, {&N.dx, "dx"}, {&N.dh_out, "dh_out"}, {&N.dh, "dh"}, {&N.dy, "dy"},
               {&N.dgate, "dgate"}, {&N.dscale, "dscale"}, {&N.dshift, "dshift"}, {&N.dpost_w, "dpost_w"},
               {&N.dpre_w, "dpre_w"}, {&N.w_gate, "w_gate"}, {&N.w_up, "w_up"}, {&N.pre_gate, "pre_gate"},
               {&N.pre_up, "pre_up"}, {&N.codes, "codes"}, {&N.scales, "scales"}, {&N.codes_t, "codes_t"},
               {&N.scales_t, "scales_t"}, {&N.exponent, "exponent"}, {&N.a_scales, "a_scales"},
               {&N.w_scales, "w_scales"}, {&N.a_exponent, "a_exponent"}, {&N.w_exponent, "w_exponent"}, {&N.p, "p"},
               {&N.g, "g"}, {&N.m, "m"}, {&N.m_scale, "m_scale"}, {&N.v_scale, "v_scale"}};
  for (const auto& e : names)
    if (!(*e.slot = PyUnicode_InternFromString(e.name))) return nullptr;
  return PyModule_Create(&module);
}
