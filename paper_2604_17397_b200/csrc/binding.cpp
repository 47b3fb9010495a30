// Argument marshalling of the dense operators for Python: what the ctypes binding does for the other entry points, compiled,
// because these calls' kernels take a few microseconds and ctypes with the checks in Python took six.  Reads tensors' types,
// shapes, strides and addresses, refuses what does not fit with ValueError, and calls the C ABI of libsdvg; no computation.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "sdvg.h"

namespace {

using at::ScalarType;
using at::Tensor;

int elem_type(ScalarType t) {
  switch (t) {
    case ScalarType::BFloat16: return SDVG_BF16;
    case ScalarType::Half: return SDVG_F16;
    case ScalarType::Float: return SDVG_F32;
    default: return -1;
  }
}

// Arguments are read left to right; the first that does not fit sets the error and everything after it is skipped.
struct Reader {
  PyObject* const* args;
  bool ok = true;
  int dev = -1;

  bool fail(const char* what, const char* why) {
    if (ok) PyErr_Format(PyExc_ValueError, "%s: %s", what, why);
    ok = false;
    return false;
  }
  // The tensor of argument i, null for None or after an error.
  const Tensor* tensor(int i, const char* what, bool optional) {
    if (!ok || (optional && args[i] == Py_None)) return nullptr;
    if (!THPVariable_Check(args[i])) {
      fail(what, "expected a tensor");
      return nullptr;
    }
    const Tensor& t = THPVariable_Unpack(args[i]);
    if (!t.is_cuda()) fail(what, "expected a CUDA tensor");
    else if (dev < 0) dev = t.get_device();
    else if (t.get_device() != dev) fail(what, "on another device than the other tensors");
    return ok ? &t : nullptr;
  }
  long long integer(int i) {
    if (!ok) return 0;
    const long long v = PyLong_AsLongLong(args[i]);
    if (v == -1 && PyErr_Occurred()) ok = false;
    return v;
  }
  int small(int i) {
    const long long v = integer(i);
    if (ok && (v < -2147483647 - 1 || v > 2147483647)) fail("argument", "does not fit 32 bits");
    return (int)v;
  }
  float number(int i) {
    if (!ok) return 0.f;
    const double v = PyFloat_AsDouble(args[i]);
    if (v == -1.0 && PyErr_Occurred()) ok = false;
    return (float)v;
  }
  void* address(int i) { return reinterpret_cast<void*>(static_cast<intptr_t>(integer(i))); }
};

struct Matrix {
  void* p = nullptr;
  int64_t ld = 0;
  int type = 0;
};

// A [rows, cols] tensor with unit column stride.
Matrix matrix(Reader& r, const Tensor* t, int64_t rows, int64_t cols, ScalarType dtype, const char* what) {
  Matrix m;
  if (!t) return m;
  if (t->dim() != 2 || t->size(0) != rows || t->size(1) != cols) {
    if (r.ok)
      PyErr_Format(PyExc_ValueError, "%s: expected shape [%lld, %lld]", what, (long long)rows, (long long)cols);
    r.ok = false;
  } else if (t->scalar_type() != dtype) {
    r.fail(what, "unexpected element type");
  } else if (t->stride(1) != 1 && cols > 1) {
    r.fail(what, "columns must be contiguous");
  }
  if (!r.ok) return m;
  m.p = t->data_ptr();
  m.ld = t->stride(0);
  m.type = elem_type(dtype);
  return m;
}

const float* vector(Reader& r, int i, int64_t n, const char* what) {
  const Tensor* t = r.tensor(i, what, true);
  if (!t) return nullptr;
  if (t->scalar_type() != ScalarType::Float || t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1)) {
    if (r.ok) PyErr_Format(PyExc_ValueError, "%s: expected contiguous float32 [%lld]", what, (long long)n);
    r.ok = false;
    return nullptr;
  }
  return static_cast<const float*>(t->data_ptr());
}

// One row of fp32 vectors per `group_rows` rows.
Matrix groups(Reader& r, int i, int64_t rows, int64_t cols, int group_rows, const char* what) {
  const Tensor* t = r.tensor(i, what, true);
  if (!t) return Matrix();
  if (group_rows < 1) {
    r.fail(what, "rows per group must be given");
    return Matrix();
  }
  return matrix(r, t, (rows + group_rows - 1) / group_rows, cols, ScalarType::Float, what);
}

// (x, w, out, workspace, bias, act, residual, gate, gate_rows, stream) -> status
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 10) return PyErr_Format(PyExc_TypeError, "linear takes 10 arguments");
  Reader r{args};
  const Tensor *x = r.tensor(0, "x", false), *w = r.tensor(1, "w", false), *out = r.tensor(2, "out", false),
               *ws = r.tensor(3, "workspace", false);
  if (!r.ok) return nullptr;
  if (x->dim() != 2 || w->dim() != 2) return r.fail("x, w", "expected matrices"), nullptr;
  const int64_t rows = x->size(0), inner = x->size(1), cols = w->size(0);
  const ScalarType in = x->scalar_type(), to = out->scalar_type();
  if ((in != ScalarType::BFloat16 && in != ScalarType::Half) || elem_type(to) < 0)
    return r.fail("x, out", "x must be bfloat16 or float16, out one of these or float32"), nullptr;
  if (rows > 0x7fffffff || cols > 0x7fffffff || inner > 0x7fffffff) return r.fail("x, w", "too large"), nullptr;
  const int act = r.small(5), gate_rows = r.small(8);
  const Matrix mx = matrix(r, x, rows, inner, in, "x"), mw = matrix(r, w, cols, inner, in, "w"),
               mo = matrix(r, out, rows, cols, to, "out"),
               res = matrix(r, r.tensor(6, "residual", true), rows, cols, to, "residual"),
               gate = groups(r, 7, rows, cols, gate_rows, "gate");
  const float* bias = vector(r, 4, cols, "bias");
  void* stream = r.address(9);
  if (!r.ok) return nullptr;
  // whatever may throw is read before the interpreter lock is released
  void* const space = ws->data_ptr();
  const size_t space_bytes = ws->nbytes();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = sdvg_linear(mx.p, mx.ld, mw.p, mw.ld, bias, act, static_cast<const float*>(gate.p), gate.ld, gate_rows, res.p, res.ld,
                   mo.p, mo.ld, (int)rows, (int)cols, (int)inner, mx.type, mo.type, space, space_bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// A matrix of codes and its scales, one per 128 columns and `block_rows` rows.
struct Coded {
  Matrix codes, scale;
};
Coded coded(Reader& r, const Tensor* codes, const Tensor* scale, int64_t rows, int64_t cols, int64_t block_rows, const char* what,
            const char* scale_what) {
  Coded c;
  c.codes = matrix(r, codes, rows, cols, ScalarType::Byte, what);
  c.scale = matrix(r, scale, (rows + block_rows - 1) / block_rows, (cols + 127) / 128, ScalarType::Byte, scale_what);
  return c;
}
// Rows per scale of a matrix of `rows` rows: 128 or 1, by the number of rows that its scales have.
int64_t block_rows_of(const Tensor& scale, int64_t rows) {
  return scale.dim() == 2 && scale.size(0) == (rows + 127) / 128 ? 128 : 1;
}

// (x8, x_scale, w8, w_scale, out, workspace, bias, act, residual, gate, gate_rows, out_scale, stream) -> status
PyObject* linear_e4m3(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 13) return PyErr_Format(PyExc_TypeError, "linear_e4m3 takes 13 arguments");
  Reader r{args};
  const Tensor *x = r.tensor(0, "x8", false), *xs = r.tensor(1, "x_scale", false), *w = r.tensor(2, "w8", false),
               *ws = r.tensor(3, "w_scale", false), *out = r.tensor(4, "out", false), *space_t = r.tensor(5, "workspace", false),
               *os = r.tensor(11, "out_scale", true);
  if (!r.ok) return nullptr;
  if (x->dim() != 2 || w->dim() != 2) return r.fail("x8, w8", "expected matrices"), nullptr;
  const int64_t rows = x->size(0), inner = x->size(1), cols = w->size(0), w_rows = block_rows_of(*ws, cols);
  const ScalarType to = out->scalar_type();
  if (os ? to != ScalarType::Byte : elem_type(to) < 0)
    return r.fail("out", "must be bfloat16, float16 or float32, or uint8 codes with out_scale"), nullptr;
  if (rows > 0x7fffffff || cols > 0x7fffffff || inner > 0x7fffffff) return r.fail("x8, w8", "too large"), nullptr;
  const int act = r.small(7), gate_rows = r.small(10);
  const Coded mx = coded(r, x, xs, rows, inner, 1, "x8", "x_scale"), mw = coded(r, w, ws, cols, inner, w_rows, "w8", "w_scale");
  Coded mo;
  if (os) mo = coded(r, out, os, rows, cols, 1, "out", "out_scale");
  else mo.codes = matrix(r, out, rows, cols, to, "out");
  const Matrix res = matrix(r, r.tensor(8, "residual", true), rows, cols, to, "residual"),
               gate = groups(r, 9, rows, cols, gate_rows, "gate");
  const float* bias = vector(r, 6, cols, "bias");
  void* stream = r.address(12);
  if (!r.ok) return nullptr;
  // whatever may throw is read before the interpreter lock is released
  void* const space = space_t->data_ptr();
  const size_t space_bytes = space_t->nbytes();
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = sdvg_linear_e4m3(mx.codes.p, mx.codes.ld, mx.scale.p, mx.scale.ld, mw.codes.p, mw.codes.ld, mw.scale.p, mw.scale.ld,
                        (int)w_rows, bias, act, static_cast<const float*>(gate.p), gate.ld, gate_rows, res.p, res.ld, mo.codes.p,
                        mo.codes.ld, mo.scale.p, mo.scale.ld, (int)rows, (int)cols, (int)inner, os ? SDVG_E4M3 : elem_type(to), space,
                        space_bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// (values, codes, scale, to_codes, stream) -> status
PyObject* e4m3_blocks(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 5) return PyErr_Format(PyExc_TypeError, "e4m3_blocks takes 5 arguments");
  Reader r{args};
  const Tensor *x = r.tensor(0, "values", false), *c = r.tensor(1, "codes", false), *s = r.tensor(2, "scale", false);
  if (!r.ok) return nullptr;
  if (x->dim() != 2 || elem_type(x->scalar_type()) < 0)
    return r.fail("values", "expected a matrix of bfloat16, float16 or float32"), nullptr;
  const int64_t rows = x->size(0), cols = x->size(1), block_rows = block_rows_of(*s, rows);
  if (rows > 0x7fffffff || cols > 0x7fffffff) return r.fail("values", "too large"), nullptr;
  const Matrix m = matrix(r, x, rows, cols, x->scalar_type(), "values");
  const Coded q = coded(r, c, s, rows, cols, block_rows, "codes", "scale");
  const int quantise = r.small(3);
  void* stream = r.address(4);
  if (!r.ok) return nullptr;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = quantise ? sdvg_quant_e4m3_blocks(m.p, m.ld, m.type, q.codes.p, q.codes.ld, q.scale.p, q.scale.ld, (int)block_rows, (int)rows,
                                         (int)cols, stream)
                : sdvg_dequant_e4m3_blocks(q.codes.p, q.codes.ld, q.scale.p, q.scale.ld, (int)block_rows, m.p, m.ld, m.type, (int)rows,
                                           (int)cols, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// (x, out, y, gate, gate_rows, post_norm, post_weight, x_out, norm, weight, bias, scale, shift, modulate_rows, eps, stream)
// -> status; with E4M3 also out_scale, after the stream
template <bool E4M3>
PyObject* gated_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != (E4M3 ? 17 : 16))
    return PyErr_Format(PyExc_TypeError, E4M3 ? "gated_norm_e4m3 takes 17 arguments" : "gated_norm takes 16 arguments");
  Reader r{args};
  const Tensor *x = r.tensor(0, "x", false), *out = r.tensor(1, "out", !E4M3), *y = r.tensor(2, "y", true);
  if (!r.ok) return nullptr;
  if (x->dim() != 2) return r.fail("x", "expected a matrix"), nullptr;
  const int64_t rows = x->size(0), cols = x->size(1);
  if (rows > 0x7fffffff || cols > 0x7fffffff) return r.fail("x", "too large"), nullptr;
  const Tensor* out_scale = E4M3 ? r.tensor(16, "out_scale", false) : nullptr;
  if (!r.ok) return nullptr;
  for (const Tensor* t : {x, E4M3 ? nullptr : out, y})
    if (t && elem_type(t->scalar_type()) < 0)
      return r.fail("x, y, out", "expected bfloat16, float16 or float32 tensors"), nullptr;
  const int gate_rows = r.small(4), post = r.small(5), norm = r.small(8), mod_rows = r.small(13);
  const Matrix mx = matrix(r, x, rows, cols, x->scalar_type(), "x"),
               mo = out ? matrix(r, out, rows, cols, E4M3 ? ScalarType::Byte : out->scalar_type(), "out") : Matrix(),
               ms = matrix(r, out_scale, rows, (cols + 127) / 128, ScalarType::Byte, "out_scale"),
               my = y ? matrix(r, y, rows, cols, y->scalar_type(), "y") : Matrix(),
               xo = matrix(r, r.tensor(7, "x_out", true), rows, cols, x->scalar_type(), "x_out"),
               gate = groups(r, 3, rows, cols, gate_rows, "gate"), scale = groups(r, 11, rows, cols, mod_rows, "scale"),
               shift = groups(r, 12, rows, cols, mod_rows, "shift");
  if (r.ok && scale.p && shift.p && scale.ld != shift.ld && rows > mod_rows)
    r.fail("scale, shift", "must have the same row stride");
  const float *post_weight = vector(r, 6, cols, "post_weight"), *weight = vector(r, 9, cols, "weight"),
              *bias = vector(r, 10, cols, "bias");
  const float eps = r.number(14);
  void* stream = r.address(15);
  if (!r.ok) return nullptr;
  int st;
  Py_BEGIN_ALLOW_THREADS
  if (E4M3)
    st = sdvg_gated_norm_e4m3(mx.p, mx.ld, mx.type, my.p, my.ld, my.type, post, post_weight, static_cast<const float*>(gate.p),
                              gate.ld, gate_rows, xo.p, xo.ld, norm, weight, bias, static_cast<const float*>(scale.p),
                              static_cast<const float*>(shift.p), scale.p ? scale.ld : shift.ld, mod_rows, eps, mo.p, mo.ld, ms.p,
                              ms.ld, (int)rows, (int)cols, stream);
  else
    st = sdvg_gated_norm(mx.p, mx.ld, mx.type, my.p, my.ld, my.type, post, post_weight, static_cast<const float*>(gate.p), gate.ld,
                         gate_rows, xo.p, xo.ld, norm, weight, bias, static_cast<const float*>(scale.p),
                         static_cast<const float*>(shift.p), scale.p ? scale.ld : shift.ld, mod_rows, eps, mo.p, mo.ld, mo.type,
                         (int)rows, (int)cols, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// (handle, block_tokens, heads, head_dim, q, k, v, q_weight, k_weight, scope, eps, q_out, k_out, frames, grid_h, grid_w,
// frame_offset, table, tab_frames, block_index, flags, stream) -> evicted block, or -1000 - status
// For an 8-bit ring q_out is codes and k_out None, and further arguments follow: (q_inv_scale, k_inv_scale, v_inv_scale) with static
// scales, (q_tile_scale, workspace) with tile scales.
enum Ring { kBf16, kStatic, kTiled };
template <Ring RING>
PyObject* qk_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  constexpr int kArgs = RING == kBf16 ? 22 : RING == kStatic ? 25 : 24;
  if (n != kArgs) return PyErr_Format(PyExc_TypeError, "qk_norm takes %d arguments", kArgs);
  Reader r{args};
  sdvg_cache* cache = static_cast<sdvg_cache*>(r.address(0));
  const int64_t tokens = r.integer(1), heads = r.integer(2), dim = r.integer(3);
  const int scope = r.small(9);
  const int64_t width = scope == SDVG_SCOPE_ROW ? heads * dim : dim;
  const float eps = r.number(10);
  // [tokens, heads, dim], contiguous within a token
  auto block = [&](int i, const char* what, bool optional, bool contiguous, ScalarType type = ScalarType::BFloat16) {
    Matrix m;
    const Tensor* t = r.tensor(i, what, optional);
    if (!t) return m;
    if (t->scalar_type() != type || t->dim() != 3 || t->size(0) != tokens || t->size(1) != heads || t->size(2) != dim) {
      PyErr_Format(PyExc_ValueError, "%s: expected %s [%lld, %lld, %lld]", what, type == ScalarType::Byte ? "uint8" : "bfloat16",
                   (long long)tokens, (long long)heads, (long long)dim);
      r.ok = false;
      return m;
    }
    m.ld = tokens == 1 ? heads * dim : t->stride(0);
    if (t->stride(2) != 1 || (heads > 1 && t->stride(1) != dim)) r.fail(what, "the heads of a token must be contiguous");
    else if (contiguous && m.ld != heads * dim) r.fail(what, "must be contiguous");
    m.p = t->data_ptr();
    return m;
  };
  const Matrix k = block(5, "k", false, false), q = block(4, "q", true, false), v = block(6, "v", false, false),
               q_out = block(11, "q_out", true, true, RING == kBf16 ? ScalarType::BFloat16 : ScalarType::Byte),
               k_out = RING == kBf16 ? block(12, "k_out", true, true) : Matrix();
  const float *qw = vector(r, 7, width, "q_weight"), *kw = vector(r, 8, width, "k_weight");
  const int frames = r.small(13), grid_h = r.small(14), grid_w = r.small(15), offset = r.small(16), tab_frames = r.small(18),
            flags = r.small(20);
  const Tensor* table = r.tensor(17, "table", false);
  if (table && (table->scalar_type() != ScalarType::Float || !table->is_contiguous()))
    r.fail("table", "expected a contiguous float32 tensor");
  // 0 for sizes that the call refuses below
  if (table && r.ok && (uint64_t)table->numel() < sdvg_rope3d_table_floats((int)dim, tab_frames, grid_h, grid_w))
    r.fail("table", "shorter than that of the block's grid and tab_frames");
  const int64_t index = r.integer(19);
  void* stream = r.address(21);
  const float *q_inv = nullptr, *k_inv = nullptr, *v_inv = nullptr;
  Matrix q_scale;
  void* space = nullptr;
  size_t space_bytes = 0;
  if (RING == kStatic) {
    q_inv = vector(r, 22, heads, "q_inv_scale");
    k_inv = vector(r, 23, heads, "k_inv_scale");
    v_inv = vector(r, 24, heads, "v_inv_scale");
  } else if (RING == kTiled) {
    const int64_t tiles = (tokens + 127) / 128;
    q_scale = matrix(r, r.tensor(22, "q_tile_scale", true), heads, tiles, ScalarType::Float, "q_tile_scale");
    if (r.ok && q_scale.p && heads > 1 && q_scale.ld != tiles) r.fail("q_tile_scale", "must be contiguous");
    if (const Tensor* t = r.tensor(23, "workspace", true)) {
      space = t->data_ptr();
      space_bytes = t->nbytes();
    }
  }
  if (!r.ok) return nullptr;
  const float* const tab = static_cast<const float*>(table->data_ptr());      // may throw: before the lock is released
  int64_t evicted = -1;
  int st;
  Py_BEGIN_ALLOW_THREADS
  if (RING == kBf16)
    st = sdvg_qk_norm_rope3d_commit(cache, q.p, q.ld, k.p, k.ld, v.p, v.ld, qw, kw, scope, eps, q_out.p, k_out.p, frames, grid_h,
                                    grid_w, offset, tab, tab_frames, index, flags, &evicted, stream);
  else if (RING == kStatic)
    st = sdvg_qk_norm_rope3d_commit_e4m3(cache, q.p, q.ld, k.p, k.ld, v.p, v.ld, qw, kw, scope, eps, q_out.p, q_inv, k_inv, v_inv,
                                         frames, grid_h, grid_w, offset, tab, tab_frames, index, flags, &evicted, stream);
  else
    st = sdvg_qk_norm_rope3d_commit_e4m3_tiled(cache, q.p, q.ld, k.p, k.ld, v.p, v.ld, qw, kw, scope, eps, q_out.p,
                                               static_cast<float*>(q_scale.p), frames, grid_h, grid_w, offset, tab, tab_frames, index,
                                               flags, &evicted, space, space_bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLongLong(st == SDVG_OK ? evicted : -1000 - st);
}

// (handle, block_tokens, heads, slot, k_out, v_out, k_descale, v_descale, stream) -> status
PyObject* read_block_e4m3(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 9) return PyErr_Format(PyExc_TypeError, "read_block_e4m3 takes 9 arguments");
  Reader r{args};
  const sdvg_cache* cache = static_cast<sdvg_cache*>(r.address(0));
  const int64_t tokens = r.integer(1), heads = r.integer(2);
  const int slot = r.small(3);
  void* outs[2] = {nullptr, nullptr};
  for (int i = 0; i < 2; ++i) {
    const char* const what = i ? "v_out" : "k_out";
    const Tensor* t = r.tensor(4 + i, what, true);
    if (!t) continue;
    if (t->scalar_type() != ScalarType::BFloat16 || t->dim() != 3 || t->size(0) != tokens || t->size(1) != heads || t->size(2) != 128 ||
        !t->is_contiguous()) {
      PyErr_Format(PyExc_ValueError, "%s: expected contiguous bfloat16 [%lld, %lld, 128]", what, (long long)tokens, (long long)heads);
      return nullptr;
    }
    outs[i] = t->data_ptr();
  }
  const float *ks = vector(r, 6, heads, "k_descale"), *vs = vector(r, 7, heads, "v_descale");
  void* stream = r.address(8);
  if (!r.ok) return nullptr;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = sdvg_cache_read_block_e4m3(cache, slot, ks, vs, outs[0], outs[1], stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// A C++ exception (a tensor without storage, say) becomes a Python one.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n) {
  try {
    return F(self, args, n);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<F>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<linear>("linear"), method<gated_norm<false>>("gated_norm"), method<qk_norm<kBf16>>("qk_norm"),
                         method<qk_norm<kStatic>>("qk_norm_e4m3"), method<qk_norm<kTiled>>("qk_norm_e4m3_tiled"),
                         method<linear_e4m3>("linear_e4m3"), method<gated_norm<true>>("gated_norm_e4m3"),
                         method<e4m3_blocks>("e4m3_blocks"), method<read_block_e4m3>("read_block_e4m3"),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
