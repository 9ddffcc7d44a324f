// Calls of the operators on rows of channels from Python: what binding.py's ctypes calls do for the other entry points - tensors to addresses and
// sizes, checks of what the C ABI cannot see - compiled, because these operators are also called for a few tokens at a time, where marshalling
// costs as much as the launch (norm of eight rows: 7.2 us a call through ctypes).  Every function returns the library's code; wrong tensors raise
// AssertionError.  Argument marshalling only.

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "abl.h"

namespace {

constexpr at::ScalarType kF32 = at::kFloat;

bool fail(const char* what, const char* why) {
  PyErr_Format(PyExc_AssertionError, "%s: %s", what, why);
  return false;
}

int dtype_of(at::ScalarType t) { return t == at::kFloat ? ABL_F32 : t == at::kBFloat16 ? ABL_BF16 : -1; }

const at::Tensor* tensor(PyObject* o, const char* what) {
  if (THPVariable_Check(o)) {
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.is_cuda()) return &t;
  }
  fail(what, "a device tensor");
  return nullptr;
}

bool whole(long& v, PyObject* o) {
  v = PyLong_AsLong(o);
  return v != -1 || PyErr_Occurred() == nullptr;
}
// A number that the library takes as 32 bits.
bool small(int& v, PyObject* o, const char* what) {
  long w;
  if (!whole(w, o)) return false;
  v = (int)w;
  return v == w || fail(what, "out of range");
}
bool number(float& v, PyObject* o) {
  const double d = PyFloat_AsDouble(o);
  v = (float)d;
  return d != -1.0 || PyErr_Occurred() == nullptr;
}

// Address of a contiguous tensor of that type with n elements at least; None: null, for the library to say where that is an error.
bool address(void*& p, PyObject* o, at::ScalarType type, int64_t n, const char* what) {
  p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o, what);
  if (t == nullptr) return false;
  if (t->scalar_type() != type) return fail(what, "of another type than it has to be");
  if (t->numel() < n) return fail(what, "too few elements");
  if (!t->is_contiguous()) return fail(what, "has to be contiguous");
  p = t->data_ptr();
  return true;
}
// A contiguous [M, C]; None as above.
bool matrix_address(void*& p, PyObject* o, at::ScalarType type, int64_t M, int64_t C, const char* what) {
  if (!address(p, o, type, M * C, what)) return false;
  if (o == Py_None) return true;
  const at::Tensor& t = THPVariable_Unpack(o);
  return (t.dim() == 2 && t.size(0) == M && t.size(1) == C) || fail(what, "of another shape than it has to be");
}
// A tensor of bytes that holds the K-bit store of [M, C].
bool store(void*& p, PyObject* o, int64_t M, int64_t C, int K, const char* what) {
  p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o, what);
  if (t == nullptr) return false;
  if (t->element_size() != 1 || !t->is_contiguous()) return fail(what, "contiguous bytes");
  const int64_t used = M * ((C + 31) / 32) * (4 * (int64_t)K + 1);
  if (t->numel() < (used + 127) / 128 * 128) return fail(what, "too few bytes");
  p = t->data_ptr();
  return true;
}
struct Matrix {
  void* p;
  int64_t M, C, ld;
  at::ScalarType type;
};
// A tensor [M, C] whose rows are contiguous.
bool matrix(Matrix& m, PyObject* o, const char* what) {
  const at::Tensor* t = tensor(o, what);
  if (t == nullptr) return false;
  if (t->dim() != 2) return fail(what, "two dimensions");
  m.M = t->size(0), m.C = t->size(1), m.type = t->scalar_type(), m.p = t->data_ptr();
  if (t->stride(1) != 1 && m.C != 1 && m.M != 0) return fail(what, "rows have to be contiguous");
  m.ld = m.M > 1 ? t->stride(0) : m.C;
  return true;
}
bool matrix_like(Matrix& m, const Matrix& of, PyObject* o, const char* what) {
  if (!matrix(m, o, what)) return false;
  if (m.type != of.type) return fail(what, "of another type than it has to be");
  if (m.M != of.M || m.C != of.C) return fail(what, "of another shape than it has to be");
  return true;
}
bool workspace(void*& p, size_t& bytes, PyObject* o) {
  p = nullptr, bytes = 0;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o, "scratch");
  if (t == nullptr) return false;
  if (!t->is_contiguous()) return fail("scratch", "has to be contiguous");
  p = t->data_ptr(), bytes = (size_t)t->numel() * t->element_size();
  return true;
}
bool channels(const Matrix& m, const char* what) { return m.C <= INT32_MAX || fail(what, "too many channels"); }

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

bool count(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments, %zd are needed", n, want);
  return false;
}

PyObject* code(int e) { return PyLong_FromLong(e); }

// (x, K, ckpt)
PyObject* ckpt_pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix x;
  int K;
  void* s;
  if (!count(n, 3) || !matrix(x, a[0], "x") || !channels(x, "x") || !small(K, a[1], "K") || !store(s, a[2], x.M, x.C, K, "ckpt")) return nullptr;
  return code(abl_ckpt_pack(stream(), dtype_of(x.type), x.p, x.ld, x.M, (int32_t)x.C, K, s));
}

// (ckpt, K, x)
PyObject* ckpt_unpack(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix x;
  int K;
  void* s;
  if (!count(n, 3) || !matrix(x, a[2], "x") || !channels(x, "x") || !small(K, a[1], "K") || !store(s, a[0], x.M, x.C, K, "ckpt")) return nullptr;
  return code(abl_ckpt_unpack(stream(), dtype_of(x.type), s, x.M, (int32_t)x.C, K, x.p, x.ld));
}

// A row for each group of `rows` rows.  (Where `rows` is below one, the library says so; a gate for no rows is not looked at.)
bool gate_address(void*& p, PyObject* o, at::ScalarType type, const Matrix& of, long rows, const char* what) {
  if (rows < 1 || of.M == 0) return address(p, o, type, 0, what);
  return matrix_address(p, o, type, (of.M - 1) / rows + 1, of.C, what);
}

// (r, b, gate, gate_rows, w_post, w_pre, r_out, n, K, ckpt_b, rstd_b, ckpt_n, rstd_n, alpha, beta, eps, flags)
PyObject* resnorm_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix r;
  abl_resnorm s;
  long rows;
  int K, flags;
  void *b, *gate, *w_post, *w_pre, *r_out, *out, *sb, *rb, *sn, *rn, *rp;
  if (!count(n, 17) || !matrix(r, a[0], "r") || !channels(r, "r") || !whole(rows, a[3]) || !small(K, a[8], "K") || !number(s.alpha, a[13]) ||
      !number(s.beta, a[14]) || !number(s.eps, a[15]) || !small(flags, a[16], "flags"))
    return nullptr;
  if (!matrix_address(rp, a[0], r.type, r.M, r.C, "r") || !matrix_address(b, a[1], r.type, r.M, r.C, "b") ||
      !gate_address(gate, a[2], r.type, r, rows, "gate") || !address(w_post, a[4], r.type, r.C, "w_post") ||
      !address(w_pre, a[5], r.type, r.C, "w_pre") || !matrix_address(r_out, a[6], r.type, r.M, r.C, "r_out") ||
      !matrix_address(out, a[7], r.type, r.M, r.C, "n") ||
      !store(sb, a[9], r.M, r.C, K, "ckpt_b") || !address(rb, a[10], kF32, r.M, "rstd_b") || !store(sn, a[11], r.M, r.C, K, "ckpt_n") ||
      !address(rn, a[12], kF32, r.M, "rstd_n"))
    return nullptr;
  s.M = r.M, s.gate_rows = rows, s.C = (int32_t)r.C, s.dtype = dtype_of(r.type), s.K = K, s.flags = (uint32_t)flags;
  return code(abl_resnorm_forward(stream(), &s, rp, b, gate, w_post, w_pre, r_out, out, sb, (float*)rb, sn, (float*)rn));
}

// (dn, dr_out, gate, gate_rows, w_post, w_pre, K, ckpt_b, rstd_b, ckpt_n, rstd_n, scratch, dr, db, dgate, dw_post, dw_pre, alpha, beta, flags, has_b)
PyObject* resnorm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix d;
  abl_resnorm s;
  long rows;
  int K, flags;
  size_t bytes;
  void *dn, *dr_out, *gate, *w_post, *w_pre, *sb, *rb, *sn, *rn, *ws, *dr, *db, *dgate, *dw_post, *dw_pre;
  if (!count(n, 21) || !matrix(d, a[0], "dn") || !channels(d, "dn") || !whole(rows, a[3]) || !small(K, a[6], "K") || !number(s.alpha, a[17]) ||
      !number(s.beta, a[18]) || !small(flags, a[19], "flags"))
    return nullptr;
  const int has_b = PyObject_IsTrue(a[20]);
  if (has_b < 0 || !matrix_address(dn, a[0], d.type, d.M, d.C, "dn") || !matrix_address(dr_out, a[1], d.type, d.M, d.C, "dr_out") ||
      !gate_address(gate, a[2], d.type, d, rows, "gate") || !address(w_post, a[4], d.type, d.C, "w_post") ||
      !address(w_pre, a[5], d.type, d.C, "w_pre") || !store(sb, a[7], d.M, d.C, K, "ckpt_b") || !address(rb, a[8], kF32, d.M, "rstd_b") ||
      !store(sn, a[9], d.M, d.C, K, "ckpt_n") || !address(rn, a[10], kF32, d.M, "rstd_n") || !workspace(ws, bytes, a[11]) ||
      !matrix_address(dr, a[12], d.type, d.M, d.C, "dr") || !matrix_address(db, a[13], d.type, d.M, d.C, "db") ||
      !gate_address(dgate, a[14], kF32, d, rows, "dgate") ||
      !address(dw_post, a[15], kF32, d.C, "dw_post") || !address(dw_pre, a[16], kF32, d.C, "dw_pre"))
    return nullptr;
  s.M = d.M, s.gate_rows = rows, s.C = (int32_t)d.C, s.dtype = dtype_of(d.type), s.K = K, s.flags = (uint32_t)flags, s.eps = 0.0f;
  return code(abl_resnorm_backward(stream(), &s, has_b, dn, dr_out, gate, w_post, w_pre, sb, (float*)rb, sn, (float*)rn, ws, bytes, dr, db,
                                   (float*)dgate, (float*)dw_post, (float*)dw_pre));
}

// (g, u, h, act, K, ckpt_g, ckpt_u)
PyObject* glu_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix g, u, h;
  int act, K;
  void *sg, *su;
  if (!count(n, 7) || !matrix(g, a[0], "g") || !channels(g, "g") || !matrix_like(u, g, a[1], "u") || !matrix_like(h, g, a[2], "h") ||
      !small(act, a[3], "act") || !small(K, a[4], "K") || !store(sg, a[5], g.M, g.C, K, "ckpt_g") || !store(su, a[6], g.M, g.C, K, "ckpt_u"))
    return nullptr;
  return code(abl_glu_forward(stream(), dtype_of(g.type), act, g.p, g.ld, u.p, u.ld, g.M, (int32_t)g.C, K, h.p, h.ld, sg, su));
}

// (dh, ckpt_g, ckpt_u, K, dg, du, act, ckpt_h)
PyObject* glu_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix d, g, u;
  int act, K;
  void *sg, *su, *sh;
  if (!count(n, 8) || !matrix(d, a[0], "dh") || !channels(d, "dh") || !small(K, a[3], "K") || !store(sg, a[1], d.M, d.C, K, "ckpt_g") ||
      !store(su, a[2], d.M, d.C, K, "ckpt_u") || !matrix_like(g, d, a[4], "dg") || !matrix_like(u, d, a[5], "du") || !small(act, a[6], "act") ||
      !store(sh, a[7], d.M, d.C, 8, "ckpt_h"))
    return nullptr;
  return code(abl_glu_backward(stream(), dtype_of(d.type), act, d.p, d.ld, sg, su, d.M, (int32_t)d.C, K, g.p, g.ld, u.p, u.ld, sh));
}

// (ckpt, K, scale, dy, scratch, dW, flags)
PyObject* ckpt_wgrad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Matrix dy, w;
  int K, flags;
  size_t bytes;
  void *s, *scale, *ws, *dW;
  if (!count(n, 7) || !small(K, a[1], "K") || !matrix(dy, a[3], "dy") || !channels(dy, "dy") || !matrix(w, a[5], "dW") || !channels(w, "dW") ||
      !small(flags, a[6], "flags"))
    return nullptr;
  if (w.C != dy.C || w.M > INT32_MAX) {
    fail("dW", "as many columns as dy");
    return nullptr;
  }
  if (!address(dW, a[5], kF32, w.M * w.C, "dW") || !store(s, a[0], dy.M, w.M, K, "ckpt") || !address(scale, a[2], dy.type, w.M, "scale") ||
      !workspace(ws, bytes, a[4]))
    return nullptr;
  return code(abl_ckpt_wgrad(stream(), dtype_of(dy.type), (uint32_t)flags, s, dy.M, (int32_t)w.M, K, scale, dy.p, dy.ld, (int32_t)dy.C, ws,
                             bytes, (float*)dW));
}

// ---- losses over a vocabulary ----
// (h, W, labels, ids, logits): sizes and addresses; ids, logits are not there for the calls without a teacher.
bool whole_numbers(void*& p, PyObject* o, int64_t n, const char* what) {
  if (!address(p, o, at::kLong, n, what)) return false;
  return o == Py_None || THPVariable_Unpack(o).numel() == n || fail(what, "of another size than it has to be");
}
bool row_numbers(void*& p, PyObject* o, int64_t n, const char* what) {
  if (!address(p, o, kF32, n, what)) return false;
  return o == Py_None || THPVariable_Unpack(o).numel() == n || fail(what, "of another size than it has to be");
}
struct HeadArgs {
  abl_head p;
  Matrix h, W;
  void *labels, *ids = nullptr, *logits = nullptr;
};
// All tensors of a call lie on the device whose stream it goes to.
bool on_this_device(PyObject* const* a, Py_ssize_t n) {
  for (Py_ssize_t i = 0; i < n; ++i)
    if (THPVariable_Check(a[i]) && THPVariable_Unpack(a[i]).is_cuda() && THPVariable_Unpack(a[i]).device().index() != c10::hip::current_device())
      return fail("tensors", "on another device than the current one");
  return true;
}
bool head_operands(HeadArgs& g, PyObject* h, PyObject* W, PyObject* labels) {
  if (!matrix(g.h, h, "h") || !channels(g.h, "h") || !matrix(g.W, W, "W")) return false;
  if (g.W.type != g.h.type) return fail("W", "of another type than it has to be");
  if (g.W.C != g.h.C) return fail("W", "as many channels as h");
  if (g.W.M > INT32_MAX) return fail("W", "too many rows");
  g.p = abl_head{};
  g.p.M = g.h.M, g.p.C = (int32_t)g.h.C, g.p.V = (int32_t)g.W.M, g.p.dtype = g.p.dw_dtype = dtype_of(g.h.type);
  return whole_numbers(g.labels, labels, g.h.M, "labels");
}
bool teacher_operands(HeadArgs& g, PyObject* ids, PyObject* logits) {
  const at::Tensor* t = tensor(ids, "top_ids");
  if (t == nullptr) return false;
  if (t->dim() != 2 || t->size(0) != g.h.M || t->size(1) > INT32_MAX) return fail("top_ids", "a row of entries for each row of h");
  g.p.T = (int32_t)t->size(1);
  return whole_numbers(g.ids, ids, g.h.M * t->size(1), "top_ids") && matrix_address(g.logits, logits, kF32, g.h.M, t->size(1), "top_logits");
}
bool head_flags(HeadArgs& g, PyObject* o) {
  int flags;
  if (!small(flags, o, "flags")) return false;
  g.p.flags = (uint32_t)flags;
  return true;
}
// dh [M, C] (rows contiguous) and dW [V, C], either None.
bool head_gradients(HeadArgs& g, PyObject* dh, PyObject* dW, Matrix& d, void*& w) {
  d.p = nullptr, d.ld = g.h.C, w = nullptr;
  if (dh != Py_None && !matrix_like(d, g.h, dh, "dh")) return false;
  if (dW == Py_None) return true;
  const at::Tensor* t = tensor(dW, "dW");
  if (t == nullptr) return false;
  if (t->scalar_type() != kF32 && t->scalar_type() != g.h.type) return fail("dW", "of another type than it has to be");
  g.p.dw_dtype = dtype_of(t->scalar_type());
  return matrix_address(w, dW, t->scalar_type(), g.W.M, g.W.C, "dW");
}

// (h, W, labels, scratch, loss, lse, scale, smoothing, z_weight, flags)
PyObject* xent_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HeadArgs g;
  size_t bytes;
  void *ws, *loss, *lse;
  if (!count(n, 10) || !on_this_device(a, n) || !head_operands(g, a[0], a[1], a[2]) || !workspace(ws, bytes, a[3]) || !row_numbers(loss, a[4], g.h.M, "loss") ||
      !row_numbers(lse, a[5], g.h.M, "lse") || !number(g.p.scale, a[6]) || !number(g.p.smoothing, a[7]) || !number(g.p.z_weight, a[8]) ||
      !head_flags(g, a[9]))
    return nullptr;
  return code(abl_xent_forward(stream(), &g.p, g.h.p, g.h.ld, g.W.p, g.W.ld, (const int64_t*)g.labels, ws, bytes, (float*)loss, (float*)lse));
}

// (h, W, labels, lse, dloss, scratch, dh, dW, scale, smoothing, z_weight, flags)
PyObject* xent_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HeadArgs g;
  Matrix dh;
  size_t bytes;
  void *ws, *lse, *dloss, *dW;
  if (!count(n, 12) || !on_this_device(a, n) || !head_operands(g, a[0], a[1], a[2]) || !row_numbers(lse, a[3], g.h.M, "lse") ||
      !row_numbers(dloss, a[4], g.h.M, "dloss") || !workspace(ws, bytes, a[5]) || !head_gradients(g, a[6], a[7], dh, dW) ||
      !number(g.p.scale, a[8]) || !number(g.p.smoothing, a[9]) || !number(g.p.z_weight, a[10]) || !head_flags(g, a[11]))
    return nullptr;
  return code(abl_xent_backward(stream(), &g.p, g.h.p, g.h.ld, g.W.p, g.W.ld, (const int64_t*)g.labels, (const float*)lse, (const float*)dloss, ws,
                                bytes, dh.p, dh.ld, dW));
}

bool distill_numbers(HeadArgs& g, PyObject* const* a) {   // scale, temperature, teacher_weight, label_weight, smoothing, z_weight, flags
  return number(g.p.scale, a[0]) && number(g.p.temperature, a[1]) && number(g.p.teacher_weight, a[2]) && number(g.p.label_weight, a[3]) &&
         number(g.p.smoothing, a[4]) && number(g.p.z_weight, a[5]) && head_flags(g, a[6]);
}

// (h, W, labels, top_ids, top_logits, scratch, loss, lse, lse_t, z_top, 7 numbers)
PyObject* distill_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HeadArgs g;
  size_t bytes;
  void *ws, *loss, *lse, *lse_t, *z_top;
  if (!count(n, 17) || !on_this_device(a, n) || !head_operands(g, a[0], a[1], a[2]) || !teacher_operands(g, a[3], a[4]) || !workspace(ws, bytes, a[5]) ||
      !row_numbers(loss, a[6], g.h.M, "loss") || !row_numbers(lse, a[7], g.h.M, "lse") || !row_numbers(lse_t, a[8], g.h.M, "lse_t") ||
      !matrix_address(z_top, a[9], kF32, g.h.M, g.p.T, "z_top") || !distill_numbers(g, a + 10))
    return nullptr;
  return code(abl_distill_forward(stream(), &g.p, g.h.p, g.h.ld, g.W.p, g.W.ld, (const int64_t*)g.labels, (const int64_t*)g.ids,
                                  (const float*)g.logits, ws, bytes, (float*)loss, (float*)lse, (float*)lse_t, (float*)z_top));
}

// (h, W, labels, top_ids, top_logits, lse, lse_t, z_top, dloss, scratch, dh, dW, 7 numbers)
PyObject* distill_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HeadArgs g;
  Matrix dh;
  size_t bytes;
  void *ws, *lse, *lse_t, *z_top, *dloss, *dW;
  if (!count(n, 19) || !on_this_device(a, n) || !head_operands(g, a[0], a[1], a[2]) || !teacher_operands(g, a[3], a[4]) || !row_numbers(lse, a[5], g.h.M, "lse") ||
      !row_numbers(lse_t, a[6], g.h.M, "lse_t") || !matrix_address(z_top, a[7], kF32, g.h.M, g.p.T, "z_top") ||
      !row_numbers(dloss, a[8], g.h.M, "dloss") || !workspace(ws, bytes, a[9]) || !head_gradients(g, a[10], a[11], dh, dW) ||
      !distill_numbers(g, a + 12))
    return nullptr;
  return code(abl_distill_backward(stream(), &g.p, g.h.p, g.h.ld, g.W.p, g.W.ld, (const int64_t*)g.labels, (const int64_t*)g.ids,
                                   (const float*)g.logits, (const float*)lse, (const float*)lse_t, (const float*)z_top, (const float*)dloss, ws,
                                   bytes, dh.p, dh.ld, dW));
}

// No C++ exception may pass into the interpreter.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  try {
    return F(self, a, n);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

#define ABL_METHOD(f) {#f, (PyCFunction)(void (*)(void))guarded<f>, METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {ABL_METHOD(ckpt_pack),   ABL_METHOD(ckpt_unpack),  ABL_METHOD(resnorm_forward), ABL_METHOD(resnorm_backward),
                          ABL_METHOD(glu_forward), ABL_METHOD(glu_backward), ABL_METHOD(ckpt_wgrad),      ABL_METHOD(xent_forward),
                          ABL_METHOD(xent_backward), ABL_METHOD(distill_forward), ABL_METHOD(distill_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_rows", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rows(void) { return PyModule_Create(&kModule); }
