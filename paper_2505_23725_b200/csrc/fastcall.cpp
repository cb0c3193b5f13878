// The operators' calls without the interpreter: argument checks, result tensors and the argument structs of the calls
// that binding.py makes, for the common case -- every argument as it should be and the caller on the
// context's own stream.  For anything else a function returns None without having done anything, and binding.py goes
// its own way, which says what is wrong or bridges the streams.  At one token the interpreter's part of a call
// costs two to four times the kernel: norm with rotation 12 us a call without this file.
//
// A function gets (context or AdamW list, library function, device, stream) as integers, then its arguments; it returns the results, None,
// or the library's status when that is an error.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/muloco.h"

namespace {

struct Call {
  muloco_ctx* ctx;                 // (or the AdamW list)
  void* fn;
  int64_t dev;
  bool ok;
};

Call call_of(PyObject* const* a) {
  Call c;
  c.ctx = reinterpret_cast<muloco_ctx*>(PyLong_AsVoidPtr(a[0]));
  c.fn = PyLong_AsVoidPtr(a[1]);
  c.dev = PyLong_AsLongLong(a[2]);
  const void* stream = PyLong_AsVoidPtr(a[3]);
  c.ok = c.ctx && c.fn && !PyErr_Occurred() &&
         c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)c.dev).stream() == (cudaStream_t)stream;
  if (PyErr_Occurred()) PyErr_Clear();
  return c;
}

// The tensor behind an argument (nullptr for None); *ok becomes false when it is neither.
const at::Tensor* tensor(PyObject* o, bool* ok) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) { *ok = false; return nullptr; }
  return &THPVariable_Unpack(o);
}

bool is(const at::Tensor& t, const Call& c, at::ScalarType type, int64_t dims) {
  return t.is_cuda() && t.get_device() == c.dev && t.scalar_type() == type && t.dim() == dims;
}
bool dense_vector(const at::Tensor& t, const Call& c, at::ScalarType type, int64_t n) {
  return is(t, c, type, 1) && t.size(0) == n && (n < 2 || t.stride(0) == 1);
}
void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

// Calls the library without the interpreter's lock: a launch waits when the queue is full, for a GPU that may be waiting for a Python
// callback.
template <typename F> int unlocked(F call) {
  PyThreadState* const state = PyEval_SaveThread();
  const int status = call();
  PyEval_RestoreThread(state);
  return status;
}

PyObject* none() { Py_RETURN_NONE; }
PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* wrap_or_none(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : none(); }

// q, k, cos, sin, positions, gain_q, gain_k, eps, interleaved
struct Qk {
  muloco_qk_norm a;
  const at::Tensor* q;
  const at::Tensor* k;
  const at::Tensor* some;
};

bool qk_of(PyObject* const* o, const Call& c, Qk* r) {
  bool ok = true;
  r->q = tensor(o[0], &ok);
  r->k = tensor(o[1], &ok);
  const at::Tensor* cs = tensor(o[2], &ok);
  const at::Tensor* sn = tensor(o[3], &ok);
  const at::Tensor* pos = tensor(o[4], &ok);
  const at::Tensor* gq = tensor(o[5], &ok);
  const at::Tensor* gk = tensor(o[6], &ok);
  const double eps = PyFloat_AsDouble(o[7]);
  const int il = PyObject_IsTrue(o[8]);
  if (PyErr_Occurred() || il < 0) { PyErr_Clear(); return false; }
  r->some = r->q ? r->q : r->k;
  if (!ok || !r->some || !cs || !sn) return false;
  const at::ScalarType type = r->some->scalar_type();
  if (type != at::kFloat && type != at::kBFloat16) return false;
  if (r->some->dim() != 3) return false;
  const int64_t T = r->some->size(0), D = r->some->size(2);
  if (!is(*cs, c, at::kFloat, 2) || !is(*sn, c, at::kFloat, 2) || cs->sizes() != sn->sizes() || !cs->is_contiguous() || !sn->is_contiguous())
    return false;
  muloco_qk_norm& a = r->a;
  a = muloco_qk_norm();
  a.tokens = T; a.head_dim = (int32_t)D;
  a.table_len = cs->size(0); a.rotary_dim = (int32_t)(2 * cs->size(1));
  a.dtype = type == at::kFloat ? MULOCO_F32 : MULOCO_BF16;
  a.interleaved = il; a.eps = (float)eps;
  for (int w = 0; w < 2; ++w) {
    const at::Tensor* t = w ? r->k : r->q;
    const at::Tensor* g = w ? gk : gq;
    if (g && !dense_vector(*g, c, at::kFloat, D)) return false;
    if (!t) continue;
    if (!is(*t, c, type, 3) || t->size(0) != T || t->size(2) != D || t->stride(2) != 1) return false;
    (w ? a.heads_k : a.heads_q) = (int32_t)t->size(1);
    (w ? a.k_token_stride : a.q_token_stride) = t->stride(0);
    (w ? a.k_head_stride : a.q_head_stride) = t->stride(1);
  }
  if (pos && !dense_vector(*pos, c, at::kLong, T)) return false;
  a.gain_q = (const float*)ptr(gq); a.gain_k = (const float*)ptr(gk);
  a.cos = (const float*)cs->data_ptr(); a.sin = (const float*)sn->data_ptr();
  a.positions = (const int64_t*)ptr(pos);
  a.q = ptr(r->q); a.k = ptr(r->k);
  return true;
}

PyObject* qk_forward(PyObject*, PyObject* const* o, Py_ssize_t n) {
  if (n != 13) return none();
  const Call c = call_of(o);
  Qk r;
  if (!c.ok || !qk_of(o + 4, c, &r)) return none();
  at::Tensor qo, ko;
  int64_t s[2][2] = {{0, 0}, {0, 0}};
  if (r.q) { qo = at::empty_like(*r.q); s[0][0] = qo.stride(0); s[0][1] = qo.stride(1); }
  if (r.k) { ko = at::empty_like(*r.k); s[1][0] = ko.stride(0); s[1][1] = ko.stride(1); }
  const auto fn = (decltype(&muloco_qk_norm_rope))c.fn;
  const int st = unlocked([&] { return fn(c.ctx, &r.a, r.q ? qo.data_ptr() : nullptr, s[0][0], s[0][1], r.k ? ko.data_ptr() : nullptr, s[1][0], s[1][1]); });
  if (st) return PyLong_FromLong(st);
  return Py_BuildValue("(NN)", wrap_or_none(qo), wrap_or_none(ko));
}

PyObject* qk_backward(PyObject*, PyObject* const* o, Py_ssize_t n) {
  if (n != 15) return none();
  const Call c = call_of(o);
  Qk r;
  if (!c.ok || !qk_of(o + 6, c, &r)) return none();
  bool ok = true;
  const at::Tensor* dy[2] = {tensor(o[4], &ok), tensor(o[5], &ok)};
  const at::Tensor* x[2] = {r.q, r.k};
  at::Tensor dx[2], dg[2];
  int64_t s[2][2] = {{0, 0}, {0, 0}};
  for (int w = 0; w < 2; ++w) {
    if (!ok || (dy[w] != nullptr) != (x[w] != nullptr)) return none();
    if (!x[w]) continue;
    if (!is(*dy[w], c, x[w]->scalar_type(), 3) || dy[w]->sizes() != x[w]->sizes() || dy[w]->stride(2) != 1) return none();
    s[w][0] = dy[w]->stride(0); s[w][1] = dy[w]->stride(1);
  }
  for (int w = 0; w < 2; ++w) {
    if (!x[w]) continue;
    dx[w] = at::empty(x[w]->sizes(), x[w]->options());
    dg[w] = at::empty({x[w]->size(2)}, x[w]->options().dtype(at::kFloat));
  }
  auto p = [](const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; };
  const auto fn = (decltype(&muloco_qk_norm_rope_backward))c.fn;
  const int st = unlocked([&] { return fn(c.ctx, &r.a, ptr(dy[0]), s[0][0], s[0][1], ptr(dy[1]), s[1][0], s[1][1], p(dx[0]), p(dx[1]),
                    (float*)p(dg[0]), (float*)p(dg[1])); });
  if (st) return PyLong_FromLong(st);
  return Py_BuildValue("(NNNN)", wrap_or_none(dx[0]), wrap_or_none(dx[1]), wrap_or_none(dg[0]), wrap_or_none(dg[1]));
}

// x, w1, w3, w2, activation number
bool ffn_of(PyObject* const* o, const Call& c, muloco_ffn* a, const at::Tensor** x) {
  bool ok = true;
  const at::Tensor* t[4];
  for (int i = 0; i < 4; ++i) {
    t[i] = tensor(o[i], &ok);
    if (!ok || !t[i] || !is(*t[i], c, at::kBFloat16, 2) || t[i]->stride(1) != 1) return false;
  }
  const long act = PyLong_AsLong(o[4]);
  if (PyErr_Occurred()) { PyErr_Clear(); return false; }
  if (act < 0) return false;
  *a = muloco_ffn();
  const int64_t T = t[0]->size(0), d = t[0]->size(1), F = t[1]->size(1);
  if (t[1]->size(0) != d || t[2]->size(0) != d || t[2]->size(1) != F || t[3]->size(0) != F || t[3]->size(1) != d) return false;
  a->tokens = T; a->d = d; a->F = F;
  a->ldx = T > 1 ? t[0]->stride(0) : d;
  a->ldw1 = t[1]->stride(0); a->ldw3 = t[2]->stride(0); a->ldw2 = t[3]->stride(0);
  a->x = t[0]->data_ptr(); a->w1 = t[1]->data_ptr(); a->w3 = t[2]->data_ptr(); a->w2 = t[3]->data_ptr();
  a->activation = (int32_t)act;
  *x = t[0];
  return true;
}

PyObject* ffn_forward(PyObject*, PyObject* const* o, Py_ssize_t n) {
  if (n != 10) return none();
  const Call c = call_of(o);
  muloco_ffn a;
  const at::Tensor* x;
  const int save = PyObject_IsTrue(o[9]);
  if (save < 0) { PyErr_Clear(); return none(); }
  if (!c.ok || !ffn_of(o + 4, c, &a, &x)) return none();
  at::Tensor y = at::empty({a.tokens, a.d}, x->options()), h = at::empty({a.tokens, a.F}, x->options()), g, u;
  if (save) {
    g = at::empty({a.tokens, a.F}, x->options());
    u = at::empty({a.tokens, a.F}, x->options());
  }
  const auto fn = (decltype(&muloco_gated_ffn))c.fn;
  const int st = unlocked([&] { return fn(c.ctx, &a, save ? g.data_ptr() : nullptr, save ? u.data_ptr() : nullptr, h.data_ptr(), y.data_ptr()); });
  if (st) return PyLong_FromLong(st);
  if (!save) return Py_BuildValue("(NO)", wrap(y), Py_None);
  return Py_BuildValue("(N(NNN))", wrap(y), wrap(g), wrap(u), wrap(h));
}

// dy, x, w1, w3, w2, activation number, g, u, h
PyObject* ffn_backward(PyObject*, PyObject* const* o, Py_ssize_t n) {
  if (n != 13) return none();
  const Call c = call_of(o);
  muloco_ffn a;
  const at::Tensor* x;
  if (!c.ok || !ffn_of(o + 5, c, &a, &x)) return none();
  bool ok = true;
  const at::Tensor* dy = tensor(o[4], &ok);
  if (!ok || !dy || !is(*dy, c, at::kBFloat16, 2) || dy->size(0) != a.tokens || dy->size(1) != a.d || dy->stride(1) != 1) return none();
  const at::Tensor* s[3];
  for (int i = 0; i < 3; ++i) {
    s[i] = tensor(o[10 + i], &ok);
    if (!ok || !s[i] || !is(*s[i], c, at::kBFloat16, 2) || s[i]->size(0) != a.tokens || s[i]->size(1) != a.F || !s[i]->is_contiguous())
      return none();
  }
  const auto opt = x->options();
  // dG and dU are scratch: one allocation (each a multiple of 16 bytes)
  at::Tensor scratch = at::empty({2, a.tokens, a.F}, opt), dx = at::empty({a.tokens, a.d}, opt),
             dw1 = at::empty({a.d, a.F}, opt), dw3 = at::empty({a.d, a.F}, opt), dw2 = at::empty({a.F, a.d}, opt);
  const auto fn = (decltype(&muloco_gated_ffn_backward))c.fn;
  const int st = unlocked([&] { return fn(c.ctx, &a, dy->data_ptr(), a.tokens > 1 ? dy->stride(0) : a.d, s[0]->data_ptr(), s[1]->data_ptr(), s[2]->data_ptr(),
                    scratch.data_ptr(), static_cast<char*>(scratch.data_ptr()) + a.tokens * a.F * 2, dx.data_ptr(), dw1.data_ptr(), dw3.data_ptr(), dw2.data_ptr()); });
  if (st) return PyLong_FromLong(st);
  return Py_BuildValue("(NNNN)", wrap(dx), wrap(dw1), wrap(dw3), wrap(dw2));
}

// (list, library function, device, stream), step number, learning-rate scale: a step with the gradients named at construction
PyObject* adamw_step(PyObject*, PyObject* const* o, Py_ssize_t n) {
  if (n != 6) return none();
  const Call c = call_of(o);
  const long long step = PyLong_AsLongLong(o[4]);
  const double scale = PyFloat_AsDouble(o[5]);
  if (PyErr_Occurred()) { PyErr_Clear(); return none(); }
  if (!c.ok) return none();
  return PyLong_FromLong(unlocked([&] {
    return ((decltype(&muloco_adamw_step))c.fn)(reinterpret_cast<muloco_adamw*>(c.ctx), nullptr, step, (float)scale);
  }));
}

// (list, library function, device, stream), a float32 tensor to make the results like, their length
PyObject* adamw_moments(PyObject*, PyObject* const* o, Py_ssize_t n) {
  if (n != 6) return none();
  const Call c = call_of(o);
  bool ok = c.ok;
  const at::Tensor* like = tensor(o[4], &ok);
  const long long len = PyLong_AsLongLong(o[5]);
  if (PyErr_Occurred()) { PyErr_Clear(); return none(); }
  if (!ok || !like) return none();
  at::Tensor m = at::empty({len}, like->options()), v = at::empty({len}, like->options());
  const int st = unlocked([&] { return ((decltype(&muloco_adamw_moments))c.fn)(reinterpret_cast<muloco_adamw*>(c.ctx), (float*)m.data_ptr(), (float*)v.data_ptr()); });
  if (st) return PyLong_FromLong(st);
  return Py_BuildValue("(NN)", wrap(m), wrap(v));
}

// No C++ exception (an allocation that fails, above all) leaves a function: it becomes a Python one.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* o, Py_ssize_t n) {
  try {
    return F(self, o, n);
  } catch (const c10::OutOfMemoryError& e) {
    PyObject* torch = PyImport_ImportModule("torch");
    PyObject* type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
    PyErr_Clear();
    PyErr_SetString(type ? type : PyExc_MemoryError, e.what_without_backtrace());
    Py_XDECREF(type);
    Py_XDECREF(torch);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

#define FAST(name, f, doc) {name, (PyCFunction)(void (*)(void))guarded<f>, METH_FASTCALL, doc}
PyMethodDef methods[] = {
    FAST("qk_norm_rope", qk_forward, "muloco_qk_norm_rope"),
    FAST("qk_norm_rope_backward", qk_backward, "muloco_qk_norm_rope_backward"),
    FAST("gated_ffn", ffn_forward, "muloco_gated_ffn"),
    FAST("gated_ffn_backward", ffn_backward, "muloco_gated_ffn_backward"),
    FAST("adamw_step", adamw_step, "muloco_adamw_step"),
    FAST("adamw_moments", adamw_moments, "muloco_adamw_moments"),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// TORCH: the version whose headers this file was compiled with; binding.py uses the module with no other.
PyMODINIT_FUNC PyInit__fastcall(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "TORCH", MULOCO_TORCH) < 0) { Py_DECREF(m); return nullptr; }
  return m;
}
