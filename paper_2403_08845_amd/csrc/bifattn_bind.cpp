// Argument checks and calls of the per-step entry points for the Python
// binding (module _bifattn_bind).
//
// A decode step of a small layer is bound by the host: checking its tensors
// attribute by attribute in Python takes 6.5 us and the whole call 10.3 us,
// where the GPU needs 4.9 us for it. Caller makes the same checks on the
// tensor objects themselves (well under 1 us).
//
// A method returns the library's status, or None when it does not take the
// call: any tensor that is not exactly what the plan expects, and any tensor
// that is not an ordinary one (a subclass with its own dispatch, a wrapped or
// non-strided tensor). The binding then goes through its Python checks, which
// raise the specific error or make the call themselves, so what is accepted
// and what is refused does not depend on this file.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <cstdint>

#include "bifattn.h"

namespace {

typedef bifattn_status_t (*decode_fn)(bifattn_plan_t, const void*, const void*, const void*,
                                      const void*, const void*, const int32_t*, const float*,
                                      const float*, float*, hipStream_t);
typedef bifattn_status_t (*append_fn)(bifattn_plan_t, const void*, const void*, void*, void*,
                                      int32_t*, hipStream_t);

struct Caller {
  PyObject_HEAD
  decode_fn decode;
  append_fn append;
  bifattn_plan_t plan;
  PyObject* current_stream;  // callable: device index -> raw stream of the calling thread
  PyObject* device_obj;      // the plan's device index as a Python int
  int device;
  int64_t b, h, g, d, m_c, m_d, n;
  int kv;
};

// The tensor's implementation, or null when this file does not take it.
const at::Tensor* plain(PyObject* o, int device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device)
    return nullptr;
  const c10::DispatchKeySet keys = t.key_set();
  if (keys.has_any(c10::python_ks) || keys.has(c10::DispatchKey::FuncTorchBatched) ||
      keys.has(c10::DispatchKey::FuncTorchGradWrapper) ||
      keys.has(c10::DispatchKey::Functionalize) || !t.has_storage())
    return nullptr;
  return &t;
}

bool shaped(const at::Tensor& t, std::initializer_list<int64_t> shape) {
  return t.sizes().equals(c10::IntArrayRef(shape.begin(), shape.size())) && t.is_contiguous();
}

// Device pointer of a tensor of this dtype and shape in *ptr.
bool take(PyObject* o, const Caller* C, at::ScalarType type, std::initializer_list<int64_t> shape,
          void** ptr) {
  const at::Tensor* t = plain(o, C->device);
  if (!t || t->scalar_type() != type || !shaped(*t, shape)) return false;
  *ptr = t->data_ptr();
  return true;
}

bool take_cache(PyObject* o, const Caller* C, std::initializer_list<int64_t> shape, void** ptr) {
  const at::Tensor* t = plain(o, C->device);
  if (!t || !shaped(*t, shape)) return false;
  const at::ScalarType s = t->scalar_type();
  const bool byte = s == at::kByte || s == at::kChar;
  const bool ok = C->kv == BIFATTN_KV_BF16   ? s == at::kBFloat16
                  : C->kv == BIFATTN_KV_INT4 ? byte
                                             : byte || s == at::kFloat8_e4m3fn;
  if (!ok) return false;
  *ptr = t->data_ptr();
  return true;
}

bool take_scale(PyObject* o, const Caller* C, void** ptr) {
  *ptr = nullptr;
  return o == Py_None || take(o, C, at::kFloat, {C->g}, ptr);
}

// The stream argument: None for the current stream of the plan's device, or
// a raw stream as a Python int. False with no Python error set otherwise.
bool take_stream(PyObject* o, const Caller* C, hipStream_t* stream) {
  PyObject* raw = o;
  if (o == Py_None) {
    raw = PyObject_CallOneArg(C->current_stream, C->device_obj);
    if (!raw) {
      PyErr_Clear();
      return false;
    }
  } else if (!PyLong_CheckExact(o)) {
    return false;
  }
  void* p = PyLong_AsVoidPtr(raw);
  if (raw != o) Py_DECREF(raw);
  if (!p && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  *stream = static_cast<hipStream_t>(p);
  return true;
}

int64_t cols(const Caller* C) { return C->kv == BIFATTN_KV_INT4 ? C->d / 2 : C->d; }

// decode(q, Kc, Vc, Kd, Vd, decode_lens, k_scale, v_scale, out, stream)
PyObject* caller_decode(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  const Caller* C = reinterpret_cast<const Caller*>(self);
  if (nargs != 10) {
    PyErr_SetString(PyExc_TypeError, "decode takes 10 arguments");
    return nullptr;
  }
  void *q, *Kc, *Vc, *Kd, *Vd, *lens, *ks, *vs, *out;
  hipStream_t stream = nullptr;
  try {
    const int64_t w = cols(C);
    const bool flat = C->n == 1 && THPVariable_CheckExact(a[0]) && THPVariable_Unpack(a[0]).dim() == 3;
    const bool qo = flat ? take(a[0], C, at::kBFloat16, {C->b, C->h, C->d}, &q) &&
                               take(a[8], C, at::kFloat, {C->b, C->h, C->d}, &out)
                         : take(a[0], C, at::kBFloat16, {C->b, C->h, C->n, C->d}, &q) &&
                               take(a[8], C, at::kFloat, {C->b, C->h, C->n, C->d}, &out);
    if (!qo || !take_cache(a[1], C, {C->g, C->m_c, w}, &Kc) ||
        !take_cache(a[2], C, {C->g, C->m_c, w}, &Vc) ||
        !take_cache(a[3], C, {C->b, C->g, C->m_d, w}, &Kd) ||
        !take_cache(a[4], C, {C->b, C->g, C->m_d, w}, &Vd) ||
        !take(a[5], C, at::kInt, {C->b}, &lens) || !take_scale(a[6], C, &ks) ||
        !take_scale(a[7], C, &vs) || !take_stream(a[9], C, &stream))
      Py_RETURN_NONE;
  } catch (...) {  // nothing C++ throws passes into the interpreter
    Py_RETURN_NONE;
  }
  bifattn_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = C->decode(C->plan, q, Kc, Vc, Kd, Vd, static_cast<const int32_t*>(lens),
                 static_cast<const float*>(ks), static_cast<const float*>(vs),
                 static_cast<float*>(out), stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// append(k_new, v_new, Kd, Vd, decode_lens, stream)
PyObject* caller_append(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  const Caller* C = reinterpret_cast<const Caller*>(self);
  if (nargs != 6) {
    PyErr_SetString(PyExc_TypeError, "append takes 6 arguments");
    return nullptr;
  }
  void *k, *v, *Kd, *Vd, *lens;
  hipStream_t stream = nullptr;
  try {
    const int64_t w = cols(C);
    if (!take_cache(a[0], C, {C->b, C->g, C->n, w}, &k) ||
        !take_cache(a[1], C, {C->b, C->g, C->n, w}, &v) ||
        !take_cache(a[2], C, {C->b, C->g, C->m_d, w}, &Kd) ||
        !take_cache(a[3], C, {C->b, C->g, C->m_d, w}, &Vd) ||
        !take(a[4], C, at::kInt, {C->b}, &lens) || !take_stream(a[5], C, &stream))
      Py_RETURN_NONE;
  } catch (...) {
    Py_RETURN_NONE;
  }
  bifattn_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = C->append(C->plan, k, v, Kd, Vd, static_cast<int32_t*>(lens), stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// Caller(decode, append, plan, current_stream, device, b, h, g, d, m_c, m_d, n, kv):
// the entry points and the plan as addresses.
PyObject* caller_new(PyTypeObject* type, PyObject* args, PyObject*) {
  unsigned long long decode, append, plan;
  PyObject* cs;
  int device, kv;
  long long b, h, g, d, m_c, m_d, n;
  if (!PyArg_ParseTuple(args, "KKKOiLLLLLLLi", &decode, &append, &plan, &cs, &device, &b, &h, &g,
                        &d, &m_c, &m_d, &n, &kv))
    return nullptr;
  Caller* C = reinterpret_cast<Caller*>(type->tp_alloc(type, 0));
  if (!C) return nullptr;
  C->device_obj = PyLong_FromLong(device);
  if (!C->device_obj) {
    Py_DECREF(C);
    return nullptr;
  }
  Py_INCREF(cs);
  C->current_stream = cs;
  C->decode = reinterpret_cast<decode_fn>(static_cast<uintptr_t>(decode));
  C->append = reinterpret_cast<append_fn>(static_cast<uintptr_t>(append));
  C->plan = reinterpret_cast<bifattn_plan_t>(static_cast<uintptr_t>(plan));
  C->device = device;
  C->b = b, C->h = h, C->g = g, C->d = d, C->m_c = m_c, C->m_d = m_d, C->n = n;
  C->kv = kv;
  return reinterpret_cast<PyObject*>(C);
}

void caller_dealloc(PyObject* self) {
  Caller* C = reinterpret_cast<Caller*>(self);
  Py_XDECREF(C->current_stream);
  Py_XDECREF(C->device_obj);
  Py_TYPE(self)->tp_free(self);
}

// --- paged caches -----------------------------------------------------------

typedef bifattn_status_t (*paged_append_fn)(bifattn_paged_plan_t, const bifattn_pages_t*, const int32_t*,
                                            const bifattn_new_rows_t*, const int32_t*, int32_t*, hipStream_t);
typedef bifattn_status_t (*paged_gather_fn)(bifattn_paged_plan_t, const bifattn_pages_t*, const int32_t*,
                                            const int32_t*, const int32_t*, int32_t, int32_t, int32_t, void*,
                                            void*, hipStream_t);
typedef bifattn_status_t (*paged_decode_fn)(bifattn_paged_plan_t, const void*, const bifattn_pages_t*,
                                            const int32_t*, const int32_t*, const int32_t*, void*, hipStream_t);
typedef bifattn_status_t (*paged_diff_fn)(bifattn_paged_plan_t, const void*, const bifattn_pages_t*,
                                          const int32_t*, const int32_t*, const int32_t*, const float*,
                                          const float*, float, float, void*, hipStream_t);

struct PagedCaller {
  Caller base;  // plan, device, stream getter, b, h, g, d, m_c, m_d, n, kv
  paged_append_fn append;
  paged_gather_fn gather;
  paged_decode_fn decode;
  paged_diff_fn diff;
  int64_t page, num_pages;
  PyObject* pages_type;  // the binding's Pages
};

bool optional(PyObject* o, const Caller* C, at::ScalarType type, std::initializer_list<int64_t> shape,
              const void** ptr) {
  void* p = nullptr;
  const bool ok = o == Py_None || take(o, C, type, shape, &p);
  *ptr = p;
  return ok;
}

// The six tensors of a Pages tuple.
bool take_pages(PyObject* o, const PagedCaller* P, bifattn_pages_t* out) {
  const Caller* C = &P->base;
  if ((PyObject*)Py_TYPE(o) != P->pages_type || !PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 6) return false;
  const bool mx = C->kv == BIFATTN_KV_MXFP4, fp8 = C->kv == BIFATTN_KV_FP8_E4M3;
  const int64_t cols = mx ? C->d / 2 : C->d;
  void** rows[2] = {&out->K, &out->V};
  for (int k = 0; k < 2; ++k) {
    const at::Tensor* t = plain(PyTuple_GET_ITEM(o, k), C->device);
    if (!t || !shaped(*t, {P->num_pages, C->g, P->page, cols})) return false;
    const at::ScalarType s = t->scalar_type();
    const bool byte = s == at::kByte || s == at::kChar;
    if (!(mx ? byte : fp8 ? byte || s == at::kFloat8_e4m3fn : s == at::kBFloat16)) return false;
    *rows[k] = t->data_ptr();
  }
  const void* p[4];
  for (int k = 0; k < 4; ++k) {
    PyObject* x = PyTuple_GET_ITEM(o, 2 + k);
    if (k < 2 ? (x == Py_None) == mx : x != Py_None && !fp8) return false;
    if (!(k < 2 ? optional(x, C, at::kByte, {P->num_pages, C->g, P->page, C->d / 32}, &p[k])
                : optional(x, C, at::kFloat, {C->g}, &p[k])))
      return false;
  }
  out->K_exp = static_cast<uint8_t*>(const_cast<void*>(p[0]));
  out->V_exp = static_cast<uint8_t*>(const_cast<void*>(p[1]));
  out->k_scale = static_cast<const float*>(p[2]);
  out->v_scale = static_cast<const float*>(p[3]);
  return true;
}

int64_t pages_of(const PagedCaller* P, bool context) {
  const int64_t rows = context ? P->base.m_c : P->base.m_d;
  return (rows + P->page - 1) / P->page;
}

// A table of page ids: [samples, pages], or [pages] too for the context's one sequence.
bool take_table(PyObject* o, const PagedCaller* P, int64_t samples, bool context, void** ptr) {
  const int64_t pages = pages_of(P, context);
  return (context && samples == 1 && take(o, &P->base, at::kInt, {pages}, ptr)) ||
         take(o, &P->base, at::kInt, {samples, pages}, ptr);
}

// The tensors that both attention calls take: q, pages, ctx_table, tables, lens, out.
struct AttentionArgs {
  void *q, *out, *ctx = nullptr, *tables = nullptr, *lens = nullptr;
  bifattn_pages_t pages;
};
bool take_attention(PyObject* const* a, PyObject* out, const PagedCaller* P, AttentionArgs* r) {
  const Caller* C = &P->base;
  const bool flat = C->n == 1 && THPVariable_CheckExact(a[0]) && THPVariable_Unpack(a[0]).dim() == 3;
  if (flat) {
    if (!take(a[0], C, at::kBFloat16, {C->b, C->h, C->d}, &r->q) ||
        !take(out, C, at::kBFloat16, {C->b, C->h, C->d}, &r->out))
      return false;
  } else if (!take(a[0], C, at::kBFloat16, {C->b, C->h, C->n, C->d}, &r->q) ||
             !take(out, C, at::kBFloat16, {C->b, C->h, C->n, C->d}, &r->out)) {
    return false;
  }
  if (!take_pages(a[1], P, &r->pages)) return false;
  if (C->m_c > 0 && !take_table(a[2], P, 1, true, &r->ctx)) return false;
  return C->m_d == 0 || (take_table(a[3], P, C->b, false, &r->tables) &&
                         take(a[4], C, at::kInt, {C->b}, &r->lens));
}

// decode(q, pages, ctx_table, tables, lens, out, stream)
PyObject* paged_decode(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  const PagedCaller* P = reinterpret_cast<const PagedCaller*>(self);
  if (nargs != 7) {
    PyErr_SetString(PyExc_TypeError, "decode takes 7 arguments");
    return nullptr;
  }
  AttentionArgs r;
  hipStream_t stream = nullptr;
  try {
    if (!take_attention(a, a[5], P, &r) || !take_stream(a[6], &P->base, &stream)) Py_RETURN_NONE;
  } catch (...) {
    Py_RETURN_NONE;
  }
  bifattn_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = P->decode(reinterpret_cast<bifattn_paged_plan_t>(P->base.plan), r.q, &r.pages,
                 static_cast<const int32_t*>(r.ctx), static_cast<const int32_t*>(r.tables),
                 static_cast<const int32_t*>(r.lens), r.out, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// diff(q, pages, ctx_table, tables, lens, out, lam, weight, eps, out_scale, stream)
PyObject* paged_diff(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  const PagedCaller* P = reinterpret_cast<const PagedCaller*>(self);
  if (nargs != 11) {
    PyErr_SetString(PyExc_TypeError, "diff takes 11 arguments");
    return nullptr;
  }
  AttentionArgs r;
  hipStream_t stream = nullptr;
  const Caller* C = &P->base;
  void* lam;
  const void* weight;
  if (!PyFloat_CheckExact(a[8]) || !PyFloat_CheckExact(a[9])) Py_RETURN_NONE;
  const float eps = (float)PyFloat_AS_DOUBLE(a[8]), scale = (float)PyFloat_AS_DOUBLE(a[9]);
  try {
    if (!take_attention(a, a[5], P, &r) || !take(a[6], C, at::kFloat, {C->h}, &lam) ||
        !optional(a[7], C, at::kFloat, {C->d}, &weight) || !take_stream(a[10], C, &stream))
      Py_RETURN_NONE;
  } catch (...) {
    Py_RETURN_NONE;
  }
  bifattn_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = P->diff(reinterpret_cast<bifattn_paged_plan_t>(C->plan), r.q, &r.pages, static_cast<const int32_t*>(r.ctx),
               static_cast<const int32_t*>(r.tables), static_cast<const int32_t*>(r.lens),
               static_cast<const float*>(lam), static_cast<const float*>(weight), eps, scale, r.out, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// New rows [s, heads, n, d] of bf16, any strides whose rows are consecutive.
bool take_rows(PyObject* o, const Caller* C, int64_t s, int64_t heads, int64_t n, const void** ptr, int64_t* stride) {
  const at::Tensor* t = plain(o, C->device);
  if (!t || t->scalar_type() != at::kBFloat16 || t->dim() != 4 || t->size(0) != s || t->size(1) != heads ||
      t->size(2) != n || t->size(3) != C->d || t->stride(3) != 1 || t->is_neg())
    return false;
  for (int k = 0; k < 3; ++k) stride[k] = t->size(k) > 1 ? t->stride(k) : 0;
  *ptr = t->data_ptr();
  return true;
}

// append(pages, table, lens, k, v, lens_out, q, q_out, counts, freqs, neighbours, context, stream)
PyObject* paged_append(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  const PagedCaller* P = reinterpret_cast<const PagedCaller*>(self);
  if (nargs != 13) {
    PyErr_SetString(PyExc_TypeError, "append takes 13 arguments");
    return nullptr;
  }
  const Caller* C = &P->base;
  bifattn_pages_t pages;
  bifattn_new_rows_t r{};
  void *table, *lens, *lens_out;
  hipStream_t stream = nullptr;
  if (!PyBool_Check(a[10]) || !PyBool_Check(a[11])) Py_RETURN_NONE;
  try {
    const at::Tensor* k = plain(a[3], C->device);
    if (!k || k->dim() != 4 || k->size(0) > INT32_MAX || k->size(2) > INT32_MAX) Py_RETURN_NONE;
    const int64_t s = k->size(0), n = k->size(2);
    r.samples = (int32_t)s;
    r.n = (int32_t)n;
    r.neighbours = a[10] == Py_True;
    r.context = a[11] == Py_True;
    const void* p;
    if (!take_rows(a[3], C, s, C->g, n, &r.k, r.k_stride) || !take_rows(a[4], C, s, C->g, n, &r.v, r.v_stride))
      Py_RETURN_NONE;
    if ((a[6] == Py_None) != (a[7] == Py_None)) Py_RETURN_NONE;
    if (a[6] != Py_None && (!take_rows(a[6], C, s, C->h, n, &r.q, r.q_stride) ||
                            !take(a[7], C, at::kBFloat16, {s, C->h, n, C->d}, &r.q_out)))
      Py_RETURN_NONE;
    if (!optional(a[8], C, at::kInt, {s}, &p)) Py_RETURN_NONE;
    r.counts = static_cast<const int32_t*>(p);
    if (a[9] != Py_None) {
      const at::Tensor* f = plain(a[9], C->device);
      if (!f || f->dim() != 1 || f->size(0) > C->d || !optional(a[9], C, at::kFloat, {f->size(0)}, &p)) Py_RETURN_NONE;
      r.freqs = static_cast<const float*>(p);
      r.rot = (int32_t)(2 * f->size(0));
    }
    if (!take_pages(a[0], P, &pages) || !take_table(a[1], P, s, r.context, &table) ||
        !take(a[2], C, at::kInt, {s}, &lens) || !take(a[5], C, at::kInt, {s}, &lens_out) ||
        !take_stream(a[12], C, &stream))
      Py_RETURN_NONE;
  } catch (...) {
    Py_RETURN_NONE;
  }
  bifattn_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = P->append(reinterpret_cast<bifattn_paged_plan_t>(C->plan), &pages, static_cast<const int32_t*>(table), &r,
                 static_cast<const int32_t*>(lens), static_cast<int32_t*>(lens_out), stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// gather(pages, table, lens, k_out, v_out, first, context, stream)
PyObject* paged_gather(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  const PagedCaller* P = reinterpret_cast<const PagedCaller*>(self);
  if (nargs != 8) {
    PyErr_SetString(PyExc_TypeError, "gather takes 8 arguments");
    return nullptr;
  }
  const Caller* C = &P->base;
  bifattn_pages_t pages;
  void *table, *lens, *k_out, *v_out;
  const void* first;
  int64_t s, rows;
  hipStream_t stream = nullptr;
  if (!PyBool_Check(a[6])) Py_RETURN_NONE;
  const bool context = a[6] == Py_True;
  try {
    const at::Tensor* k = plain(a[3], C->device);
    if (!k || k->dim() != 4 || k->size(0) > INT32_MAX || k->size(2) > INT32_MAX) Py_RETURN_NONE;
    s = k->size(0), rows = k->size(2);
    if (!take(a[3], C, at::kBFloat16, {s, C->g, rows, C->d}, &k_out) ||
        !take(a[4], C, at::kBFloat16, {s, C->g, rows, C->d}, &v_out) || !take_pages(a[0], P, &pages) ||
        !take_table(a[1], P, s, context, &table) || !take(a[2], C, at::kInt, {s}, &lens) ||
        !optional(a[5], C, at::kInt, {s}, &first) || !take_stream(a[7], C, &stream))
      Py_RETURN_NONE;
  } catch (...) {
    Py_RETURN_NONE;
  }
  bifattn_status_t st;
  Py_BEGIN_ALLOW_THREADS
  st = P->gather(reinterpret_cast<bifattn_paged_plan_t>(C->plan), &pages, static_cast<const int32_t*>(table),
                 static_cast<const int32_t*>(first), static_cast<const int32_t*>(lens), (int32_t)s, (int32_t)rows,
                 context, k_out, v_out, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// PagedCaller(append, gather, decode, diff, plan, current_stream, device, b, h, g, d, m_c, m_d, n,
// kv, page, num_pages, Pages): the entry points and the plan as addresses.
PyObject* paged_new(PyTypeObject* type, PyObject* args, PyObject*) {
  unsigned long long append, gather, decode, diff, plan;
  PyObject *cs, *pages;
  int device, kv;
  long long b, h, g, d, m_c, m_d, n, page, num_pages;
  if (!PyArg_ParseTuple(args, "KKKKKOiLLLLLLLiLLO", &append, &gather, &decode, &diff, &plan, &cs, &device, &b, &h, &g,
                        &d, &m_c, &m_d, &n, &kv, &page, &num_pages, &pages))
    return nullptr;
  PagedCaller* P = reinterpret_cast<PagedCaller*>(type->tp_alloc(type, 0));
  if (!P) return nullptr;
  Caller* C = &P->base;
  C->device_obj = PyLong_FromLong(device);
  if (!C->device_obj) {
    Py_DECREF(P);
    return nullptr;
  }
  Py_INCREF(cs);
  C->current_stream = cs;
  Py_INCREF(pages);
  P->pages_type = pages;
  C->plan = reinterpret_cast<bifattn_plan_t>(static_cast<uintptr_t>(plan));
  C->device = device;
  C->b = b, C->h = h, C->g = g, C->d = d, C->m_c = m_c, C->m_d = m_d, C->n = n;
  C->kv = kv;
  P->append = reinterpret_cast<paged_append_fn>(static_cast<uintptr_t>(append));
  P->gather = reinterpret_cast<paged_gather_fn>(static_cast<uintptr_t>(gather));
  P->decode = reinterpret_cast<paged_decode_fn>(static_cast<uintptr_t>(decode));
  P->diff = reinterpret_cast<paged_diff_fn>(static_cast<uintptr_t>(diff));
  P->page = page, P->num_pages = num_pages;
  return reinterpret_cast<PyObject*>(P);
}

void paged_dealloc(PyObject* self) {
  Py_XDECREF(reinterpret_cast<PagedCaller*>(self)->pages_type);
  caller_dealloc(self);
}

#define BIFATTN_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL
PyMethodDef paged_methods[] = {
    {"decode", BIFATTN_FAST(paged_decode), "status of bifattn_paged_decode, or None when the call is not taken"},
    {"diff", BIFATTN_FAST(paged_diff), "status of bifattn_paged_decode_diff, or None when the call is not taken"},
    {"append", BIFATTN_FAST(paged_append), "status of bifattn_paged_append, or None when the call is not taken"},
    {"gather", BIFATTN_FAST(paged_gather), "status of bifattn_paged_gather, or None when the call is not taken"},
    {nullptr, nullptr, 0, nullptr}};
#undef BIFATTN_FAST
PyTypeObject paged_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

PyMethodDef caller_methods[] = {
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(caller_decode)),
     METH_FASTCALL, "status of bifattn_decode_scaled, or None when the call is not taken"},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(caller_append)),
     METH_FASTCALL, "status of bifattn_append_kv, or None when the call is not taken"},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject caller_type = {PyVarObject_HEAD_INIT(nullptr, 0)};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_bifattn_bind", nullptr, -1, nullptr,
                          nullptr,               nullptr,          nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bifattn_bind() {
  caller_type.tp_name = "_bifattn_bind.Caller";
  caller_type.tp_basicsize = sizeof(Caller);
  caller_type.tp_flags = Py_TPFLAGS_DEFAULT;
  caller_type.tp_new = caller_new;
  caller_type.tp_dealloc = caller_dealloc;
  caller_type.tp_methods = caller_methods;
  if (PyType_Ready(&caller_type) < 0) return nullptr;
  PyObject* m = PyModule_Create(&module_def);
  if (!m) return nullptr;
  Py_INCREF(&caller_type);
  if (PyModule_AddObject(m, "Caller", reinterpret_cast<PyObject*>(&caller_type)) < 0) {
    Py_DECREF(&caller_type);
    Py_DECREF(m);
    return nullptr;
  }
  paged_type.tp_name = "_bifattn_bind.PagedCaller";
  paged_type.tp_basicsize = sizeof(PagedCaller);
  paged_type.tp_flags = Py_TPFLAGS_DEFAULT;
  paged_type.tp_new = paged_new;
  paged_type.tp_dealloc = paged_dealloc;
  paged_type.tp_methods = paged_methods;
  if (PyType_Ready(&paged_type) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  Py_INCREF(&paged_type);
  if (PyModule_AddObject(m, "PagedCaller", reinterpret_cast<PyObject*>(&paged_type)) < 0) {
    Py_DECREF(&paged_type);
    Py_DECREF(m);
    return nullptr;
  }
  // The tensor layouts read above are this version's.
  if (PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
