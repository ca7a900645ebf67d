// The Python binding's call path in native code: argument checks, workspace lookup and
// the C ABI call of one DecodeAttention method, without a Python statement per check.
//
// A method takes a call only when every argument is what the Python checks of
// paper_2607_09207_amd/__init__.py accept, and answers None for any other call (tensor
// subclasses, active modes, a workspace that is not allocated yet, a mismatch): the
// Python code then runs its own checks, which raise or go through ctypes.  Nothing is
// kept from one call for the next.
//
// Why: issuing a call took 16.2 us on the host (12.4 us of it checks in Python, 1 us the
// ctypes conversion) against 6 to 12 us of kernel time for the small calls; it takes
// 3.9 us here, nearly all of it the launch.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/TensorSubclassLikeUtils.h>
#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include "rl_decode_attn.h"

namespace {

using at::Tensor;

// Entry points of the library, found by the caller (addresses) so that both bindings use
// the one that is loaded.
decltype(&rl_decode_attn_run) g_run;
decltype(&rl_decode_attn_run_grouped) g_grouped;
decltype(&rl_decode_attn_run_multi) g_multi;
decltype(&rl_decode_attn_run_noalloc) g_noalloc;
decltype(&rl_decode_attn_append) g_append;
decltype(&rl_decode_attn_run_scored) g_scored;
decltype(&rl_decode_attn_rotate) g_rotate;
decltype(&rl_decode_attn_append_rotary) g_append_rotary;
decltype(&rl_decode_attn_page_grow) g_page_grow;
decltype(&rl_decode_attn_page_release) g_page_release;
decltype(&rl_decode_attn_page_fork) g_page_fork;
decltype(&rl_decode_attn_page_compact) g_page_compact;
decltype(&rl_decode_attn_page_bounds) g_page_bounds;
decltype(&rl_decode_attn_select_pages) g_select_pages;
decltype(&rl_decode_attn_run_selected) g_selected;
decltype(&rl_decode_attn_weighed_workspace_size) g_weighed_size;
decltype(&rl_decode_attn_run_weighed) g_weighed;
decltype(&rl_decode_attn_page_evict) g_page_evict;
PyObject* g_raw_stream;   // device index -> current stream (an int)

constexpr int kMaxDevices = 64;
PyObject* g_device_key[kMaxDevices];   // "cuda:0", ... : keys of the workspace dict

struct Layer {
  PyObject_HEAD
  rl_decode_attn_t handle;
  PyObject* workspaces;   // dict: device string -> uint8 tensor (the Python object's own)
  PyObject* page_workspaces;   // dict: (device string, pages) -> uint8 tensor (its own too)
  PyObject* weighed_workspaces;   // dict: device string -> uint8 tensor (its own too)
  int64_t hq, hkv, d, page, max_batch, max_pages;
  int64_t stride[3];
  int64_t ws_bytes, grouped_ws_bytes;   // as allocated, alignment room included
  at::ScalarType q_dtype, kv_dtype, out_dtype;
  bool fp8;
};

at::ScalarType scalar_of(int code) {
  return code == RLDA_F32 ? at::kFloat : code == RLDA_BF16 ? at::kBFloat16 : at::kFloat8_e4m3fn;
}

// The tensor of an argument, or null: not a plain strided tensor.
const Tensor* tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.layout() != at::kStrided || !t.has_storage() || at::isTensorSubclassLike(t)) return nullptr;
  return &t;
}

bool plain(const Tensor* t, int dev, at::ScalarType type) {
  return t && t->is_cuda() && t->get_device() == dev && t->scalar_type() == type;
}
bool shaped(const Tensor* t, int dev, at::ScalarType type, at::IntArrayRef shape) {
  return plain(t, dev, type) && t->sizes() == shape && t->is_contiguous();
}

// One call's arguments that every method shares.
struct Call {
  int dev = -1;
  int64_t npages = 0;
  const Tensor *k = nullptr, *v = nullptr, *ks = nullptr, *vs = nullptr, *bt = nullptr, *lens = nullptr;
  Tensor ws;   // held: the dict's entry may be replaced while the call is without the GIL
  char* ws_ptr = nullptr;
  size_t ws_room = 0;
  void* stream = nullptr;
};

bool cache_ok(const Layer* L, const Tensor* t, int dev, int64_t npages) {
  if (!plain(t, dev, L->kv_dtype) || t->dim() != 4) return false;
  const auto sz = t->sizes(), st = t->strides();
  if (sz[1] != L->hkv || sz[2] != L->page || sz[3] != L->d || sz[0] < npages) return false;
  for (int i = 0; i < 3; ++i)
    if (sz[i] > 1 && st[i] != L->stride[i]) return false;
  return sz[3] <= 1 || st[3] == 1;
}

bool scale_ok(const Layer* L, const Tensor* t, int dev, int64_t npages) {
  return plain(t, dev, at::kFloat) && t->dim() == 2 && t->size(1) == L->hkv && t->size(0) >= npages &&
         t->is_contiguous();
}

// An int argument, or `none` for None; false: neither.
bool as_int(PyObject* o, int64_t none, int64_t* out) {
  if (o == Py_None) {
    *out = none;
    return true;
  }
  if (!PyLong_CheckExact(o)) return false;
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  *out = x;
  return true;
}

// The stream of an argument: None (the device's current one), a raw handle or an object
// that holds one.
bool stream_of(PyObject* o, int dev, void** out) {
  int64_t s = 0;
  PyObject* r = nullptr;
  if (o == Py_None) {
    PyObject* idx = PyLong_FromLong(dev);
    r = idx ? PyObject_CallFunctionObjArgs(g_raw_stream, idx, nullptr) : nullptr;
    Py_XDECREF(idx);
  } else if (as_int(o, 0, &s)) {
    *out = (void*)(intptr_t)s;
    return true;
  } else {
    r = PyObject_GetAttrString(o, "cuda_stream");   // a torch.cuda.Stream
  }
  const bool ok = r && as_int(r, 0, &s);
  Py_XDECREF(r);
  if (!ok) PyErr_Clear();
  *out = (void*)(intptr_t)s;
  return ok;
}

// The arguments common to the methods, in order: k, v, block table, lengths, k scale,
// v scale, stream, page count; `batch` sequences on device `dev`.
bool common(const Layer* L, Call& c, PyObject* const* a, int dev, int64_t batch) {
  c.dev = dev;
  c.k = tensor(a[0]);
  c.v = tensor(a[1]);
  c.bt = tensor(a[2]);
  c.lens = tensor(a[3]);
  if (!c.k || !c.v || c.k->dim() != 4 || !as_int(a[7], c.k->size(0), &c.npages)) return false;
  if (c.npages < 0 || c.npages > INT32_MAX || batch < 0 || batch > L->max_batch) return false;
  if (!cache_ok(L, c.k, dev, c.npages) || !cache_ok(L, c.v, dev, c.npages)) return false;
  if (!shaped(c.bt, dev, at::kInt, {batch, L->max_pages}) || !shaped(c.lens, dev, at::kInt, {batch})) return false;
  if (L->fp8) {
    c.ks = tensor(a[4]);
    c.vs = tensor(a[5]);
    if (!scale_ok(L, c.ks, dev, c.npages) || !scale_ok(L, c.vs, dev, c.npages)) return false;
  } else if (a[4] != Py_None || a[5] != Py_None) {
    return false;
  }
  return stream_of(a[6], dev, &c.stream);
}

bool use_workspace(Call& c, const Tensor* t) {
  if (!plain(t, c.dev, at::kByte) || !t->is_contiguous()) return false;
  c.ws = *t;
  char* p = (char*)t->mutable_data_ptr();
  c.ws_ptr = (char*)(((uintptr_t)p + 255) / 256 * 256);
  const int64_t room = t->numel() - (c.ws_ptr - p);
  if (room < 0) return false;
  c.ws_room = (size_t)room;
  return true;
}

// The workspace given, or the one the Python object keeps for the device.
bool workspace(const Layer* L, Call& c, PyObject* given, bool grouped) {
  const Tensor* t = nullptr;
  if (given != Py_None) {
    t = tensor(given);
  } else {
    if (c.dev >= kMaxDevices) return false;
    PyObject* o = PyDict_GetItem(L->workspaces, g_device_key[c.dev]);   // borrowed
    t = o ? tensor(o) : nullptr;
    if (t && t->numel() < (grouped ? L->grouped_ws_bytes : L->ws_bytes)) return false;
  }
  return use_workspace(c, t);
}

void* ptr(const Tensor* t) { return t ? t->mutable_data_ptr() : nullptr; }

// A tensor that a call on `stream` writes and the caller then has (`given`: the stream as the
// caller gave it).  On another stream than the current one, memory of that stream's own:
// memory of the current stream's might still be in use by what is queued there.  And it is
// not given out again before what is then queued on the current stream is done.
Tensor empty_on(at::IntArrayRef shape, at::TensorOptions how, int dev, PyObject* given, void* stream) {
  void* now = stream;
  if (given != Py_None && !stream_of(Py_None, dev, &now)) throw std::runtime_error("no current stream");
  if (now == stream) return at::empty(shape, how);
  const c10::impl::VirtualGuardImpl impl(c10::DeviceType::CUDA);
  // A stream's handle names it, as torch.cuda.ExternalStream does (0: the default stream).
  struct Guard {
    const c10::impl::VirtualGuardImpl& impl;
    c10::Stream old;
    ~Guard() { impl.exchangeStream(old); }
  } guard{impl, impl.exchangeStream(c10::Stream::unpack3((int64_t)(intptr_t)stream, (c10::DeviceIndex)dev, c10::DeviceType::CUDA))};
  Tensor t = at::empty(shape, how);
  t.record_stream(guard.old);
  return t;
}

// The output given, or a new tensor (rows, Hq, d) held by `fresh`.
const Tensor* output(const Layer* L, PyObject* given, const Tensor& q, int64_t rows, PyObject* stream, const Call& c, Tensor& fresh) {
  if (given == Py_None) {
    fresh = empty_on({rows, L->hq, L->d}, at::TensorOptions().dtype(L->out_dtype).device(q.device()), c.dev, stream, c.stream);
    return &fresh;
  }
  const Tensor* o = tensor(given);
  return shaped(o, q.get_device(), L->out_dtype, {rows, L->hq, L->d}) ? o : nullptr;
}

// The call's answer: the output tensor, or the status of a call that failed.
PyObject* answer(rlda_status st, PyObject* given, const Tensor& fresh) {
  if (st != RLDA_OK) return PyLong_FromLong((long)st);
  if (given != Py_None) {
    Py_INCREF(given);
    return given;
  }
  return THPVariable_Wrap(fresh);
}

// Runs `body` with C++ exceptions (a tensor without data, no memory) turned into "not
// taken": the Python path then meets, and reports, the same condition.
template <class F>
PyObject* guarded(F body) {
  try {
    PyObject* r = body();
    if (r) return r;
    if (PyErr_Occurred()) return nullptr;
  } catch (const std::exception&) {
  }
  Py_RETURN_NONE;
}

#define WITHOUT_GIL(call)    \
  rlda_status st;            \
  Py_BEGIN_ALLOW_THREADS     \
  st = (call);               \
  Py_END_ALLOW_THREADS

// run(q, k, v, block_table, seq_lens, k_scale, v_scale, stream, num_pages, out, workspace)
PyObject* layer_run(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 11) return PyErr_Format(PyExc_TypeError, "run takes 11 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    const Tensor* q = tensor(a[0]);
    if (!q || !q->is_cuda() || q->dim() != 3) return nullptr;
    const int dev = q->get_device();
    const int64_t B = q->size(0);
    Call c;
    if (!shaped(q, dev, L->q_dtype, {B, L->hq, L->d}) || !common(L, c, a + 1, dev, B) || !workspace(L, c, a[10], false))
      return nullptr;
    Tensor fresh;
    const Tensor* o = output(L, a[9], *q, B, a[7], c, fresh);
    if (!o) return nullptr;
    void *qp = ptr(q), *kp = ptr(c.k), *vp = ptr(c.v), *ksp = ptr(c.ks), *vsp = ptr(c.vs), *bp = ptr(c.bt),
         *lp = ptr(c.lens), *op = ptr(o);
    WITHOUT_GIL(g_run(L->handle, (int32_t)B, (int32_t)c.npages, qp, kp, vp, (const float*)ksp, (const float*)vsp,
                      (const int32_t*)bp, (const int32_t*)lp, op, c.ws_ptr, c.ws_room, c.stream));
    return answer(st, a[9], fresh);
  });
}

// grouped(q, k, v, block_table, seq_lens, k_scale, v_scale, stream, num_pages, out, workspace,
//         group_size, prefix_pages, prompt_pages_hint)
PyObject* layer_grouped(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 14) return PyErr_Format(PyExc_TypeError, "grouped takes 14 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    const Tensor* q = tensor(a[0]);
    if (!q || !q->is_cuda() || q->dim() != 3) return nullptr;
    const int dev = q->get_device();
    const int64_t B = q->size(0);
    Call c;
    int64_t gs = 0, hint = -1;
    const Tensor* pp = tensor(a[12]);
    if (!as_int(a[11], 0, &gs) || a[13] == Py_None || !as_int(a[13], -1, &hint) || gs < 1 || gs > INT32_MAX ||
        hint < INT32_MIN || hint > INT32_MAX)
      return nullptr;
    if (!shaped(q, dev, L->q_dtype, {B, L->hq, L->d}) || !common(L, c, a + 1, dev, B) ||
        !shaped(pp, dev, at::kInt, {(B + gs - 1) / gs}) || !workspace(L, c, a[10], true))
      return nullptr;
    Tensor fresh;
    const Tensor* o = output(L, a[9], *q, B, a[7], c, fresh);
    if (!o) return nullptr;
    void *qp = ptr(q), *kp = ptr(c.k), *vp = ptr(c.v), *ksp = ptr(c.ks), *vsp = ptr(c.vs), *bp = ptr(c.bt),
         *lp = ptr(c.lens), *op = ptr(o), *ppp = ptr(pp);
    WITHOUT_GIL(g_grouped(L->handle, (int32_t)B, (int32_t)c.npages, (int32_t)gs, (const int32_t*)ppp, (int32_t)hint, qp,
                          kp, vp, (const float*)ksp, (const float*)vsp, (const int32_t*)bp, (const int32_t*)lp, op,
                          c.ws_ptr, c.ws_room, c.stream, nullptr, nullptr));
    return answer(st, a[9], fresh);
  });
}

// multi(q, k, v, block_table, seq_lens, k_scale, v_scale, stream, num_pages, out, workspace,
//       q_start, max_q_len)
PyObject* layer_multi(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 13) return PyErr_Format(PyExc_TypeError, "multi takes 13 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    const Tensor *q = tensor(a[0]), *qs = tensor(a[11]);
    if (!q || !q->is_cuda() || q->dim() != 3 || !qs || qs->dim() != 1) return nullptr;
    const int dev = q->get_device();
    const int64_t total = q->size(0), B = qs->size(0) - 1;
    Call c;
    int64_t mq = 0;
    if (total > INT32_MAX || a[12] == Py_None || !as_int(a[12], 0, &mq) || mq < INT32_MIN || mq > INT32_MAX)
      return nullptr;
    if (!shaped(q, dev, L->q_dtype, {total, L->hq, L->d}) || !shaped(qs, dev, at::kInt, {B + 1}) ||
        !common(L, c, a + 1, dev, B) || !workspace(L, c, a[10], false))
      return nullptr;
    Tensor fresh;
    const Tensor* o = output(L, a[9], *q, total, a[7], c, fresh);
    if (!o) return nullptr;
    void *qp = ptr(q), *kp = ptr(c.k), *vp = ptr(c.v), *ksp = ptr(c.ks), *vsp = ptr(c.vs), *bp = ptr(c.bt),
         *lp = ptr(c.lens), *op = ptr(o), *qsp = ptr(qs);
    WITHOUT_GIL(g_multi(L->handle, (int32_t)B, (int32_t)c.npages, (int32_t)total, (int32_t)mq, qp, kp, vp,
                        (const float*)ksp, (const float*)vsp, (const int32_t*)bp, (const int32_t*)lp,
                        (const int32_t*)qsp, op, c.ws_ptr, c.ws_room, c.stream, nullptr, nullptr));
    return answer(st, a[9], fresh);
  });
}

// noalloc(q, k, v, block_table, seq_lens, k_scale, v_scale, stream, num_pages, out, flags)
PyObject* layer_noalloc(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 11) return PyErr_Format(PyExc_TypeError, "noalloc takes 11 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    const Tensor* q = tensor(a[0]);
    if (!q || !q->is_cuda() || q->dim() != 3) return nullptr;
    const int dev = q->get_device();
    const int64_t B = q->size(0);
    Call c;
    const Tensor* flags = nullptr;
    if (a[10] != Py_None && !shaped(flags = tensor(a[10]), dev, at::kInt, {1})) return nullptr;
    if (!shaped(q, dev, L->q_dtype, {B, L->hq, L->d}) || !common(L, c, a + 1, dev, B)) return nullptr;
    Tensor fresh;
    const Tensor* o = output(L, a[9], *q, B, a[7], c, fresh);
    if (!o) return nullptr;
    void *qp = ptr(q), *kp = ptr(c.k), *vp = ptr(c.v), *ksp = ptr(c.ks), *vsp = ptr(c.vs), *bp = ptr(c.bt),
         *lp = ptr(c.lens), *op = ptr(o), *fp = ptr(flags);
    WITHOUT_GIL(g_noalloc(L->handle, (int32_t)B, (int32_t)c.npages, qp, kp, vp, (const float*)ksp, (const float*)vsp,
                          (const int32_t*)bp, (const int32_t*)lp, op, (uint32_t*)fp, c.stream));
    return answer(st, a[9], fresh);
  });
}

// append(k_new, k, v, block_table, seq_lens, k_scale, v_scale, stream, num_pages, v_new, workspace):
// the status, or None (not taken).
PyObject* layer_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 11) return PyErr_Format(PyExc_TypeError, "append takes 11 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    const Tensor *kn = tensor(a[0]), *vn = tensor(a[9]);
    if (!kn || !kn->is_cuda() || kn->dim() != 3) return nullptr;
    const int dev = kn->get_device();
    const int64_t B = kn->size(0);
    Call c;
    if (!shaped(kn, dev, L->q_dtype, {B, L->hkv, L->d}) || !shaped(vn, dev, L->q_dtype, {B, L->hkv, L->d}) ||
        !common(L, c, a + 1, dev, B) || !workspace(L, c, a[10], false))
      return nullptr;
    void *knp = ptr(kn), *vnp = ptr(vn), *kp = ptr(c.k), *vp = ptr(c.v), *ksp = ptr(c.ks), *vsp = ptr(c.vs),
         *bp = ptr(c.bt), *lp = ptr(c.lens);
    WITHOUT_GIL(g_append(L->handle, (int32_t)B, (int32_t)c.npages, knp, vnp, kp, vp, (float*)ksp, (float*)vsp,
                         (const int32_t*)bp, (const int32_t*)lp, c.ws_ptr, c.ws_room, c.stream));
    return PyLong_FromLong((long)st);
  });
}

// ------------------------------------------------------------------ modified scores, rotary positions, pages

// The new calls launch on the current device: one on another is left to Python, which
// makes it the current one.
bool current(int dev) { return c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index() == dev; }

bool as_double(PyObject* o, double* out) {
  if (PyFloat_CheckExact(o)) {
    *out = PyFloat_AS_DOUBLE(o);
    return true;
  }
  int64_t i = 0;
  if (o == Py_None || !as_int(o, 0, &i)) return false;
  *out = (double)i;
  return true;
}
bool as_bool(PyObject* o, int* out) {
  *out = o == Py_True;
  return o == Py_True || o == Py_False;
}
// A vector argument of n elements, or None (null).
bool vector_or_none(PyObject* o, int dev, at::ScalarType type, int64_t n, const Tensor** out) {
  *out = nullptr;
  return o == Py_None || shaped(*out = tensor(o), dev, type, {n});
}

// Rows [n][heads][d] as the C ABI takes them.
bool rows_of(const Tensor* t, int dev, at::ScalarType type, int64_t n, int64_t heads, int64_t d, rl_decode_attn_rows* out) {
  if (!plain(t, dev, type) || t->dim() != 3) return false;
  const auto sz = t->sizes(), st = t->strides();
  if (sz[0] != n || sz[1] != heads || sz[2] != d || (d > 1 && st[2] != 1)) return false;
  const int64_t per = 16 / (int64_t)t->element_size();
  void* p = t->mutable_data_ptr();
  if (((uintptr_t)p & 15) || (n > 1 && st[0] % per) || (heads > 1 && st[1] % per)) return false;
  *out = {p, n > 1 ? st[0] : 0, heads > 1 ? st[1] : 0};
  return true;
}

// A tensor whose derivatives are asked for, by either mode: Python notes it or refuses it.
bool derived(const Tensor& t) {
  return (t.requires_grad() && c10::GradMode::is_enabled()) ||
         (c10::AutogradState::get_tls_state().get_fw_grad_mode() && t._fw_grad(0).defined());
}

// A backward pass that saved a tensor written here is to notice.
void mark_written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

bool rotary_of(PyObject* freqs, PyObject* interleaved, PyObject* amplitude, int inverse, int dev, int64_t d,
               rl_decode_attn_rotary* out) {
  const Tensor* f = tensor(freqs);
  int il = 0;
  double a = 1.0;
  if (!plain(f, dev, at::kDouble) || derived(*f) || f->dim() != 1 || !f->is_contiguous() || !as_bool(interleaved, &il) ||
      !as_double(amplitude, &a))
    return false;
  const int64_t half = f->size(0);
  if (half < 8 || 2 * half > d || half % 8) return false;
  *out = {(const double*)f->mutable_data_ptr(), (int32_t)(2 * half), il, (float)a, inverse};
  return true;
}

// scored(q, k, v, block_table, seq_lens, k_scale, v_scale, stream, num_pages, out, workspace,
//        q_start, max_q_len, score_cap, slopes, window, key_start, prefix_lens)
PyObject* layer_scored(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 18) return PyErr_Format(PyExc_TypeError, "scored takes 18 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    const Tensor* q = tensor(a[0]);
    if (!q || !q->is_cuda() || q->dim() != 3 || (a[9] == Py_None && a[7] != Py_None)) return nullptr;
    const int dev = q->get_device();
    const int64_t total = q->size(0);
    const Tensor *qs = nullptr, *slopes, *ks, *pl;
    int64_t B = total, mq = 0, window = 0;
    double cap = 0.0;
    if (a[11] != Py_None) {
      qs = tensor(a[11]);
      if (!qs || qs->dim() != 1) return nullptr;
      B = qs->size(0) - 1;
      if (!shaped(qs, dev, at::kInt, {B + 1})) return nullptr;
    }
    if (total > INT32_MAX || a[12] == Py_None || !as_int(a[12], 0, &mq) || mq < INT32_MIN || mq > INT32_MAX ||
        !as_double(a[13], &cap) || (cap != 0.0 && (float)cap == 0.f) || a[15] == Py_None || !as_int(a[15], 0, &window) || window < INT32_MIN || window > INT32_MAX)
      return nullptr;
    Call c;
    if (!shaped(q, dev, L->q_dtype, {total, L->hq, L->d}) || !vector_or_none(a[14], dev, at::kFloat, L->hq, &slopes) ||
        !vector_or_none(a[16], dev, at::kInt, total, &ks) || !common(L, c, a + 1, dev, B) ||
        !vector_or_none(a[17], dev, at::kInt, B, &pl) || !workspace(L, c, a[10], false) || !current(dev))
      return nullptr;
    Tensor fresh;
    const Tensor* o = output(L, a[9], *q, total, a[7], c, fresh);
    if (!o) return nullptr;
    const rl_decode_attn_scores sc = {(float)cap, (int32_t)window, (const float*)ptr(slopes), (const int32_t*)ptr(ks),
                                      (const int32_t*)ptr(pl)};
    void *qp = ptr(q), *kp = ptr(c.k), *vp = ptr(c.v), *ksp = ptr(c.ks), *vsp = ptr(c.vs), *bp = ptr(c.bt),
         *lp = ptr(c.lens), *op = ptr(o), *qsp = ptr(qs);
    WITHOUT_GIL(g_scored(L->handle, &sc, (int32_t)B, (int32_t)c.npages, (int32_t)total, (int32_t)mq, qp, kp, vp,
                         (const float*)ksp, (const float*)vsp, (const int32_t*)bp, (const int32_t*)lp, (const int32_t*)qsp,
                         op, c.ws_ptr, c.ws_room, c.stream, nullptr, nullptr));
    return answer(st, a[9], fresh);
  });
}

// append_rotary(q, k, v, block_table, seq_lens, k_scale, v_scale, stream, num_pages, out, workspace,
//               k_new, v_new, freqs, q_start, positions, interleaved, amplitude)
PyObject* layer_append_rotary(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 18) return PyErr_Format(PyExc_TypeError, "append_rotary takes 18 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    const Tensor* q = tensor(a[0]);
    if (!q || !q->is_cuda() || q->dim() != 3 || (a[9] == Py_None && a[7] != Py_None)) return nullptr;
    const int dev = q->get_device();
    const int64_t total = q->size(0);
    const Tensor *qs = nullptr, *pos;
    int64_t B = total;
    if (a[14] != Py_None) {
      qs = tensor(a[14]);
      if (!qs || qs->dim() != 1) return nullptr;
      B = qs->size(0) - 1;
      if (!shaped(qs, dev, at::kInt, {B + 1})) return nullptr;
    }
    Call c;
    rl_decode_attn_rows rq, rk, rv, ro;
    rl_decode_attn_rotary rot;
    const Tensor *kn = tensor(a[11]), *vn = tensor(a[12]), *given = a[9] == Py_None ? nullptr : tensor(a[9]);
    if (total > INT32_MAX || !rows_of(q, dev, L->q_dtype, total, L->hq, L->d, &rq) ||
        !rows_of(kn, dev, L->q_dtype, total, L->hkv, L->d, &rk) ||
        !rows_of(vn, dev, L->q_dtype, total, L->hkv, L->d, &rv) || derived(*q) || derived(*kn) || derived(*vn) ||
        !rotary_of(a[13], a[16], a[17], 0, dev, L->d, &rot) || !vector_or_none(a[15], dev, at::kInt, total, &pos) ||
        !common(L, c, a + 1, dev, B) || !workspace(L, c, a[10], false) || !current(dev))
      return nullptr;
    Tensor fresh;
    if (a[9] == Py_None) fresh = at::empty({total, L->hq, L->d}, q->options());
    if (!rows_of(a[9] == Py_None ? &fresh : given, dev, L->q_dtype, total, L->hq, L->d, &ro) || (given && derived(*given)))
      return nullptr;
    if (given) mark_written(*given);
    void *kp = ptr(c.k), *vp = ptr(c.v), *ksp = ptr(c.ks), *vsp = ptr(c.vs), *bp = ptr(c.bt), *lp = ptr(c.lens),
         *qsp = ptr(qs), *pp = ptr(pos);
    WITHOUT_GIL(g_append_rotary(L->handle, (int32_t)B, (int32_t)c.npages, (int32_t)total, &rot, &rq, &rk, &rv,
                                (const int32_t*)qsp, (const int32_t*)pp, kp, vp, (float*)ksp, (float*)vsp,
                                (const int32_t*)bp, (const int32_t*)lp, &ro, c.ws_ptr, c.ws_room, c.stream));
    return answer(st, a[9], fresh);
  });
}

// rotate(x, positions, freqs, interleaved, amplitude, inverse, out, stream)
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 8) return PyErr_Format(PyExc_TypeError, "rotate takes 8 arguments");
  return guarded([&]() -> PyObject* {
    const Tensor* x = tensor(a[0]);
    if (!x || !x->is_cuda() || x->dim() != 3 || (a[6] == Py_None && a[7] != Py_None)) return nullptr;
    const auto type = x->scalar_type();
    if (type != at::kBFloat16 && type != at::kFloat) return nullptr;
    if (derived(*x)) return nullptr;
    const int dev = x->get_device();
    const int64_t rows = x->size(0), heads = x->size(1), d = x->size(2);
    int inverse = 0;
    rl_decode_attn_rows rx, ro;
    rl_decode_attn_rotary rot;
    void* stream = nullptr;
    const Tensor* pos = tensor(a[1]);
    if (rows > INT32_MAX || heads > INT32_MAX || d > INT32_MAX || !as_bool(a[5], &inverse) ||
        !rows_of(x, dev, type, rows, heads, d, &rx) || !shaped(pos, dev, at::kInt, {rows}) ||
        !rotary_of(a[2], a[3], a[4], inverse, dev, d, &rot) || !stream_of(a[7], dev, &stream) || !current(dev))
      return nullptr;
    Tensor fresh;
    const Tensor* out = &fresh;
    if (a[6] == Py_None) {
      fresh = at::empty({rows, heads, d}, x->options());
    } else {
      out = tensor(a[6]);
      if (!out || derived(*out)) return nullptr;
    }
    if (!rows_of(out, dev, type, rows, heads, d, &ro)) return nullptr;
    if (a[6] != Py_None) mark_written(*out);
    const int32_t* pp = (const int32_t*)ptr(pos);
    WITHOUT_GIL(g_rotate(type == at::kFloat ? RLDA_F32 : RLDA_BF16, (int32_t)rows, (int32_t)heads, (int32_t)d, &rx, pp, &rot,
                         &ro, stream));
    return answer(st, a[6], fresh);
  });
}

// What the page operations share: (refs, block_table, seq_lens), workspace, stream.
bool page_common(const Layer* L, Call& c, PyObject* const* a, PyObject* ws, PyObject* stream, const Tensor** refs, int64_t* batch) {
  const Tensor* r = tensor(a[0]);
  if (!r || !r->is_cuda() || r->dim() != 1) return false;
  c.dev = r->get_device();
  c.npages = r->size(0);
  c.bt = tensor(a[1]);
  c.lens = tensor(a[2]);
  if (!c.lens || c.lens->dim() != 1) return false;
  *batch = c.lens->size(0);
  if (c.npages > INT32_MAX || *batch > L->max_batch || !shaped(r, c.dev, at::kInt, {c.npages}) ||
      !shaped(c.bt, c.dev, at::kInt, {*batch, L->max_pages}) || !shaped(c.lens, c.dev, at::kInt, {*batch}))
    return false;
  *refs = r;
  const Tensor* t = nullptr;
  if (ws != Py_None) {
    t = tensor(ws);
  } else {
    if (c.dev >= kMaxDevices) return false;
    PyObject* pages = PyLong_FromLongLong(c.npages);
    PyObject* key = pages ? PyTuple_Pack(2, g_device_key[c.dev], pages) : nullptr;
    PyObject* o = key ? PyDict_GetItem(L->page_workspaces, key) : nullptr;   // borrowed
    Py_XDECREF(key);
    Py_XDECREF(pages);
    t = o ? tensor(o) : nullptr;
  }
  return use_workspace(c, t) && stream_of(stream, c.dev, &c.stream) && current(c.dev);
}

PyObject* status(rlda_status st) { return PyLong_FromLong((long)st); }

// The caches of a set: their number, the address of the C array, pages, device.
bool caches_of(PyObject* const* a, const Call& c, int32_t* n, const rl_decode_attn_cache** array) {
  int64_t num = 0, addr = 0, pages = 0, dev = 0;
  if (a[0] == Py_None || !as_int(a[0], 0, &num) || num < 0 || num > INT32_MAX) return false;
  *n = (int32_t)num;
  if (num == 0) return true;
  if (!as_int(a[1], 0, &addr) || addr == 0 || !as_int(a[2], -1, &pages) || !as_int(a[3], -1, &dev) || pages < c.npages || dev != c.dev)
    return false;
  *array = (const rl_decode_attn_cache*)(intptr_t)addr;
  return true;
}

// page_grow(refs, block_table, seq_lens, add, workspace, stream): the status, or None (not taken).
PyObject* layer_page_grow(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) return PyErr_Format(PyExc_TypeError, "page_grow takes 6 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    Call c;
    const Tensor *refs, *add;
    int64_t B;
    if (!page_common(L, c, a, a[4], a[5], &refs, &B) || !vector_or_none(a[3], c.dev, at::kInt, B, &add)) return nullptr;
    void *rp = ptr(refs), *bp = ptr(c.bt), *lp = ptr(c.lens), *ap = ptr(add);
    WITHOUT_GIL(g_page_grow(L->handle, (int32_t)B, (int32_t)c.npages, (int32_t*)rp, (int32_t*)bp, (int32_t*)lp,
                            (const int32_t*)ap, c.ws_ptr, c.ws_room, c.stream));
    return status(st);
  });
}

// page_release(refs, block_table, seq_lens, rows, workspace, stream)
PyObject* layer_page_release(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 6) return PyErr_Format(PyExc_TypeError, "page_release takes 6 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    Call c;
    const Tensor *refs, *rows = tensor(a[3]);
    int64_t B;
    if (!rows || rows->dim() != 1 || rows->size(0) > INT32_MAX || !page_common(L, c, a, a[4], a[5], &refs, &B) ||
        !shaped(rows, c.dev, at::kInt, {rows->size(0)}))
      return nullptr;
    const int32_t count = (int32_t)rows->size(0);
    void *rp = ptr(refs), *bp = ptr(c.bt), *lp = ptr(c.lens), *wp = ptr(rows);
    WITHOUT_GIL(g_page_release(L->handle, (int32_t)B, (int32_t)c.npages, (int32_t*)rp, (int32_t*)bp, (int32_t*)lp, count,
                               (const int32_t*)wp, c.ws_ptr, c.ws_room, c.stream));
    return status(st);
  });
}

// page_fork(refs, block_table, seq_lens, parents, children, caches: number, address, pages, device, workspace, stream)
PyObject* layer_page_fork(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 11) return PyErr_Format(PyExc_TypeError, "page_fork takes 11 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    Call c;
    const Tensor *refs, *par = tensor(a[3]), *kid = tensor(a[4]);
    int64_t B;
    int32_t nc = 0;
    const rl_decode_attn_cache* caches = nullptr;
    if (!par || par->dim() != 1 || par->size(0) > INT32_MAX || !page_common(L, c, a, a[9], a[10], &refs, &B) ||
        !shaped(par, c.dev, at::kInt, {par->size(0)}) || !shaped(kid, c.dev, at::kInt, {par->size(0)}) ||
        !caches_of(a + 5, c, &nc, &caches))
      return nullptr;
    const int32_t count = (int32_t)par->size(0);
    void *rp = ptr(refs), *bp = ptr(c.bt), *lp = ptr(c.lens), *pp = ptr(par), *kp = ptr(kid);
    WITHOUT_GIL(g_page_fork(L->handle, (int32_t)B, (int32_t)c.npages, (int32_t*)rp, (int32_t*)bp, (int32_t*)lp, count,
                            (const int32_t*)pp, (const int32_t*)kp, nc, caches, c.ws_ptr, c.ws_room, c.stream));
    return status(st);
  });
}

// page_compact(refs, block_table, seq_lens, caches: number, address, pages, device, live, workspace, stream):
// the live tensor, a status, or None
PyObject* layer_page_compact(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 10) return PyErr_Format(PyExc_TypeError, "page_compact takes 10 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    Call c;
    const Tensor* refs;
    int64_t B;
    int32_t nc = 0;
    const rl_decode_attn_cache* caches = nullptr;
    if ((a[7] == Py_None && a[9] != Py_None) || !page_common(L, c, a, a[8], a[9], &refs, &B) || !caches_of(a + 3, c, &nc, &caches))
      return nullptr;
    Tensor fresh;
    if (a[7] == Py_None) fresh = at::empty({1}, refs->options());
    const Tensor* live = a[7] == Py_None ? &fresh : tensor(a[7]);
    if (!shaped(live, c.dev, at::kInt, {1})) return nullptr;
    void *rp = ptr(refs), *bp = ptr(c.bt), *lp = ptr(c.lens), *vp = ptr(live);
    WITHOUT_GIL(g_page_compact(L->handle, (int32_t)B, (int32_t)c.npages, (int32_t*)rp, (int32_t*)bp, (int32_t*)lp, nc, caches,
                               (int32_t*)vp, c.ws_ptr, c.ws_room, c.stream));
    return answer(st, a[7], fresh);
  });
}

// ------------------------------------------------------------------ a cache read and kept in part

// q [total][Hq][d] of `batch` sequences, one row each or by q_start.
bool rows_call(const Layer* L, PyObject* q_arg, PyObject* qs_arg, const Tensor** q, const Tensor** qs, int* dev, int64_t* total,
               int64_t* batch) {
  const Tensor* t = *q = tensor(q_arg);
  *qs = nullptr;
  if (!t || !t->is_cuda() || t->dim() != 3 || t->size(0) > INT32_MAX || derived(*t)) return false;
  *dev = t->get_device();
  *total = *batch = t->size(0);
  if (qs_arg != Py_None) {
    const Tensor* s = *qs = tensor(qs_arg);
    if (!s || s->dim() != 1) return false;
    *batch = s->size(0) - 1;
    if (!shaped(s, *dev, at::kInt, {*batch + 1})) return false;
  }
  return shaped(t, *dev, L->q_dtype, {*total, L->hq, L->d}) && current(*dev);
}

bool bounds_ok(const Layer* L, const Tensor* b, const Tensor* s, int dev, int64_t npages) {
  return plain(b, dev, at::kChar) && b->dim() == 4 && b->size(0) >= npages && b->size(1) == L->hkv && b->size(2) == 2 &&
         b->size(3) == L->d && b->is_contiguous() && scale_ok(L, s, dev, npages);
}

bool host_int(PyObject* o, int32_t* out) {
  int64_t x = 0;
  if (o == Py_None || !as_int(o, 0, &x) || x < INT32_MIN || x > INT32_MAX) return false;
  *out = (int32_t)x;
  return true;
}
bool budget_of(PyObject* const* a, int32_t* budget, int32_t* sink, int32_t* recent) {
  return host_int(a[0], budget) && host_int(a[1], sink) && host_int(a[2], recent) && *sink >= 0 && *recent >= 1 &&
         (int64_t)*sink + *recent <= *budget;
}

// page_bounds(k, block_table, seq_lens, k_scale, stream, num_pages, workspace, bounds, bound_scale, first): the
// status, or None (not taken).
PyObject* layer_page_bounds(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 10) return PyErr_Format(PyExc_TypeError, "page_bounds takes 10 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    const Tensor *lens = tensor(a[2]), *k = tensor(a[0]), *bounds = tensor(a[7]), *bscale = tensor(a[8]), *first;
    if (!k || !k->is_cuda() || !lens || lens->dim() != 1) return nullptr;
    const int dev = k->get_device();
    const int64_t B = lens->size(0);
    PyObject* const args[8] = {a[0], a[0], a[1], a[2], a[3], a[3], a[4], a[5]};   // (K alone)
    Call c;
    if (!common(L, c, args, dev, B) || !bounds_ok(L, bounds, bscale, dev, c.npages) || !vector_or_none(a[9], dev, at::kInt, B, &first) ||
        !workspace(L, c, a[6], false) || !current(dev))
      return nullptr;
    mark_written(*bounds);
    mark_written(*bscale);
    void *kp = ptr(c.k), *ksp = ptr(c.ks), *bp = ptr(c.bt), *lp = ptr(c.lens), *fp = ptr(first), *op = ptr(bounds), *sp = ptr(bscale);
    WITHOUT_GIL(g_page_bounds(L->handle, (int32_t)B, (int32_t)c.npages, kp, (const float*)ksp, (const int32_t*)bp, (const int32_t*)lp,
                              (const int32_t*)fp, (int8_t*)op, (float*)sp, c.ws_ptr, c.ws_room, c.stream));
    return status(st);
  });
}

// select_pages(q, bounds, bound_scale, block_table, seq_lens, stream, num_pages, pages, counts, workspace, q_start,
//              budget, sink, recent): (pages, counts), a status, or None
PyObject* layer_select_pages(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 14) return PyErr_Format(PyExc_TypeError, "select_pages takes 14 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    const Tensor *q, *qs, *bounds = tensor(a[1]), *bscale = tensor(a[2]);
    int dev;
    int64_t total, B;
    int32_t budget, sink, recent;
    Call c;
    if (!rows_call(L, a[0], a[10], &q, &qs, &dev, &total, &B) || !budget_of(a + 11, &budget, &sink, &recent) || !bounds ||
        bounds->dim() != 4 || !as_int(a[6], bounds->size(0), &c.npages) || c.npages < 0 || c.npages > INT32_MAX ||
        !bounds_ok(L, bounds, bscale, dev, c.npages) || B < 0 || B > L->max_batch)
      return nullptr;
    c.dev = dev;
    c.bt = tensor(a[3]);
    c.lens = tensor(a[4]);
    if (!shaped(c.bt, dev, at::kInt, {B, L->max_pages}) || !shaped(c.lens, dev, at::kInt, {B}) || !stream_of(a[5], dev, &c.stream) ||
        !workspace(L, c, a[9], false))
      return nullptr;
    Tensor fresh[2];
    const Tensor* out[2];
    const std::vector<int64_t> shape[2] = {{total, L->hkv, budget}, {total, L->hkv}};
    for (int i = 0; i < 2; ++i) {
      if (a[7 + i] == Py_None) {
        fresh[i] = empty_on(shape[i], c.lens->options(), dev, a[5], c.stream);
        out[i] = &fresh[i];
      } else if (!shaped(out[i] = tensor(a[7 + i]), dev, at::kInt, shape[i])) {
        return nullptr;
      }
    }
    for (int i = 0; i < 2; ++i)
      if (a[7 + i] != Py_None) mark_written(*out[i]);
    void *qp = ptr(q), *op = ptr(bounds), *sp = ptr(bscale), *bp = ptr(c.bt), *lp = ptr(c.lens), *qsp = ptr(qs), *pp = ptr(out[0]),
         *cp = ptr(out[1]);
    WITHOUT_GIL(g_select_pages(L->handle, (int32_t)B, (int32_t)c.npages, (int32_t)total, budget, sink, recent, qp, (const int8_t*)op,
                               (const float*)sp, (const int32_t*)bp, (const int32_t*)lp, (const int32_t*)qsp, (int32_t*)pp,
                               (int32_t*)cp, c.ws_ptr, c.ws_room, c.stream));
    if (st != RLDA_OK) return status(st);
    PyObject* r[2];
    for (int i = 0; i < 2; ++i) r[i] = answer(st, a[7 + i], fresh[i]);
    PyObject* both = r[0] && r[1] ? PyTuple_Pack(2, r[0], r[1]) : nullptr;
    Py_XDECREF(r[0]);
    Py_XDECREF(r[1]);
    return both;
  });
}

// selected(q, k, v, block_table, seq_lens, k_scale, v_scale, stream, num_pages, out, workspace, q_start, pages, counts)
PyObject* layer_selected(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 14) return PyErr_Format(PyExc_TypeError, "selected takes 14 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    const Tensor *q, *qs, *pages = tensor(a[12]), *counts = tensor(a[13]);
    int dev;
    int64_t total, B;
    Call c;
    if (!rows_call(L, a[0], a[11], &q, &qs, &dev, &total, &B) || !pages || pages->dim() != 3 || pages->size(2) > INT32_MAX ||
        !shaped(pages, dev, at::kInt, {total, L->hkv, pages->size(2)}) || !shaped(counts, dev, at::kInt, {total, L->hkv}) ||
        !common(L, c, a + 1, dev, B) || !workspace(L, c, a[10], false))
      return nullptr;
    Tensor fresh;
    const Tensor* o = output(L, a[9], *q, total, a[7], c, fresh);
    if (!o) return nullptr;
    if (a[9] != Py_None) mark_written(*o);
    const int32_t budget = (int32_t)pages->size(2);
    void *qp = ptr(q), *kp = ptr(c.k), *vp = ptr(c.v), *ksp = ptr(c.ks), *vsp = ptr(c.vs), *bp = ptr(c.bt), *lp = ptr(c.lens),
         *op = ptr(o), *qsp = ptr(qs), *pp = ptr(pages), *cp = ptr(counts);
    WITHOUT_GIL(g_selected(L->handle, (int32_t)B, (int32_t)c.npages, (int32_t)total, budget, (const int32_t*)pp, (const int32_t*)cp,
                           qp, kp, vp, (const float*)ksp, (const float*)vsp, (const int32_t*)bp, (const int32_t*)lp,
                           (const int32_t*)qsp, op, c.ws_ptr, c.ws_room, c.stream, nullptr, nullptr));
    return answer(st, a[9], fresh);
  });
}

// weighed(q, k, v, block_table, seq_lens, k_scale, v_scale, stream, num_pages, out, workspace, q_start, weights, decay)
PyObject* layer_weighed(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 14) return PyErr_Format(PyExc_TypeError, "weighed takes 14 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    const Tensor *q, *qs, *weights = tensor(a[12]);
    int dev;
    int64_t total, B;
    double decay = 0.0;
    Call c;
    size_t need = 0;
    if (!rows_call(L, a[0], a[11], &q, &qs, &dev, &total, &B) || !as_double(a[13], &decay) || !(decay >= 0.0 && decay <= 1.0) ||
        !shaped(weights, dev, at::kFloat, {B, L->max_pages}) || derived(*weights) || !common(L, c, a + 1, dev, B) ||
        dev >= kMaxDevices || g_weighed_size(L->handle, (int32_t)total, &need) != RLDA_OK)
      return nullptr;
    const Tensor* ws = nullptr;
    if (a[10] != Py_None) {
      ws = tensor(a[10]);
    } else {
      PyObject* o = PyDict_GetItem(L->weighed_workspaces, g_device_key[dev]);   // borrowed
      ws = o ? tensor(o) : nullptr;
      if (ws && ws->numel() < (int64_t)need + 256) return nullptr;
    }
    if (!use_workspace(c, ws)) return nullptr;
    Tensor fresh;
    const Tensor* o = output(L, a[9], *q, total, a[7], c, fresh);
    if (!o) return nullptr;
    if (a[9] != Py_None) mark_written(*o);
    mark_written(*weights);
    void *qp = ptr(q), *kp = ptr(c.k), *vp = ptr(c.v), *ksp = ptr(c.ks), *vsp = ptr(c.vs), *bp = ptr(c.bt), *lp = ptr(c.lens),
         *op = ptr(o), *qsp = ptr(qs), *wp = ptr(weights);
    WITHOUT_GIL(g_weighed(L->handle, (int32_t)B, (int32_t)c.npages, (int32_t)total, (float*)wp, (float)decay, qp, kp, vp,
                          (const float*)ksp, (const float*)vsp, (const int32_t*)bp, (const int32_t*)lp, (const int32_t*)qsp, op,
                          c.ws_ptr, c.ws_room, c.stream, nullptr, nullptr));
    return answer(st, a[9], fresh);
  });
}

// page_evict(refs, block_table, seq_lens, weights, budget, sink, recent, dropped, workspace, stream): the dropped
// tensor, a status, or None
PyObject* layer_page_evict(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  if (n != 10) return PyErr_Format(PyExc_TypeError, "page_evict takes 10 arguments");
  const Layer* L = (const Layer*)self;
  return guarded([&]() -> PyObject* {
    Call c;
    const Tensor *refs, *weights = tensor(a[3]);
    int64_t B;
    int32_t budget, sink, recent;
    if (!budget_of(a + 4, &budget, &sink, &recent) || !page_common(L, c, a, a[8], a[9], &refs, &B) ||
        !shaped(weights, c.dev, at::kFloat, {B, L->max_pages}) || derived(*weights))
      return nullptr;
    Tensor fresh;
    if (a[7] == Py_None) fresh = empty_on({B}, refs->options(), c.dev, a[9], c.stream);
    const Tensor* dropped = a[7] == Py_None ? &fresh : tensor(a[7]);
    if (!shaped(dropped, c.dev, at::kInt, {B})) return nullptr;
    if (a[7] != Py_None) mark_written(*dropped);
    mark_written(*weights);
    void *rp = ptr(refs), *bp = ptr(c.bt), *lp = ptr(c.lens), *wp = ptr(weights), *dp = ptr(dropped);
    WITHOUT_GIL(g_page_evict(L->handle, (int32_t)B, (int32_t)c.npages, (int32_t*)rp, (int32_t*)bp, (int32_t*)lp, (float*)wp, budget,
                             sink, recent, (int32_t*)dp, c.ws_ptr, c.ws_room, c.stream));
    return answer(st, a[7], fresh);
  });
}

PyMethodDef layer_methods[] = {
    {"run", (PyCFunction)(void*)layer_run, METH_FASTCALL, nullptr},
    {"grouped", (PyCFunction)(void*)layer_grouped, METH_FASTCALL, nullptr},
    {"multi", (PyCFunction)(void*)layer_multi, METH_FASTCALL, nullptr},
    {"noalloc", (PyCFunction)(void*)layer_noalloc, METH_FASTCALL, nullptr},
    {"append", (PyCFunction)(void*)layer_append, METH_FASTCALL, nullptr},
    {"scored", (PyCFunction)(void*)layer_scored, METH_FASTCALL, nullptr},
    {"append_rotary", (PyCFunction)(void*)layer_append_rotary, METH_FASTCALL, nullptr},
    {"page_grow", (PyCFunction)(void*)layer_page_grow, METH_FASTCALL, nullptr},
    {"page_release", (PyCFunction)(void*)layer_page_release, METH_FASTCALL, nullptr},
    {"page_fork", (PyCFunction)(void*)layer_page_fork, METH_FASTCALL, nullptr},
    {"page_compact", (PyCFunction)(void*)layer_page_compact, METH_FASTCALL, nullptr},
    {"page_bounds", (PyCFunction)(void*)layer_page_bounds, METH_FASTCALL, nullptr},
    {"select_pages", (PyCFunction)(void*)layer_select_pages, METH_FASTCALL, nullptr},
    {"selected", (PyCFunction)(void*)layer_selected, METH_FASTCALL, nullptr},
    {"weighed", (PyCFunction)(void*)layer_weighed, METH_FASTCALL, nullptr},
    {"page_evict", (PyCFunction)(void*)layer_page_evict, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

void layer_dealloc(PyObject* self) {
  Py_XDECREF(((Layer*)self)->workspaces);
  Py_XDECREF(((Layer*)self)->page_workspaces);
  Py_XDECREF(((Layer*)self)->weighed_workspaces);
  Py_TYPE(self)->tp_free(self);
}

// Layer(handle, workspaces, page workspaces, workspaces of weighed, (Hq, Hkv, d, page, max_batch, max_pages), (q, kv, out dtype codes),
//       (page, head, slot strides), workspace bytes, grouped workspace bytes)
PyObject* layer_new(PyTypeObject* type, PyObject* args, PyObject*) {
  unsigned long long handle = 0;
  PyObject *dict = nullptr, *pages = nullptr, *weighed = nullptr;
  long long v[6], s[3], ws = 0, gws = 0;
  int q = 0, kv = 0, out = 0;
  if (!PyArg_ParseTuple(args, "KO!O!O!(LLLLLL)(iii)(LLL)LL", &handle, &PyDict_Type, &dict, &PyDict_Type, &pages, &PyDict_Type,
                        &weighed, &v[0], &v[1], &v[2], &v[3], &v[4],
                        &v[5], &q, &kv, &out, &s[0], &s[1], &s[2], &ws, &gws))
    return nullptr;
  Layer* L = (Layer*)type->tp_alloc(type, 0);
  if (!L) return nullptr;
  L->handle = (rl_decode_attn_t)(uintptr_t)handle;
  Py_INCREF(dict);
  L->workspaces = dict;
  Py_INCREF(pages);
  L->page_workspaces = pages;
  Py_INCREF(weighed);
  L->weighed_workspaces = weighed;
  L->hq = v[0], L->hkv = v[1], L->d = v[2], L->page = v[3], L->max_batch = v[4], L->max_pages = v[5];
  for (int i = 0; i < 3; ++i) L->stride[i] = s[i];
  L->ws_bytes = ws;
  L->grouped_ws_bytes = gws;
  L->q_dtype = scalar_of(q);
  L->kv_dtype = scalar_of(kv);
  L->out_dtype = scalar_of(out);
  L->fp8 = kv == RLDA_FP8_E4M3FN;
  return (PyObject*)L;
}

PyTypeObject layer_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

// bind(raw_stream, run, grouped, multi, noalloc, append, scored, rotate, append_rotary, page_grow,
// page_release, page_fork, page_compact, page_bounds, select_pages, selected, weighed_size,
// weighed, page_evict): the stream lookup and the addresses of the loaded
// library's entry points.
PyObject* bind(PyObject*, PyObject* args) {
  PyObject* raw = nullptr;
  unsigned long long f[18];
  if (!PyArg_ParseTuple(args, "OKKKKKKKKKKKKKKKKKK", &raw, &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6], &f[7], &f[8], &f[9],
                        &f[10], &f[11], &f[12], &f[13], &f[14], &f[15], &f[16], &f[17]))
    return nullptr;
  Py_INCREF(raw);
  Py_XDECREF(g_raw_stream);
  g_raw_stream = raw;
  g_run = (decltype(g_run))(uintptr_t)f[0];
  g_grouped = (decltype(g_grouped))(uintptr_t)f[1];
  g_multi = (decltype(g_multi))(uintptr_t)f[2];
  g_noalloc = (decltype(g_noalloc))(uintptr_t)f[3];
  g_append = (decltype(g_append))(uintptr_t)f[4];
  g_scored = (decltype(g_scored))(uintptr_t)f[5];
  g_rotate = (decltype(g_rotate))(uintptr_t)f[6];
  g_append_rotary = (decltype(g_append_rotary))(uintptr_t)f[7];
  g_page_grow = (decltype(g_page_grow))(uintptr_t)f[8];
  g_page_release = (decltype(g_page_release))(uintptr_t)f[9];
  g_page_fork = (decltype(g_page_fork))(uintptr_t)f[10];
  g_page_compact = (decltype(g_page_compact))(uintptr_t)f[11];
  g_page_bounds = (decltype(g_page_bounds))(uintptr_t)f[12];
  g_select_pages = (decltype(g_select_pages))(uintptr_t)f[13];
  g_selected = (decltype(g_selected))(uintptr_t)f[14];
  g_weighed_size = (decltype(g_weighed_size))(uintptr_t)f[15];
  g_weighed = (decltype(g_weighed))(uintptr_t)f[16];
  g_page_evict = (decltype(g_page_evict))(uintptr_t)f[17];
  Py_RETURN_NONE;
}

PyMethodDef module_methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                                {"rotate", (PyCFunction)(void*)rotate, METH_FASTCALL, nullptr},
                                {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, module_methods};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) {
  layer_type.tp_name = "paper_2607_09207_amd._fastcall.Layer";
  layer_type.tp_basicsize = sizeof(Layer);
  layer_type.tp_flags = Py_TPFLAGS_DEFAULT;
  layer_type.tp_new = layer_new;
  layer_type.tp_dealloc = layer_dealloc;
  layer_type.tp_methods = layer_methods;
  if (PyType_Ready(&layer_type) < 0) return nullptr;
  for (int i = 0; i < kMaxDevices; ++i) {
    g_device_key[i] = PyUnicode_InternFromString(("cuda:" + std::to_string(i)).c_str());
    if (!g_device_key[i]) return nullptr;
  }
  PyObject* m = PyModule_Create(&module_def);
  if (!m) return nullptr;
  Py_INCREF(&layer_type);
  if (PyModule_AddObject(m, "Layer", (PyObject*)&layer_type) < 0) return nullptr;
  return m;
}
