// The short way from torch tensors to the calls of wf_kv.h, for sound arguments: checks,
// outputs and call without an interpreter step between.  Every function returns None
// where an argument is not plainly as wanted (the caller's Python path then takes it, or
// says what is wrong), a status where the call failed, else the outputs.
#include <Python.h>

#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <climits>
#include <cstdint>

#include "wf_kv.h"

namespace {

// The library's calls, by address: the binding loads it itself.
decltype(&wf_kv_step) g_step;
decltype(&wf_kv_store) g_store;
decltype(&wf_kv_load) g_load;
decltype(&wf_kv_attend) g_attend;
decltype(&wf_kv_fork) g_fork;
decltype(&wf_kv_release) g_release;
decltype(&wf_kv_compact) g_compact;
decltype(&wf_kv_copy) g_copy;

struct Geometry {
  wf_kv_ctx* ctx;
  int64_t device, q_heads, kv_heads, d, n_blocks, max_blocks, cache_bytes;
  at::ScalarType type;
};

constexpr const char* kName = "wf_kv.Geometry";

// Positional arguments, taken in order; `ok` falls where one is not as wanted.
struct Args {
  PyObject* const* at;
  const Geometry* g;
  bool ok;
  Args(PyObject* const* args, Py_ssize_t given, Py_ssize_t wanted) : at(args), g(nullptr), ok(given == wanted) {
    if (ok) g = static_cast<const Geometry*>(PyCapsule_GetPointer(*at++, kName));
    if (!g) ok = false;
  }
  int64_t integer(int64_t low, int64_t high) {
    if (!ok) return 0;
    PyObject* x = *at++;
    if (!PyLong_CheckExact(x)) return ok = false;
    int over = 0;
    const int64_t n = PyLong_AsLongLongAndOverflow(x, &over);
    if (over || n < low || n > high) ok = false;
    return n;
  }
  int32_t count() { return (int32_t)integer(0, INT32_MAX); }
  void* address() {
    if (!ok) return nullptr;
    PyObject* x = *at++;
    if (!PyLong_CheckExact(x)) return ok = false, nullptr;
    const unsigned long long p = PyLong_AsUnsignedLongLong(x);
    if (PyErr_Occurred()) ok = false;
    return reinterpret_cast<void*>((uintptr_t)p);
  }
  float real() {
    if (!ok) return 0;
    PyObject* x = *at++;
    if (!PyFloat_CheckExact(x)) return ok = false;
    return (float)PyFloat_AS_DOUBLE(x);
  }
  bool truth() {
    if (!ok) return false;
    PyObject* x = *at++;
    if (!PyBool_Check(x)) return ok = false;
    return x == Py_True;
  }
  // A tensor of the context's device; null with `ok` kept for None where that is allowed.
  const at::Tensor* tensor(at::ScalarType type, bool optional = false) {
    if (!ok) return nullptr;
    PyObject* x = *at++;
    if (optional && x == Py_None) return nullptr;
    if (!THPVariable_Check(x)) return ok = false, nullptr;
    const at::Tensor& t = THPVariable_Unpack(x);
    if (t.layout() != at::kStrided || t.scalar_type() != type || !t.is_cuda() || t.get_device() != g->device)
      return ok = false, nullptr;
    return &t;
  }
  // ... that is dense and has `numel` elements at least.
  const at::Tensor* dense(at::ScalarType type, bool optional = false) {
    const at::Tensor* t = tensor(type, optional);
    if (t && !t->is_contiguous()) ok = false;
    return t;
  }
  void holds(const at::Tensor* t, int64_t numel) {
    if (ok && t && t->numel() < numel) ok = false;
  }
  // ... whose rows, where it has several axes, are `pitch` elements apart.
  void rows(const at::Tensor* t, int64_t pitch) {
    if (ok && t && t->dim() > 1 && t->numel() != t->size(0) * pitch) ok = false;
  }
  // ... of `layers` caches, one after the other (axes that say otherwise, or nothing, are for the caller).
  void caches(const at::Tensor* t, int64_t layers) {
    holds(t, std::max<int64_t>(layers, 1) * g->cache_bytes);
    if (!ok || layers < 2 || t->dim() < 2 || t->numel() == layers * g->cache_bytes) return;
    ok = false;
    for (const int64_t apart : t->strides()) ok |= apart == g->cache_bytes;
  }
  // [n, heads, D] with dense heads; its token stride.
  int64_t tokens(const at::Tensor* t, int64_t n, int64_t heads) {
    if (!ok) return 0;
    if (t->dim() != 3 || t->size(0) != n || t->size(1) != heads || t->size(2) != g->d || t->stride(2) != 1 ||
        t->stride(1) != g->d)
      return ok = false;
    return n > 1 ? t->stride(0) : heads * g->d;
  }
};

void* data(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

PyObject* none() {
  if (PyErr_Occurred()) PyErr_Clear();
  Py_RETURN_NONE;
}

// A call of the library, which may wait for a place in a full queue: other threads of the
// interpreter go on meanwhile.
template <class F, class... A>
wf_status queued(F call, A... args) {
  PyThreadState* thread = PyEval_SaveThread();
  const wf_status st = call(args...);
  PyEval_RestoreThread(thread);
  return st;
}

at::Tensor fresh(const at::Tensor& like, at::IntArrayRef shape, at::ScalarType type) {
  return at::empty(shape, like.options().dtype(type));
}

// A part of an array of one dimension as a tensor of its own: what narrow() and view() give, without their dispatch (a fork and
// its copies 10.0 -> 8.9 us from Python, a compaction 10.3 -> 9.2).
at::Tensor part(const at::Tensor& flat, int64_t from, at::IntArrayRef shape) {
  at::Tensor out = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(flat.storage()), flat.key_set(), flat.dtype());
  c10::TensorImpl* impl = out.unsafeGetTensorImpl();
  impl->set_storage_offset(flat.storage_offset() + from);
  impl->set_sizes_contiguous(shape);
  return out;
}

// The outputs as a tuple.
template <size_t N>
PyObject* wrapped(const at::Tensor (&out)[N]) {
  PyObject* tuple = PyTuple_New(N);
  if (!tuple) return nullptr;
  for (size_t i = 0; i < N; ++i) {
    PyObject* x = THPVariable_Wrap(out[i]);
    if (!x) {
      Py_DECREF(tuple);
      return nullptr;
    }
    PyTuple_SET_ITEM(tuple, i, x);
  }
  return tuple;
}

// new, n_tokens, lens, pool, ring, table -> (lens, pool, q_off, slot, pos, granted)
PyObject* step(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 8);
  void* stream = a.address();
  const at::Tensor* new_tokens = a.dense(at::kInt);
  const int32_t tokens = a.count();
  const at::Tensor *lens = a.dense(at::kInt), *pool = a.dense(at::kInt), *ring = a.dense(at::kInt), *table = a.dense(at::kInt);
  if (!a.ok || new_tokens->dim() != 1 || new_tokens->size(0) > WF_KV_MAX_ROWS) return none();
  const int64_t r = new_tokens->size(0);
  a.holds(lens, r);
  a.holds(pool, 2);
  a.holds(ring, a.g->n_blocks);
  a.holds(table, r * a.g->max_blocks);
  a.rows(table, a.g->max_blocks);
  if (!a.ok) return none();
  at::AutoDispatchBelowADInplaceOrView plain;
  const at::Tensor flat = fresh(*new_tokens, {2 * r + 3 + tokens}, at::kInt);
  const at::Tensor out[6] = {flat.narrow(0, 0, r), flat.narrow(0, r, 2), flat.narrow(0, r + 2, r + 1),
                             fresh(*new_tokens, {tokens}, at::kLong), flat.narrow(0, 2 * r + 3, tokens),
                             fresh(*new_tokens, {r}, at::kByte)};
  int32_t* base = static_cast<int32_t*>(flat.data_ptr());
  const wf_status st =
      queued(g_step, a.g->ctx, (const int32_t*)data(new_tokens), (int32_t)r, tokens, (const int32_t*)data(lens), base,
             (const int32_t*)data(pool), base + r, (int32_t*)data(ring), (int32_t*)data(table), base + r + 2,
             (int64_t*)data(&out[3]), base + 2 * r + 3, (uint8_t*)data(&out[5]), stream);
  if (st != WF_OK) return PyLong_FromLong(st);
  return wrapped(out);
  END_HANDLE_TH_ERRORS
}

// q, k, v, pos, slot, cache, cos_sin, rot_dim, interleaved, q_weight, k_weight, eps -> q
PyObject* store(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 14);
  if (!a.ok) return none();
  void* stream = a.address();
  const at::Tensor *q = a.tensor(a.g->type), *k = a.tensor(a.g->type), *v = a.tensor(a.g->type);
  const at::Tensor *pos = a.dense(at::kInt, true), *slot = a.dense(at::kLong), *cache = a.dense(at::kByte);
  const at::Tensor* cos_sin = a.dense(at::kFloat, true);
  const int32_t rot = a.count();
  const bool interleaved = a.truth();
  const at::Tensor *qw = a.dense(a.g->type, true), *kw = a.dense(a.g->type, true);
  const float eps = a.real();
  if (!a.ok || q->dim() != 3 || q->size(0) > INT32_MAX || (cos_sin && (cos_sin->dim() < 1 || cos_sin->size(0) > INT32_MAX)))
    return none();
  const int64_t t = q->size(0), qs = a.tokens(q, t, a.g->q_heads), ks = a.tokens(k, t, a.g->kv_heads),
                vs = a.tokens(v, t, a.g->kv_heads), n_pos = cos_sin ? cos_sin->size(0) : 0;
  a.holds(pos, t);
  a.holds(slot, t);
  a.holds(cache, a.g->cache_bytes);
  a.holds(cos_sin, n_pos * rot);
  if (rot) a.rows(cos_sin, rot);
  a.holds(qw, a.g->d);
  a.holds(kw, a.g->d);
  if (!a.ok) return none();
  at::AutoDispatchBelowADInplaceOrView plain;
  const at::Tensor out = fresh(*q, {t, a.g->q_heads, a.g->d}, a.g->type);
  const wf_kv_norm_rope how = {data(qw), data(kw), eps, rot, interleaved, (int32_t)n_pos, (const float*)data(cos_sin)};
  const wf_status st = queued(g_store, a.g->ctx, data(q), data(k), data(v), qs, ks, vs, (int32_t)t, &how, (const int32_t*)data(pos),
                               (const int64_t*)data(slot), data(&out), (uint8_t*)data(cache), stream);
  if (st != WF_OK) return PyLong_FromLong(st);
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// cache, slot -> (k, v)
PyObject* load(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 4);
  void* stream = a.address();
  const at::Tensor *cache = a.dense(at::kByte), *slot = a.dense(at::kLong);
  if (!a.ok || slot->dim() != 1 || slot->size(0) > INT32_MAX) return none();
  a.holds(cache, a.g->cache_bytes);
  if (!a.ok) return none();
  const int64_t t = slot->size(0);
  at::AutoDispatchBelowADInplaceOrView plain;
  const at::Tensor k = fresh(*slot, {t, a.g->kv_heads, a.g->d}, a.g->type), v = fresh(*slot, {t, a.g->kv_heads, a.g->d}, a.g->type);
  const wf_status st = queued(g_load, a.g->ctx, (const uint8_t*)data(cache), (const int64_t*)data(slot), (int32_t)t, data(&k), data(&v), stream);
  if (st != WF_OK) return PyLong_FromLong(st);
  PyObject *x = THPVariable_Wrap(k), *y = THPVariable_Wrap(v);
  PyObject* pair = x && y ? PyTuple_Pack(2, x, y) : nullptr;
  Py_XDECREF(x);
  Py_XDECREF(y);
  return pair;
  END_HANDLE_TH_ERRORS
}

// q, cache, table, kv_len, q_off, pos, scale, window, max_q, max_kv -> out
PyObject* attend(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 12);
  if (!a.ok) return none();
  void* stream = a.address();
  const at::Tensor *q = a.tensor(a.g->type), *cache = a.dense(at::kByte), *table = a.dense(at::kInt);
  const at::Tensor *kv_len = a.dense(at::kInt), *q_off = a.dense(at::kInt), *pos = a.dense(at::kInt);
  const float scale = a.real();
  const int32_t window = a.count(), max_q = a.count(), max_kv = a.count();
  if (!a.ok || q->dim() != 3 || q->size(0) > INT32_MAX || kv_len->dim() != 1 || kv_len->size(0) > WF_KV_MAX_ROWS) return none();
  const int64_t t = q->size(0), r = kv_len->size(0), qs = a.tokens(q, t, a.g->q_heads);
  a.holds(cache, a.g->cache_bytes);
  a.holds(table, r * a.g->max_blocks);
  a.rows(table, a.g->max_blocks);
  a.holds(q_off, r + 1);
  a.holds(pos, t);
  if (!a.ok) return none();
  at::AutoDispatchBelowADInplaceOrView plain;
  const at::Tensor out = fresh(*q, {t, a.g->q_heads, a.g->d}, a.g->type);
  const wf_status st = queued(g_attend, a.g->ctx, data(q), qs, (int32_t)t, (const uint8_t*)data(cache), (const int32_t*)data(table),
                                (const int32_t*)data(kv_len), (const int32_t*)data(q_off), (const int32_t*)data(pos), (int32_t)r,
                                scale, window, max_q, max_kv, data(&out), stream);
  if (st != WF_OK) return PyLong_FromLong(st);
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// The arrays of a batch that shares blocks: lens, pool, ring, table, shared, as the calls take them.
struct Batch {
  const at::Tensor *lens, *pool, *ring, *table, *shared;
  int64_t rows = 0;
  explicit Batch(Args& a)
      : lens(a.dense(at::kInt)), pool(a.dense(at::kInt)), ring(a.dense(at::kInt)), table(a.dense(at::kInt)), shared(a.dense(at::kInt)) {
    if (!a.ok) return;
    if (lens->dim() != 1 || lens->size(0) > WF_KV_MAX_ROWS) {
      a.ok = false;
      return;
    }
    rows = lens->size(0);
    a.holds(pool, 2);
    a.holds(ring, a.g->n_blocks);
    a.holds(table, rows * a.g->max_blocks);
    a.rows(table, a.g->max_blocks);
    a.holds(shared, a.g->n_blocks);
  }
  static const int32_t* in(const at::Tensor* t) { return (const int32_t*)data(t); }
  static int32_t* out(const at::Tensor* t) { return (int32_t*)data(t); }
};

// src, dst, tokens, lens, pool, ring, table, shared -> (lens, pool, shared, granted, moves)
PyObject* fork(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 10);
  void* stream = a.address();
  const at::Tensor *src = a.dense(at::kInt), *dst = a.dense(at::kInt), *tokens = a.dense(at::kInt);
  const Batch b(a);
  if (!a.ok || src->dim() != 1 || dst->dim() != 1 || tokens->dim() != 1 || src->size(0) > WF_KV_MAX_FORKS ||
      dst->size(0) != src->size(0) || tokens->size(0) != src->size(0))
    return none();
  const int64_t f = src->size(0), r = b.rows, blocks = a.g->n_blocks;
  at::AutoDispatchBelowADInplaceOrView plain;
  const at::Tensor flat = fresh(*b.lens, {r + 2 + blocks + 2 * f}, at::kInt);
  int32_t* base = static_cast<int32_t*>(flat.data_ptr());
  int32_t *pool = base + r, *shared = pool + 2, *moves = shared + blocks;
  const at::Tensor out[5] = {part(flat, 0, {r}), part(flat, r, {2}), part(flat, r + 2, {blocks}), fresh(*b.lens, {f}, at::kByte),
                             part(flat, r + 2 + blocks, {2, f})};
  const wf_status st = queued(g_fork, a.g->ctx, Batch::in(src), Batch::in(dst), Batch::in(tokens), (int32_t)f, (int32_t)r, Batch::in(b.lens), base,
                              Batch::in(b.pool), pool, Batch::in(b.ring), Batch::out(b.table), Batch::in(b.shared), shared, moves, moves + f,
                              (uint8_t*)data(&out[3]), (int32_t*)nullptr, stream);
  if (st != WF_OK) return PyLong_FromLong(st);
  return wrapped(out);
  END_HANDLE_TH_ERRORS
}

// release, lens, pool, ring, table, shared -> (lens, pool, shared)
PyObject* release(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 8);
  void* stream = a.address();
  const at::Tensor* ends = a.dense(at::kByte);
  const Batch b(a);
  a.holds(ends, b.rows);
  if (!a.ok) return none();
  const int64_t r = b.rows, blocks = a.g->n_blocks;
  at::AutoDispatchBelowADInplaceOrView plain;
  const at::Tensor flat = fresh(*b.lens, {r + 2 + blocks + WF_KV_PAGES_WORK}, at::kInt);
  int32_t* base = static_cast<int32_t*>(flat.data_ptr());
  const at::Tensor out[3] = {part(flat, 0, {r}), part(flat, r, {2}), part(flat, r + 2, {blocks})};
  const wf_status st = queued(g_release, a.g->ctx, (const uint8_t*)data(ends), (int32_t)r, Batch::in(b.lens), base, Batch::in(b.pool), base + r,
                              Batch::out(b.ring), Batch::in(b.table), Batch::in(b.shared), base + r + 2, base + r + 2 + blocks, stream);
  if (st != WF_OK) return PyLong_FromLong(st);
  return wrapped(out);
  END_HANDLE_TH_ERRORS
}

// keep, lens, pool, ring, table, shared -> (pool, ring, shared, done, moves)
PyObject* compact(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 8);
  if (!a.ok) return none();
  void* stream = a.address();
  const int64_t k = a.integer(1, a.g->n_blocks - 1);
  const Batch b(a);
  if (!a.ok) return none();
  const int64_t blocks = a.g->n_blocks, m = k < blocks - k ? k : blocks - k;
  at::AutoDispatchBelowADInplaceOrView plain;
  const at::Tensor flat = fresh(*b.lens, {2 + 2 * k + 2 * m + 1 + blocks + WF_KV_PAGES_WORK}, at::kInt);
  int32_t* base = static_cast<int32_t*>(flat.data_ptr());
  int32_t *ring = base + 2, *shared = ring + k, *moves = shared + k, *done = moves + 2 * m, *ids = done + 1, *work = ids + blocks;
  const at::Tensor out[5] = {part(flat, 0, {2}), part(flat, 2, {k}), part(flat, 2 + k, {k}), part(flat, 2 + 2 * k + 2 * m, {1}),
                             part(flat, 2 + 2 * k, {2, m})};
  const wf_status st = queued(g_compact, a.g->ctx, (int32_t)k, (int32_t)b.rows, Batch::in(b.lens), Batch::in(b.pool), base, Batch::in(b.ring), ring,
                              Batch::out(b.table), Batch::in(b.shared), shared, moves, moves + m, done, ids, work, stream);
  if (st != WF_OK) return PyLong_FromLong(st);
  return wrapped(out);
  END_HANDLE_TH_ERRORS
}

// cache, moves, layers -> True
PyObject* copy(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 5);
  if (!a.ok) return none();
  void* stream = a.address();
  const at::Tensor *cache = a.dense(at::kByte), *moves = a.dense(at::kInt);
  const int64_t layers = a.integer(0, WF_KV_MAX_LAYERS);
  if (!a.ok || moves->dim() != 2 || moves->size(0) != 2 || moves->size(1) > WF_KV_MAX_BLOCKS) return none();
  a.caches(cache, layers);
  if (!a.ok) return none();
  const int64_t m = moves->size(1);
  const wf_status st = queued(g_copy, a.g->ctx, (uint8_t*)data(cache), a.g->cache_bytes, (int32_t)layers, Batch::in(moves), Batch::in(moves) + m,
                              (int32_t)m, stream);
  if (st != WF_OK) return PyLong_FromLong(st);
  Py_RETURN_TRUE;
  END_HANDLE_TH_ERRORS
}

void drop(PyObject* capsule) { delete static_cast<Geometry*>(PyCapsule_GetPointer(capsule, kName)); }

// geometry(ctx, device, q_heads, kv_heads, head_dim, n_blocks, max_blocks, cache_bytes, f16): what the
// calls take first.  Not to be used once the context is destroyed.
PyObject* geometry(PyObject*, PyObject* args) {
  unsigned long long ctx;
  long long device, hq, hk, d, n, width, bytes;
  int f16;
  if (!PyArg_ParseTuple(args, "KLLLLLLLp", &ctx, &device, &hq, &hk, &d, &n, &width, &bytes, &f16)) return nullptr;
  Geometry* g = new (std::nothrow) Geometry{reinterpret_cast<wf_kv_ctx*>((uintptr_t)ctx), device, hq, hk, d, n, width, bytes,
                                            f16 ? at::kHalf : at::kBFloat16};
  if (!g) return PyErr_NoMemory();
  PyObject* c = PyCapsule_New(g, kName, drop);
  if (!c) delete g;
  return c;
}

// calls(step, store, load, attend): their addresses in the loaded library.
PyObject* calls(PyObject*, PyObject* args) {
  unsigned long long s, t, l, a;
  if (!PyArg_ParseTuple(args, "KKKK", &s, &t, &l, &a)) return nullptr;
  g_step = reinterpret_cast<decltype(g_step)>((uintptr_t)s);
  g_store = reinterpret_cast<decltype(g_store)>((uintptr_t)t);
  g_load = reinterpret_cast<decltype(g_load)>((uintptr_t)l);
  g_attend = reinterpret_cast<decltype(g_attend)>((uintptr_t)a);
  Py_RETURN_NONE;
}

// page_calls(fork, release, compact, copy): likewise.
PyObject* page_calls(PyObject*, PyObject* args) {
  unsigned long long f, r, c, k;
  if (!PyArg_ParseTuple(args, "KKKK", &f, &r, &c, &k)) return nullptr;
  g_fork = reinterpret_cast<decltype(g_fork)>((uintptr_t)f);
  g_release = reinterpret_cast<decltype(g_release)>((uintptr_t)r);
  g_compact = reinterpret_cast<decltype(g_compact)>((uintptr_t)c);
  g_copy = reinterpret_cast<decltype(g_copy)>((uintptr_t)k);
  Py_RETURN_NONE;
}

template <class F>
PyCFunction fast(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f));
}

PyMethodDef g_methods[] = {{"step", fast(step), METH_FASTCALL, nullptr},
                           {"store", fast(store), METH_FASTCALL, nullptr},
                           {"load", fast(load), METH_FASTCALL, nullptr},
                           {"attend", fast(attend), METH_FASTCALL, nullptr},
                           {"fork", fast(fork), METH_FASTCALL, nullptr},
                           {"release", fast(release), METH_FASTCALL, nullptr},
                           {"compact", fast(compact), METH_FASTCALL, nullptr},
                           {"copy", fast(copy), METH_FASTCALL, nullptr},
                           {"geometry", geometry, METH_VARARGS, nullptr},
                           {"calls", calls, METH_VARARGS, nullptr},
                           {"page_calls", page_calls, METH_VARARGS, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_kvbind", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__kvbind() { return PyModule_Create(&g_module); }
