// Native marshalling of the calls a decode step makes many times: the argument
// checks of the Python binding (device placement, dtype, contiguity, element
// counts) and the call into liboasis.so in one extension call.
//
// Each function takes the arguments of the binding's function of that name and
// returns the library's status, or None when it does not accept them exactly as
// they are (an argument of another type, a tensor subclass, a failed check, a
// null argument that some sizes allow): the binding's Python code then handles
// the call, so that every error and every unusual form stays there. Nothing is
// kept between calls. Measured on the host of an MI355X, the attention call's
// marshalling takes 6.2 us in Python and 0.4 us here, more than a launch.
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "oasis.h"

namespace {

decltype(&oasis_sparse_decode_attn) f_attn;
decltype(&oasis_score_blocks) f_score;
decltype(&oasis_select_topk) f_topk;
decltype(&oasis_score_select) f_score_select;
decltype(&oasis_stage_blocks) f_stage;
decltype(&oasis_tree_attn) f_tree;
decltype(&oasis_sparse_tree_attn) f_sparse_tree;
decltype(&oasis_verify_drafts) f_verify;
decltype(&oasis_append_tokens) f_append;

enum Kind { kBf16, kI32, kF32, kU8 };

bool dtype_is(at::ScalarType t, Kind k) {
  switch (k) {
    case kBf16: return t == at::kBFloat16 || t == at::kUInt16 || t == at::kShort;  // bf16 bits in any 16-bit dtype
    case kI32: return t == at::kInt;
    case kF32: return t == at::kFloat;
    default: return t == at::kByte;
  }
}

// Product of counts; -1, which no tensor matches, with a negative factor or past 63 bits.
int64_t count(std::initializer_list<int64_t> factors) {
  int64_t n = 1;
  bool bad = false;
  for (const int64_t f : factors) bad |= f < 0 || __builtin_mul_overflow(n, f, &n);
  return bad ? -1 : n;
}

// The data of a plain contiguous tensor on the device or, where pinned memory is
// allowed, pinned; false: not such a tensor.
bool any_count(PyObject* o, Kind kind, void** p, bool pinned_ok = false) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!dtype_is(t.scalar_type(), kind) || !t.is_contiguous()) return false;
  if (!t.is_cuda() && !(pinned_ok && t.is_pinned())) return false;
  *p = t.data_ptr();
  return true;
}
// The same, of exactly n elements.
bool tensor(PyObject* o, int64_t n, Kind kind, void** p, bool pinned_ok = false) {
  return THPVariable_CheckExact(o) && THPVariable_Unpack(o).numel() == n && any_count(o, kind, p, pinned_ok);
}

bool int32(PyObject* o, int32_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int overflow = 0;
  const long long x = PyLong_AsLongLongAndOverflow(o, &overflow);
  if (overflow || x < INT32_MIN || x > INT32_MAX) return false;
  *v = (int32_t)x;
  return true;
}

// The dims structure (its address, taken by the binding) and the stream: a handle or None, the current stream.
const oasis_dims* dims_at(PyObject* o) { return static_cast<const oasis_dims*>(PyLong_AsVoidPtr(o)); }
bool stream_at(PyObject* o, void** s) {
  if (o == Py_None) {
    *s = c10::hip::getCurrentHIPStream().stream();
    return true;
  }
  if (!PyLong_CheckExact(o)) return false;
  *s = PyLong_AsVoidPtr(o);
  return !PyErr_Occurred();
}

#define FALLBACK             \
  do {                       \
    if (PyErr_Occurred()) PyErr_Clear(); \
    Py_RETURN_NONE;          \
  } while (0)

// Runs `call` without the GIL (a full queue blocks the launch) and returns its status.
template <typename F>
PyObject* run(F&& call) {
  oasis_status st;
  Py_BEGIN_ALLOW_THREADS
  st = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong((long)st);
}

// No C++ exception (a tensor without storage throws) leaves an entry.
template <typename F>
PyObject* guarded(F&& body) {
  try {
    return body();
  } catch (...) {
    FALLBACK;
  }
}

using Args = PyObject* const*;

// dims, q, num_q_tokens, pool_k, pool_v, slot_map, k_slots, ctx_len, scale, out, lse, workspace, stream
PyObject* sparse_decode_attn(PyObject*, Args a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 13) FALLBACK;
    const oasis_dims* d = dims_at(a[0]);
    int32_t T, k;
    if (!d || !int32(a[2], &T) || !int32(a[6], &k)) FALLBACK;
    const int64_t R = d->num_reqs, H = d->num_kv_heads, D = d->head_dim;
    const int64_t rows = count({R, T, d->num_q_heads}), qn = count({R, T, d->num_q_heads, D});
    const int64_t pool = count({R, (int64_t)k + 1, H, d->block_size, D});
    void *q, *pk, *pv, *map, *ctx, *out, *lse = nullptr, *ws, *s;
    float scale;
    if (D <= 0) FALLBACK;  // no default scale
    if (a[8] == Py_None) scale = (float)(1.0 / std::sqrt((double)D));
    else if (PyFloat_CheckExact(a[8])) scale = (float)PyFloat_AS_DOUBLE(a[8]);
    else FALLBACK;
    if (!tensor(a[1], qn, kBf16, &q) || !tensor(a[3], pool, kBf16, &pk) || !tensor(a[4], pool, kBf16, &pv) ||
        !tensor(a[5], count({R, H, k}), kI32, &map) || !tensor(a[7], R, kI32, &ctx) || !tensor(a[9], qn, kBf16, &out) ||
        (a[10] != Py_None && !tensor(a[10], rows, kF32, &lse)) || !any_count(a[11], kU8, &ws) ||
        !stream_at(a[12], &s))
      FALLBACK;
    const size_t bytes = (size_t)THPVariable_Unpack(a[11]).numel();
    return run([&] {
      return f_attn(d, (const uint16_t*)q, T, (const uint16_t*)pk, (const uint16_t*)pv, (const int32_t*)map, k,
                    (const int32_t*)ctx, scale, (uint16_t*)out, (float*)lse, ws, bytes, s);
    });
  });
}

struct Score {
  int32_t T, first, num;
  void *q, *kmax, *kmin, *ctx, *scores;
};
// q, num_q_tokens, first_draft, num_draft, kmax, kmin, ctx_len at a[1..7]; scores at a[scores]
bool score_args(const oasis_dims* d, Args a, int scores, Score* s) {
  if (!d || !int32(a[2], &s->T) || !int32(a[3], &s->first) || !int32(a[4], &s->num)) return false;
  const int64_t R = d->num_reqs, H = d->num_kv_heads, NB = d->max_blocks, D = d->head_dim;
  const int64_t summary = count({R, H, NB, D});
  return tensor(a[1], count({R, s->T, d->num_q_heads, D}), kBf16, &s->q) && tensor(a[5], summary, kBf16, &s->kmax) &&
         tensor(a[6], summary, kBf16, &s->kmin) && tensor(a[7], R, kI32, &s->ctx) &&
         tensor(a[scores], count({R, H, NB}), kF32, &s->scores);
}

// dims, q, num_q_tokens, first_draft, num_draft, kmax, kmin, ctx_len, scores, stream
PyObject* score_blocks(PyObject*, Args a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 10) FALLBACK;
    const oasis_dims* d = dims_at(a[0]);
    Score c;
    void* s;
    if (!score_args(d, a, 8, &c) || !stream_at(a[9], &s)) FALLBACK;
    return run([&] {
      return f_score(d, (const uint16_t*)c.q, c.T, c.first, c.num, (const uint16_t*)c.kmax, (const uint16_t*)c.kmin,
                     (const int32_t*)c.ctx, (float*)c.scores, s);
    });
  });
}

// dims, scores, ctx_len, k, sel, sel_count, stream
PyObject* select_topk(PyObject*, Args a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 7) FALLBACK;
    const oasis_dims* d = dims_at(a[0]);
    int32_t k;
    void *scores, *ctx, *sel, *cnt, *s;
    if (!d || !int32(a[3], &k)) FALLBACK;
    const int64_t R = d->num_reqs, RH = count({R, d->num_kv_heads});
    if (!tensor(a[1], count({RH, d->max_blocks}), kF32, &scores) || !tensor(a[2], R, kI32, &ctx) ||
        !tensor(a[4], count({RH, k}), kI32, &sel) || !tensor(a[5], RH, kI32, &cnt) || !stream_at(a[6], &s))
      FALLBACK;
    return run([&] {
      return f_topk(d, (const float*)scores, (const int32_t*)ctx, k, (int32_t*)sel, (int32_t*)cnt, s);
    });
  });
}

// dims, q, num_q_tokens, first_draft, num_draft, kmax, kmin, ctx_len, k, scores, sel, sel_count, stream
PyObject* score_select(PyObject*, Args a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 13) FALLBACK;
    const oasis_dims* d = dims_at(a[0]);
    Score c;
    int32_t k;
    void *sel, *cnt, *s;
    if (!score_args(d, a, 9, &c) || !int32(a[8], &k)) FALLBACK;
    const int64_t RH = count({d->num_reqs, d->num_kv_heads});
    if (!tensor(a[10], count({RH, k}), kI32, &sel) || !tensor(a[11], RH, kI32, &cnt) || !stream_at(a[12], &s)) FALLBACK;
    return run([&] {
      return f_score_select(d, (const uint16_t*)c.q, c.T, c.first, c.num, (const uint16_t*)c.kmax,
                            (const uint16_t*)c.kmin, (const int32_t*)c.ctx, k, (float*)c.scores, (int32_t*)sel,
                            (int32_t*)cnt, s);
    });
  });
}

// dims, host_k, host_v, num_pages, host_block_table, ctx_len, sel, sel_count, scores, k, slot_map, slot_stamp, step,
// fetch_cap, copy_local, pool_k, pool_v, moved, stream
PyObject* stage_blocks(PyObject*, Args a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 19) FALLBACK;
    const oasis_dims* d = dims_at(a[0]);
    int32_t pages, k, step, cap;
    if (!d || !int32(a[3], &pages) || !int32(a[9], &k) || !int32(a[12], &step) || !int32(a[13], &cap) ||
        (a[14] != Py_True && a[14] != Py_False))
      FALLBACK;
    const int64_t R = d->num_reqs, H = d->num_kv_heads, RH = count({R, H});
    const int64_t tier = count({pages, H, d->block_size, d->head_dim});
    const int64_t pool = count({RH, (int64_t)k + 1, d->block_size, d->head_dim}), items = count({RH, k});
    void *hk, *hv, *table, *ctx, *sel, *cnt, *scores, *map, *stamp, *pk, *pv, *moved, *s;
    if (!tensor(a[1], tier, kBf16, &hk, true) || !tensor(a[2], tier, kBf16, &hv, true) ||
        !tensor(a[4], count({R, d->max_blocks}), kI32, &table) || !tensor(a[5], R, kI32, &ctx) ||
        !tensor(a[6], items, kI32, &sel) || !tensor(a[7], RH, kI32, &cnt) ||
        !tensor(a[8], count({RH, d->max_blocks}), kF32, &scores) || !tensor(a[10], items, kI32, &map) ||
        !tensor(a[11], items, kI32, &stamp) || !tensor(a[15], pool, kBf16, &pk) ||
        !tensor(a[16], pool, kBf16, &pv) || !tensor(a[17], RH, kI32, &moved) || !stream_at(a[18], &s))
      FALLBACK;
    const int32_t copy_local = a[14] == Py_True;
    return run([&] {
      return f_stage(d, (const uint16_t*)hk, (const uint16_t*)hv, pages, (const int32_t*)table, (const int32_t*)ctx,
                     (const int32_t*)sel, (const int32_t*)cnt, (const float*)scores, k, (int32_t*)map,
                     (int32_t*)stamp, step, cap, copy_local, (uint16_t*)pk, (uint16_t*)pv, (int32_t*)moved, s);
    });
  });
}

// The calls of the speculative step take tensors of the current device alone.
bool on_current(Args a, std::initializer_list<int> which) {
  const auto dev = c10::hip::current_device();
  for (const int i : which) {
    if (a[i] == Py_None) continue;
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    if (t.is_cuda() && t.device().index() != dev) return false;
  }
  return true;
}

// As tensor(), or None.
bool optional(PyObject* o, int64_t n, Kind kind, void** p) {
  *p = nullptr;
  return o == Py_None || tensor(o, n, kind, p);
}

// A workspace or None.
bool workspace_at(PyObject* o, void** p, size_t* bytes) {
  *p = nullptr;
  *bytes = 0;
  if (o == Py_None) return true;
  if (!any_count(o, kU8, p)) return false;
  *bytes = (size_t)THPVariable_Unpack(o).numel();
  return true;
}

bool scale_at(PyObject* o, int64_t D, float* scale) {
  if (D <= 0) return false;  // no default scale
  if (o == Py_None) *scale = (float)(1.0 / std::sqrt((double)D));
  else if (PyFloat_CheckExact(o)) *scale = (float)PyFloat_AS_DOUBLE(o);
  else return false;
  return true;
}

// Two tiers of the same shape, of whole pages [Hkv][B][d]: their number.
bool tier_at(PyObject* ko, PyObject* vo, const oasis_dims* d, void** k, void** v, int64_t* pages) {
  if (!any_count(ko, kBf16, k, true) || !any_count(vo, kBf16, v, true)) return false;
  const at::Tensor &kt = THPVariable_Unpack(ko), &vt = THPVariable_Unpack(vo);
  const int64_t per = count({d->num_kv_heads, d->block_size, d->head_dim});
  if (per < 1 || kt.dim() < 1 || kt.sizes() != vt.sizes() || kt.numel() % per) return false;
  *pages = kt.numel() / per;
  return true;
}

struct Tree {
  void *ctx, *tk, *tv, *parent, *len, *out, *lse, *ws, *s;
  size_t bytes;
  float scale;
};
// ctx_len, tree_k, tree_v, parent, tree_len, scale, out, lse, workspace, stream from a[0] on
bool tree_args(const oasis_dims* d, int32_t T, Args a, Tree* t) {
  const int64_t R = d->num_reqs, D = d->head_dim, rows = count({R, T, d->num_q_heads}), kv = count({R, T, d->num_kv_heads, D});
  return tensor(a[0], R, kI32, &t->ctx) && tensor(a[1], kv, kBf16, &t->tk) && tensor(a[2], kv, kBf16, &t->tv) &&
         optional(a[3], count({R, T}), kI32, &t->parent) && optional(a[4], R, kI32, &t->len) &&
         scale_at(a[5], D, &t->scale) && tensor(a[6], count({rows, D}), kBf16, &t->out) &&
         optional(a[7], rows, kF32, &t->lse) && workspace_at(a[8], &t->ws, &t->bytes) && stream_at(a[9], &t->s) &&
         on_current(a, {0, 1, 2, 3, 4, 6, 7, 8});
}

// dims, q, num_q_tokens, k_pages, v_pages, block_table, ctx_len, tree_k, tree_v, parent, tree_len, scale, out, lse,
// workspace, stream
PyObject* tree_attn(PyObject*, Args a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 16) FALLBACK;
    const oasis_dims* d = dims_at(a[0]);
    int32_t T;
    int64_t pages;
    void *q, *k, *v, *table;
    Tree t;
    if (!d || !int32(a[2], &T) || !tensor(a[1], count({d->num_reqs, T, d->num_q_heads, d->head_dim}), kBf16, &q) ||
        !tier_at(a[3], a[4], d, &k, &v, &pages) || !tensor(a[5], count({d->num_reqs, d->max_blocks}), kI32, &table) ||
        !tree_args(d, T, a + 6, &t) || !on_current(a, {1, 3, 4, 5}))
      FALLBACK;
    return run([&] {
      return f_tree(d, (const uint16_t*)q, T, (const uint16_t*)k, (const uint16_t*)v, pages, (const int32_t*)table,
                    (const int32_t*)t.ctx, (const uint16_t*)t.tk, (const uint16_t*)t.tv, (const int32_t*)t.parent,
                    (const int32_t*)t.len, t.scale, (uint16_t*)t.out, (float*)t.lse, t.ws, t.bytes, t.s);
    });
  });
}

// dims, q, num_q_tokens, pool_k, pool_v, slot_map, k_slots, ctx_len, tree_k, tree_v, parent, tree_len, scale, out, lse,
// workspace, stream
PyObject* sparse_tree_attn(PyObject*, Args a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 17) FALLBACK;
    const oasis_dims* d = dims_at(a[0]);
    int32_t T, ks;
    void *q, *k, *v, *map;
    Tree t;
    if (!d || !int32(a[2], &T) || !int32(a[6], &ks)) FALLBACK;
    const int64_t R = d->num_reqs, H = d->num_kv_heads;
    const int64_t pool = count({R, (int64_t)ks + 1, H, d->block_size, d->head_dim});
    if (!tensor(a[1], count({R, T, d->num_q_heads, d->head_dim}), kBf16, &q) || !tensor(a[3], pool, kBf16, &k) ||
        !tensor(a[4], pool, kBf16, &v) || !tensor(a[5], count({R, H, ks}), kI32, &map) ||
        !tree_args(d, T, a + 7, &t) || !on_current(a, {1, 3, 4, 5}))
      FALLBACK;
    return run([&] {
      return f_sparse_tree(d, (const uint16_t*)q, T, (const uint16_t*)k, (const uint16_t*)v, (const int32_t*)map, ks,
                           (const int32_t*)t.ctx, (const uint16_t*)t.tk, (const uint16_t*)t.tv, (const int32_t*)t.parent,
                           (const int32_t*)t.len, t.scale, (uint16_t*)t.out, (float*)t.lse, t.ws, t.bytes, t.s);
    });
  });
}

// Probabilities [R][T][V] of dense rows, evenly spaced: their address and row stride.
bool prob_rows(PyObject* o, int64_t R, int64_t T, int64_t V, void** p, int64_t* row) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.scalar_type() != at::kFloat || t.dim() != 3 || t.size(0) != R || t.size(1) != T || t.size(2) != V)
    return false;
  *row = T > 1 ? t.stride(1) : (R > 1 ? t.stride(0) : V);
  if ((V > 1 && t.stride(2) != 1) || *row < V || (R > 1 && t.stride(0) != T * *row)) return false;
  *p = t.data_ptr();
  return true;
}

// target_probs, draft_probs, tokens, parent, tree_len, accept_u, sample_u, path, path_len, out_tokens, workspace, stream
PyObject* verify_drafts(PyObject*, Args a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 12 || !THPVariable_CheckExact(a[0])) FALLBACK;
    const at::Tensor& target = THPVariable_Unpack(a[0]);
    if (target.dim() != 3) FALLBACK;
    const int64_t R = target.size(0), T = target.size(1), V = target.size(2), RT = count({R, T});
    if (R > INT32_MAX || T > INT32_MAX || V > INT32_MAX) FALLBACK;
    void *tp, *dp = nullptr, *tok, *par, *len, *ua, *us, *path, *plen, *out, *ws, *s;
    int64_t ts, ds = 0;
    size_t bytes;
    if (!prob_rows(a[0], R, T, V, &tp, &ts) || (a[1] != Py_None && !prob_rows(a[1], R, T, V, &dp, &ds)) ||
        !tensor(a[2], RT, kI32, &tok) || !optional(a[3], RT, kI32, &par) || !optional(a[4], R, kI32, &len) ||
        !tensor(a[5], RT, kF32, &ua) || !tensor(a[6], R, kF32, &us) || !tensor(a[7], RT, kI32, &path) ||
        !tensor(a[8], R, kI32, &plen) || !tensor(a[9], RT, kI32, &out) || !workspace_at(a[10], &ws, &bytes) ||
        !stream_at(a[11], &s) || !on_current(a, {0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10}))
      FALLBACK;
    return run([&] {
      return f_verify((int32_t)R, (int32_t)T, (int32_t)V, (const float*)tp, ts, (const float*)dp, ds, (const int32_t*)tok,
                      (const int32_t*)par, (const int32_t*)len, (const float*)ua, (const float*)us, (int32_t*)path,
                      (int32_t*)plen, (int32_t*)out, ws, bytes, s);
    });
  });
}

// dims, new_k, new_v, num_tokens, path, path_len, k_pages, v_pages, block_table, ctx_len, new_ctx_len, stream
PyObject* append_tokens(PyObject*, Args a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 12) FALLBACK;
    const oasis_dims* d = dims_at(a[0]);
    int32_t N;
    int64_t pages;
    if (!d || !int32(a[3], &N)) FALLBACK;
    const int64_t R = d->num_reqs, kv = count({R, N, d->num_kv_heads, d->head_dim});
    void *nk, *nv, *path, *plen, *k, *v, *table, *ctx, *end, *s;
    if (!tensor(a[1], kv, kBf16, &nk) || !tensor(a[2], kv, kBf16, &nv) || !optional(a[4], count({R, N}), kI32, &path) ||
        !optional(a[5], R, kI32, &plen) || !tier_at(a[6], a[7], d, &k, &v, &pages) ||
        !tensor(a[8], count({R, d->max_blocks}), kI32, &table) || !tensor(a[9], R, kI32, &ctx) ||
        !optional(a[10], R, kI32, &end) || !stream_at(a[11], &s) || !on_current(a, {1, 2, 4, 5, 6, 7, 8, 9, 10}))
      FALLBACK;
    return run([&] {
      return f_append(d, (const uint16_t*)nk, (const uint16_t*)nv, N, (const int32_t*)path, (const int32_t*)plen,
                      (uint16_t*)k, (uint16_t*)v, pages, (const int32_t*)table, (const int32_t*)ctx, (int32_t*)end, s);
    });
  });
}

// bind(attn, score, topk, score_select, stage): addresses of the library's entry points
PyObject* bind(PyObject*, Args a, Py_ssize_t n) {
  void* p[5];
  if (n != 5) return PyErr_Format(PyExc_TypeError, "bind takes 5 addresses");
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "bind: null address");
  }
  f_attn = reinterpret_cast<decltype(f_attn)>(p[0]);
  f_score = reinterpret_cast<decltype(f_score)>(p[1]);
  f_topk = reinterpret_cast<decltype(f_topk)>(p[2]);
  f_score_select = reinterpret_cast<decltype(f_score_select)>(p[3]);
  f_stage = reinterpret_cast<decltype(f_stage)>(p[4]);
  Py_RETURN_NONE;
}

// bind_drafts(tree_attn, sparse_tree_attn, verify, append): addresses of the library's entry points
PyObject* bind_drafts(PyObject*, Args a, Py_ssize_t n) {
  void* p[4];
  if (n != 4) return PyErr_Format(PyExc_TypeError, "bind_drafts takes 4 addresses");
  for (int i = 0; i < 4; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "bind_drafts: null address");
  }
  f_tree = reinterpret_cast<decltype(f_tree)>(p[0]);
  f_sparse_tree = reinterpret_cast<decltype(f_sparse_tree)>(p[1]);
  f_verify = reinterpret_cast<decltype(f_verify)>(p[2]);
  f_append = reinterpret_cast<decltype(f_append)>(p[3]);
  Py_RETURN_NONE;
}

#define METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind),         METHOD(sparse_decode_attn), METHOD(score_blocks), METHOD(select_topk),
                         METHOD(score_select), METHOD(stage_blocks),       METHOD(bind_drafts),  METHOD(tree_attn),
                         METHOD(sparse_tree_attn), METHOD(verify_drafts),  METHOD(append_tokens), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) {
  PyObject* m = PyModule_Create(&module);
  // the signatures the calls above were compiled with; the binding compares it with the loaded library's
  if (m && PyModule_AddIntConstant(m, "abi_version", OASIS_ABI_VERSION) < 0) Py_CLEAR(m);
  return m;
}
