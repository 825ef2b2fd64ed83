// C ABI of the speculative step: argument checks, workspace carving and kernel
// launches (conventions of api.hip: nothing here allocates memory or throws).
#include <cmath>
#include <initializer_list>

#include "drafts_internal.h"

namespace oasis {

constexpr float kLog2e = 1.4426950408889634f;

namespace {

oasis_status need(const void* p, const char* name, const char* fn) {
  return p ? OASIS_OK : fail(OASIS_ERR_INVALID_ARG, "%s: %s is NULL", fn, name);
}
// for 16-byte loads and stores
oasis_status need16(const void* p, const char* name, const char* fn) {
  if ((uintptr_t)p & 15) return fail(OASIS_ERR_INVALID_ARG, "%s: %s is not 16-byte aligned", fn, name);
  return need(p, name, fn);
}
#define REQUIRE_AS(check, p, name, fn)                                    \
  do {                                                                    \
    const oasis_status require_st = ::oasis::check(p, name, fn);            \
    if (require_st != OASIS_OK) return require_st;                        \
  } while (0)
#define REQUIRE_PTR(p, fn) REQUIRE_AS(need, p, #p, fn)
#define REQUIRE_ALIGNED(p, fn) REQUIRE_AS(need16, p, #p, fn)

// What a call writes must not be what it reads, or writes elsewhere: the waves and
// workgroups of a launch read at times of their own.
struct Buffer {
  const void* at;
  long long bytes;
  const char* name;
};
oasis_status apart(std::initializer_list<Buffer> written, std::initializer_list<Buffer> read, const char* fn) {
  auto meet = [](const Buffer& x, const Buffer& y) {
    const uintptr_t a = (uintptr_t)x.at, b = (uintptr_t)y.at;
    return a && b && a < b + (uintptr_t)y.bytes && b < a + (uintptr_t)x.bytes;
  };
  for (const Buffer* w = written.begin(); w != written.end(); ++w) {
    for (const Buffer* o = written.begin(); o != w; ++o)
      if (meet(*w, *o)) return fail(OASIS_ERR_INVALID_ARG, "%s: %s overlaps %s", fn, w->name, o->name);
    for (const Buffer& r : read)
      if (meet(*w, r)) return fail(OASIS_ERR_INVALID_ARG, "%s: %s overlaps %s", fn, w->name, r.name);
  }
  return OASIS_OK;
}

// Sizes of a tree of drafted tokens over any cache.
oasis_status check_tree(const oasis_dims* d, int32_t T, const char* fn) {
  const oasis_status st = check_dims(d, fn);
  if (st != OASIS_OK) return st;
  if (T < 1) return fail(OASIS_ERR_INVALID_ARG, "%s: num_q_tokens < 1", fn);
  if (T > kTreeMaxTokens)
    return fail(OASIS_ERR_UNSUPPORTED, "%s: num_q_tokens %d (at most %d)", fn, T, kTreeMaxTokens);
  const long long rows = (long long)T * (d->num_q_heads / d->num_kv_heads);
  if (rows > kTreeMaxRows)
    return fail(OASIS_ERR_UNSUPPORTED, "%s: G * num_q_tokens = %lld rows per KV head (at most %d)", fn, rows,
                kTreeMaxRows);
  if ((long long)d->max_blocks * d->block_size > INT32_MAX - 32)  // positions are rounded up to units of 32
    return fail(OASIS_ERR_UNSUPPORTED, "%s: max_blocks * block_size past 31 bits", fn);
  return OASIS_OK;
}

oasis_status check_slots(const oasis_dims* d, int32_t k_slots, const char* fn) {
  if (k_slots < 0) return fail(OASIS_ERR_INVALID_ARG, "%s: k_slots < 0", fn);
  if (((long long)k_slots + 2) * d->block_size > INT32_MAX)
    return fail(OASIS_ERR_UNSUPPORTED, "%s: k_slots * block_size past 31 bits", fn);
  return OASIS_OK;
}

TreePlan paged_plan(const oasis_dims* d, int32_t T) {
  return tree_plan((long long)d->num_reqs * d->num_kv_heads, d->num_q_heads / d->num_kv_heads, T,
                   (int)(((long long)d->max_blocks * d->block_size + 31) / 32), true);
}
TreePlan sparse_plan(const oasis_dims* d, int32_t T, int32_t k_slots) {
  return tree_plan((long long)d->num_reqs * d->num_kv_heads, d->num_q_heads / d->num_kv_heads, T,
                   (int)((((long long)k_slots + 1) * d->block_size + 31) / 32), false);
}

struct TreeCall {
  const oasis_dims* dims;
  const uint16_t* q;
  int32_t T;
  const uint16_t *tree_k, *tree_v;
  const int32_t *parent, *tree_len, *ctx_len;
  float scale;
  uint16_t* out;
  float* lse;
  void* workspace;
  size_t workspace_bytes;
};

// Checks and fills what both caches share.
oasis_status make_tree_args(const TreeCall& c, const TreePlan& p, TreeAttnArgs* a, const char* fn) {
  REQUIRE_AS(need16, c.q, "q", fn);
  REQUIRE_AS(need16, c.tree_k, "tree_k", fn);
  REQUIRE_AS(need16, c.tree_v, "tree_v", fn);
  REQUIRE_AS(need, c.ctx_len, "ctx_len", fn);
  REQUIRE_AS(need16, c.out, "out", fn);
  if (p.bytes > 0 && (!c.workspace || c.workspace_bytes < p.bytes))
    return fail(OASIS_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, c.workspace_bytes, p.bytes);
  if (p.bytes > 0 && (uintptr_t)c.workspace & 15)
    return fail(OASIS_ERR_INVALID_ARG, "%s: workspace is not 16-byte aligned", fn);
  TreeAttnArgs t{};
  t.q = c.q;
  t.ctx_len = c.ctx_len;
  t.tree_k = c.tree_k;
  t.tree_v = c.tree_v;
  t.parent = c.parent;
  t.tree_len = c.tree_len;
  t.out = c.out;
  t.lse = c.lse;
  t.part_o = static_cast<float*>(c.workspace);
  t.part_ml = static_cast<float*>(c.workspace) + p.part_o_floats;
  t.R = c.dims->num_reqs;
  t.Hq = c.dims->num_q_heads;
  t.Hkv = c.dims->num_kv_heads;
  t.G = t.Hq / t.Hkv;
  t.T = c.T;
  t.B = c.dims->block_size;
  t.NBmax = c.dims->max_blocks;
  t.scale_log2 = c.scale == 0.f ? 1.f : std::fabs(c.scale) * kLog2e;
  t.q_and = c.scale == 0.f ? 0u : ~0u;
  t.q_xor = c.scale < 0.f ? 0x80008000u : 0u;
  t.top = std::ldexp(1.f, 8 - tree_lift(p.units));
  t.rows = p.rows;
  t.tiles = p.tiles;
  t.groups = p.groups;
  t.nsplit = p.nsplit;
  t.by_groups = fast_div(p.groups);
  t.by_nsplit = fast_div(p.nsplit);
  t.by_hkv = fast_div(t.Hkv);
  t.by_g = fast_div(t.G);
  *a = t;
  return OASIS_OK;
}

}  // namespace
}  // namespace oasis

using oasis::fail;
using oasis::hip_status;
using oasis::kLog2e;
using oasis::ok;

extern "C" {

size_t oasis_tree_attn_workspace_bytes(const oasis_dims* dims, int32_t num_q_tokens) {
  if (oasis::check_tree(dims, num_q_tokens, "oasis_tree_attn_workspace_bytes") != OASIS_OK) return 0;
  return oasis::paged_plan(dims, num_q_tokens).bytes;
}

oasis_status oasis_tree_attn(const oasis_dims* dims, const uint16_t* q, int32_t num_q_tokens, const uint16_t* k_pages,
                             const uint16_t* v_pages, int64_t num_pages, const int32_t* block_table,
                             const int32_t* ctx_len, const uint16_t* tree_k, const uint16_t* tree_v,
                             const int32_t* parent, const int32_t* tree_len, float scale, uint16_t* out, float* lse,
                             void* workspace, size_t workspace_bytes, void* stream) {
  static const char* fn = "oasis_tree_attn";
  oasis_status st = oasis::check_tree(dims, num_q_tokens, fn);
  if (st != OASIS_OK) return st;
  if (num_pages < 1 || num_pages > INT32_MAX) return fail(OASIS_ERR_INVALID_ARG, "%s: num_pages out of range", fn);
  if (!std::isfinite(scale * kLog2e)) return fail(OASIS_ERR_INVALID_ARG, "%s: scale is not finite", fn);
  if (dims->num_reqs == 0) return ok();
  REQUIRE_ALIGNED(k_pages, fn);
  REQUIRE_ALIGNED(v_pages, fn);
  REQUIRE_PTR(block_table, fn);
  const oasis::TreePlan plan = oasis::paged_plan(dims, num_q_tokens);
  oasis::TreeAttnArgs a{};
  st = oasis::make_tree_args({dims, q, num_q_tokens, tree_k, tree_v, parent, tree_len, ctx_len, scale, out, lse,
                              workspace, workspace_bytes},
                             plan, &a, fn);
  if (st != OASIS_OK) return st;
  const void *kp = nullptr, *vp = nullptr;
  if ((st = oasis::device_view(k_pages, &kp, "k_pages", fn)) != OASIS_OK) return st;
  if ((st = oasis::device_view(v_pages, &vp, "v_pages", fn)) != OASIS_OK) return st;
  a.k = static_cast<const uint16_t*>(kp);
  a.v = static_cast<const uint16_t*>(vp);
  a.table = block_table;
  a.num_pages = num_pages;
  a.by_length = oasis::tree_by_length(plan, dims->num_reqs, dims->num_kv_heads);
  return hip_status(oasis::launch_tree_attn(a, true, static_cast<hipStream_t>(stream)), fn);
}

size_t oasis_sparse_tree_attn_workspace_bytes(const oasis_dims* dims, int32_t num_q_tokens, int32_t k_slots) {
  static const char* fn = "oasis_sparse_tree_attn_workspace_bytes";
  if (oasis::check_tree(dims, num_q_tokens, fn) != OASIS_OK || oasis::check_slots(dims, k_slots, fn) != OASIS_OK)
    return 0;
  return oasis::sparse_plan(dims, num_q_tokens, k_slots).bytes;
}

oasis_status oasis_sparse_tree_attn(const oasis_dims* dims, const uint16_t* q, int32_t num_q_tokens,
                                    const uint16_t* pool_k, const uint16_t* pool_v, const int32_t* slot_map,
                                    int32_t k_slots, const int32_t* ctx_len, const uint16_t* tree_k,
                                    const uint16_t* tree_v, const int32_t* parent, const int32_t* tree_len,
                                    float scale, uint16_t* out, float* lse, void* workspace, size_t workspace_bytes,
                                    void* stream) {
  static const char* fn = "oasis_sparse_tree_attn";
  oasis_status st = oasis::check_tree(dims, num_q_tokens, fn);
  if (st != OASIS_OK) return st;
  if ((st = oasis::check_slots(dims, k_slots, fn)) != OASIS_OK) return st;
  if (!std::isfinite(scale * kLog2e)) return fail(OASIS_ERR_INVALID_ARG, "%s: scale is not finite", fn);
  if (dims->num_reqs == 0) return ok();
  REQUIRE_ALIGNED(pool_k, fn);
  REQUIRE_ALIGNED(pool_v, fn);
  if (k_slots > 0) REQUIRE_PTR(slot_map, fn);
  oasis::TreeAttnArgs a{};
  st = oasis::make_tree_args({dims, q, num_q_tokens, tree_k, tree_v, parent, tree_len, ctx_len, scale, out, lse,
                              workspace, workspace_bytes},
                             oasis::sparse_plan(dims, num_q_tokens, k_slots), &a, fn);
  if (st != OASIS_OK) return st;
  a.k = pool_k;
  a.v = pool_v;
  a.table = slot_map;
  a.k_slots = k_slots;
  return hip_status(oasis::launch_tree_attn(a, false, static_cast<hipStream_t>(stream)), fn);
}

size_t oasis_verify_workspace_bytes(int32_t num_reqs, int32_t num_q_tokens, int32_t vocab) {
  if (num_reqs < 1 || num_q_tokens < 1 || vocab < 1) return 0;
  return oasis::verify_ws_bytes(num_reqs);
}

oasis_status oasis_verify_drafts(int32_t num_reqs, int32_t num_q_tokens, int32_t vocab, const float* target_probs,
                                 int64_t target_stride, const float* draft_probs, int64_t draft_stride,
                                 const int32_t* tokens, const int32_t* parent, const int32_t* tree_len,
                                 const float* accept_u, const float* sample_u, int32_t* path, int32_t* path_len,
                                 int32_t* out_tokens, void* workspace, size_t workspace_bytes, void* stream) {
  static const char* fn = "oasis_verify_drafts";
  if (num_reqs < 0) return fail(OASIS_ERR_INVALID_ARG, "%s: num_reqs < 0", fn);
  if (num_reqs > 65535) return fail(OASIS_ERR_UNSUPPORTED, "%s: num_reqs > 65535", fn);
  if (num_q_tokens < 1) return fail(OASIS_ERR_INVALID_ARG, "%s: num_q_tokens < 1", fn);
  if (num_q_tokens > oasis::kTreeMaxTokens)
    return fail(OASIS_ERR_UNSUPPORTED, "%s: num_q_tokens %d (at most %d)", fn, num_q_tokens, oasis::kTreeMaxTokens);
  if (vocab < 1) return fail(OASIS_ERR_INVALID_ARG, "%s: vocab < 1", fn);
  if (vocab > (1 << 28)) return fail(OASIS_ERR_UNSUPPORTED, "%s: vocab %d", fn, vocab);
  if (target_stride < vocab || (draft_probs && draft_stride < vocab))
    return fail(OASIS_ERR_INVALID_ARG, "%s: a row stride below vocab", fn);
  if (num_reqs == 0) return ok();
  REQUIRE_PTR(target_probs, fn);
  REQUIRE_PTR(tokens, fn);
  REQUIRE_PTR(accept_u, fn);
  REQUIRE_PTR(sample_u, fn);
  REQUIRE_PTR(path, fn);
  REQUIRE_PTR(path_len, fn);
  REQUIRE_PTR(out_tokens, fn);
  const size_t bytes = oasis::verify_ws_bytes(num_reqs);
  if (!workspace || workspace_bytes < bytes)
    return fail(OASIS_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, workspace_bytes, bytes);
  if ((uintptr_t)workspace & 15) return fail(OASIS_ERR_INVALID_ARG, "%s: workspace is not 16-byte aligned", fn);
  const long long ints = 4ll * num_reqs * num_q_tokens, reqs = 4ll * num_reqs;
  const oasis_status st = oasis::apart(
      {{path, ints, "path"}, {path_len, reqs, "path_len"}, {out_tokens, ints, "out_tokens"}},
      {{tokens, ints, "tokens"}, {parent, ints, "parent"}, {tree_len, reqs, "tree_len"},
       {accept_u, ints, "accept_u"}, {sample_u, reqs, "sample_u"}, {workspace, (long long)bytes, "workspace"}},
      fn);
  if (st != OASIS_OK) return st;
  oasis::VerifyArgs a{};
  a.target = target_probs;
  a.draft = draft_probs;
  a.target_stride = target_stride;
  a.draft_stride = draft_stride;
  a.tokens = tokens;
  a.parent = parent;
  a.tree_len = tree_len;
  a.accept_u = accept_u;
  a.sample_u = sample_u;
  a.path = path;
  a.path_len = path_len;
  a.out_tokens = out_tokens;
  a.R = num_reqs;
  a.T = num_q_tokens;
  a.V = vocab;
  a.cut = oasis::verify_cut(vocab);
  a.groups = oasis::verify_groups(num_reqs, vocab, draft_probs != nullptr);
  a.part = static_cast<double*>(workspace);
  a.state = reinterpret_cast<oasis::VerifyState*>(a.part + (size_t)num_reqs * oasis::kVerifyBlocks);
  return hip_status(oasis::launch_verify(a, static_cast<hipStream_t>(stream)), fn);
}

oasis_status oasis_append_tokens(const oasis_dims* dims, const uint16_t* new_k, const uint16_t* new_v,
                                 int32_t num_tokens, const int32_t* path, const int32_t* path_len, uint16_t* k_pages,
                                 uint16_t* v_pages, int64_t num_pages, const int32_t* block_table,
                                 const int32_t* ctx_len, int32_t* new_ctx_len, void* stream) {
  static const char* fn = "oasis_append_tokens";
  oasis_status st = oasis::check_dims(dims, fn);
  if (st != OASIS_OK) return st;
  if (num_tokens < 1) return fail(OASIS_ERR_INVALID_ARG, "%s: num_tokens < 1", fn);
  if ((long long)num_tokens * dims->num_kv_heads > (1 << 26))
    return fail(OASIS_ERR_UNSUPPORTED, "%s: num_tokens * num_kv_heads > 2^26", fn);
  if (num_pages < 1 || num_pages > INT32_MAX) return fail(OASIS_ERR_INVALID_ARG, "%s: num_pages out of range", fn);
  if ((long long)dims->max_blocks * dims->block_size > INT32_MAX)
    return fail(OASIS_ERR_UNSUPPORTED, "%s: max_blocks * block_size past 31 bits", fn);
  if (dims->num_reqs == 0) return ok();
  REQUIRE_ALIGNED(new_k, fn);
  REQUIRE_ALIGNED(new_v, fn);
  REQUIRE_ALIGNED(k_pages, fn);
  REQUIRE_ALIGNED(v_pages, fn);
  REQUIRE_PTR(block_table, fn);
  REQUIRE_PTR(ctx_len, fn);
  if (path && !path_len) return fail(OASIS_ERR_INVALID_ARG, "%s: path without path_len", fn);
  if (new_ctx_len == ctx_len) return fail(OASIS_ERR_INVALID_ARG, "%s: new_ctx_len is ctx_len", fn);
  const long long reqs = 4ll * dims->num_reqs;
  st = oasis::apart({{new_ctx_len, reqs, "new_ctx_len"}},
                    {{ctx_len, reqs, "ctx_len"}, {path_len, reqs, "path_len"}, {path, reqs * num_tokens, "path"},
                     {block_table, reqs * dims->max_blocks, "block_table"}},
                    fn);
  if (st != OASIS_OK) return st;
  const void *kp = nullptr, *vp = nullptr;
  if ((st = oasis::device_view(k_pages, &kp, "k_pages", fn)) != OASIS_OK) return st;
  if ((st = oasis::device_view(v_pages, &vp, "v_pages", fn)) != OASIS_OK) return st;
  const oasis::AppendArgs a{new_k, new_v, path, path_len, static_cast<uint16_t*>(const_cast<void*>(kp)),
                            static_cast<uint16_t*>(const_cast<void*>(vp)), num_pages, block_table, ctx_len, new_ctx_len,
                            dims->num_reqs, dims->num_kv_heads, num_tokens, dims->block_size, dims->max_blocks,
                            oasis::fast_div(dims->num_kv_heads)};
  return hip_status(oasis::launch_append(a, static_cast<hipStream_t>(stream)), fn);
}

}  // extern "C"
