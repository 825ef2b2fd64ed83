// Argument checks that the entry points of the speculative step and of the 4-bit cache
// share.
#pragma once

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

// Checks and fills what the caches share. cache_only: there may be no tree's keys and
// values (both NULL), the rows attend the cache alone.
oasis_status make_tree_args(const TreeCall& c, const TreePlan& p, TreeAttnArgs* a, const char* fn,
                            bool cache_only = false) {
  REQUIRE_AS(need16, c.q, "q", fn);
  if (!cache_only || c.tree_k || c.tree_v) {
    REQUIRE_AS(need16, c.tree_k, "tree_k", fn);
    REQUIRE_AS(need16, c.tree_v, "tree_v", fn);
  }
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
