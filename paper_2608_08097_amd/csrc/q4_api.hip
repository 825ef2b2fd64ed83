// C ABI of the 4-bit cache: argument checks, workspace carving and kernel launches
// (conventions of api.hip: nothing here allocates memory or throws).
#include "api_checks.h"
#include "q4_internal.h"

namespace oasis {
namespace {

constexpr double kTwoPi = 6.283185307179586476925286766559;

// Checks and fills a rotation (rotary NULL: none).
oasis_status make_rotary(const oasis_rotary* rotary, bool inverse, RotaryArgs* a, const char* fn) {
  *a = RotaryArgs{};
  if (!rotary) return OASIS_OK;
  if (rotary->rotary_dim < 2 || rotary->rotary_dim > kHeadDim || rotary->rotary_dim % 2)
    return fail(OASIS_ERR_INVALID_ARG, "%s: rotary_dim %d (even, from 2 to %d)", fn, rotary->rotary_dim, kHeadDim);
  if (rotary->interleaved != 0 && rotary->interleaved != 1)
    return fail(OASIS_ERR_INVALID_ARG, "%s: interleaved is %d", fn, rotary->interleaved);
  if (!std::isfinite(rotary->amplitude)) return fail(OASIS_ERR_INVALID_ARG, "%s: amplitude is not finite", fn);
  REQUIRE_AS(need, rotary->turns, "turns", fn);
  if ((uintptr_t)rotary->turns & 7) return fail(OASIS_ERR_INVALID_ARG, "%s: turns is not 8-byte aligned", fn);
  a->turns = rotary->turns;
  a->half = rotary->rotary_dim / 2;
  a->interleaved = rotary->interleaved;
  a->cos_amplitude = rotary->amplitude;
  a->sin_amplitude = inverse ? -rotary->amplitude : rotary->amplitude;
  return OASIS_OK;
}

// Rows of `heads` heads, `stride` elements apart.
struct Rows {
  const void* at;
  long long stride, rows, heads;
  const char* name;
  long long width() const { return heads * kHeadDim * 2; }
  long long extent() const { return at ? ((rows - 1) * stride + heads * kHeadDim) * 2 : 0; }
};
oasis_status check_rows(const Rows& r, const char* fn) {
  REQUIRE_AS(need16, r.at, r.name, fn);
  if (r.stride < r.heads * kHeadDim || r.stride % 8 || r.stride > INT64_MAX / 4 / r.rows)
    return fail(OASIS_ERR_INVALID_ARG, "%s: the rows of %s are %lld elements apart (a multiple of 8, at least %lld)", fn,
                r.name, r.stride, r.heads * kHeadDim);
  return OASIS_OK;
}
// Whether two sets of rows share memory; those of one stride may lie side by side.
bool rows_meet(const Rows& x, const Rows& y) {
  const uintptr_t a = (uintptr_t)x.at, b = (uintptr_t)y.at;
  if (!a || !b || a >= b + (uintptr_t)y.extent() || b >= a + (uintptr_t)x.extent()) return false;
  if (x.stride != y.stride) return true;
  const long long row = x.stride * 2;
  long long off = (long long)(b - a) % row;  // of y's row in x's
  if (off < 0) off += row;
  return off < x.width() || off + y.width() > row;
}
Buffer buffer_of(const Rows& r) { return Buffer{r.at, r.extent(), r.name}; }

oasis_status check_pages(const oasis_dims* d, int64_t num_pages, const char* fn) {
  if (num_pages < 1 || num_pages > INT32_MAX) return fail(OASIS_ERR_INVALID_ARG, "%s: num_pages out of range", fn);
  if ((long long)d->max_blocks * d->block_size > INT32_MAX - 64)  // positions are rounded up to units of 64
    return fail(OASIS_ERR_UNSUPPORTED, "%s: max_blocks * block_size past 31 bits", fn);
  if (q4_page_bytes(d->num_kv_heads, d->block_size) > INT32_MAX)
    return fail(OASIS_ERR_UNSUPPORTED, "%s: pages of more than 31 bits", fn);
  return OASIS_OK;
}

oasis_status check_attn_q4(const oasis_dims* d, int32_t T, int32_t k, const char* fn) {
  oasis_status st = check_tree(d, T, fn);
  if (st == OASIS_OK) st = check_pages(d, 1, fn);
  if (st != OASIS_OK) return st;
  if (k < 0) return fail(OASIS_ERR_INVALID_ARG, "%s: k < 0", fn);
  if (k > 65536) return fail(OASIS_ERR_UNSUPPORTED, "%s: k = %d (at most 65536)", fn, k);
  return OASIS_OK;
}

TreePlan attn_q4_plan(const oasis_dims* d, int32_t T, int32_t k) {
  const long long attended = k > 0 ? k + 1 : d->max_blocks;
  const long long blocks = attended < d->max_blocks ? attended : d->max_blocks;
  auto units = [&](long long n) { return (int)((n * d->block_size + kQ4Unit - 1) / kQ4Unit); };
  return q4_plan((long long)d->num_reqs * d->num_kv_heads, d->num_q_heads / d->num_kv_heads, T, units(blocks),
                 units(attended));
}

}  // namespace
}  // namespace oasis

using oasis::Buffer;
using oasis::fail;
using oasis::hip_status;
using oasis::kHeadDim;
using oasis::kLog2e;
using oasis::ok;
using oasis::Rows;

extern "C" {

size_t oasis_q4_page_bytes(const oasis_dims* dims) {
  if (oasis::check_dims(dims, "oasis_q4_page_bytes") != OASIS_OK) return 0;
  return (size_t)oasis::q4_page_bytes(dims->num_kv_heads, dims->block_size);
}

oasis_status oasis_rotary_turns(int32_t rotary_dim, double base, int32_t scaling, double factor, double first_len,
                                double low, double high, double* turns, double* amplitude) {
  static const char* fn = "oasis_rotary_turns";
  if (rotary_dim < 2 || rotary_dim > kHeadDim || rotary_dim % 2)
    return fail(OASIS_ERR_INVALID_ARG, "%s: rotary_dim %d (even, from 2 to %d)", fn, rotary_dim, kHeadDim);
  if (!(base > 0) || !std::isfinite(base)) return fail(OASIS_ERR_INVALID_ARG, "%s: base", fn);
  if (scaling < OASIS_ROTARY_PLAIN || scaling > OASIS_ROTARY_BY_INDEX)
    return fail(OASIS_ERR_INVALID_ARG, "%s: scaling %d", fn, scaling);
  if (scaling != OASIS_ROTARY_PLAIN && (!(factor > 0) || !std::isfinite(factor)))
    return fail(OASIS_ERR_INVALID_ARG, "%s: factor", fn);
  const bool ramps = scaling == OASIS_ROTARY_BY_TURNS || scaling == OASIS_ROTARY_BY_INDEX;
  if (ramps && !(std::isfinite(first_len) && first_len > 0 && std::isfinite(low) && low > 0 && std::isfinite(high) && high > low))
    return fail(OASIS_ERR_INVALID_ARG, "%s: first_len, low and high have to be positive, low below high", fn);
  if (scaling == OASIS_ROTARY_BY_INDEX && !(base > 1)) return fail(OASIS_ERR_INVALID_ARG, "%s: base", fn);
  REQUIRE_PTR(turns, fn);
  const double dim = rotary_dim;
  if (scaling == OASIS_ROTARY_STRETCHED && rotary_dim > 2) base *= std::pow(factor, dim / (dim - 2));
  // pair at which a pair makes x turns over the first contexts
  auto pair_of = [&](double x) { return dim * std::log(first_len / (x * oasis::kTwoPi)) / (2 * std::log(base)); };
  double from = 0, to = 0;
  if (scaling == OASIS_ROTARY_BY_INDEX) {
    from = std::fmax(std::floor(pair_of(high)), 0.0);
    to = std::fmin(std::ceil(pair_of(low)), dim - 1);
    if (to <= from) to = from + 0.001;
  }
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / dim) / oasis::kTwoPi;
    double kept = 0;  // share of the unscaled frequency
    if (scaling == OASIS_ROTARY_BY_TURNS) kept = (first_len * f - low) / (high - low);
    if (scaling == OASIS_ROTARY_BY_INDEX) kept = 1 - (i - from) / (to - from);
    kept = std::fmin(std::fmax(kept, 0.0), 1.0);
    if (scaling == OASIS_ROTARY_LINEAR || ramps) f = f * kept + f / factor * (1 - kept);
    turns[i] = f;
  }
  if (amplitude) *amplitude = scaling == OASIS_ROTARY_BY_INDEX && factor > 1 ? 0.1 * std::log(factor) + 1 : 1;
  return ok();
}

oasis_status oasis_rotate(const oasis_dims* dims, const oasis_rotary* rotary, int32_t num_tokens,
                          const int32_t* positions, const int32_t* ctx_len, int32_t inverse, const uint16_t* q,
                          int64_t q_stride, uint16_t* q_out, int64_t q_out_stride, const uint16_t* k, int64_t k_stride,
                          uint16_t* k_out, int64_t k_out_stride, void* stream) {
  static const char* fn = "oasis_rotate";
  oasis_status st = oasis::check_dims(dims, fn);
  if (st != OASIS_OK) return st;
  if (num_tokens < 1) return fail(OASIS_ERR_INVALID_ARG, "%s: num_tokens < 1", fn);
  if (!rotary) return fail(OASIS_ERR_INVALID_ARG, "%s: rotary is NULL", fn);
  oasis::RotateArgs a{};
  if ((st = oasis::make_rotary(rotary, inverse != 0, &a.rot, fn)) != OASIS_OK) return st;
  const long long rows = (long long)dims->num_reqs * num_tokens;
  // (a launch has fewer than 2^32 threads: 256 for every two rows)
  if (rows > 1 << 24 || (long long)dims->num_q_heads + dims->num_kv_heads > 65536)
    return fail(OASIS_ERR_UNSUPPORTED, "%s: %lld rows of %d and %d heads", fn, rows, dims->num_q_heads,
                dims->num_kv_heads);
  if (dims->num_reqs == 0) return ok();
  if (!q && !k) return fail(OASIS_ERR_INVALID_ARG, "%s: q and k are NULL", fn);
  if (!positions) REQUIRE_PTR(ctx_len, fn);
  const Rows in[2] = {{q, q_stride, rows, dims->num_q_heads, "q"}, {k, k_stride, rows, dims->num_kv_heads, "k"}};
  const Rows out[2] = {{q_out, q_out_stride, rows, dims->num_q_heads, "q_out"},
                       {k_out, k_out_stride, rows, dims->num_kv_heads, "k_out"}};
  const long long reqs = 4ll * dims->num_reqs;
  for (int x = 0; x < 2; ++x) {
    if (!in[x].at) continue;
    if ((st = oasis::check_rows(in[x], fn)) != OASIS_OK || (st = oasis::check_rows(out[x], fn)) != OASIS_OK) return st;
    for (int y = 0; y < 2; ++y) {
      if (!in[y].at) continue;
      const bool in_place = x == y && out[x].at == in[y].at && out[x].stride == in[y].stride;
      if (!in_place && oasis::rows_meet(out[x], in[y]))
        return fail(OASIS_ERR_INVALID_ARG, "%s: %s overlaps %s", fn, out[x].name, in[y].name);
      if (y < x && oasis::rows_meet(out[x], out[y]))
        return fail(OASIS_ERR_INVALID_ARG, "%s: %s overlaps %s", fn, out[x].name, out[y].name);
    }
    st = oasis::apart({oasis::buffer_of(out[x])},
                      {{positions, 4 * rows, "positions"}, {ctx_len, reqs, "ctx_len"},
                       {rotary->turns, 4ll * rotary->rotary_dim, "turns"}}, fn);
    if (st != OASIS_OK) return st;
  }
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  a.positions = positions;
  a.ctx_len = ctx_len;
  a.T = num_tokens;
  a.Hq = q ? dims->num_q_heads : 0;
  a.Hkv = k ? dims->num_kv_heads : 0;
  a.rows = rows;
  a.by_heads = oasis::fast_div(a.Hq + a.Hkv);
  a.by_t = oasis::fast_div(num_tokens);
  return hip_status(oasis::launch_rotate(a, static_cast<hipStream_t>(stream)), fn);
}

oasis_status oasis_append_tokens_q4(const oasis_dims* dims, const oasis_rotary* rotary, const uint16_t* new_k,
                                    int64_t k_stride, const uint16_t* new_v, int64_t v_stride, int32_t num_tokens,
                                    const int32_t* path, const int32_t* path_len, uint8_t* k_pages, uint8_t* v_pages,
                                    int64_t num_pages, const int32_t* block_table, const int32_t* ctx_len,
                                    int32_t* new_ctx_len, uint16_t* read_k, uint16_t* read_v, void* stream) {
  static const char* fn = "oasis_append_tokens_q4";
  oasis_status st = oasis::check_dims(dims, fn);
  if (st != OASIS_OK) return st;
  if (num_tokens < 1) return fail(OASIS_ERR_INVALID_ARG, "%s: num_tokens < 1", fn);
  if ((long long)num_tokens * dims->num_kv_heads > (1 << 26))
    return fail(OASIS_ERR_UNSUPPORTED, "%s: num_tokens * num_kv_heads > 2^26", fn);
  if ((st = oasis::check_pages(dims, num_pages, fn)) != OASIS_OK) return st;
  oasis::AppendQ4Args a{};
  if ((st = oasis::make_rotary(rotary, false, &a.rot, fn)) != OASIS_OK) return st;
  if (dims->num_reqs == 0) return ok();
  const long long H = dims->num_kv_heads, rows = (long long)dims->num_reqs * num_tokens;
  const Rows nk{new_k, k_stride, rows, H, "new_k"}, nv{new_v, v_stride, rows, H, "new_v"};
  if ((st = oasis::check_rows(nk, fn)) != OASIS_OK || (st = oasis::check_rows(nv, fn)) != OASIS_OK) return st;
  REQUIRE_ALIGNED(k_pages, fn);
  REQUIRE_ALIGNED(v_pages, fn);
  REQUIRE_PTR(block_table, fn);
  REQUIRE_PTR(ctx_len, fn);
  if (read_k) REQUIRE_ALIGNED(read_k, fn);
  if (read_v) REQUIRE_ALIGNED(read_v, fn);
  if (path && !path_len) return fail(OASIS_ERR_INVALID_ARG, "%s: path without path_len", fn);
  const long long reqs = 4ll * dims->num_reqs, page = oasis::q4_page_bytes(H, dims->block_size);
  const long long read = rows * H * kHeadDim * 2;
  st = oasis::apart({{k_pages, num_pages * page, "k_pages"}, {v_pages, num_pages * page, "v_pages"},
                     {new_ctx_len, reqs, "new_ctx_len"}, {read_k, read, "read_k"}, {read_v, read, "read_v"}},
                    {oasis::buffer_of(nk), oasis::buffer_of(nv), {ctx_len, reqs, "ctx_len"},
                     {path_len, reqs, "path_len"}, {path, reqs * num_tokens, "path"},
                     {block_table, reqs * dims->max_blocks, "block_table"},
                     {a.rot.turns, 8ll * a.rot.half, "turns"}}, fn);
  if (st != OASIS_OK) return st;
  const void *kp = nullptr, *vp = nullptr;
  if ((st = oasis::device_view(k_pages, &kp, "k_pages", fn)) != OASIS_OK) return st;
  if ((st = oasis::device_view(v_pages, &vp, "v_pages", fn)) != OASIS_OK) return st;
  a.new_k = new_k;
  a.new_v = new_v;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.path = path;
  a.path_len = path_len;
  a.k = static_cast<uint8_t*>(const_cast<void*>(kp));
  a.v = static_cast<uint8_t*>(const_cast<void*>(vp));
  a.num_pages = num_pages;
  a.page_bytes = page;
  a.table = block_table;
  a.ctx_len = ctx_len;
  a.new_ctx_len = new_ctx_len;
  a.read_k = read_k;
  a.read_v = read_v;
  a.R = dims->num_reqs;
  a.Hkv = dims->num_kv_heads;
  a.T = num_tokens;
  a.B = dims->block_size;
  a.NBmax = dims->max_blocks;
  a.by_heads = oasis::fast_div(2 * a.Hkv);
  return hip_status(oasis::launch_append_q4(a, static_cast<hipStream_t>(stream)), fn);
}

oasis_status oasis_update_summaries_q4(const oasis_dims* dims, const uint8_t* k_pages, int64_t num_pages,
                                       const int32_t* block_table, const int32_t* prev_ctx_len, const int32_t* ctx_len,
                                       int32_t max_new_blocks, uint16_t* kmax, uint16_t* kmin, void* stream) {
  static const char* fn = "oasis_update_summaries_q4";
  oasis_status st = oasis::check_dims(dims, fn);
  if (st != OASIS_OK) return st;
  if ((st = oasis::check_pages(dims, num_pages, fn)) != OASIS_OK) return st;
  if (prev_ctx_len && max_new_blocks < 1) return fail(OASIS_ERR_INVALID_ARG, "%s: max_new_blocks < 1", fn);
  if ((long long)dims->max_blocks * dims->num_kv_heads > (1 << 27))
    return fail(OASIS_ERR_UNSUPPORTED, "%s: max_blocks * num_kv_heads > 2^27", fn);
  if (dims->num_reqs == 0) return ok();
  REQUIRE_ALIGNED(k_pages, fn);
  REQUIRE_PTR(block_table, fn);
  REQUIRE_PTR(ctx_len, fn);
  REQUIRE_ALIGNED(kmax, fn);
  REQUIRE_ALIGNED(kmin, fn);
  const long long reqs = 4ll * dims->num_reqs, page = oasis::q4_page_bytes(dims->num_kv_heads, dims->block_size);
  const long long bytes = (long long)dims->num_reqs * dims->num_kv_heads * dims->max_blocks * kHeadDim * 2;
  st = oasis::apart({{kmax, bytes, "kmax"}, {kmin, bytes, "kmin"}},
                    {{k_pages, num_pages * page, "k_pages"}, {block_table, reqs * dims->max_blocks, "block_table"},
                     {prev_ctx_len, reqs, "prev_ctx_len"}, {ctx_len, reqs, "ctx_len"}}, fn);
  if (st != OASIS_OK) return st;
  const void* kp = nullptr;
  if ((st = oasis::device_view(k_pages, &kp, "k_pages", fn)) != OASIS_OK) return st;
  const oasis::SummaryQ4Args a{static_cast<const uint8_t*>(kp), num_pages, page, block_table, prev_ctx_len, ctx_len,
                               max_new_blocks, kmax, kmin, dims->num_reqs, dims->num_kv_heads, dims->block_size,
                               dims->max_blocks, oasis::fast_div(dims->num_kv_heads)};
  return hip_status(oasis::launch_summaries_q4(a, static_cast<hipStream_t>(stream)), fn);
}

size_t oasis_tree_attn_q4_workspace_bytes(const oasis_dims* dims, int32_t num_q_tokens, int32_t k) {
  if (oasis::check_attn_q4(dims, num_q_tokens, k, "oasis_tree_attn_q4_workspace_bytes") != OASIS_OK) return 0;
  return oasis::attn_q4_plan(dims, num_q_tokens, k).bytes;
}

oasis_status oasis_tree_attn_q4(const oasis_dims* dims, const uint16_t* q, int32_t num_q_tokens, const uint8_t* k_pages,
                                const uint8_t* v_pages, int64_t num_pages, const int32_t* block_table,
                                const int32_t* ctx_len, const int32_t* sel, const int32_t* sel_count, int32_t k,
                                const uint16_t* tree_k, const uint16_t* tree_v, const int32_t* parent,
                                const int32_t* tree_len, float scale, uint16_t* out, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream) {
  static const char* fn = "oasis_tree_attn_q4";
  oasis_status st = oasis::check_attn_q4(dims, num_q_tokens, k, fn);
  if (st != OASIS_OK) return st;
  if ((st = oasis::check_pages(dims, num_pages, fn)) != OASIS_OK) return st;
  if (!std::isfinite(scale * kLog2e)) return fail(OASIS_ERR_INVALID_ARG, "%s: scale is not finite", fn);
  if ((sel != nullptr) != (k > 0) || (sel != nullptr) != (sel_count != nullptr))
    return fail(OASIS_ERR_INVALID_ARG, "%s: sel, sel_count and k go together (all blocks: NULL, NULL and 0)", fn);
  if (dims->num_reqs == 0) return ok();
  REQUIRE_ALIGNED(k_pages, fn);
  REQUIRE_ALIGNED(v_pages, fn);
  REQUIRE_PTR(block_table, fn);
  const oasis::TreePlan plan = oasis::attn_q4_plan(dims, num_q_tokens, k);
  oasis::AttnQ4Args a{};
  st = oasis::make_tree_args({dims, q, num_q_tokens, tree_k, tree_v, parent, tree_len, ctx_len, scale, out, lse,
                              workspace, workspace_bytes},
                             plan, &a, fn, true);
  if (st != OASIS_OK) return st;
  const long long reqs = 4ll * dims->num_reqs, page = oasis::q4_page_bytes(dims->num_kv_heads, dims->block_size);
  const long long rows = (long long)dims->num_reqs * num_q_tokens * dims->num_q_heads;
  const long long tree = (long long)dims->num_reqs * num_q_tokens * dims->num_kv_heads * kHeadDim * 2;
  st = oasis::apart({{out, rows * kHeadDim * 2, "out"}, {lse, rows * 4, "lse"},
                     {workspace, (long long)plan.bytes, "workspace"}},
                    {{q, rows * kHeadDim * 2, "q"}, {k_pages, num_pages * page, "k_pages"},
                     {v_pages, num_pages * page, "v_pages"}, {block_table, reqs * dims->max_blocks, "block_table"},
                     {ctx_len, reqs, "ctx_len"}, {sel, reqs * dims->num_kv_heads * k, "sel"},
                     {sel_count, reqs * dims->num_kv_heads, "sel_count"}, {tree_k, tree, "tree_k"},
                     {tree_v, tree, "tree_v"}, {parent, reqs * num_q_tokens, "parent"}, {tree_len, reqs, "tree_len"}}, fn);
  if (st != OASIS_OK) return st;
  const void *kp = nullptr, *vp = nullptr;
  if ((st = oasis::device_view(k_pages, &kp, "k_pages", fn)) != OASIS_OK) return st;
  if ((st = oasis::device_view(v_pages, &vp, "v_pages", fn)) != OASIS_OK) return st;
  a.k4 = static_cast<const uint8_t*>(kp);
  a.v4 = static_cast<const uint8_t*>(vp);
  a.page_bytes = page;
  a.num_pages = num_pages;
  a.table = block_table;
  a.sel = sel;
  a.sel_count = sel_count;
  a.k_sel = k;
  a.by_length = !sel && oasis::tree_by_length(plan, dims->num_reqs, dims->num_kv_heads);
  return hip_status(oasis::launch_attn_q4(a, static_cast<hipStream_t>(stream)), fn);
}

}  // extern "C"
