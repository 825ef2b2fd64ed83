// Attention of a drafted token tree over a cache, and the tree's own tokens.
//
// Row t of a request's tree attends every cached token (the pages of a paged
// cache, or the slots and local block of the working set) and the drafted tokens
// on its path to the root, itself among them: out = softmax(scale q K^T) V over
// the two sets together, one pass with a running maximum and sum.
//
// One 32-token unit of keys and values for one 16-row tile is, as in the working
// set's attention,
//   S^T (tokens x rows) = K . Q^T     8 of v_mfma_f32_16x16x32_bf16
//   O^T (d x rows)     += V^T . P^T   8 of them
// with the tokens dealt to MFMA rows so that lane (g, n) holds row n's scores of
// unit tokens 8g .. 8g+7, which makes the probabilities directly the B operand of
// the second product: no cross-lane movement and no LDS for P. The A operand of
// that product is 8 tokens of one dim in a lane. The working set keeps V
// transposed, so it is one load; pages keep V token-major.
//
// Two forms. Up to two row tiles (G * T <= 32) bandwidth bounds everything and
// tree_attn_kernel streams K and V from HBM straight into MFMA registers, four
// waves a workgroup, every wave a strided subset of the units with its own online
// softmax; token-major V is transposed in registers, 8 x 8 blocks, 32 byte
// permutes a unit. With more rows every unit is needed by several waves, and
// tree_attn_rows_kernel brings its K and V into LDS once for them; token-major V
// is read back with the transposing LDS read. Small calls with more rows take the
// first form in several groups of rows (kTreeSmallUnits). Both forms compute whole
// tiles, the second one four or eight of them: 2 x 8 x 65,536 tokens take 107 to 112 us
// with 5 to 8 tiles and 155 to 160 with 9 to 16.
//
// Measured (2 x 256 bytes a token and KV head; 4 d operations a row and token):
//   8 requests x 8 heads x 131,072 tokens, 20 rows   653 us  6.6 TB/s
//   64 x 8 x up to 2,064 of a working set, 28 rows   73-75 us  HBM, and 7 us of a workgroup's start and end
//   8 x 8 x 2,064 of a working set, 20 rows          18.8 us  two launches, and 10 of the bytes
//   24 x 8 x 1 to 32,768, 64 rows                    213-328 us a draw, 5.5 TB/s
//   16 x 8 x 4,128 of a working set, 256 rows        82-89 us  780-840 TFLOP/s
//   2 x 8 x 65,000 to 65,536, 512 rows               276-297 us  920-990 TFLOP/s
//   1 x 8 x 2,000, 8 rows                            8.9-9.2 us  two launches (7.4) and three loads in turn
// (a 16,384-cubed bf16 product of the library runs at 1,360 to 1,600 TFLOP/s here.) These
// block tables fit the contexts. The cut goes by the table's width, not by the lengths:
// with one for 131,072 tokens 8 x 8 x 2,064 paged tokens take 29 us instead of 20 (20
// rows) or 55 instead of 40 (256 rows).
//
// The tree's own tokens are one or two more units, with a mask per row, in the
// last split of every pair. Splits leave partials that a second kernel merges.
#include "tree_core.h"

namespace oasis {
namespace {

constexpr int kTW = kTreeWaves;

struct TreeUnit {
  u32x4 k[2][4];
  u32x4 v[8];
};

// Scores of one unit for one tile, before the scale: lane (g, n) gets row n against
// tokens 8g .. 8g+7.
__device__ __forceinline__ void unit_scores(const u32x4 (&k)[2][4], const bf16x8 (&qb)[4], f32x4 (&sc)[2]) {
  sc[0] = sc[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int st = 0; st < 4; ++st)
#pragma unroll
    for (int tau = 0; tau < 2; ++tau)
      sc[tau] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(k[tau][st]), qb[st], sc[tau], 0, 0, 0);
}

__device__ __forceinline__ void unit_pv(const u32x4 (&v)[8], bf16x8 pb, f32x4 (&acc)[8]) {
#pragma unroll
  for (int dt = 0; dt < 8; ++dt)
    acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v[dt]), pb, acc[dt], 0, 0, 0);
}

// What a workgroup works on.
struct TreeItem {
  int r, h, rh, split, row0, tlen, ctx;
  long long unit_elems;   // of a page or a slot
  const uint16_t *kb, *vb;  // this head's part of the pages, or of the request's slots
  const int32_t* tab;     // the request's block table, or the pair's slot map
  long long tree_row, tree_base;  // elements between the tree's rows, and to this head's first one
};
template <int BS, bool PAGED>
__device__ __forceinline__ bool tree_setup(const TreeAttnArgs& a, int group_rows, TreeItem& t) {
  int group, rs;
  if (PAGED && a.by_length) {
    rs = tree_item_spread(blockIdx.x, a, a.R * a.Hkv * a.nsplit, group);
    if (rs < 0) return false;
  } else {
    const int item = tree_item(blockIdx.x, a.R * a.Hkv * a.nsplit * a.groups);
    if (item < 0) return false;
    rs = a.by_groups(item);
    group = item - rs * a.groups;
  }
  t.row0 = group * group_rows;
  t.rh = a.by_nsplit(rs);
  t.split = rs - t.rh * a.nsplit;
  t.r = a.by_hkv(t.rh);
  t.h = t.rh - t.r * a.Hkv;
  if (PAGED && a.by_length) {
    t.r = request_of_rank(a.ctx_len, a.R, t.r, t.ctx);
    t.rh = t.r * a.Hkv + t.h;
  } else {
    t.ctx = a.ctx_len[t.r];  // read beside the tree's length
  }
  t.unit_elems = (long long)a.Hkv * BS * kHeadDim;
  const long long base = (PAGED ? 0 : (long long)t.r * (a.k_slots + 1) * t.unit_elems) + (long long)t.h * BS * kHeadDim;
  t.kb = a.k + base;
  t.vb = a.v + base;
  t.tab = a.table + (PAGED ? (long long)t.r * a.NBmax : (long long)t.rh * a.k_slots);
  t.tree_row = (long long)a.Hkv * kHeadDim;
  t.tree_base = (long long)t.r * a.T * t.tree_row + (long long)t.h * kHeadDim;
  t.tlen = tree_length(a, t.r);
  return t.row0 < t.tlen * a.G;  // else no row of this group is in the tree
}

// The cached tokens of request r and the units [begin, end) of a split of them.
template <int BS, bool PAGED>
__device__ __forceinline__ Ctx tree_units(const TreeAttnArgs& a, const TreeItem& t, int& L, int& begin, int& end) {
  const Ctx c = ctx_blocks(t.ctx, BS, a.NBmax);
  L = c.nb ? c.n_cand * BS + c.local_len : 0;
  const int nu = PAGED ? (L + 31) / 32 : (BS == 16 ? (a.k_slots + 2) / 2 : a.k_slots + 1);
  const int each = a.by_nsplit(nu), more = nu - each * a.nsplit;  // the first `more` splits have one more
  begin = t.split * each + min(t.split, more);
  end = begin + each + (t.split < more);
  return c;
}

// Table entry of block b: its place (page or slot; a valid one where nothing of it
// is attended) and its attended tokens.
template <int BS, bool PAGED>
__device__ __forceinline__ int block_raw(const TreeAttnArgs& a, const TreeItem& t, const Ctx& c, int b) {
  if constexpr (PAGED) return b < c.nb ? t.tab[b] : -1;
  else return b < a.k_slots ? t.tab[b] : (b == a.k_slots ? 0 : -1);
}
template <int BS, bool PAGED>
__device__ __forceinline__ void block_entry(const TreeAttnArgs& a, const Ctx& c, int L, int b, int raw, int& place,
                                            int& count) {
  if constexpr (PAGED) {
    const bool ok = raw >= 0 && raw < a.num_pages;
    const int n = L - b * BS;
    place = ok ? raw : 0;
    count = ok ? (n < BS ? n : BS) : 0;
  } else {
    place = b <= a.k_slots ? b : 0;
    count = raw < 0 ? 0 : (b == a.k_slots ? c.local_len : BS);
  }
}

// Q^T operand of the tile whose first row is `first`: lane (g, i) holds row first + i.
// A negative scale's sign is taken into the queries, and so is a scale of 0 (q_and,
// q_xor), so that the scale that the scores meet is positive.
__device__ __forceinline__ void load_q(const TreeAttnArgs& a, const TreeItem& t, int first, int g, int i, bf16x8 (&qb)[4]) {
  const int row = first + i;
  const int tq = row < a.rows ? a.by_g(row) : 0;
  const int qh = t.h * a.G + (row < a.rows ? row - tq * a.G : 0);
  const uint16_t* qrow = a.q + (((long long)t.r * a.T + tq) * a.Hq + qh) * kHeadDim;
#pragma unroll
  for (int st = 0; st < 4; ++st) {
    const u32x4 x = ldg16(qrow + st * 32 + g * 8);
    u32x4 y;
#pragma unroll
    for (int w = 0; w < 4; ++w) y[w] = row < a.rows ? (x[w] & a.q_and) ^ a.q_xor : 0u;
    qb[st] = as_bf16x8(y);
  }
}

// Up to two row tiles. Every load of a unit is issued a unit ahead into the registers
// that the present one has just left, 16 KB a wave on their way; two workgroups a CU
// (at most 256 registers) hide what that leaves. The tree's unit comes first, before the
// registers have a next one: as the last one, loaded in the same order, it cost copies of
// all of them in every step (the first case above 726 us).
template <int NT, int BS, bool PAGED, bool STREAM>
__global__ __launch_bounds__(kTW * 64) void tree_attn_kernel(TreeAttnArgs a) {
  static_assert(NT <= 2, "three or more row tiles take tree_attn_rows_kernel");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int g = lane >> 4;
  const int i = lane & 15;
  TreeItem t;
  if (!tree_setup<BS, PAGED>(a, NT * 16, t)) return;
  int L, u_begin, u_end;
  const Ctx c = tree_units<BS, PAGED>(a, t, L, u_begin, u_end);

  // A wave's units are u_begin + wave + n * kTW. For kChunk of them at a time, lane
  // e holds the place and the attended tokens of one block: block e % 2 of unit
  // e / 2 at B = 16, of unit e at B = 32. The next chunk's table entries are on
  // their way while a chunk is attended.
  constexpr int kPer = 32 / BS;  // blocks per unit
  constexpr int kChunk = 64 / kPer;
  const int u_first = u_begin + wave;
  const int nt = u_first < u_end ? (u_end - u_first + kTW - 1) / kTW : 0;
  auto entry_block = [&](int n0) { return (u_first + (n0 + lane / kPer) * kTW) * kPer + lane % kPer; };
  auto entry_load = [&](int n0) -> int {
    return n0 + lane / kPer < nt ? block_raw<BS, PAGED>(a, t, c, entry_block(n0)) : -1;
  };
  int n0 = 0, place, count;  // of this lane's block of the current chunk
  uint64_t live;             // blocks of the chunk with an attended token, not yet taken
  int raw = entry_load(0);
  auto chunk_set = [&]() __attribute__((always_inline)) {
    block_entry<BS, PAGED>(a, c, L, entry_block(n0), raw, place, count);
    raw = entry_load(n0 + kChunk);
    live = __builtin_amdgcn_ballot_w64(count > 0);
  };
  struct Next {
    int p0, p1, n0, n1;
    bool any;
  };
  // The wave's next unit with an attended token.
  auto next = [&]() __attribute__((always_inline)) {
    while (!live && n0 + kChunk < nt) {
      n0 += kChunk;
      chunk_set();
    }
    if (!live) return Next{0, 0, 0, 0, false};
    const int p = __builtin_ctzll(live) / kPer * kPer;
    live &= ~(((1ull << kPer) - 1) << p);
    return Next{__builtin_amdgcn_readlane(place, p), __builtin_amdgcn_readlane(place, p + kPer - 1),
                __builtin_amdgcn_readlane(count, p), __builtin_amdgcn_readlane(count, p + kPer - 1), true};
  };
  const uint32_t tok = 8 * (i >> 2) + (i & 3);  // K: token tile tau -> unit token tok + 4 tau
  const uint32_t ko = (BS == 16 ? tok & 15 : tok) * kHeadDim + g * 8;
  const uint32_t vo = PAGED ? (uint32_t)((BS == 16 ? g & 1 : g) * 8 * kHeadDim + i * 8)
                            : (uint32_t)(i * BS + (BS == 16 ? g & 1 : g) * 8);
  // Loads are issued for a wave without a next unit too, every lane on the first
  // bytes of place 0: the same number on every path keeps the compiler's wait
  // counts exact, so that waiting for one half of a unit never drains what is behind it.
  TreeUnit u;
  auto load_k = [&](const Next& n) __attribute__((always_inline)) {
    const uint16_t* ku = t.kb + (long long)(BS == 16 && i >= 8 ? n.p1 : n.p0) * t.unit_elems + (n.any ? ko : 0u);
#pragma unroll
    for (int tau = 0; tau < 2; ++tau)
#pragma unroll
      for (int st = 0; st < 4; ++st) u.k[tau][st] = ldg16(ku + tau * 4 * kHeadDim + st * 32);
  };
  auto load_v = [&](const Next& n) __attribute__((always_inline)) {
    const uint16_t* vu = t.vb + (long long)(BS == 16 && g >= 2 ? n.p1 : n.p0) * t.unit_elems + (n.any ? vo : 0u);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) u.v[dt] = ldg16_once<STREAM>(vu + (PAGED ? dt * kHeadDim : dt * 16 * BS));
  };

  bf16x8 qb[NT][4];
#pragma unroll
  for (int v = 0; v < NT; ++v) load_q(a, t, t.row0 + v * 16, g, i, qb[v]);
  float m_neg[NT], l_run[NT];
  f32x4 acc[NT][8];
#pragma unroll
  for (int v = 0; v < NT; ++v) {
    m_neg[v] = INFINITY;
    l_run[v] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[v][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  constexpr int kRows = NT * 16;
  constexpr int kPad = kHeadDim + 4;
  __shared__ float s_m[kTW][kRows], s_l[kTW][kRows], s_ml[2][kRows];
  __shared__ uint64_t s_anc[kTreeMaxTokens];
  __shared__ int s_wild[kTW];
  __shared__ __align__(16) float s_o[kTW][kRows][kPad];

  // ---- the tree's own tokens, unit tu of them in the last split: to the last waves,
  // which have a unit less of the cache than the first where they have not as many
  const int tu = kTW - 1 - wave;
  const bool tree = t.split == a.nsplit - 1 && tu * 32 < t.tlen;
  int wild = 0;
  if (tree) {
#pragma unroll
    for (int tau = 0; tau < 2; ++tau) {
      const int j = min(tu * 32 + (int)tok + 4 * tau, t.tlen - 1);
#pragma unroll
      for (int st = 0; st < 4; ++st) u.k[tau][st] = ldg16(a.tree_k + t.tree_base + j * t.tree_row + st * 32 + g * 8);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = min(tu * 32 + 8 * g + e, t.tlen - 1);
      u.v[e] = ldg16(a.tree_v + t.tree_base + j * t.tree_row + i * 8);
    }
    const uint64_t anc = ancestors(tree_parent(a, t.r, t.tlen, lane), t.tlen, lane);
    if (tu == 0) s_anc[lane] = anc;
    transpose8(u.v);
    const int n = t.tlen - tu * 32 - 8 * g;
    clear_tokens(u.v, n < 0 ? 0 : (n > 8 ? 8 : n));
    wild = take_wild(u.v);
    if constexpr (!PAGED) {
      // the working set's accumulators hold d-tile dt = dims 16 dt + i: through LDS,
      // [dim][32 tokens], each wave in its own part of the merge area
      u32x4* sv = reinterpret_cast<u32x4*>(&s_o[wave][0][0]);
#pragma unroll
      for (int j = 0; j < 8; ++j) sv[(8 * i + j) * 4 + g] = u.v[j];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) u.v[dt] = sv[(16 * dt + i) * 4 + g];
    }
#pragma unroll
    for (int v = 0; v < NT; ++v) {
      const int row = t.row0 + v * 16 + i;
      const int tq = row < a.rows ? a.by_g(row) : 0;
      const uint32_t half = __shfl((uint32_t)(anc >> (tu * 32)), tq);
      f32x4 sc[2];
      unit_scores(u.k, qb[v], sc);
      mask_scores(sc, half >> (8 * g) & 0xFF);
      unit_pv(u.v, unit_softmax(sc, a.scale_log2, a.top, m_neg[v], l_run[v], acc[v]), acc[v]);
    }
  }
  if (lane == 0) s_wild[wave] = wild;

  // ---- the cache: the next unit's K is loaded once this one's scores are known, its V
  // once this one's is used, into the same registers. Two workgroups of a CU hide what
  // that leaves of the latency.
  chunk_set();
  Next cur = next();
  load_k(cur);
  load_v(cur);
  while (cur.any) {
    const Next nxt = next();
    f32x4 sc[NT][2];
#pragma unroll
    for (int v = 0; v < NT; ++v) unit_scores(u.k, qb[v], sc[v]);
    __builtin_amdgcn_sched_barrier(0);
    load_k(nxt);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (PAGED) transpose8(u.v);
    if (cur.n0 < BS || (BS == 16 && cur.n1 < BS)) {
      const int n = BS == 16 ? (g < 2 ? cur.n0 : cur.n1) - (g & 1) * 8 : cur.n0 - g * 8;
      const int keep = n < 0 ? 0 : (n > 8 ? 8 : n);
      clear_tokens(u.v, keep);  // 0 times what an unused place holds must stay 0
#pragma unroll
      for (int v = 0; v < NT; ++v) mask_scores(sc[v], (1u << keep) - 1);
    }
#pragma unroll
    for (int v = 0; v < NT; ++v) unit_pv(u.v, unit_softmax(sc[v], a.scale_log2, a.top, m_neg[v], l_run[v], acc[v]), acc[v]);
    __builtin_amdgcn_sched_barrier(0);
    load_v(nxt);
    cur = nxt;
  }
  float m_run[NT];
#pragma unroll
  for (int v = 0; v < NT; ++v) m_run[v] = finish_row(m_neg[v], l_run[v]);

  // ---- merge the waves through LDS ----
  if (g == 0) {
#pragma unroll
    for (int v = 0; v < NT; ++v) {
      s_m[wave][v * 16 + i] = m_run[v];
      s_l[wave][v * 16 + i] = l_run[v];
    }
  }
  __syncthreads();  // the tree units' LDS reads are done too
#pragma unroll
  for (int v = 0; v < NT; ++v) {
    const int row = v * 16 + i;
    float M = s_m[0][row];
#pragma unroll
    for (int w = 1; w < kTW; ++w) M = fmaxf(M, s_m[w][row]);
    float S = 0.f;
#pragma unroll
    for (int w = 0; w < kTW; ++w) S += s_m[w][row] == -INFINITY ? 0.f : s_l[w][row] * fast_exp2(s_m[w][row] - M);
    const float f = m_run[v] == -INFINITY ? 0.f : fast_exp2(m_run[v] - M);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[v][dt] *= f;
    if (wave == 0 && g == 0) {
      s_ml[0][row] = M;
      s_ml[1][row] = S;
    }
    if constexpr (PAGED) {  // dims 32 g + 8 e + dt
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int q = 0; q < 2; ++q)
          *reinterpret_cast<f32x4*>(&s_o[wave][row][32 * g + 8 * e + 4 * q]) =
              f32x4{acc[v][4 * q][e], acc[v][4 * q + 1][e], acc[v][4 * q + 2][e], acc[v][4 * q + 3][e]};
    } else {  // dims 16 dt + 4 g + e
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f32x4*>(&s_o[wave][row][16 * dt + 4 * g]) = acc[v][dt];
    }
  }
  __syncthreads();

  const long long pbase = ((long long)t.rh * a.nsplit + t.split) * a.rows + t.row0;
  const int last = min(t.tlen * a.G, a.rows) - t.row0;  // rows of this group in the tree
  for (int pos = threadIdx.x; pos < kRows * (kHeadDim / 4); pos += kTW * 64) {
    const int row = pos >> 5;
    const int c4 = pos & 31;
    if (row >= last) break;
    f32x4 o = *reinterpret_cast<const f32x4*>(&s_o[0][row][c4 * 4]);
#pragma unroll
    for (int w = 1; w < kTW; ++w) o += *reinterpret_cast<const f32x4*>(&s_o[w][row][c4 * 4]);
    if (s_wild[kTW - 1] | s_wild[kTW - 2]) add_wild(a, t, s_anc[a.by_g(t.row0 + row)], c4, o);
    if (a.nsplit == 1) {
      write_row(a, t.r, t.h, t.row0 + row, c4, o, s_ml[0][row], s_ml[1][row]);
    } else {
      *reinterpret_cast<f32x4*>(a.part_o + (pbase + row) * kHeadDim + c4 * 4) = o;
      if (c4 == 0) *reinterpret_cast<float2*>(a.part_ml + (pbase + row) * 2) = make_float2(s_ml[0][row], s_ml[1][row]);
    }
  }
}

// 16 bytes a lane from global memory straight into LDS: lane L's bytes land at
// offset lds + 16 L, lds being the same in every lane. In assembly for the reason
// given at the working set's attention (lds_dma16): the compiler would drain every
// earlier load before each one; the waits are the kernel's own counts instead.
template <bool STREAM>
__device__ __forceinline__ void tree_dma16(const void* src, uint32_t lds) {
  uint32_t saved;
  if constexpr (STREAM)
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %2\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %1, off nt\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(src), "s"(lds)
        : "memory");
  else
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %2\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %1, off\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(src), "s"(lds)
        : "memory");
}
__device__ __forceinline__ uint32_t lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
template <int N>
__device__ __forceinline__ void tree_wait() {  // s_waitcnt vmcnt(N) alone
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

// More than two row tiles. Eight waves in two teams: a wave holds one or two of a
// team's (up to) eight row tiles, and a team takes every other unit. A step is two
// units, one for each team; a ring of kRingSteps steps in LDS is filled by loads that
// go straight there, four a wave and step; one barrier a step publishes it and frees
// the one before. Two tiles a wave: each unit is read from LDS by four waves, 64 KB,
// which takes as long as their products do.
//
// The units of a split are listed first, up to kListUnits at a time, the ones without
// an attended token left out: whole ones ahead, which a loop without masks takes, then
// the others, then the tree's. A load takes four tokens of K or of token-major V, whole
// rows of them, and leaves their 32-byte pieces in turn (token p's piece c at 128 c +
// 32 p): an MFMA operand of K is a 16-byte read a lane, one of V the transposing read of
// 4 tokens x 16 dims a group of 16 lanes, 128 bytes in a row, where lane (g, i) names
// dims 4 (i % 4) .. +3 of token i / 4 and receives dim i of the four. The working set's
// transposed V is put there in operand layout.
//
// A unit's order is: V is read, scores; the next unit's K is read; softmax, second
// product. So LDS reads run beside the products, in the registers that these leave.
//
// With two tiles a wave a step takes some 2,000 cycles, 1,024 of them the matrix unit's;
// the softmax of the other wave of the SIMD runs beside about half of these. Without the
// barrier (each team waiting on a count of its own in LDS) or with the loads spread over
// the step it is 9 % slower. With one tile a wave (three and four row tiles) the loads
// bound it, and those of caches that no cache of the chip holds go past them: 228 us
// where they do not, 208 where they do.
constexpr int kRingSteps = 4;
constexpr int kListUnits = 1024;
constexpr int kListPad = 4 + 2 * kRingSteps;  // the tree's units, and none behind them
constexpr int kRowsThreads = 512;
constexpr int kRowPlaces = 4;  // waves of a team
// A unit in LDS: K, then V, 8 KB each and a skew after every two pieces, so that the
// lanes of one read meet no bank twice.
constexpr int kSkewK = 128, kSkewV = 128;
constexpr int kUnitV = 8 * 1024 + 4 * kSkewK;
constexpr int kUnitBytes = kUnitV + 8 * 1024 + 4 * kSkewV;

template <int NT, int BS, bool PAGED, bool STREAM>
__global__ __launch_bounds__(kRowsThreads) void tree_attn_rows_kernel(TreeAttnArgs a) {
  constexpr int kRows = NT * kRowPlaces * 16;
  constexpr int kPad = kHeadDim + 4;
  __shared__ __align__(16) char s_ring[kRingSteps * 2 * kUnitBytes];
  // places and attended tokens of a unit's blocks; x: which, z = -1: a unit of the tree; z = -2: none
  __shared__ __align__(16) int4 s_list[kListUnits + kListPad];
  __shared__ uint64_t s_anc[kTreeMaxTokens];
  __shared__ float s_ml[2][kRows];
  __shared__ int s_wave[8][2], s_wild;
  static_assert(sizeof(float) * kRows * kPad <= sizeof(s_ring), "a team's rows fit the ring");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int g = lane >> 4;
  const int i = lane & 15;
  const int team = wave / kRowPlaces;
  const int rt = wave % kRowPlaces;  // this wave's tiles: rt and rt + 4 of the group's
  TreeItem t;
  if (!tree_setup<BS, PAGED>(a, a.tiles * 16, t)) return;
  int L, u_begin, u_end;
  const Ctx c = tree_units<BS, PAGED>(a, t, L, u_begin, u_end);
  const bool last_split = t.split == a.nsplit - 1;

  bf16x8 qb[NT][4];
#pragma unroll
  for (int v = 0; v < NT; ++v) load_q(a, t, t.row0 + (rt + v * kRowPlaces) * 16, g, i, qb[v]);
  const int parent = last_split && wave == 0 ? tree_parent(a, t.r, t.tlen, lane) : -1;
  if (threadIdx.x == 0) s_wild = 0;
  float m_neg[NT], l_run[NT];
  f32x4 acc[NT][8];
#pragma unroll
  for (int v = 0; v < NT; ++v) {
    m_neg[v] = INFINITY;
    l_run[v] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[v][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // What this wave loads: of unit `half` of a step, pieces j0 .. j0 + 3 of K or of V,
  // tokens 4 j .. 4 j + 3 in piece j (of transposed V d-tile j). A lane's element
  // offset within the unit's block lo or hi, piece jj being jj * step further.
  const int half = wave >> 2;
  const bool load_v = wave & 2;
  const int j0 = (wave & 1) * 4;
  const bool by_row = PAGED || !load_v;  // token-major
  int off;
  bool hi;
  if (by_row) {
    const int row = 4 * j0 + (lane >> 1 & 3);
    off = (BS == 16 ? row & 15 : row) * kHeadDim + (lane >> 3) * 16 + (lane & 1) * 8;
    hi = BS == 16 && j0 >= 4;
  } else {
    off = (j0 * 16 + i) * BS + (BS == 16 ? g & 1 : g) * 8;
    hi = BS == 16 && g >= 2;
  }
  const int step = by_row ? 4 * kHeadDim : 16 * BS;
  const uint16_t* src0 = load_v ? t.vb : t.kb;
  const uint32_t ring = lds_offset(s_ring);
  const int tree_units_n = last_split ? (t.tlen + 31) / 32 : 0;

  for (int seg = u_begin; seg == u_begin || seg < u_end; seg += kListUnits) {
    // ---- list this segment's units: whole ones from the front, others from the back ----
    const int n_seg = min(kListUnits, u_end - seg);
    const bool final_seg = seg + kListUnits >= u_end;
    int n_full = 0, n_part = 0;
    for (int b0 = 0; b0 < n_seg; b0 += kRowsThreads) {
      const int n = b0 + (int)threadIdx.x;
      int4 e = make_int4(0, 0, 0, 0);
      if (n < n_seg) {
        const int b = (seg + n) * (32 / BS);
        block_entry<BS, PAGED>(a, c, L, b, block_raw<BS, PAGED>(a, t, c, b), e.x, e.z);
        if (BS == 16) block_entry<BS, PAGED>(a, c, L, b + 1, block_raw<BS, PAGED>(a, t, c, b + 1), e.y, e.w);
        e.w = max(e.w, 0);  // a block past the context
      }
      const bool full = e.z == BS && (BS == 32 || e.w == BS);
      const bool part = !full && (e.z > 0 || e.w > 0);
      const uint64_t fulls = __builtin_amdgcn_ballot_w64(full), parts = __builtin_amdgcn_ballot_w64(part);
      if (lane == 0) {
        s_wave[wave][0] = __popcll(fulls);
        s_wave[wave][1] = __popcll(parts);
      }
      __syncthreads();
      const uint64_t below = (1ull << lane) - 1;
      int at_f = n_full + __popcll(fulls & below), at_p = n_part + __popcll(parts & below);
      for (int w = 0; w < 8; ++w) {
        const int kf = s_wave[w][0], kp = s_wave[w][1];
        at_f += w < wave ? kf : 0;
        at_p += w < wave ? kp : 0;
        n_full += kf;
        n_part += kp;
      }
      if (full) s_list[at_f] = e;
      if (part) s_list[kListUnits - 1 - at_p] = e;
      __syncthreads();
    }
    n_full = __builtin_amdgcn_readfirstlane(n_full);
    n_part = __builtin_amdgcn_readfirstlane(n_part);
    const int total = n_full + n_part;
    const int units = total + (final_seg ? tree_units_n : 0);
    const int steps = (units + 1) / 2;
    if (threadIdx.x < kListPad)
      s_list[kListUnits + threadIdx.x] =
          total + (int)threadIdx.x < units ? make_int4((int)threadIdx.x, 0, -1, 0) : make_int4(0, 0, -2, 0);
    __syncthreads();
    auto entry_read = [&](int n) __attribute__((always_inline)) {
      return s_list[n < n_full ? n : (n < total ? kListUnits - 1 - (n - n_full) : kListUnits + (n - total))];
    };
    auto uniform = [&](int4 e) __attribute__((always_inline)) {
      return make_int4(__builtin_amdgcn_readfirstlane(e.x), __builtin_amdgcn_readfirstlane(e.y),
                       __builtin_amdgcn_readfirstlane(e.z), __builtin_amdgcn_readfirstlane(e.w));
    };
    // This wave's loads of step s, whose list entry is `raw`.
    auto issue = [&](int s, int4 raw) __attribute__((always_inline)) {
      const int4 e = uniform(raw);
      const uint32_t dst = ring + (uint32_t)((s % kRingSteps * 2 + half) * kUnitBytes + (load_v ? kUnitV : 0) + j0 * 1024);
      const uint32_t skew = load_v ? (PAGED || e.z == -1 ? kSkewV : 0) : kSkewK;  // per two pieces
      if (e.z != -1) {
        const uint16_t* src = src0 + (long long)(hi ? e.y : e.x) * t.unit_elems + off;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) tree_dma16<STREAM>(src + jj * step, dst + jj * 1024 + (j0 + jj) / 2 * skew);
      } else {  // the tree's rows
        int ll = lane;
        asm volatile("" : "+v"(ll));  // its terms are not worth registers through the loop
        const uint16_t* src = (load_v ? a.tree_v : a.tree_k) + t.tree_base + (ll >> 3) * 16 + (ll & 1) * 8;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          const int row = e.x * 32 + 4 * (j0 + jj) + (ll >> 1 & 3);
          tree_dma16<false>(src + min(row, t.tlen - 1) * t.tree_row, dst + jj * 1024 + (j0 + jj) / 2 * skew);
        }
      }
    };
    TreeUnit u;
    auto unit_at = [&](int s) __attribute__((always_inline)) { return s_ring + (s % kRingSteps * 2 + team) * kUnitBytes; };
    auto read_k = [&](int s) __attribute__((always_inline)) {
      // token tile tau, k-step st: token 4 (2 (i / 4) + tau) + i % 4, dims 32 st + 8 g .. +7
      const char* at = unit_at(s) + (i >> 2) * (2048 + kSkewK) + (g >> 1) * 128 + (i & 3) * 32 + (g & 1) * 16;
#pragma unroll
      for (int tau = 0; tau < 2; ++tau)
#pragma unroll
        for (int st = 0; st < 4; ++st)
          u.k[tau][st] = *reinterpret_cast<const u32x4*>(at + tau * 1024 + st * 256);
    };
    auto read_v = [&](int s, bool by_row) __attribute__((always_inline)) {
      if (by_row) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        // tokens 8 g + 4 q .. +3 at load 2 g + q
        char* at = unit_at(s) + kUnitV + g * (2048 + kSkewV) + (i >> 2) * 32 + (i & 3) * 8;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const u32x2 w = __builtin_bit_cast(
                u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                           (__attribute__((address_space(3))) s16x4*)(at + q * 1024 + dt * 128)));
            u.v[dt][2 * q] = w[0];
            u.v[dt][2 * q + 1] = w[1];
          }
      } else {
        const u32x4* at = reinterpret_cast<const u32x4*>(unit_at(s) + kUnitV) + lane;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) u.v[dt] = at[dt * 64];
      }
    };
    // Between the barriers of steps s - 1 and s the units of steps s and s + 1 are in
    // LDS, and the loads of step s + 3 go out, into the place of step s - 1. Behind
    // barrier s step s + 2 is there too: this wave's loads of it are in by then, and
    // the barrier publishes every wave's and tells that step s is no longer read.
    auto leave = [&]() __attribute__((always_inline)) {
      tree_wait<4>();
      __syncthreads();
    };
#pragma unroll 1
    for (int s = 0; s < 3; ++s) issue(s, entry_read(s * 2 + half));
    if (last_split && wave == 0 && seg == u_begin) s_anc[lane] = ancestors(parent, t.tlen, lane);
    leave();
    read_k(0);
    f32x4 sc[NT][2];
    auto attend = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int v = 0; v < NT; ++v) unit_pv(u.v, unit_softmax(sc[v], a.scale_log2, a.top, m_neg[v], l_run[v], acc[v]), acc[v]);
      __builtin_amdgcn_sched_barrier(0);  // no reads ahead of it, into registers that are then spilled
    };
    // The two waves of a SIMD are of different teams, and do a step's parts in
    // different order, so that one's products run beside the other's softmax: team 0
    // leaves a unit's softmax and second product to the next step.
    const int whole = n_full / 2;  // steps of two whole units
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
      // (32 loads at once, behind the barrier, would hold every wave up for some 500
      // cycles: each team's go out at another time, the list entry read ahead)
      const int4 ahead = entry_read((s + 3) * 2 + half);
      if (team == 0) {
        issue(s + 3, ahead);
        __builtin_amdgcn_sched_barrier(0);
        if (s > 0) attend();
      }
      read_v(s, PAGED);
#pragma unroll
      for (int v = 0; v < NT; ++v) unit_scores(u.k, qb[v], sc[v]);
      __builtin_amdgcn_sched_barrier(0);
      read_k(s + 1);
      if constexpr (PAGED) {  // the halves of the reads above are one operand from here on, in every branch
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) asm volatile("" : "+v"(u.v[dt]));
      }
      if (s >= whole) {  // masks
        const int4 e = uniform(entry_read(s * 2 + team));
        const bool tree = e.z == -1;
        if (tree && !PAGED) read_v(s, true);
        const int n = tree ? t.tlen - e.x * 32 - 8 * g : (BS == 16 ? (g < 2 ? e.z : e.w) - (g & 1) * 8 : e.z - g * 8);
        const int keep = n < 0 ? 0 : (n > 8 ? 8 : n);
        clear_tokens(u.v, keep);  // 0 times what an unused place holds must stay 0
        if (tree) {
          if (take_wild(u.v)) s_wild = 1;
        }
#pragma unroll
        for (int v = 0; v < NT; ++v) {
          uint32_t bits = (1u << keep) - 1;
          if (tree) {
            const int row = t.row0 + (rt + v * kRowPlaces) * 16 + i;
            bits = (uint32_t)(s_anc[row < a.rows ? a.by_g(row) : 0] >> (e.x * 32 + 8 * g));
          }
          mask_scores(sc[v], bits);
        }
      }
      if (team == 1) {
        issue(s + 3, ahead);
        __builtin_amdgcn_sched_barrier(0);
        attend();
      }
      leave();
    }
    if (team == 0 && steps > 0) attend();
    tree_wait<0>();   // the loads past the last step land before the ring and the list are reused
    __syncthreads();
  }

  // ---- merge the teams: the second one's rows through LDS, the sums back there ----
  float(*s_o)[kPad] = reinterpret_cast<float(*)[kPad]>(s_ring);  // [row of the group]
#pragma unroll
  for (int v = 0; v < NT; ++v) m_neg[v] = -finish_row(m_neg[v], l_run[v]);
  if (team == 1) {
#pragma unroll
    for (int v = 0; v < NT; ++v) {
      const int row = (rt + v * kRowPlaces) * 16 + i;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f32x4*>(&s_o[row][16 * dt + 4 * g]) = acc[v][dt];
      if (g == 0) {
        s_ml[0][row] = -m_neg[v];
        s_ml[1][row] = l_run[v];
      }
    }
  }
  __syncthreads();
  if (team == 0) {
#pragma unroll
    for (int v = 0; v < NT; ++v) {
      const int row = (rt + v * kRowPlaces) * 16 + i;
      const float m0 = -m_neg[v], m1 = s_ml[0][row], M = fmaxf(m0, m1);
      const float f0 = m0 == -INFINITY ? 0.f : fast_exp2(m0 - M), f1 = m1 == -INFINITY ? 0.f : fast_exp2(m1 - M);
      const float S = l_run[v] * f0 + s_ml[1][row] * f1;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
        f32x4& o = *reinterpret_cast<f32x4*>(&s_o[row][16 * dt + 4 * g]);
        o = acc[v][dt] * f0 + o * f1;
      }
      if (g == 0) {  // the row's other lanes have read them
        s_ml[0][row] = M;
        s_ml[1][row] = S;
      }
    }
  }
  __syncthreads();
  const long long pbase = ((long long)t.rh * a.nsplit + t.split) * a.rows + t.row0;
  const int last = min(min(t.tlen * a.G, a.rows) - t.row0, a.tiles * 16);  // rows of this group in the tree
  for (int pos = threadIdx.x; pos < kRows * (kHeadDim / 4); pos += kRowsThreads) {
    const int row = pos >> 5;
    const int c4 = pos & 31;
    if (row >= last) break;
    f32x4 o = *reinterpret_cast<const f32x4*>(&s_o[row][c4 * 4]);
    if (s_wild) add_wild(a, t, s_anc[a.by_g(t.row0 + row)], c4, o);
    if (a.nsplit == 1) {
      write_row(a, t.r, t.h, t.row0 + row, c4, o, s_ml[0][row], s_ml[1][row]);
    } else {
      *reinterpret_cast<f32x4*>(a.part_o + (pbase + row) * kHeadDim + c4 * 4) = o;
      if (c4 == 0) *reinterpret_cast<float2*>(a.part_ml + (pbase + row) * 2) = make_float2(s_ml[0][row], s_ml[1][row]);
    }
  }
}

// Merge of the splits: 8 rows of one pair per workgroup, 32 threads a row, 4 dims a
// thread; the splits are read kBatch at a time.
constexpr int kTreeMergeRows = 8;

__global__ __launch_bounds__(kTreeMergeRows * 32) void tree_merge_kernel(TreeAttnArgs a) {
  const int item = tree_item(blockIdx.x, a.R * a.Hkv * a.groups);  // a.groups, by_groups: of kTreeMergeRows rows
  if (item < 0) return;
  const int rh = a.by_groups(item);
  const int row = (item - rh * a.groups) * kTreeMergeRows + (threadIdx.x >> 5);
  const int r = a.by_hkv(rh);
  if (row >= tree_length(a, r) * a.G) return;
  const int c4 = threadIdx.x & 31;
  const long long base = (long long)rh * a.nsplit * a.rows + row;
  float M = -INFINITY, S = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  constexpr int kBatch = 8;
  for (int s0 = 0; s0 < a.nsplit; s0 += kBatch) {
    float2 ml[kBatch];
    f32x4 os[kBatch];
#pragma unroll
    for (int s = 0; s < kBatch; ++s) {
      const long long idx = base + (long long)min(s0 + s, a.nsplit - 1) * a.rows;
      ml[s] = *reinterpret_cast<const float2*>(a.part_ml + idx * 2);
      os[s] = *reinterpret_cast<const f32x4*>(a.part_o + idx * kHeadDim + c4 * 4);
    }
    float mn = M;
#pragma unroll
    for (int s = 0; s < kBatch; ++s) mn = fmaxf(mn, s0 + s < a.nsplit ? ml[s].x : -INFINITY);
    const float keep = M == -INFINITY ? 0.f : fast_exp2(M - mn);
    S *= keep;
    o *= keep;
#pragma unroll
    for (int s = 0; s < kBatch; ++s) {
      if (s0 + s < a.nsplit) {
        // a split without an attended token (maximum -inf) weighs nothing
        const float f = ml[s].x == -INFINITY ? 0.f : fast_exp2(ml[s].x - mn);
        S += ml[s].y * f;
        o += os[s] * f;
      }
    }
    M = mn;
  }
  // An infinity in a split whose weight is too small for a float meets a factor of 0
  // above, and is NaN: its weight is positive, so the row takes it up as it is, as it
  // does where one split holds everything. Rare, and so read again.
  if (__builtin_amdgcn_ballot_w64(o[0] != o[0] || o[1] != o[1] || o[2] != o[2] || o[3] != o[3])) {
    f32x4 w = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.nsplit; ++s) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(a.part_o + (base + (long long)s * a.rows) * kHeadDim + c4 * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] += wild_f32(x[e]) ? x[e] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = wild_f32(w[e]) ? w[e] : o[e];
  }
  write_row(a, r, rh - r * a.Hkv, row, c4, o, M, S);
}

// A scale of 0 takes the queries' bits away (q_and), and with them infinities and NaN, 0
// times which is a NaN score of every token: the rows of such queries, after the others.
// (Looked at where the queries are read, or where rows are written, every call of wide
// trees paid 1 to 3 % for it.)
//
// A row that attends nothing keeps its 0 and -infinity. With a tree it attends itself;
// without one (the 4-bit cache) it attends a token where a block of the context, or of the
// selection and the local one, has a page of the tier: its 32 lanes look at as many blocks
// at a time.
__device__ __forceinline__ uint32_t of_row(bool x) {
  return (uint32_t)(__builtin_amdgcn_ballot_w64(x) >> (threadIdx.x & 32));
}
__device__ bool cache_attended(const TreeAttnArgs& a, const CacheSelection& sel, int r, int h) {
  const Ctx c = ctx_blocks(a.ctx_len[r], a.B, a.NBmax);
  if (c.nb == 0) return false;
  int selected = c.n_cand;
  const int32_t* ids = nullptr;
  if (sel.ids) {
    const long long rh = (long long)r * a.Hkv + h;
    selected = min(max(sel.count[rh], 0), sel.k);
    ids = sel.ids + rh * sel.k;
  }
  const int32_t* table = a.table + (long long)r * a.NBmax;
  for (int b0 = 0; b0 <= selected; b0 += 32) {  // the local block last
    const int b = b0 + (threadIdx.x & 31);
    int id = c.n_cand;
    bool in = b <= selected;
    if (ids && b < selected) {
      id = ids[b];
      in = id >= 0 && id < c.n_cand;
    } else if (b < selected) {
      id = b;
    }
    const int page = in ? table[id] : -1;
    if (of_row(page >= 0 && page < a.num_pages)) return true;
  }
  return false;
}

__global__ __launch_bounds__(kTreeWildRows * 32) void wild_queries_kernel(TreeAttnArgs a, CacheSelection sel) {
  const int c4 = threadIdx.x & 31;
  const int rows = a.R * a.T * a.Hq;  // at most 2^28
  for (int row = blockIdx.x * kTreeWildRows + (threadIdx.x >> 5); row < rows; row += gridDim.x * kTreeWildRows) {
    const int rt = row / a.Hq, r = rt / a.T;
    if (rt - r * a.T >= tree_length(a, r)) continue;
    const long long at = (long long)row * kHeadDim + c4 * 4;
    const uint2 w = *reinterpret_cast<const uint2*>(a.q + at);
    if (!of_row(wild_bf16(w.x) || wild_bf16(w.x >> 16) || wild_bf16(w.y) || wild_bf16(w.y >> 16))) continue;
    if (!a.tree_k && !cache_attended(a, sel, r, a.by_g(row - rt * a.Hq))) continue;
    *reinterpret_cast<uint2*>(a.out + at) = make_uint2(0x7FC07FC0u, 0x7FC07FC0u);
    if (c4 == 0 && a.lse) a.lse[row] = __builtin_nanf("");
  }
}

template <int BS, bool PAGED>
void launch_bs(const TreeAttnArgs& a, hipStream_t s) {
  const long long runs = (long long)a.R * a.Hkv * a.nsplit;  // of keys and values
  const dim3 grid((unsigned)(a.by_length ? (runs + 7) / 8 * 8 * a.groups : (runs * a.groups + 7) / 8 * 8));
  // What the tables and pools hold at most: past kStreamBytes V, whose loads take whole
  // lines, is read past the caches (8 x 131,072 tokens, 4.3 GB, 711 and 640 us; 64 x
  // 2,064, 541 MB, half of it attended, 80.8 and 76.5; 68 MB, in the Infinity Cache, 21.2
  // and 21.3; K as well 639, 80.1), and with one tile a wave of the form for more rows both
  // are; with two tiles several workgroups read them, through the L2.
  const long long blocks = PAGED ? a.NBmax : (a.k_slots + 1ll < a.NBmax ? a.k_slots + 1ll : a.NBmax);
  const bool stream = (long long)a.R * a.Hkv * blocks * BS * (2 * kHeadDim * 2) >= kStreamBytes;
  if (a.tiles == 1)
    hipLaunchKernelGGL((stream ? tree_attn_kernel<1, BS, PAGED, true> : tree_attn_kernel<1, BS, PAGED, false>), grid,
                       dim3(kTW * 64), 0, s, a);
  else if (a.tiles == 2)
    hipLaunchKernelGGL((stream ? tree_attn_kernel<2, BS, PAGED, true> : tree_attn_kernel<2, BS, PAGED, false>), grid,
                       dim3(kTW * 64), 0, s, a);
  else if (a.tiles <= kRowPlaces)
    hipLaunchKernelGGL((stream ? tree_attn_rows_kernel<1, BS, PAGED, true> : tree_attn_rows_kernel<1, BS, PAGED, false>),
                       grid, dim3(kRowsThreads), 0, s, a);
  else
    hipLaunchKernelGGL((tree_attn_rows_kernel<2, BS, PAGED, false>), grid, dim3(kRowsThreads), 0, s, a);
}

}  // namespace

hipError_t launch_tree_finish(const TreeAttnArgs& a, const CacheSelection& sel, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (a.nsplit > 1) {
    TreeAttnArgs m = a;
    m.groups = (a.rows + kTreeMergeRows - 1) / kTreeMergeRows;
    m.by_groups = fast_div(m.groups);
    const long long items = (long long)a.R * a.Hkv * m.groups;
    hipLaunchKernelGGL(tree_merge_kernel, dim3((unsigned)((items + 7) / 8 * 8)), dim3(kTreeMergeRows * 32), 0, s, m);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.q_and != 0) return e;
  hipLaunchKernelGGL(wild_queries_kernel, dim3(tree_wild_groups((long long)a.R * a.T * a.Hq)), dim3(kTreeWildRows * 32), 0, s,
                     a, sel);
  return hipGetLastError();
}

hipError_t launch_tree_attn(const TreeAttnArgs& a, bool paged, hipStream_t s) {
  if (a.B == 16)
    paged ? launch_bs<16, true>(a, s) : launch_bs<16, false>(a, s);
  else
    paged ? launch_bs<32, true>(a, s) : launch_bs<32, false>(a, s);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_tree_finish(a, CacheSelection{}, s);
}

}  // namespace oasis
