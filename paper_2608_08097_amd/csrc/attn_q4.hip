// Attention of a step's rows, a drafted tree or not, over the 4-bit paged cache: over
// every cached token, or over the blocks selected for each KV head, read where they lie.
//
// out = softmax(scale q K^T) V in one pass with a running maximum and sum, as tree_attn.hip,
// whose row references, merge and treatment of the tree's wild values are used here. A unit
// is 64 tokens of one KV head, four sub-blocks of 16; for one 16-row tile
//   S^T (tokens x rows) = K . Q^T     16 of v_mfma_f32_16x16x32_bf16
//   O^T (d x rows)     += V^T . P^T   16 of them
//
// Codes become bf16 exactly, two a conversion with their power of two, and both products are
// those of tree_attn.hip over the values that the cache stands for. The probabilities are
// rounded to bf16 for the second one, their sums are not (unit_softmax in tree_core.h). Two
// forms.
//
// Up to two row tiles every wave streams units of its own. Of a sub-block a lane has 32 dims of
// a token in 16 bytes, with one power: keys are the first product's operand as soon as they are
// turned, the queries being dealt to the same dims. The second product needs 8 tokens of one
// dim in a lane: values go through LDS, 16 KB a wave, and come back through the transposing
// read. (Left as codes there, with the powers taken up by the probabilities, they took 249 us
// instead of 220 in the second case below.) With more rows eight waves share what is turned.
//
// The tree's rows, keys and values in bf16, are a unit of their own in the last split of
// every pair.
//
// Measured (136 bytes a token and KV head; 4 d operations a row and token):
//   8 requests x 8 heads x 131,072 tokens, 4 rows    180 us  6.3 TB/s
//   8 x 8 x 131,072, 20 rows                         201-208 us  5.6 TB/s; its loads alone take 174 and the
//                                                    clock falls from 2.4 to 2.2 GHz with the products
//   24 x 8 x 1 to 32,768, 64 rows                    151-173 us a draw; of its 768 workgroups on 512 places
//                                                    the last ends at 1.3 times a place's share of the units
//   2 x 8 x 65,000 to 65,536, 512 rows               297-307 us  890-920 TFLOP/s
//   16 x 8 x 4,128 selected, 72 rows                 52 us
//   8 x 8 x 2,064 selected, 20 rows                  16.1 us  two launches (7.4), four loads in turn
//   1 x 8 x 2,000, 4 rows                            8.8-9.5 us  the same
// A read of 1 KB pieces in any order reaches 6.7 TB/s here past the caches and 5.9 through
// them, hence the loads of large caches.
#include "tree_core.h"
#include "q4_internal.h"

namespace oasis {
namespace {

constexpr int kQW = kQ4Waves;
constexpr int kUnitTokens = kQ4Unit;  // four sub-blocks of 16

struct Q4Item {
  int r, h, rh, split, row0, tlen, ctx;
  const int32_t* tab;   // the request's block table
  const int32_t* sel;   // the pair's selection, `selected` of them
  int selected;
  long long tree_row, tree_base;  // elements between the tree's rows, and to this head's first one
};

template <bool SELECT>
__device__ __forceinline__ bool q4_setup(const AttnQ4Args& a, int group_rows, Q4Item& t) {
  int group, rs;
  if (!SELECT && a.by_length) {
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
  if (!SELECT && a.by_length) {
    t.r = request_of_rank(a.ctx_len, a.R, t.r, t.ctx);
    t.rh = t.r * a.Hkv + t.h;
  } else {
    t.ctx = a.ctx_len[t.r];
  }
  t.tab = a.table + (long long)t.r * a.NBmax;
  t.selected = 0;
  if constexpr (SELECT) {
    t.sel = a.sel + (long long)t.rh * a.k_sel;
    const int n = a.sel_count[t.rh];
    t.selected = n < 0 ? 0 : (n > a.k_sel ? a.k_sel : n);
  }
  t.tree_row = (long long)a.Hkv * kHeadDim;
  t.tree_base = (long long)t.r * a.T * t.tree_row + (long long)t.h * kHeadDim;
  t.tlen = tree_length(a, t.r);
  return t.row0 < t.tlen * a.G;  // else no row of this group is in use
}

// Entry b of the pair's list of blocks: its page, and in `count` its attended tokens (0: none
// such, and page 0 stands in).
template <int BS, bool SELECT>
__device__ __forceinline__ void q4_block(const AttnQ4Args& a, const Q4Item& t, const Ctx& c, int b, int& page, int& count) {
  int id = b;
  bool ok;
  if constexpr (SELECT) {
    ok = b < t.selected;
    id = ok ? t.sel[b] : c.n_cand;
    ok = ok ? id >= 0 && id < c.n_cand : b == t.selected && c.nb > 0;
  } else {
    ok = b < c.nb;
  }
  const int raw = ok ? t.tab[id] : -1;
  ok = raw >= 0 && raw < a.num_pages;
  page = ok ? raw : 0;
  count = ok ? (id == c.n_cand ? c.local_len : BS) : 0;
}

template <int SEL>
__device__ __forceinline__ uint32_t two_bf16(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}
__device__ __forceinline__ bf16x8 eight_bf16(uint32_t codes, float scale) {
  const u32x4 v = {two_bf16<0>(codes, scale), two_bf16<1>(codes, scale), two_bf16<2>(codes, scale),
                   two_bf16<3>(codes, scale)};
  return as_bf16x8(v);
}

// Q^T operand of the tile whose first row is `first`: lane (g, n) holds row first + n, dims
// 32 g + 8 st .. +7 of step st (signs and a scale of 0 as load_q of tree_attn.hip).
__device__ __forceinline__ void load_q4_queries(const TreeAttnArgs& a, const Q4Item& t, int first, int g, int n,
                                                bf16x8 (&qb)[4]) {
  const int row = first + n;
  const int tq = row < a.rows ? a.by_g(row) : 0;
  const int qh = t.h * a.G + (row < a.rows ? row - tq * a.G : 0);
  const uint16_t* qrow = a.q + (((long long)t.r * a.T + tq) * a.Hq + qh) * kHeadDim;
#pragma unroll
  for (int st = 0; st < 4; ++st) {
    const u32x4 x = ldg16(qrow + g * 32 + st * 8);
    u32x4 y;
#pragma unroll
    for (int w = 0; w < 4; ++w) y[w] = row < a.rows ? (x[w] & a.q_and) ^ a.q_xor : 0u;
    qb[st] = as_bf16x8(y);
  }
}

// The online softmax of tree_attn.hip over a lane's 4 U scores of the first `used` tiles, with
// one branch for all: probabilities not yet rounded.
template <int U>
__device__ __forceinline__ float exp_of(const f32x4 (&s)[U], float scale, float m_neg, float (&p)[4 * U]) {
  float sum[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int e = 0; e < 4; ++e) p[4 * u + e] = fast_exp2(__builtin_fmaf(s[u][e], scale, m_neg));
    sum[u] = (p[4 * u] + p[4 * u + 1]) + (p[4 * u + 2] + p[4 * u + 3]);
  }
  if constexpr (U == 4) return (sum[0] + sum[1]) + (sum[2] + sum[3]);
  else return sum[0] + sum[1];
}
template <int NT, int U>
__device__ __forceinline__ void softmax_of(const f32x4 (&s)[NT][U], float scale, float top, float (&m_neg)[NT],
                                           float (&l_part)[NT], f32x4 (&acc)[NT][8], float (&p)[NT][4 * U], int used = NT) {
  float psum[NT];
  bool over = false;
#pragma unroll
  for (int v = 0; v < NT; ++v) {
    if (v >= used) continue;
    psum[v] = exp_of(s[v], scale, m_neg[v], p[v]);
    over |= !(psum[v] <= top);
  }
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(over) != 0, 0)) {
#pragma unroll
    for (int v = 0; v < NT; ++v) {
      if (v >= used) continue;
      const uint64_t past = __builtin_amdgcn_ballot_w64(!(psum[v] <= top));
      const uint64_t rows = past | past >> 16 | past >> 32 | past >> 48;
      const bool mine = rows >> (threadIdx.x & 15) & 1;
      float m = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u) m = fmaxf(m, fmaxf(fmaxf(s[v][u][0], s[v][u][1]), fmaxf(s[v][u][2], s[v][u][3])));
      m *= scale;
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(fmaxf(m, __shfl_xor(m, 32)) + tree_lift_of(top), -m_neg[v]);
      m = mine ? m : -m_neg[v];
      const float alpha = m == -INFINITY ? 1.f : fast_exp2(-m_neg[v] - m);
      l_part[v] *= alpha;
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) acc[v][dt] *= alpha;
      m_neg[v] = -m;
      psum[v] = exp_of(s[v], scale, m == -INFINITY ? 0.f : m_neg[v], p[v]);
    }
  }
#pragma unroll
  for (int v = 0; v < NT; ++v)
    if (v < used) l_part[v] += psum[v];
}

template <int NT, int BS, bool SELECT, bool STREAM>
__global__ __launch_bounds__(kQW * 64) void q4_attn_kernel(AttnQ4Args a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int g = lane >> 4;
  const int i = lane & 15;
  Q4Item t;
  if (!q4_setup<SELECT>(a, NT * 16, t)) return;
  const Ctx c = ctx_blocks(t.ctx, BS, a.NBmax);
  constexpr int kPer = kUnitTokens / BS;  // blocks of a unit
  const int blocks = SELECT ? t.selected + (c.nb > 0) : c.nb;
  const int nu = (blocks + kPer - 1) / kPer;
  const int each = a.by_nsplit(nu), more = nu - each * a.nsplit;  // the first `more` splits have one more
  const int u_begin = t.split * each + min(t.split, more);
  const int u_end = u_begin + each + (t.split < more);

  // A wave's units are u_begin + wave + n * kQW; for kChunk of them at a time lane e holds
  // block e % kPer of unit e / kPer.
  constexpr int kChunk = 64 / kPer;
  const int u_first = u_begin + wave;
  const int nt = u_first < u_end ? (u_end - u_first + kQW - 1) / kQW : 0;
  int n0 = 0, place, count;
  uint64_t live;
  auto chunk_set = [&]() __attribute__((always_inline)) {
    const int n = n0 + lane / kPer;
    if (n < nt) q4_block<BS, SELECT>(a, t, c, (u_first + n * kQW) * kPer + lane % kPer, place, count);
    else place = count = 0;
    live = __builtin_amdgcn_ballot_w64(count > 0);
  };
  // The wave's next unit with an attended token: where its first block's lane is, -1 without one.
  auto next = [&]() __attribute__((always_inline)) {
    while (!live && n0 + kChunk < nt) {
      n0 += kChunk;
      chunk_set();
    }
    if (!live) return -1;
    const int p = __builtin_ctzll(live) / kPer * kPer;
    live &= ~(((1ull << kPer) - 1) << p);
    return p;
  };
  // Of sub-block q lane (g, i) holds token i, dims 32 g .. +31: each load stays in a page, and
  // lane (g, n) gets row n's scores of tokens 4 g .. 4 g + 3 of each.
  struct Loaded {
    u32x4 k[4], v[4];              // codes
    uint32_t k_pow[4], v_pow[4];
  };
  const uint32_t codes_at = t.h * BS * kQ4Codes, power_at = a.Hkv * BS * kQ4Codes + t.h * BS * kQ4Powers;
  const uint32_t code_of = i * kQ4Codes + g * 16, power_of = ((i & 3) * 4 + g) * 4 + (i >> 2);
  Loaded u;
  // where the next unit's sub-blocks are, and their attended tokens (for a wave without a next
  // unit the first bytes of page 0 stand in)
  long long page_at[kPer];
  int keeps;  // five bits each
  auto find = [&](int p) __attribute__((always_inline)) {
    keeps = 0;
#pragma unroll
    for (int b = 0; b < kPer; ++b) {
      page_at[b] = p < 0 ? 0 : (long long)__builtin_amdgcn_readlane(place, p + b) * a.page_bytes;
      const int n = p < 0 ? 0 : __builtin_amdgcn_readlane(count, p + b);
      if constexpr (BS == 16) keeps |= n << (5 * b);
      else keeps |= (n > 16 ? 16 | (n - 16) << 5 : n) << (10 * b);
    }
  };
  auto load = [&](const uint8_t* pages, int q, u32x4& codes, uint32_t& power) __attribute__((always_inline)) {
    const uint8_t* at = pages + page_at[BS == 16 ? q : q >> 1] + (BS == 16 ? 0 : q & 1) * 1024;
    codes = ldg16_once<STREAM>(at + codes_at + code_of);
    at -= (BS == 16 ? 0 : q & 1) * (1024 - 64);
    power = at[power_at + power_of];
  };
  constexpr int kWhole = 16 | 16 << 5 | 16 << 10 | 16 << 15;

  bf16x8 qb[NT][4];
#pragma unroll
  for (int v = 0; v < NT; ++v) load_q4_queries(a, t, t.row0 + v * 16, g, i, qb[v]);
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
  __shared__ float s_m[kQW][kRows], s_l[kQW][kRows], s_ml[2][kRows];
  __shared__ uint64_t s_anc[kTreeMaxTokens];
  __shared__ int s_wild;
  // a wave's values of a unit, its part of the tree's, and its rows at the end
  constexpr int kValues = kUnitTokens * kHeadDim * 2, kMerge = (int)sizeof(float) * kRows * kPad;
  constexpr int kWaveBytes = kValues > kMerge ? kValues : kMerge;
  __shared__ __align__(16) char s_wave[kQW][kWaveBytes];
  auto s_o = [&](int w, int row, int dim) __attribute__((always_inline)) {
    return reinterpret_cast<f32x4*>(&s_wave[w][(row * kPad + dim) * sizeof(float)]);
  };

  // ---- the tree's own rows: one unit, of the last wave of the last split ----
  const bool tree_split = t.split == a.nsplit - 1 && a.tree_k != nullptr;
  bool wild = false;
  if (tree_split && wave == kQW - 1) {
    u32x4 tk[4][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int j = min(16 * q + i, t.tlen - 1);
#pragma unroll
      for (int st = 0; st < 4; ++st) tk[q][st] = ldg16(a.tree_k + t.tree_base + j * t.tree_row + g * 32 + st * 8);
    }
    const uint64_t anc = ancestors(tree_parent(a, t.r, t.tlen, lane), t.tlen, lane);
    s_anc[lane] = anc;
    float p[NT][16];
    f32x4 sc[NT][4];
#pragma unroll
    for (int v = 0; v < NT; ++v) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        sc[v][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < 4; ++st)
          sc[v][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(tk[q][st]), qb[v][st], sc[v][q], 0, 0, 0);
      }
      const int row = t.row0 + v * 16 + i;
      const int tq = row < a.rows ? a.by_g(row) : 0;
      const uint32_t lo = __shfl((uint32_t)anc, tq), hi = __shfl((uint32_t)(anc >> 32), tq);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sc[v][q][e] = (q < 2 ? lo : hi) >> (16 * (q & 1) + 4 * g + e) & 1 ? sc[v][q][e] : -INFINITY;
    }
    softmax_of(sc, a.scale_log2, a.top, m_neg, l_run, acc, p);
    u32x4* sv = reinterpret_cast<u32x4*>(s_wave[wave]);  // [dim][group of tokens], 8 tokens each
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      u32x4 tv[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int j = 32 * half + 16 * (e >> 2) + 4 * g + (e & 3);
        tv[e] = ldg16(a.tree_v + t.tree_base + min(j, t.tlen - 1) * t.tree_row + i * 8);
        if (j >= t.tlen) tv[e] = u32x4{0, 0, 0, 0};
      }
      transpose8(tv);
      wild |= take_wild(tv);
#pragma unroll
      for (int j = 0; j < 8; ++j) sv[(8 * i + j) * 4 + g] = tv[j];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) tv[dt] = sv[(16 * dt + i) * 4 + g];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int v = 0; v < NT; ++v) {
        bf16x8 pb;
#pragma unroll
        for (int e = 0; e < 8; ++e) pb[e] = (__bf16)p[v][8 * half + e];
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
          acc[v][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(tv[dt]), pb, acc[v][dt], 0, 0, 0);
      }
    }
  }
  if (threadIdx.x == (kQW - 1) * 64) s_wild = wild;

  // ---- the cache ----
  // Values in LDS: [32 dims][16 dims][tile q][lane i] of 32 bytes, the two halves swapped in
  // every other four lanes, so that the lanes of a write meet no bank twice.
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  char* const put = s_wave[wave] + g * 4096 + i * 32;
  char* const get = s_wave[wave] + (4 * g + (i >> 2)) * 32 + ((((i & 3) >> 1) ^ (g & 1)) << 4) + (i & 1) * 8;
  const int swap = (i >> 2 & 1) << 4;
  chunk_set();
  int cur = next();
  find(cur);
#pragma unroll
  for (int q = 0; q < 4; ++q) load(a.v4, q, u.v[q], u.v_pow[q]);
#pragma unroll
  for (int q = 0; q < 4; ++q) load(a.k4, q, u.k[q], u.k_pow[q]);
  while (cur >= 0) {
    // A sub-block's registers take the next unit's codes as soon as this one's are turned: the
    // time to the next use is what hides the latency, 8.5 KB a wave on their way.
    const int nxt = next();
    const int keep = keeps;
    find(nxt);
    if (keep != kWhole) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (i >= (keep >> (5 * q) & 31)) {  // 0 times what an unused place holds must stay 0
          u.v_pow[q] = 127;
          u.v[q] = u32x4{0, 0, 0, 0};
        }
    }
    f32x4 sc[NT][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      // values into LDS
      const float sv = __uint_as_float(u.v_pow[q] << 23);
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<bf16x8*>(put + (c >> 1) * 2048 + q * 512 + (((c & 1) << 4) ^ swap)) = eight_bf16(u.v[q][c], sv);
      // scores
      const float sk = __uint_as_float(u.k_pow[q] << 23);
#pragma unroll
      for (int v = 0; v < NT; ++v) sc[v][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        const bf16x8 kb = eight_bf16(u.k[q][st], sk);
#pragma unroll
        for (int v = 0; v < NT; ++v) sc[v][q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qb[v][st], sc[v][q], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      load(a.v4, q, u.v[q], u.v_pow[q]);
      load(a.k4, q, u.k[q], u.k_pow[q]);
    }
    if (keep != kWhole) {
#pragma unroll
      for (int v = 0; v < NT; ++v)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[v][q][e] = 4 * g + e < (keep >> (5 * q) & 31) ? sc[v][q][e] : -INFINITY;
    }
    float p[NT][16];
    softmax_of(sc, a.scale_log2, a.top, m_neg, l_run, acc, p);
    bf16x8 pb[NT][2];
#pragma unroll
    for (int v = 0; v < NT; ++v)
#pragma unroll
      for (int e = 0; e < 16; ++e) pb[v][e >> 3][e & 7] = (__bf16)p[v][e];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
      u32x4 vf[2];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const u32x2 w = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                       (__attribute__((address_space(3))) s16x4*)(get + (dt >> 1) * 4096 + (dt & 1) * 2048 + q * 512)));
        vf[q >> 1][2 * (q & 1)] = w[0];
        vf[q >> 1][2 * (q & 1) + 1] = w[1];
      }
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int v = 0; v < NT; ++v)
          acc[v][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vf[half]), pb[v][half], acc[v][dt], 0, 0, 0);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
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
  __syncthreads();
#pragma unroll
  for (int v = 0; v < NT; ++v) {
    const int row = v * 16 + i;
    float M = s_m[0][row];
#pragma unroll
    for (int w = 1; w < kQW; ++w) M = fmaxf(M, s_m[w][row]);
    float S = 0.f;
#pragma unroll
    for (int w = 0; w < kQW; ++w) S += s_m[w][row] == -INFINITY ? 0.f : s_l[w][row] * fast_exp2(s_m[w][row] - M);
    const float f = m_run[v] == -INFINITY ? 0.f : fast_exp2(m_run[v] - M);
    if (wave == 0 && g == 0) {
      s_ml[0][row] = M;
      s_ml[1][row] = S;
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) *s_o(wave, row, 16 * dt + 4 * g) = acc[v][dt] * f;
  }
  __syncthreads();
  const long long pbase = ((long long)t.rh * a.nsplit + t.split) * a.rows + t.row0;
  const int last = min(t.tlen * a.G, a.rows) - t.row0;  // rows of this group in use
  for (int pos = threadIdx.x; pos < kRows * (kHeadDim / 4); pos += kQW * 64) {
    const int row = pos >> 5;
    const int c4 = pos & 31;
    if (row >= last) break;
    f32x4 o = *s_o(0, row, c4 * 4);
#pragma unroll
    for (int w = 1; w < kQW; ++w) o += *s_o(w, row, c4 * 4);
    if (s_wild) add_wild(a, t, s_anc[a.by_g(t.row0 + row)], c4, o);
    if (a.nsplit == 1) {
      write_row(a, t.r, t.h, t.row0 + row, c4, o, s_ml[0][row], s_ml[1][row]);
    } else {
      *reinterpret_cast<f32x4*>(a.part_o + (pbase + row) * kHeadDim + c4 * 4) = o;
      if (c4 == 0) *reinterpret_cast<float2*>(a.part_ml + (pbase + row) * 2) = make_float2(s_ml[0][row], s_ml[1][row]);
    }
  }
}

// More than two row tiles. Eight waves in two teams share every unit: each wave turns a
// sixteenth of its codes, 16 tokens of keys or of values, into bf16 in LDS, and then attends
// with its own one or two of the group's row tiles, team 0 the unit's first 32 tokens and
// team 1 the others. Keys lie there as the first product's operand, values a token after the
// other, 16 dims (32 bytes, the halves swapped as above) apart, for the transposing read. One
// barrier a unit.
//
// With two tiles a wave (512 rows over 65,536 tokens, 296 us) the barrier takes 38 us, the LDS
// reads 40, turning the codes and their loads 41, and the rest 177, about what the products
// take at the library's rate; with the teams out of step, as in tree_attn.hip, it was slower
// (308), with a barrier for every two units in four buffers too (303), with loads two and
// three units ahead the same. With one tile a wave 42 % of a wave's
// time is waiting; keys read by each wave as codes, from LDS (166 us for the ragged case) or
// from memory (199), were no faster than through LDS in bf16 (164), nor were two tiles a wave
// in four teams over 128 tokens a step, with 0.6 of the LDS traffic and one workgroup a CU
// (407 and 382 us for 8 x 8 x 131,072 tokens with 64 rows, 43 and 41 for 16 x 8 x 4,128).
constexpr int kRowsThreads = 512;
constexpr int kRowPlaces = 4;   // waves of a team
// Groups of five or six tiles leave out the products and exponentials of the places without a
// second one, tile by tile (FULL false). Measured, us with and without, 512 pairs over 2,064
// selected tokens: five tiles 95 and 102, six 100 and 105, seven 110 and 108; 16 pairs over
// 65,536: 85 and 87, 87 and 89, 96 and 90.
constexpr int kUnevenTiles = 6;
constexpr int kListBlocks = 1024;
constexpr int kKeysBytes = 16 * 1024;
constexpr int kValuesPart = 4 * 1024;  // 32 dims of the unit's tokens
constexpr int kUnitBytes = kKeysBytes + 4 * kValuesPart;

template <int NT, int BS, bool SELECT, bool FULL>
__global__ __launch_bounds__(kRowsThreads, NT == 1 ? 4 : 2) void q4_attn_rows_kernel(AttnQ4Args a) {
  constexpr int kRows = NT * kRowPlaces * 16;
  constexpr int kPad = kHeadDim + 4;
  constexpr int kPer = kUnitTokens / BS;
  constexpr int kBuffers = NT == 1 ? 2 : 3;
  constexpr int kMerge = (int)sizeof(float) * kRows * kPad;
  __shared__ __align__(16) char s_buf[kBuffers * kUnitBytes > kMerge ? kBuffers * kUnitBytes : kMerge];
  __shared__ int2 s_list[kListBlocks];  // page and attended tokens of the segment's blocks
  __shared__ uint64_t s_anc[kTreeMaxTokens];
  __shared__ float s_ml[2][kRows];
  __shared__ int s_wild;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int g = lane >> 4;
  const int i = lane & 15;
  const int team = wave / kRowPlaces;
  // this wave's tiles: rt and rt + 4 of the group's; not FULL: the second one may be none of
  // the group's (the waves with two tiles of the teams are on different SIMDs)
  const int rt = (wave + (FULL ? 0 : 2 * team)) % kRowPlaces;
  const int used = FULL ? NT : (rt + kRowPlaces < a.tiles ? 2 : 1);
  Q4Item t;
  if (!q4_setup<SELECT>(a, a.tiles * 16, t)) return;
  const Ctx c = ctx_blocks(t.ctx, BS, a.NBmax);
  const int blocks = SELECT ? t.selected + (c.nb > 0) : c.nb;
  const int nu = (blocks + kPer - 1) / kPer;
  const int each = a.by_nsplit(nu), more = nu - each * a.nsplit;
  const int u_begin = t.split * each + min(t.split, more);
  const int u_end = u_begin + each + (t.split < more);

  bf16x8 qb[NT][4];
#pragma unroll
  for (int v = 0; v < NT; ++v) load_q4_queries(a, t, t.row0 + (rt + v * kRowPlaces) * 16, g, i, qb[v]);
  float m_neg[NT], l_run[NT];
  f32x4 acc[NT][8];
#pragma unroll
  for (int v = 0; v < NT; ++v) {
    m_neg[v] = INFINITY;
    l_run[v] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[v][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (threadIdx.x == 0) s_wild = 0;

  // ---- what this wave converts: sub-block `sub` of keys or of values, lane (g, i) its token
  // i, dims 32 g .. +31
  const bool is_v = wave >= 4;
  const int sub = wave & 3;
  const uint8_t* const src = is_v ? a.v4 : a.k4;
  const int sub_in = BS == 16 ? 0 : sub & 1;  // of its block
  const long long codes_at = (long long)t.h * BS * kQ4Codes + sub_in * 1024 + i * kQ4Codes + g * 16;
  const long long power_at = (long long)a.Hkv * BS * kQ4Codes + (long long)t.h * BS * kQ4Powers + sub_in * 64 +
                             ((i & 3) * 4 + g) * 4 + (i >> 2);
  // 32 dims of a token (quads of 8) to their place
  const uint32_t put_at = is_v ? kKeysBytes + g * kValuesPart + (sub * 16 + i) * 32 : sub * 4096 + g * 256 + i * 16;
  auto put = [&](int buf, int q, u32x4 x) __attribute__((always_inline)) {
    *reinterpret_cast<u32x4*>(s_buf + buf * kUnitBytes + put_at + (is_v ? (q >> 1) * 2048 + ((q & 1) ^ (i >> 2 & 1)) * 16 : q * 1024)) = x;
  };
  struct Codes {
    u32x4 x;
    uint32_t power;
    int keep;  // attended tokens
  };
  // ---- the products of one unit
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  u32x4 kf[2][4], vf[8];
  auto read_k = [&](int buf) __attribute__((always_inline)) {
    const char* kb = s_buf + buf * kUnitBytes + team * 8192 + lane * 16;
#pragma unroll
    for (int tau = 0; tau < 2; ++tau)
#pragma unroll
      for (int st = 0; st < 4; ++st) kf[tau][st] = *reinterpret_cast<const u32x4*>(kb + tau * 4096 + st * 1024);
  };
  auto read_v = [&](int buf) __attribute__((always_inline)) {
    char* vb = s_buf + buf * kUnitBytes + kKeysBytes + (team * 32 + 4 * g + (i >> 2)) * 32 +
               ((((i & 3) >> 1) ^ (g & 1)) << 4) + (i & 1) * 8;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const u32x2 w = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(
                       vb + (dt >> 1) * kValuesPart + (dt & 1) * 2048 + q * 512)));
        vf[dt][2 * q] = w[0];
        vf[dt][2 * q + 1] = w[1];
      }
  };
  f32x4 sc[NT][2];
  auto scores = [&]() __attribute__((always_inline)) {
    if constexpr (FULL) {
#pragma unroll
      for (int v = 0; v < NT; ++v) sc[v][0] = sc[v][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int v = 0; v < NT; ++v)
#pragma unroll
          for (int tau = 0; tau < 2; ++tau)
            sc[v][tau] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[tau][st]), qb[v][st], sc[v][tau], 0, 0, 0);
    } else {
#pragma unroll
      for (int v = 0; v < NT; ++v) {
        if (v >= used) continue;
        sc[v][0] = sc[v][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
          for (int tau = 0; tau < 2; ++tau)
            sc[v][tau] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[tau][st]), qb[v][st], sc[v][tau], 0, 0, 0);
      }
    }
  };
  // `keep` attended tokens of the team's two sub-blocks (16: all), or the tree's rows
  auto mask = [&](int keep0, int keep1, bool tree) __attribute__((always_inline)) {
    if (keep0 >= 16 && keep1 >= 16 && !tree) return;
#pragma unroll
    for (int v = 0; v < NT; ++v) {
      if (v >= used) continue;
      const int k0 = keep0 - 4 * g, k1 = keep1 - 4 * g;
      uint32_t bits = (k0 <= 0 ? 0u : k0 >= 4 ? 15u : (1u << k0) - 1) | (k1 <= 0 ? 0u : k1 >= 4 ? 15u : (1u << k1) - 1) << 4;
      if (tree) {
        const int row = t.row0 + (rt + v * kRowPlaces) * 16 + i;
        const uint64_t anc = s_anc[row < a.rows ? a.by_g(row) : 0];
        bits = (uint32_t)(anc >> (team * 32 + 4 * g)) & 15u;
        bits |= ((uint32_t)(anc >> (team * 32 + 16 + 4 * g)) & 15u) << 4;
      }
      mask_scores(sc[v], bits);
    }
  };
  bf16x8 pb[NT];
  auto softmax = [&]() __attribute__((always_inline)) {
    float p[NT][8];
    softmax_of(sc, a.scale_log2, a.top, m_neg, l_run, acc, p, used);
#pragma unroll
    for (int v = 0; v < NT; ++v) {
      if (v >= used) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) pb[v][e] = (__bf16)p[v][e];
    }
  };
  auto values = [&](int dt) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < NT; ++v)
      acc[v][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vf[dt]), pb[v], acc[v][dt], 0, 0, 0);
  };
  auto attend = [&]() __attribute__((always_inline)) {
    softmax();
    if constexpr (FULL) {
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) values(dt);
    } else {
#pragma unroll
      for (int v = 0; v < NT; ++v) {
        if (v >= used) continue;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
          acc[v][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vf[dt]), pb[v], acc[v][dt], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  for (int seg = u_begin; seg < u_end; seg += kListBlocks / kPer) {
    const int units = min(kListBlocks / kPer, u_end - seg);
    for (int n = threadIdx.x; n < units * kPer; n += kRowsThreads) {
      int2 e;
      q4_block<BS, SELECT>(a, t, c, seg * kPer + n, e.x, e.y);
      s_list[n] = e;
    }
    __syncthreads();
    auto load = [&](int s) __attribute__((always_inline)) {
      const int2 e = s_list[min(s, units - 1) * kPer + (BS == 16 ? sub : sub >> 1)];
      const int page = __builtin_amdgcn_readfirstlane(e.x);
      Codes x;
      x.keep = __builtin_amdgcn_readfirstlane(e.y) - sub_in * 16;
      const uint8_t* at = src + page * a.page_bytes;
      x.x = ldg16(at + codes_at);
      x.power = at[power_at];
      return x;
    };
    auto convert = [&](int buf, const Codes& x) __attribute__((always_inline)) {
      float s = __uint_as_float(x.power << 23);
      u32x4 codes = x.x;
      if (x.keep < 16 && i >= x.keep) {  // what an unused place holds may be NaN
        s = 1.f;
        codes = u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const u32x4 y = {two_bf16<0>(codes[q], s), two_bf16<1>(codes[q], s), two_bf16<2>(codes[q], s), two_bf16<3>(codes[q], s)};
        put(buf, q, y);
      }
    };
    auto keep_of = [&](int s, int b) __attribute__((always_inline)) {  // sub-block b of unit s
      const int n = __builtin_amdgcn_readfirstlane(s_list[s * kPer + (BS == 16 ? b : b >> 1)].y) - (BS == 16 ? 0 : (b & 1) * 16);
      return n > 16 ? 16 : n;
    };
    if constexpr (NT == 1) {
      // Two workgroups share a CU, and hide each other's waits: two units in LDS, loads three
      // units ahead of their conversion.
      constexpr int kAhead = 3;
      Codes x[kAhead];
#pragma unroll
      for (int p = 0; p < kAhead; ++p) x[p] = load(p);
      convert(0, x[0]);
      x[0] = load(kAhead);
      __syncthreads();
      for (int s0 = 0; s0 < units; s0 += kAhead) {
#pragma unroll
        for (int p = 0; p < kAhead; ++p) {
          const int s = s0 + p;
          if (s >= units) break;
          if (s + 1 < units) {
            convert((s + 1) & 1, x[(p + 1) % kAhead]);
            x[(p + 1) % kAhead] = load(s + 1 + kAhead);
          }
          read_k(s & 1);
          scores();
          mask(keep_of(s, 2 * team), keep_of(s, 2 * team + 1), false);
          __builtin_amdgcn_sched_barrier(0);  // no reads of values ahead of it, into more registers
          softmax();
          __builtin_amdgcn_sched_barrier(0);
          read_v(s & 1);
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) values(dt);
          __syncthreads();
        }
      }
    } else {
      // One workgroup a CU: LDS reads run beside the products, V ahead of the scores and the
      // next unit's K behind them, so three units are in LDS.
      convert(0, load(0));
      convert(1, load(1));
      Codes x = load(2);
      __syncthreads();
      read_k(0);
      int buf = 0;  // of unit s
      for (int s = 0; s < units; ++s) {
        const int next = buf < 2 ? buf + 1 : 0, after = next < 2 ? next + 1 : 0;
        convert(after, x);
        x = load(s + 3);
        __builtin_amdgcn_sched_barrier(0);
        read_v(buf);
        scores();
        __builtin_amdgcn_sched_barrier(0);
        read_k(next);
        mask(keep_of(s, 2 * team), keep_of(s, 2 * team + 1), false);
        attend();
        __syncthreads();
        buf = next;
      }
    }
  }

  // ---- the tree's own rows: a unit of the last split ----
  __syncthreads();  // team 0's last unit is read, and s_wild is set where there was none
  if (t.split == a.nsplit - 1 && a.tree_k) {
    if (wave == 0) s_anc[lane] = ancestors(tree_parent(a, t.r, t.tlen, lane), t.tlen, lane);
    const int j = sub * 16 + i;
    const uint16_t* row = (is_v ? a.tree_v : a.tree_k) + t.tree_base + min(j, t.tlen - 1) * t.tree_row + g * 32;
    u32x4 y[8];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      y[q] = ldg16(row + 8 * q);
      y[4 + q] = u32x4{0, 0, 0, 0};
      if (j >= t.tlen) y[q] = y[4 + q];
    }
    if (is_v && take_wild(y)) s_wild = 1;
#pragma unroll
    for (int q = 0; q < 4; ++q) put(0, q, y[q]);
    __syncthreads();
    if (team * 32 < t.tlen) {
      read_k(0);
      read_v(0);
      scores();
      mask(16, 16, true);
      attend();
    }
    __syncthreads();
  }

  // ---- merge the teams: the second one's rows through LDS, the sums back there ----
  float(*s_o)[kPad] = reinterpret_cast<float(*)[kPad]>(s_buf);  // [row of the group]
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
  const int last = min(min(t.tlen * a.G, a.rows) - t.row0, a.tiles * 16);  // rows of this group in use
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

template <int BS, bool SELECT>
void launch_bs_q4(const AttnQ4Args& a, hipStream_t s) {
  const long long runs = (long long)a.R * a.Hkv * a.nsplit;
  const dim3 grid((unsigned)(a.by_length ? (runs + 7) / 8 * 8 * a.groups : (runs * a.groups + 7) / 8 * 8));
  // What the tables and selections hold at most: past kStreamBytes the codes are read past
  // the caches (whole lines a load).
  const long long blocks = SELECT && a.k_sel + 1ll < a.NBmax ? a.k_sel + 1ll : a.NBmax;
  const bool stream = (long long)a.R * a.Hkv * blocks * BS * 2 * (kQ4Codes + kQ4Powers) >= kStreamBytes;
  if (a.tiles == 1)
    hipLaunchKernelGGL((stream ? q4_attn_kernel<1, BS, SELECT, true> : q4_attn_kernel<1, BS, SELECT, false>), grid,
                       dim3(kQW * 64), 0, s, a);
  else if (a.tiles == 2)
    hipLaunchKernelGGL((stream ? q4_attn_kernel<2, BS, SELECT, true> : q4_attn_kernel<2, BS, SELECT, false>), grid,
                       dim3(kQW * 64), 0, s, a);
  else if (a.tiles <= kRowPlaces)
    hipLaunchKernelGGL((q4_attn_rows_kernel<1, BS, SELECT, true>), grid, dim3(kRowsThreads), 0, s, a);
  else if (a.tiles <= kUnevenTiles)
    hipLaunchKernelGGL((q4_attn_rows_kernel<2, BS, SELECT, false>), grid, dim3(kRowsThreads), 0, s, a);
  else
    hipLaunchKernelGGL((q4_attn_rows_kernel<2, BS, SELECT, true>), grid, dim3(kRowsThreads), 0, s, a);
}

}  // namespace

hipError_t launch_attn_q4(const AttnQ4Args& a, hipStream_t s) {
  if (a.B == 16)
    a.sel ? launch_bs_q4<16, true>(a, s) : launch_bs_q4<16, false>(a, s);
  else
    a.sel ? launch_bs_q4<32, true>(a, s) : launch_bs_q4<32, false>(a, s);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_tree_finish(a, CacheSelection{a.sel, a.sel_count, a.k_sel}, s);
}

}  // namespace oasis
