// Attention of a drafted token tree over a cache, and the tree's own tokens.
//
// Row t of a request's tree attends every cached token (the pages of a paged
// cache, or the slots and local block of the working set) and the drafted tokens
// on its path to the root, itself among them: out = softmax(scale q K^T) V over
// the two sets together, one pass with a running maximum and sum.
//
// Work decomposition. Cached tokens come in units of 32; a workgroup of four
// waves takes a run of a (request, KV head) pair's units for up to four 16-row
// tiles, every wave a strided subset of the units with its own online softmax.
// The tree's tokens are one or two more units, with a mask per row, that the last
// split's waves take after their own. The waves merge through LDS, the splits
// through the workspace and a second kernel.
//
// One unit for one 16-row tile is, as in the working set's attention,
//   S^T (tokens x rows) = K . Q^T     8 of v_mfma_f32_16x16x32_bf16
//   O^T (d x rows)     += V^T . P^T   8 of them
// with the tokens dealt to MFMA rows so that lane (g, n) holds row n's scores of
// unit tokens 8g .. 8g+7, which makes the probabilities directly the B operand of
// the second product: no cross-lane movement and no LDS for P. The A operand of
// that product needs V[8g .. 8g+7][one d] in a lane. The working set keeps V
// transposed, so it is one load per d-tile (d = 16 dt + i). Pages keep V
// token-major: there lane (g, i) loads dims 8i .. 8i+7 of each of its 8 tokens (a
// wave reads whole rows) and transposes the 8 x 8 block in registers, 32 byte
// permutes a unit; d-tile j is then the dims d = 8i + j, and a lane's outputs of
// one row are 32 consecutive dims.
#include "drafts_internal.h"

namespace oasis {
namespace {

constexpr int kTW = kTreeWaves;
constexpr float kTreeLazy = 8.f;  // as kLazyTh of the working set's attention: exponents stay below 2^8

// Contiguous runs of the items on each XCD (workgroup ids go round the 8 XCDs): a
// pair's splits and row groups share one L2.
__device__ __forceinline__ int tree_item(int wg, int items) {
  const int item = (wg & 7) * ((items + 7) >> 3) + (wg >> 3);
  return (wg >> 3) < ((items + 7) >> 3) && item < items ? item : -1;
}

struct TreeUnit {
  u32x4 k[2][4];
  u32x4 v[8];
};

// 8 tokens x 8 dims of 16-bit values, a token per register quad, into a dim per quad.
__device__ __forceinline__ void transpose8(u32x4 (&v)[8]) {
  u32x4 t[8];
#pragma unroll
  for (int w = 0; w < 4; ++w)
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      t[2 * w][p] = __builtin_amdgcn_perm(v[2 * p + 1][w], v[2 * p][w], 0x05040100);
      t[2 * w + 1][p] = __builtin_amdgcn_perm(v[2 * p + 1][w], v[2 * p][w], 0x07060302);
    }
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = t[j];
}

// Clears the values of tokens from `keep` on (8 tokens along each quad).
__device__ __forceinline__ void clear_tokens(u32x4 (&v)[8], int keep) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t m = (2 * w < keep ? 0x0000FFFFu : 0u) | (2 * w + 1 < keep ? 0xFFFF0000u : 0u);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j][w] &= m;
  }
}

__device__ __forceinline__ bool odd_bf16(uint32_t b) { return (b & 0x7F80u) == 0x7F80u; }  // infinity or NaN

// First dim of the 4 that element quad dt of a lane's accumulators holds, and
// whether the quad runs over e (dims d0 + e) or over tiles: see store_dims.
template <bool PAGED>
__device__ __forceinline__ int acc_dim(int dt, int g, int e) {
  return PAGED ? 32 * g + 8 * e + dt : 16 * dt + 4 * g + e;
}

// Scores of one unit for one tile: lane (g, n) gets row n against tokens 8g .. 8g+7.
__device__ __forceinline__ void unit_scores(const TreeUnit& u, const bf16x8 (&qb)[4], float scale_log2, float (&x)[8]) {
  f32x4 sc[2];
#pragma unroll
  for (int tau = 0; tau < 2; ++tau) {
    sc[tau] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < 4; ++st)
      sc[tau] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(u.k[tau][st]), qb[st], sc[tau], 0, 0, 0);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = sc[e >> 2][e & 3] * scale_log2;
}

// Online softmax of one tile's scores: probabilities in bf16 (the second
// product's operand; 2^-8 of each at most, unbiased, and the sum takes them
// unrounded), the row reference and the lane's partial sum updated. The
// accumulators are rescaled only when a score passes its row's reference by 2^8.
__device__ __forceinline__ bf16x8 unit_softmax(const float (&x)[8], float& m_ref, float& l_part, f32x4 (&acc)[8]) {
  const float lmax = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
  if (__builtin_amdgcn_ballot_w64(lmax > m_ref + kTreeLazy)) {
    float rmax = fmaxf(lmax, __shfl_xor(lmax, 16));
    rmax = fmaxf(rmax, __shfl_xor(rmax, 32));
    const float m_new = fmaxf(m_ref, rmax);
    const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(m_ref - m_new);
    l_part *= alpha;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[dt] *= alpha;
    m_ref = m_new;
  }
  const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
  bf16x8 pb;
  float psum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float pe = fast_exp2(x[e] - m_use);
    psum += pe;
    pb[e] = (__bf16)pe;
  }
  l_part += psum;
  return pb;
}

__device__ __forceinline__ void unit_pv(const TreeUnit& u, bf16x8 pb, f32x4 (&acc)[8]) {
#pragma unroll
  for (int dt = 0; dt < 8; ++dt)
    acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(u.v[dt]), pb, acc[dt], 0, 0, 0);
}

// Ancestor masks of a request's tree, lane t: row t's (its own bit among them).
// Pointer doubling: after n rounds a mask holds 2^n rows of the path. A parent
// outside [0, t) makes the row a root; lanes past the tree hold 0.
__device__ __forceinline__ uint64_t ancestors(const int32_t* parent, int T, int len, int lane) {
  int up = -1;
  if (lane < len && lane > 0) up = parent ? parent[lane] : lane - 1;
  if (up >= lane || up < 0) up = -1;
  uint64_t m = lane < len ? 1ull << lane : 0;
#pragma unroll
  for (int n = 0; n < 6; ++n) {
    const int src = up < 0 ? lane : up;
    const uint32_t lo = __shfl((uint32_t)m, src), hi = __shfl((uint32_t)(m >> 32), src);
    const int next = __shfl(up, src);
    if (up >= 0) {
      m |= (uint64_t)hi << 32 | lo;
      up = next;
    }
  }
  return m;
}

// Normalised bf16 output of 4 dims of one row, and its log-sum-exp.
__device__ __forceinline__ void write_row(const TreeAttnArgs& a, int r, int h, int row, int c4, f32x4 o, float M, float L) {
  const int t = row / a.G;
  const int qh = h * a.G + (row - t * a.G);
  const long long orow = ((long long)r * a.T + t) * a.Hq + qh;
  const float inv = L == 0.f ? 0.f : 1.f / L;  // a NaN sum stays one
  uint32_t w[2];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const __bf16 lo = (__bf16)(o[2 * p] * inv), hi = (__bf16)(o[2 * p + 1] * inv);
    w[p] = __builtin_bit_cast(uint16_t, lo) | (uint32_t)__builtin_bit_cast(uint16_t, hi) << 16;
  }
  *reinterpret_cast<uint2*>(a.out + orow * kHeadDim + c4 * 4) = make_uint2(w[0], w[1]);
  if (c4 == 0 && a.lse) a.lse[orow] = L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.69314718055994531f;
}

__device__ __forceinline__ int tree_length(const TreeAttnArgs& a, int r) {
  const int n = a.tree_len ? a.tree_len[r] : a.T;
  return n < 0 ? 0 : (n > a.T ? a.T : n);
}

template <int NT, int BS, bool PAGED>
__global__ __launch_bounds__(kTW * 64) void tree_attn_kernel(TreeAttnArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int g = lane >> 4;
  const int i = lane & 15;
  const int item = tree_item(blockIdx.x, a.R * a.Hkv * a.nsplit * a.groups);
  if (item < 0) return;
  const int rg = item % a.groups;
  const int rs = item / a.groups;
  const int split = rs % a.nsplit;
  const int rh = rs / a.nsplit;
  const int r = rh / a.Hkv;
  const int h = rh - r * a.Hkv;
  const int tlen = tree_length(a, r);
  const int row0 = rg * NT * 16;
  if (row0 >= tlen * a.G) return;  // no row of this group is in the tree

  const long long unit_elems = (long long)a.Hkv * BS * kHeadDim;  // a page, or a slot
  const int ks = a.k_slots;
  const Ctx c = ctx_blocks(a.ctx_len[r], BS, a.NBmax);
  const int L = c.nb ? c.n_cand * BS + c.local_len : 0;
  const int nu = PAGED ? (L + 31) / 32 : (BS == 16 ? (ks + 2) / 2 : ks + 1);
  const int u_begin = (int)((long long)nu * split / a.nsplit);
  const int u_end = (int)((long long)nu * (split + 1) / a.nsplit);
  const long long base = (PAGED ? 0 : (long long)r * (ks + 1) * unit_elems) + (long long)h * BS * kHeadDim;
  const uint16_t* kb = a.k + base;
  const uint16_t* vb = a.v + base;
  const int32_t* tab = a.table + (PAGED ? (long long)r * a.NBmax : (long long)rh * ks);

  bf16x8 qb[NT][4];
#pragma unroll
  for (int v = 0; v < NT; ++v) {
    const int row = row0 + v * 16 + i;
    if (row < a.rows) {
      const int tq = row / a.G;
      const int qh = h * a.G + (row - tq * a.G);
      const uint16_t* qrow = a.q + (((long long)r * a.T + tq) * a.Hq + qh) * kHeadDim;
#pragma unroll
      for (int st = 0; st < 4; ++st) qb[v][st] = as_bf16x8(ldg16(qrow + st * 32 + g * 8));
    } else {
#pragma unroll
      for (int st = 0; st < 4; ++st) qb[v][st] = as_bf16x8(u32x4{0, 0, 0, 0});
    }
  }
  float m_run[NT], l_run[NT];
  f32x4 acc[NT][8];
#pragma unroll
  for (int v = 0; v < NT; ++v) {
    m_run[v] = -INFINITY;
    l_run[v] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[v][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // A wave's units are u_begin + wave + t * kTW. For kChunk of them at a time, lane
  // e holds the place (page or slot) and the attended tokens of one block: block
  // e % 2 of unit e / 2 at B = 16, of unit e at B = 32.
  constexpr int kPer = 32 / BS;  // blocks per unit
  constexpr int kChunk = 64 / kPer;
  const int u_first = u_begin + wave;
  const int nt = u_first < u_end ? (u_end - u_first + kTW - 1) / kTW : 0;
  auto entry_block = [&](int t0) { return (u_first + (t0 + lane / kPer) * kTW) * kPer + lane % kPer; };
  auto entry_load = [&](int t0) -> int {
    const int b = entry_block(t0);
    if (t0 + lane / kPer >= nt) return -1;
    if constexpr (PAGED) return b < c.nb ? tab[b] : -1;
    else return b < ks ? tab[b] : (b == ks ? 0 : -1);
  };
  int place = 0, count = 0;  // of this lane's block of the current chunk
  auto entry_set = [&](int t0, int raw) {
    const int b = entry_block(t0);
    if constexpr (PAGED) {
      const bool ok = raw >= 0 && raw < a.num_pages;
      place = ok ? raw : 0;
      const int n = L - b * BS;
      count = ok ? (n < BS ? n : BS) : 0;
    } else {
      place = b <= ks ? b : 0;
      count = raw < 0 ? 0 : (b == ks ? c.local_len : BS);
    }
  };
  // units with an attended token, bit per block
  auto next_live = [&](uint64_t live, int p) -> int {  // first unit >= p of the chunk, kChunk: none
    const uint64_t rest = p < kChunk ? live >> (p * kPer) : 0;
    return rest ? p + __builtin_ctzll(rest) / kPer : kChunk;
  };
  const uint32_t tok = 8 * (i >> 2) + (i & 3);
  const uint32_t ko = ((BS == 16 ? tok & 15 : tok) * kHeadDim + g * 8);
  const uint32_t vo = PAGED ? (uint32_t)((BS == 16 ? g & 1 : g) * 8 * kHeadDim + i * 8)
                            : (uint32_t)(i * BS + (BS == 16 ? g & 1 : g) * 8);
  auto load = [&](TreeUnit& u, int p0, int p1) __attribute__((always_inline)) {
    const uint16_t* ku = kb + (long long)(BS == 16 && i >= 8 ? p1 : p0) * unit_elems + ko;
    const uint16_t* vu = vb + (long long)(BS == 16 && g >= 2 ? p1 : p0) * unit_elems + vo;
#pragma unroll
    for (int tau = 0; tau < 2; ++tau)
#pragma unroll
      for (int st = 0; st < 4; ++st) u.k[tau][st] = ldg16(ku + tau * 4 * kHeadDim + st * 32);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) u.v[dt] = ldg16(vu + (PAGED ? dt * kHeadDim : dt * 16 * BS));
  };
  auto run = [&](TreeUnit& u, int n0, int n1) __attribute__((always_inline)) {
    if constexpr (PAGED) transpose8(u.v);
    const int n = BS == 16 ? (g < 2 ? n0 : n1) - (g & 1) * 8 : n0 - g * 8;
    const int keep = n < 0 ? 0 : (n > 8 ? 8 : n);
    const bool partial = __builtin_amdgcn_ballot_w64(keep < 8) != 0;
    if (partial) clear_tokens(u.v, keep);  // 0 times what an unused place holds must stay 0
#pragma unroll
    for (int v = 0; v < NT; ++v) {
      float x[8];
      unit_scores(u, qb[v], a.scale_log2, x);
      if (partial) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < keep ? x[e] : -INFINITY;
      }
      unit_pv(u, unit_softmax(x, m_run[v], l_run[v], acc[v]), acc[v]);
    }
  };

  for (int t0 = 0; t0 < nt; t0 += kChunk) {
    entry_set(t0, entry_load(t0));
    const uint64_t live = __builtin_amdgcn_ballot_w64(count > 0);
    for (int p = next_live(live, 0); p < kChunk; p = next_live(live, p + 1)) {
      TreeUnit u;
      const int p0 = __builtin_amdgcn_readlane(place, p * kPer), p1 = __builtin_amdgcn_readlane(place, p * kPer + kPer - 1);
      const int n0 = __builtin_amdgcn_readlane(count, p * kPer), n1 = __builtin_amdgcn_readlane(count, p * kPer + kPer - 1);
      load(u, p0, p1);
      run(u, n0, n1);
    }
  }

  constexpr int kRows = NT * 16;
  constexpr int kPad = kHeadDim + 4;
  __shared__ float s_m[kTW][kRows], s_l[kTW][kRows], s_ml[2][kRows];
  __shared__ __align__(16) float s_o[kTW][kRows][kPad];

  // ---- the tree's own tokens: unit tu of them to wave tu of the last split ----
  const int tu = wave;
  if (split == a.nsplit - 1 && tu * 32 < tlen) {
    const uint64_t anc = ancestors(a.parent ? a.parent + (long long)r * a.T : nullptr, a.T, tlen, lane);
    const long long row_elems = (long long)a.Hkv * kHeadDim;
    const long long tb = (long long)r * a.T * row_elems + (long long)h * kHeadDim;
    TreeUnit u;
#pragma unroll
    for (int tau = 0; tau < 2; ++tau) {
      const int j = min(tu * 32 + (int)tok + 4 * tau, tlen - 1);
#pragma unroll
      for (int st = 0; st < 4; ++st) u.k[tau][st] = ldg16(a.tree_k + tb + j * row_elems + st * 32 + g * 8);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = min(tu * 32 + 8 * g + e, tlen - 1);
      u.v[e] = ldg16(a.tree_v + tb + j * row_elems + i * 8);
    }
    transpose8(u.v);
    const int n = tlen - tu * 32 - 8 * g;
    clear_tokens(u.v, n < 0 ? 0 : (n > 8 ? 8 : n));
    // A value that is not finite counts for the rows that attend it alone: it is
    // taken out of the product (where 0 times it would spoil every row) and added to
    // those rows below.
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (odd_bf16(u.v[j][w])) odd = true, u.v[j][w] &= 0xFFFF0000u;
        if (odd_bf16(u.v[j][w] >> 16)) odd = true, u.v[j][w] &= 0x0000FFFFu;
      }
    const uint64_t any_odd = __builtin_amdgcn_ballot_w64(odd);
    if constexpr (!PAGED) {
      // the working set's accumulators hold d-tile dt = dims 16 dt + i: through LDS,
      // [dim][32 tokens], each wave in its own part of the merge area
      u32x4* sv = reinterpret_cast<u32x4*>(&s_o[wave][0][0]);
#pragma unroll
      for (int j = 0; j < 8; ++j) sv[(8 * i + j) * 4 + g] = u.v[j];
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) u.v[dt] = sv[(16 * dt + i) * 4 + g];
    }
#pragma unroll
    for (int v = 0; v < NT; ++v) {
      const int row = row0 + v * 16 + i;
      const int t = row < a.rows ? row / a.G : 0;
      const uint64_t mine = (uint64_t)__shfl((uint32_t)(anc >> 32), t) << 32 | (uint32_t)__shfl((uint32_t)anc, t);
      const uint32_t bits = (uint32_t)(mine >> (tu * 32 + 8 * g)) & 0xFF;
      float x[8];
      unit_scores(u, qb[v], a.scale_log2, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = bits >> e & 1 ? x[e] : -INFINITY;
      const bf16x8 pb = unit_softmax(x, m_run[v], l_run[v], acc[v]);
      unit_pv(u, pb, acc[v]);
      if (any_odd) {
        const float m_use = m_run[v] == -INFINITY ? 0.f : m_run[v];
        for (int e = 0; e < 8; ++e)
          for (int gg = 0; gg < 4; ++gg) {
            const int j = tu * 32 + 8 * gg + e;
            if (j >= tlen) break;
            float xe = x[0];
#pragma unroll
            for (int f = 1; f < 8; ++f) xe = e == f ? x[f] : xe;
            const float p = __shfl(fast_exp2(xe - m_use), gg * 16 + i);
            if (!(mine >> j & 1)) continue;
            const uint16_t* vr = a.tree_v + tb + j * row_elems;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
#pragma unroll
              for (int f = 0; f < 4; ++f) {
                const uint32_t b = vr[acc_dim<PAGED>(dt, g, f)];
                if (odd_bf16(b)) acc[v][dt][f] += p * bf16_bits_to_f32(b);
              }
          }
      }
    }
  }
#pragma unroll
  for (int v = 0; v < NT; ++v) {
    l_run[v] += __shfl_xor(l_run[v], 16);
    l_run[v] += __shfl_xor(l_run[v], 32);
    if (l_run[v] != l_run[v] && m_run[v] == -INFINITY) m_run[v] = 0.f;  // a NaN sum is not an empty one
  }

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
    if constexpr (PAGED) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int q = 0; q < 2; ++q)
          *reinterpret_cast<f32x4*>(&s_o[wave][row][32 * g + 8 * e + 4 * q]) =
              f32x4{acc[v][4 * q][e], acc[v][4 * q + 1][e], acc[v][4 * q + 2][e], acc[v][4 * q + 3][e]};
    } else {
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f32x4*>(&s_o[wave][row][16 * dt + 4 * g]) = acc[v][dt];
    }
  }
  __syncthreads();

  const long long pbase = ((long long)rh * a.nsplit + split) * a.rows;
  const int last = min(tlen * a.G, a.rows) - row0;  // rows of this group in the tree
  for (int pos = threadIdx.x; pos < kRows * (kHeadDim / 4); pos += kTW * 64) {
    const int row = pos >> 5;
    const int c4 = pos & 31;
    if (row >= last) break;
    f32x4 o = *reinterpret_cast<const f32x4*>(&s_o[0][row][c4 * 4]);
#pragma unroll
    for (int w = 1; w < kTW; ++w) o += *reinterpret_cast<const f32x4*>(&s_o[w][row][c4 * 4]);
    if (a.nsplit == 1) {
      write_row(a, r, h, row0 + row, c4, o, s_ml[0][row], s_ml[1][row]);
    } else {
      *reinterpret_cast<f32x4*>(a.part_o + (pbase + row0 + row) * kHeadDim + c4 * 4) = o;
      if (c4 == 0)
        *reinterpret_cast<float2*>(a.part_ml + (pbase + row0 + row) * 2) = make_float2(s_ml[0][row], s_ml[1][row]);
    }
  }
}

// Merge of the splits: 8 rows of one pair per workgroup, 32 threads a row, 4 dims a
// thread; the splits are read kMergeBatch at a time.
constexpr int kTreeMergeRows = 8;

__global__ __launch_bounds__(kTreeMergeRows * 32) void tree_merge_kernel(TreeAttnArgs a) {
  const int groups = (a.rows + kTreeMergeRows - 1) / kTreeMergeRows;
  const int item = tree_item(blockIdx.x, a.R * a.Hkv * groups);
  if (item < 0) return;
  const int rh = item / groups;
  const int row = (item - rh * groups) * kTreeMergeRows + (threadIdx.x >> 5);
  const int r = rh / a.Hkv;
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
      // a split without an attended token (maximum -inf) weighs nothing
      if (s0 + s < a.nsplit && ml[s].x != -INFINITY) {
        const float f = fast_exp2(ml[s].x - mn);
        S += ml[s].y * f;
        o += os[s] * f;
      }
    }
    M = mn;
  }
  write_row(a, r, rh - r * a.Hkv, row, c4, o, M, S);
}

template <int NT, int BS, bool PAGED>
void launch_nt(const TreeAttnArgs& a, hipStream_t s) {
  const long long items = (long long)a.R * a.Hkv * a.nsplit * a.groups;
  hipLaunchKernelGGL((tree_attn_kernel<NT, BS, PAGED>), dim3((unsigned)((items + 7) / 8 * 8)), dim3(kTW * 64), 0, s, a);
}

template <int BS, bool PAGED>
void launch_bs(const TreeAttnArgs& a, hipStream_t s) {
  switch (a.tiles) {
    case 1: return launch_nt<1, BS, PAGED>(a, s);
    case 2: return launch_nt<2, BS, PAGED>(a, s);
    case 3: return launch_nt<3, BS, PAGED>(a, s);
    default: return launch_nt<4, BS, PAGED>(a, s);
  }
}

}  // namespace

hipError_t launch_tree_attn(const TreeAttnArgs& a, bool paged, hipStream_t s) {
  if (a.B == 16)
    paged ? launch_bs<16, true>(a, s) : launch_bs<16, false>(a, s);
  else
    paged ? launch_bs<32, true>(a, s) : launch_bs<32, false>(a, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  const long long items = (long long)a.R * a.Hkv * ((a.rows + kTreeMergeRows - 1) / kTreeMergeRows);
  hipLaunchKernelGGL(tree_merge_kernel, dim3((unsigned)((items + 7) / 8 * 8)), dim3(kTreeMergeRows * 32), 0, s, a);
  return hipGetLastError();
}

}  // namespace oasis
