// What the attention kernels of a drafted tree share, over bf16 caches and over the
// 4-bit one: how work items lie on the chip, the online softmax, the tree's ancestors and
// wild values, and the rows' ends.
#pragma once

#include "drafts_internal.h"

namespace oasis {
namespace {

// Contiguous runs of the items on each XCD (workgroup ids go round the 8 XCDs): a
// pair's splits and row groups share one L2.
__device__ __forceinline__ int tree_item(int wg, int items) {
  const int item = (wg & 7) * ((items + 7) >> 3) + (wg >> 3);
  return (wg >> 3) < ((items + 7) >> 3) && item < items ? item : -1;
}

// The same where the requests are taken by length (tree_by_length): the n-th of `count`
// runs of keys and values goes to XCD n % 8, its row groups one after the other there.
__device__ __forceinline__ int tree_item_spread(int wg, const TreeAttnArgs& a, int count, int& group) {
  const int n = wg >> 3, run = a.by_groups(n);
  const int item = run * 8 + (wg & 7);
  group = n - run * a.groups;
  return item < count ? item : -1;
}
// The request of rank k by length, and in `len` its length: the longest first, equal ones
// in order. At most 64 of them, one a lane.
__device__ __forceinline__ int request_of_rank(const int32_t* ctx_len, int R, int k, int& len) {
  const int lane = threadIdx.x & 63;
  const int mine = lane < R ? ctx_len[lane] : INT32_MIN;
  int rank = lane < R ? 0 : R;
  for (int r = 0; r < R; ++r) {
    const int other = __builtin_amdgcn_readlane(mine, r);
    rank += other > mine || (other == mine && r < lane);
  }
  const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(rank == k));
  len = __builtin_amdgcn_readlane(mine, at);
  return at;
}

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

// The tree's values: a row that attends a token takes up its infinities and NaN,
// the other rows must not, but 0 times them is NaN in the product. So they are
// taken out of the product (true: there were some) and added to the rows that
// attend them when those are written (add_wild).
__device__ __forceinline__ bool wild_bf16(uint32_t b) { return (b & 0x7F80u) == 0x7F80u; }
__device__ __forceinline__ bool wild_f32(float x) {
  return (__builtin_bit_cast(uint32_t, x) & 0x7F800000u) == 0x7F800000u;
}
__device__ __forceinline__ bool take_wild(u32x4 (&v)[8]) {
  uint32_t any = 0;  // an exponent of ones carries into the sign's place
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int p = 0; p < 4; ++p) any |= (v[j][p] & 0x7F807F80u) + 0x00800080u;
  if (!__builtin_amdgcn_ballot_w64((any & 0x80008000u) != 0)) return false;
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      uint32_t x = v[j][p];
      asm volatile("" : "+v"(x));  // one at a time: the test's terms are not kept for this
      v[j][p] = x & ~(((((x & 0x7F807F80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xFFFFu);
    }
  return true;
}

// A tile's scores of 32 tokens, 8 a lane; those of the lane's bits stay.
__device__ __forceinline__ void mask_scores(f32x4 (&sc)[2], uint32_t bits) {
#pragma unroll
  for (int e = 0; e < 8; ++e) sc[e >> 2][e & 3] = bits >> e & 1 ? sc[e >> 2][e & 3] : -INFINITY;
}

// Online softmax of one tile's scores (scale > 0: load_q): probabilities in bf16
// (the second product's operand; 2^-8 of each at most, unbiased, and the sum takes
// them unrounded), the row's reference (negated: +inf before its first token) and
// the lane's partial sum updated. A probability is 2^(score - reference), and the
// reference follows the row's maximum only when a lane's eight probabilities pass
// `top` together: that needs no maximum of every unit's scores, and values far
// above the reference show as large, infinite or NaN sums. The accumulators are
// rescaled then, in a branch that is rare after a wave's first unit. The reference
// lies a lift above the maximum that it was taken from, and `top` as far below 2^8
// (tree_lift): the sums of all the tokens that the call can attend stay below 1/2,
// so that no finite value overflows in them.
// (Taken from `top` where it is needed: with it as an argument of its own, live through
// the loops, wide trees took 1 % more.)
__device__ __forceinline__ float tree_lift_of(float top) { return (float)(9 - __builtin_amdgcn_frexp_expf(top)); }

__device__ __forceinline__ float unit_exp(const f32x4 (&s)[2], float scale, float m_neg, float (&p)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) p[e] = fast_exp2(__builtin_fmaf(s[e >> 2][e & 3], scale, m_neg));
  return ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
}

__device__ __forceinline__ bf16x8 unit_softmax(const f32x4 (&s)[2], float scale, float top, float& m_neg, float& l_part,
                                               f32x4 (&acc)[8]) {
  float p[8];
  float psum = unit_exp(s, scale, m_neg, p);
  const uint64_t past = __builtin_amdgcn_ballot_w64(!(psum <= top));
  if (__builtin_expect(past != 0, 0)) {
    // the rows that passed it in one of their four lanes; the others stay as they are
    const uint64_t rows = past | past >> 16 | past >> 32 | past >> 48;
    const bool mine = rows >> (threadIdx.x & 15) & 1;
    const float lmax = scale * fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                                     fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    float m = fmaxf(lmax, __shfl_xor(lmax, 16));
    m = fmaxf(fmaxf(m, __shfl_xor(m, 32)) + tree_lift_of(top), -m_neg);
    m = mine ? m : -m_neg;
    const float alpha = m == -INFINITY ? 1.f : fast_exp2(-m_neg - m);
    l_part *= alpha;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[dt] *= alpha;
    m_neg = -m;
    psum = unit_exp(s, scale, m == -INFINITY ? 0.f : m_neg, p);
  }
  bf16x8 pb;
#pragma unroll
  for (int e = 0; e < 8; ++e) pb[e] = (__bf16)p[e];
  l_part += psum;
  return pb;
}

// A row's maximum and, in l, its sum, from its four lanes' parts.
__device__ __forceinline__ float finish_row(float m_neg, float& l) {
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  return l != l && m_neg == INFINITY ? 0.f : -m_neg;  // a NaN sum is not an empty one
}

// A lane's parent in a request's tree, -1 for a root: row t's in lane t.
__device__ __forceinline__ int tree_parent(const TreeAttnArgs& a, int r, int len, int lane) {
  if (lane < 1 || lane >= len) return -1;
  const int up = a.parent ? a.parent[(long long)r * a.T + lane] : lane - 1;
  return up >= 0 && up < lane ? up : -1;
}
// Ancestor masks, lane t: row t's (its own bit among them); lanes past the tree hold
// 0. Pointer doubling: after n rounds a mask holds 2^n rows of the path, so it ends
// by the sixth.
__device__ __forceinline__ uint64_t ancestors(int up, int len, int lane) {
  uint64_t m = lane < len ? 1ull << lane : 0;
  while (__builtin_amdgcn_ballot_w64(up >= 0)) {
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

constexpr float kBf16Max = 0x1.fep127f;

// Normalised bf16 output of 4 dims of one row, and its log-sum-exp.
__device__ __forceinline__ void write_row(const TreeAttnArgs& a, int r, int h, int row, int c4, f32x4 o, float M, float L) {
  const int t = a.by_g(row);
  const int qh = h * a.G + (row - t * a.G);
  const long long orow = ((long long)r * a.T + t) * a.Hq + qh;
  const float inv = L == 0.f ? 0.f : 1.f / L;  // a NaN sum stays one
  // a mean of finite values is no larger than they are: where the rounded probabilities
  // weigh more than their sum, it must not pass the largest value
  auto mean = [&](float x) __attribute__((always_inline)) {
    const float y = x * inv;
    return (__bf16)(wild_f32(y) ? y : __builtin_amdgcn_fmed3f(y, -kBf16Max, kBf16Max));
  };
  uint32_t w[2];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const __bf16 lo = mean(o[2 * p]), hi = mean(o[2 * p + 1]);
    w[p] = __builtin_bit_cast(uint16_t, lo) | (uint32_t)__builtin_bit_cast(uint16_t, hi) << 16;
  }
  *reinterpret_cast<uint2*>(a.out + orow * kHeadDim + c4 * 4) = make_uint2(w[0], w[1]);
  if (c4 == 0 && a.lse) a.lse[orow] = L == 0.f ? -INFINITY : (M + __log2f(L)) * 0.69314718055994531f;
}

__device__ __forceinline__ int tree_length(const TreeAttnArgs& a, int r) {
  const int n = a.tree_len ? a.tree_len[r] : a.T;
  return n < 0 ? 0 : (n > a.T ? a.T : n);
}

// The infinities and NaN that row `row` attends in the tree, in dims 4 c4 .. +3 (t:
// elements to the head's first tree row and between them).
template <typename Item>
__device__ __forceinline__ void add_wild(const TreeAttnArgs& a, const Item& t, uint64_t anc, int c4, f32x4& o) {
  for (; anc; anc &= anc - 1) {
    const int j = __builtin_ctzll(anc);
    const uint2 w = *reinterpret_cast<const uint2*>(a.tree_v + t.tree_base + j * t.tree_row + c4 * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t b = (e < 2 ? w.x : w.y) >> (e & 1) * 16 & 0xFFFFu;
      if (wild_bf16(b)) o[e] += bf16_bits_to_f32(b);
    }
  }
}

}  // namespace
}  // namespace oasis
