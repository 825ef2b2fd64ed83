// What the attention kernels of a drafted tree share, over bf16 caches and over the
// 4-bit one: how work items lie on the chip, the tree's ancestors and wild values, and
// the rows' ends.
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
