// Compressed keys of the 4-bit cache: per block and head the coordinate-wise maximum and
// minimum of the keys as the cache holds them (summaries.hip), exact in bf16.
//
// Eight threads a (request, block, head), 16 dims each: a token's 8 bytes, two codes a
// conversion with the token's power, then a maximum and a minimum a value.
#include <type_traits>

#include "q4_internal.h"

namespace oasis {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

template <int SEL>
__device__ __forceinline__ f32x2 pair_of(uint32_t w, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, SEL);
}

template <int BS>
__global__ __launch_bounds__(256) void q4_summaries_kernel(SummaryQ4Args a) {
  const int r = blockIdx.y;
  const uint32_t item = blockIdx.x * 256 + threadIdx.x;  // below 2^31 (the entry point)
  const int w = item & 7;
  const int bh = item >> 3, at = a.by_hkv(bh), h = bh - at * a.Hkv;
  const Ctx c = ctx_blocks(a.ctx_len[r], BS, a.NBmax);
  const int lo = a.prev_ctx_len ? ctx_blocks(a.prev_ctx_len[r], BS, a.NBmax).n_cand : 0;
  if (a.prev_ctx_len && at >= a.max_new) return;
  const long long b = (long long)lo + at;
  if (b >= c.n_cand) return;
  const int page = a.table[(long long)r * a.NBmax + b];
  if (page < 0 || page >= a.num_pages) return;
  const uint8_t* base = a.k + page * a.page_bytes;
  const uint8_t* codes = base + h * BS * kQ4Codes + w * 8;
  const uint32_t* powers = reinterpret_cast<const uint32_t*>(base + a.Hkv * BS * kQ4Codes + h * BS * kQ4Powers) + (w >> 1);
  uint2 x[BS];
  uint32_t p[BS / 4];
#pragma unroll
  for (int t = 0; t < BS; ++t) x[t] = *reinterpret_cast<const uint2*>(codes + t * kQ4Codes);
#pragma unroll
  for (int q = 0; q < BS / 4; ++q) p[q] = powers[(q >> 2) * 16 + (q & 3) * 4];  // tokens q % 4 + 4 u of 16
  float mx[16], mn[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    mx[j] = -INFINITY;
    mn[j] = INFINITY;
  }
#pragma unroll
  for (int t = 0; t < BS; ++t) {
    const float s = __uint_as_float((p[(t >> 4) * 4 + (t & 3)] >> (8 * ((t >> 2) & 3)) & 255u) << 23);
    const f32x2 v[8] = {pair_of<0>(x[t].x, s), pair_of<1>(x[t].x, s), pair_of<2>(x[t].x, s), pair_of<3>(x[t].x, s),
                        pair_of<0>(x[t].y, s), pair_of<1>(x[t].y, s), pair_of<2>(x[t].y, s), pair_of<3>(x[t].y, s)};
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      mx[j] = fmaxf(mx[j], v[j >> 1][j & 1]);
      mn[j] = fminf(mn[j], v[j >> 1][j & 1]);
    }
  }
  const long long o = (((long long)r * a.Hkv + h) * a.NBmax + b) * kHeadDim + w * 16;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    u32x4 omx, omn;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int j = half * 8 + 2 * q;  // exact: the values are bf16
      omx[q] = (__float_as_uint(mx[j]) >> 16) | (__float_as_uint(mx[j + 1]) & 0xFFFF0000u);
      omn[q] = (__float_as_uint(mn[j]) >> 16) | (__float_as_uint(mn[j + 1]) & 0xFFFF0000u);
    }
    *reinterpret_cast<u32x4*>(a.kmax + o + half * 8) = omx;
    *reinterpret_cast<u32x4*>(a.kmin + o + half * 8) = omn;
  }
}

}  // namespace

hipError_t launch_summaries_q4(const SummaryQ4Args& a, hipStream_t s) {
  const long long blocks = a.prev_ctx_len ? (a.max_new < a.NBmax ? a.max_new : a.NBmax) : a.NBmax;
  const long long items = blocks * a.Hkv * 8;
  const dim3 grid((unsigned)((items + 255) / 256), (unsigned)a.R);
  if (a.B == 16)
    hipLaunchKernelGGL(q4_summaries_kernel<16>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(q4_summaries_kernel<32>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace oasis
