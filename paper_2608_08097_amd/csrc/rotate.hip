// Rotary positions of a step's query and key rows (rotary.h), in one launch for both.
//
// A workgroup takes some rows with all their heads: first their cosines and sines, 64 bits
// rounded to 32, into LDS, then eight threads a head, 16 elements each: the two halves of
// eight pairs, or eight pairs side by side, or 16 elements that do not turn. Products and
// sums are in 32 bits, rounded to bf16 once: the rounding to bf16 is 2^15 times theirs.
//
// It is a copy: 32,768 rows of 40 heads (671 MB both ways) 120 us, 5.6 TB/s, with two rows a
// workgroup (four 125, eight 137); 320 rows the time of a launch.
#include "rotary.h"

namespace oasis {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotTokens = 2;  // rows of a workgroup at most

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint16_t, (__bf16)lo) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)hi) << 16;
}

// EIGHTS: halves of a multiple of 8 pairs, or pairs side by side.
template <bool EIGHTS>
__global__ __launch_bounds__(kRotThreads) void rotate_kernel(RotateArgs a) {
  __shared__ float2 s_cs[kRotTokens][kHeadDim / 2];
  const long long row0 = (long long)blockIdx.x * a.tokens;
  const int n = (int)(a.rows - row0 < a.tokens ? a.rows - row0 : a.tokens);
  const int half = a.rot.half;
  for (int e = threadIdx.x; e < n * 64; e += kRotThreads) {
    const int t = e >> 6, pair = e & 63;
    if (pair >= half) continue;
    const long long row = row0 + t;
    long long pos;
    if (a.positions) {
      pos = a.positions[row];
    } else {
      const int r = a.by_t((uint32_t)row);
      const int ctx = a.ctx_len[r];
      pos = (long long)(ctx < 0 ? 0 : ctx) + ((int)row - r * a.T);
    }
    const double2 cs = rotary_cos_sin(a.rot, pos, pair);
    s_cs[t][pair] = make_float2((float)cs.x, (float)cs.y);
  }
  __syncthreads();
  const int heads = a.Hq + a.Hkv;
  const int per = EIGHTS ? 8 : 64;  // threads of a head
  for (int e = threadIdx.x; e < n * heads * per; e += kRotThreads) {
    const int w = e & (per - 1), th = e / per;
    const int t = a.by_heads(th), hh = th - t * heads;
    const bool is_k = hh >= a.Hq;
    const int h = is_k ? hh - a.Hq : hh;
    const uint16_t* src = (is_k ? a.k + (row0 + t) * a.k_stride : a.q + (row0 + t) * a.q_stride) + h * kHeadDim;
    uint16_t* dst = (is_k ? a.k_out + (row0 + t) * a.k_out_stride : a.q_out + (row0 + t) * a.q_out_stride) + h * kHeadDim;
    const float2* cs = s_cs[t];
    if constexpr (!EIGHTS) {  // one pair, or two elements that do not turn
      const int i = w < half ? w : 2 * w, j = w < half ? w + half : 2 * w + 1;
      const float x = bf16_bits_to_f32(src[i]), y = bf16_bits_to_f32(src[j]);
      if (w < half) {
        const float2 c = cs[w];
        dst[i] = __builtin_bit_cast(uint16_t, (__bf16)(x * c.x - y * c.y));
        dst[j] = __builtin_bit_cast(uint16_t, (__bf16)(y * c.x + x * c.y));
      } else if (src != dst) {
        dst[i] = src[i];
        dst[j] = src[j];
      }
    } else if (a.rot.interleaved) {
      u32x4 v[2] = {ldg16(src + 8 * w), ldg16(src + 64 + 8 * w)};  // whole lines (32 bytes a lane: 8 % slower)
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        const int pair = (p >> 2) * 32 + 4 * w + (p & 3);
        const uint32_t x = v[p >> 2][p & 3];
        const float2 c = cs[pair];  // (past the pairs: not used)
        const float lo = bf16_lo(x), hi = bf16_hi(x);
        const uint32_t y = pack_bf16(lo * c.x - hi * c.y, hi * c.x + lo * c.y);
        v[p >> 2][p & 3] = pair < half ? y : x;
      }
      *reinterpret_cast<u32x4*>(dst + 8 * w) = v[0];
      *reinterpret_cast<u32x4*>(dst + 64 + 8 * w) = v[1];
    } else {
      const bool turns = 8 * w < half;
      const int i = turns ? 8 * w : 16 * w, j = turns ? i + half : i + 8;
      if (!turns && src == dst) continue;
      u32x4 x = ldg16(src + i), y = ldg16(src + j);
      if (turns) {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const float2 c0 = cs[i + 2 * p], c1 = cs[i + 2 * p + 1];
          const float x0 = bf16_lo(x[p]), x1 = bf16_hi(x[p]), y0 = bf16_lo(y[p]), y1 = bf16_hi(y[p]);
          x[p] = pack_bf16(x0 * c0.x - y0 * c0.y, x1 * c1.x - y1 * c1.y);
          y[p] = pack_bf16(y0 * c0.x + x0 * c0.y, y1 * c1.x + x1 * c1.y);
        }
      }
      *reinterpret_cast<u32x4*>(dst + i) = x;
      *reinterpret_cast<u32x4*>(dst + j) = y;
    }
  }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& args, hipStream_t s) {
  RotateArgs a = args;
  a.tokens = kRotTokens;
  while (a.tokens > 1 && a.rows < 1024ll * a.tokens) a.tokens >>= 1;
  const unsigned grid = (unsigned)((a.rows + a.tokens - 1) / a.tokens);
  if (a.rot.interleaved || a.rot.half % 8 == 0)
    hipLaunchKernelGGL(rotate_kernel<true>, dim3(grid), dim3(kRotThreads), 0, s, a);
  else
    hipLaunchKernelGGL(rotate_kernel<false>, dim3(grid), dim3(kRotThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace oasis
