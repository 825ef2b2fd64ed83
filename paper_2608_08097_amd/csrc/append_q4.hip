// Append to the 4-bit paged cache: row path[r][i] of the new keys and values, the keys
// turned to position ctx_len[r] + i on the way (rotary.h), quantised and written there.
//
// A (token, head) entry is 16 lanes of 8 dims; four lanes share a power of two. The power
// is the smallest 2^e whose seven-fold reaches the group's largest value, so that no value
// is off by more than half of the step at it (6 rounds up to 7); e stays in [-126, 125], so
// that every value read back is finite. The codes are the nearest, ties to an even code
// (the hardware's conversion). A NaN or an infinity makes its 32 values NaN.
//
// Turned keys are held in 64 bits up to their code: with 32, one value in some 10^7 lies
// close enough to a border between two codes to fall on the other side. On the way to the
// conversion, which takes 32 bits, they are rounded to odd, which keeps them on their side.
//
// Four chunks of 8,192 tokens (306 MB with the rows read back): 77 us, 65 without the
// rotation, 60 at the rate of a copy. Heads of keys and values alternate between the waves:
// with all keys in two of the four, on two of the SIMDs, 87; with the pages looked up row by
// row 100. A batch's accepted rows take the time of a launch (4.3 us).
#include "rotary.h"

namespace oasis {
namespace {

constexpr int kQAThreads = 256;
constexpr int kQATokens = 8;  // of a workgroup at most

// A float on the same side of every value of 23 significant bits and fewer as x.
__device__ __forceinline__ float round_to_odd(double x) {
  float f = (float)x;
  const double back = (double)f;
  uint32_t b = __float_as_uint(f);
  if (fabs(back) > fabs(x)) --b;          // towards zero (an infinity from a finite x: the largest value)
  if (back != x) b |= 1;
  return back != back ? f : __uint_as_float(b);
}

// Largest of the four lanes of a group.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true);  // quad_perm 1,0,3,2
  x = x > y ? x : y;
  const uint32_t z = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true);  // quad_perm 2,3,0,1
  return x > z ? x : z;
}

template <bool ROTATE>
__global__ __launch_bounds__(kQAThreads) void q4_append_kernel(AppendQ4Args a) {
  __shared__ double2 s_cs[ROTATE ? kQATokens : 1][kHeadDim / 2];
  __shared__ int2 s_at[kQATokens];  // a token's row of the new ones (-1: it is not written) and its page
  const int r = blockIdx.y;
  const long long cap = (long long)a.NBmax * a.B;
  long long ctx = a.ctx_len[r];
  ctx = ctx < 0 ? 0 : (ctx > cap ? cap : ctx);
  int n = a.path_len ? a.path_len[r] : a.T;
  n = n < 0 ? 0 : (n > a.T ? a.T : n);
  if (n > cap - ctx) n = (int)(cap - ctx);
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.new_ctx_len) a.new_ctx_len[r] = (int)(ctx + n);
  const int i0 = blockIdx.x * a.tokens;
  const int mine = min(n - i0, a.tokens);
  if (mine <= 0) return;
  if ((int)threadIdx.x < mine) {
    const int i = i0 + threadIdx.x;
    const int row = a.path ? a.path[(long long)r * a.T + i] : i;
    const int page = a.table[(long long)r * a.NBmax + ((ctx + i) >> (a.B == 16 ? 4 : 5))];
    const bool ok = row >= 0 && row < a.T && page >= 0 && page < a.num_pages;
    s_at[threadIdx.x] = make_int2(ok ? row : -1, page);
  }
  __syncthreads();
  const int heads = 2 * a.Hkv;
  const int w = threadIdx.x & 15, d0 = 8 * w;  // this lane's dims
  // whole waves stay together: the quads exchange their maxima
  const int end = (mine * heads + 3) / 4 * 4;
  struct Entry {
    int t, h, row, page;
    bool is_v;
    const uint16_t* src;
    u32x4 x;
  };
  auto fetch = [&](int e) __attribute__((always_inline)) {
    Entry y;
    const bool in = e < mine * heads;
    y.t = in ? a.by_heads(e) : 0;
    const int hh = in ? e - y.t * heads : 0;
    const bool upper = hh >= a.Hkv;
    y.is_v = upper != (bool)(y.t & 1);  // in turn, so that every SIMD has its share of the rotations
    y.h = upper ? hh - a.Hkv : hh;
    const int2 at = s_at[y.t];
    y.row = in ? at.x : -1;
    y.page = at.y;
    const long long from = (long long)r * a.T + (y.row < 0 ? 0 : y.row);
    y.src = (y.is_v ? a.new_v + from * a.v_stride : a.new_k + from * a.k_stride) + y.h * kHeadDim;
    y.x = ldg16(y.src + d0);
    return y;
  };
  Entry ahead{};
  if ((int)threadIdx.x >> 4 < end) ahead = fetch(threadIdx.x >> 4);
  if constexpr (ROTATE) {  // behind the first loads
    for (int e = threadIdx.x; e < mine * 64; e += kQAThreads) {
      const int t = e >> 6, pair = e & 63;
      if (pair < a.rot.half) s_cs[t][pair] = rotary_cos_sin(a.rot, ctx + i0 + t, pair);
    }
    __syncthreads();
  }
  for (int e = threadIdx.x >> 4; e < end; e += kQAThreads / 16) {
    const Entry cur = ahead;
    if (e + kQAThreads / 16 < end) ahead = fetch(e + kQAThreads / 16);
    const int t = cur.t, h = cur.h, i = i0 + t, tok = (int)((ctx + i) & (a.B - 1));
    const bool is_v = cur.is_v, ok = cur.row >= 0;
    const uint16_t* src = cur.src;
    const u32x4 x = cur.x;
    float f[8];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      f[2 * p] = bf16_bits_to_f32(x[p] & 0xFFFFu);
      f[2 * p + 1] = __uint_as_float(x[p] & 0xFFFF0000u);
    }
    if constexpr (ROTATE) {
      if (!is_v && d0 < 2 * a.rot.half) {
        const double2* cs = s_cs[t];
        if (a.rot.interleaved) {
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const int pair = d0 / 2 + p;
            if (pair < a.rot.half) {
              const double2 c = cs[pair];
              const double lo = f[2 * p], hi = f[2 * p + 1];
              f[2 * p] = round_to_odd(lo * c.x - hi * c.y);
              f[2 * p + 1] = round_to_odd(hi * c.x + lo * c.y);
            }
          }
        } else {
          const int half = a.rot.half;
          float g[8];  // the other ends of the pairs
          if (half % 8 == 0) {
            const u32x4 y = ldg16(src + (d0 < half ? d0 + half : d0 - half));
#pragma unroll
            for (int p = 0; p < 4; ++p) {
              g[2 * p] = bf16_bits_to_f32(y[p] & 0xFFFFu);
              g[2 * p + 1] = __uint_as_float(y[p] & 0xFFFF0000u);
            }
          } else {
#pragma unroll
            for (int p = 0; p < 8; ++p) {
              const int d = d0 + p;
              g[p] = d < 2 * half ? bf16_bits_to_f32(src[d < half ? d + half : d - half]) : 0.f;
            }
          }
#pragma unroll
          for (int p = 0; p < 8; ++p) {
            const int d = d0 + p;
            if (d < half) {
              const double2 c = cs[d];
              f[p] = round_to_odd((double)f[p] * c.x - (double)g[p] * c.y);
            } else if (d < 2 * half) {
              const double2 c = cs[d - half];
              f[p] = round_to_odd((double)f[p] * c.x + (double)g[p] * c.y);
            }
          }
        }
      }
    }
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const uint32_t b = __float_as_uint(f[p]) & 0x7FFFFFFFu;
      top = top > b ? top : b;
    }
    top = quad_max(top);
    const bool wild = top >= 0x7F800000u;
    // exponent of the largest value, one more past 1.75 of its power, less 2
    int byte = (int)((top + 0x1FFFFFu) >> 23) - 2;
    byte = wild ? kQ4NaN : (byte < 1 ? 1 : (byte > 252 ? 252 : byte));
    const float scale = __uint_as_float((uint32_t)byte << 23);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[0], f[1], scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[2], f[3], scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[4], f[5], scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, f[6], f[7], scale, 3);
    codes = wild ? 0 : codes;
    if (!ok) continue;
    uint8_t* dst = (is_v ? a.v : a.k) + cur.page * a.page_bytes;
    *reinterpret_cast<uint32_t*>(dst + (h * a.B + tok) * kQ4Codes + 4 * w) = codes;
    if ((w & 3) == 0) dst[a.Hkv * a.B * kQ4Codes + q4_power_at(h, a.B, tok, w >> 2)] = (uint8_t)byte;
    uint16_t* read = is_v ? a.read_v : a.read_k;
    if (read) {
      u32x4 y;
      y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
      y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
      y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
      y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
      // past the caches: whole lines (92 -> 87 us)
      __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(read + (((long long)r * a.T + i) * a.Hkv + h) * kHeadDim + d0));
    }
  }
}

}  // namespace

hipError_t launch_append_q4(const AppendQ4Args& args, hipStream_t s) {
  AppendQ4Args a = args;
  a.tokens = kQATokens;
  while (a.tokens > 1 && (long long)a.R * a.T < 1024ll * a.tokens) a.tokens >>= 1;
  const dim3 grid((unsigned)((a.T + a.tokens - 1) / a.tokens), (unsigned)a.R);
  if (a.rot.turns)
    hipLaunchKernelGGL(q4_append_kernel<true>, grid, dim3(kQAThreads), 0, s, a);
  else
    hipLaunchKernelGGL(q4_append_kernel<false>, grid, dim3(kQAThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace oasis
