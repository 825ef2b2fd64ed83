// Compressed keys of the 4-bit cache: per block and head the coordinate-wise maximum and
// minimum of the keys as the cache holds them (summaries.hip), exact in bf16.
//
// A wave takes eight sub-blocks, 16 tokens of one head each: their codes come in whole lines,
// a kilobyte a load, and pass through LDS to eight threads a sub-block, 16 dims each (8 of
// the first 64 and 8 of the others, so that a row is written in whole lines): two codes a
// conversion with their token's power, then a maximum and a minimum a value.
//
// 8 x 131,072 tokens (570 MB read, 268 written): 160 us, 5.24 TB/s, a copy's rate; with eight
// bytes a lane straight from memory, in half lines, 169. A step's new blocks take the time of
// a launch (3.7 us).
#include <type_traits>

#include "q4_internal.h"

namespace oasis {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kSubs = 8;             // sub-blocks of a wave
constexpr int kSubStride = 1024 + 32;  // of a sub-block in LDS: the eight of a read meet no bank twice

__device__ __forceinline__ void eight_f32(uint32_t w, float s, f32x2 (&v)[4]) {
  v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0);
  v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1);
  v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2);
  v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
}
__device__ __forceinline__ float across_eight(float x) {  // the value of the lane 8 further in its row of 16
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xF, 0xF, false));
}

template <int BS>
__global__ __launch_bounds__(256, 4) void q4_summaries_kernel(SummaryQ4Args a) {
  __shared__ __align__(16) char s_codes[4][kSubs * kSubStride];
  __shared__ uint32_t s_powers[4][kSubs * 16];
  constexpr int kPer = BS / 16;  // sub-blocks of an item (block, head)
  const int r = blockIdx.y;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const Ctx c = ctx_blocks(a.ctx_len[r], BS, a.NBmax);
  const int lo = a.prev_ctx_len ? ctx_blocks(a.prev_ctx_len[r], BS, a.NBmax).n_cand : 0;
  long long n = c.n_cand - lo;
  if (a.prev_ctx_len && n > a.max_new) n = a.max_new;
  const int item0 = (blockIdx.x * 4 + wave) * (kSubs / kPer);  // below 2^28 (the entry point)
  if ((int)a.by_hkv(item0) >= n) return;
  // this lane's item, in the lanes of its sub-block
  const int sub = lane >> 3, w = lane & 7;
  const int item = item0 + sub / kPer;
  const int at = a.by_hkv(item), h = item - at * a.Hkv, b = lo + at;
  int page = at < n ? a.table[(long long)r * a.NBmax + b] : -1;
  const bool ok = page >= 0 && page < a.num_pages;
  page = ok ? page : 0;
  const long long from = page * a.page_bytes;
  const int codes_at = (h * BS + sub % kPer * 16) * kQ4Codes;
  const int powers_at = a.Hkv * BS * kQ4Codes + (h * BS + sub % kPer * 16) * kQ4Powers;
  const bool stream = (long long)a.R * n * a.Hkv * (BS * (kQ4Codes + kQ4Powers)) >= kStreamBytes;
  u32x4 x[kSubs];
  auto load = [&](auto past) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < kSubs; ++q) {
      const long long f = __shfl(from, 8 * q);
      const int o = __shfl(codes_at, 8 * q);
      x[q] = ldg16_once<decltype(past)::value>(a.k + f + o + lane * 16);
    }
  };
  // (the marks keep the compiler from folding the two forms into one)
  if (stream) {
    asm volatile("; read past the caches");
    load(std::true_type{});
    asm volatile("; read past the caches");
  } else {
    load(std::false_type{});
  }
  const uint2 pw = *reinterpret_cast<const uint2*>(a.k + from + powers_at + w * 8);
  char* const s = s_codes[wave];
#pragma unroll
  for (int q = 0; q < kSubs; ++q) *reinterpret_cast<u32x4*>(s + q * kSubStride + lane * 16) = x[q];
  *reinterpret_cast<uint2*>(&s_powers[wave][lane * 2]) = pw;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  float mx[16], mn[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    mx[j] = -INFINITY;
    mn[j] = INFINITY;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {  // tokens e + 4 u
    const uint32_t p0 = s_powers[wave][sub * 16 + e * 4 + (w >> 2)], p1 = s_powers[wave][sub * 16 + e * 4 + 2 + (w >> 2)];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const char* row = s + sub * kSubStride + (e + 4 * u) * kQ4Codes + w * 4;
      f32x2 v[2][4];
      eight_f32(*reinterpret_cast<const uint32_t*>(row), __uint_as_float((p0 >> (8 * u) & 255u) << 23), v[0]);
      eight_f32(*reinterpret_cast<const uint32_t*>(row + 32), __uint_as_float((p1 >> (8 * u) & 255u) << 23), v[1]);
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        mx[j] = fmaxf(mx[j], v[j >> 3][j >> 1 & 3][j & 1]);
        mn[j] = fminf(mn[j], v[j >> 3][j >> 1 & 3][j & 1]);
      }
    }
  }
  if constexpr (BS == 32) {  // the item's other sub-block
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      mx[j] = fmaxf(mx[j], across_eight(mx[j]));
      mn[j] = fminf(mn[j], across_eight(mn[j]));
    }
  }
  if (!ok) return;
  const long long o = (((long long)r * a.Hkv + h) * a.NBmax + b) * kHeadDim + w * 8;
  u32x4 rows[2][2];  // kmax, kmin; the first and the other 64 dims
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int j = half * 8 + 2 * q;  // exact: the values are bf16
      rows[0][half][q] = (__float_as_uint(mx[j]) >> 16) | (__float_as_uint(mx[j + 1]) & 0xFFFF0000u);
      rows[1][half][q] = (__float_as_uint(mn[j]) >> 16) | (__float_as_uint(mn[j + 1]) & 0xFFFF0000u);
    }
  auto store = [&](uint16_t* to, u32x4 v) __attribute__((always_inline)) {
    if (stream) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(to));
    else *reinterpret_cast<u32x4*>(to) = v;
  };
  if constexpr (BS == 16) {
    store(a.kmax + o, rows[0][0]);
    store(a.kmax + o + 64, rows[0][1]);
    store(a.kmin + o, rows[1][0]);
    store(a.kmin + o + 64, rows[1][1]);
  } else {  // a sub-block's lanes each write one of the two
    const int which = sub & 1;
    uint16_t* const to = which ? a.kmin : a.kmax;
    store(to + o, which ? rows[1][0] : rows[0][0]);
    store(to + o + 64, which ? rows[1][1] : rows[0][1]);
  }
}

}  // namespace

hipError_t launch_summaries_q4(const SummaryQ4Args& a, hipStream_t s) {
  const long long blocks = a.prev_ctx_len ? (a.max_new < a.NBmax ? a.max_new : a.NBmax) : a.NBmax;
  const long long per_group = 4 * kSubs / (a.B / 16);  // (block, head) items of a workgroup
  const dim3 grid((unsigned)((blocks * a.Hkv + per_group - 1) / per_group), (unsigned)a.R);
  if (a.B == 16)
    hipLaunchKernelGGL(q4_summaries_kernel<16>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(q4_summaries_kernel<32>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace oasis
