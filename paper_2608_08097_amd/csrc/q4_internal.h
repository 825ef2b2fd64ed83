// Internal declarations of the 4-bit cache: its pages, rotary positions, the append that
// quantises, compressed keys, attention.
//
// A page holds, for B tokens of every KV head, codes [Hkv][B][64] and then powers of two
// [Hkv][B / 16][4][4][4], a byte each. A code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4,
// 6 (dims 2 j and 2 j + 1 of a token in the low and high half of its byte j); the power of
// 32 dims, byte s, is 2^(s - 127), s up to 252 (the conversions read the exponent of a float
// whose bits are s << 23, 2^-127 for 0). The powers of 16 tokens are indexed by t % 4, the group
// of dims and t / 4: a lane of the attention has tokens 4 apart, and finds their powers in
// one dword.
#pragma once

#include "drafts_internal.h"
#include "q4_plan.h"

namespace oasis {

constexpr int kQ4Group = 32;                       // dims that share a power of two
constexpr int kQ4Codes = kHeadDim / 2;             // bytes of a token and head
constexpr int kQ4Powers = kHeadDim / kQ4Group;
constexpr int kQ4NaN = 255;                        // power of 32 NaN (their codes are 0)
inline long long q4_page_bytes(long long Hkv, long long B) { return Hkv * B * (kQ4Codes + kQ4Powers); }

// Byte offset, behind a page's codes, of the power of token t (of B) and group g of head h.
__host__ __device__ __forceinline__ int q4_power_at(int h, int B, int t, int g) {
  return h * B * kQ4Powers + (t >> 4) * 64 + ((t & 3) * 4 + g) * 4 + ((t >> 2) & 3);
}

struct RotaryArgs {
  const double* turns;  // [half], of a pair a position; NULL: no rotation
  int half;             // pairs
  int interleaved;      // pair i: dims 2 i and 2 i + 1, else i and i + half
  double cos_amplitude, sin_amplitude;  // (a negative one of the sine turns back)
};

struct RotateArgs {
  RotaryArgs rot;
  const uint16_t *q, *k;  // rows of heads, q_stride and k_stride elements apart; NULL: none
  uint16_t *q_out, *k_out;
  long long q_stride, k_stride, q_out_stride, k_out_stride;
  const int32_t* positions;  // [R][T]; NULL: ctx_len[r] + t
  const int32_t* ctx_len;
  int T, Hq, Hkv;            // heads: 0 where there are no such rows
  long long rows;            // R * T
  int tokens;                // rows of a workgroup
  FastDiv by_heads, by_t;
};
hipError_t launch_rotate(const RotateArgs& a, hipStream_t s);

struct AppendQ4Args {
  RotaryArgs rot;
  const uint16_t *new_k, *new_v;  // rows of [Hkv][d], k_stride and v_stride elements apart
  long long k_stride, v_stride;
  const int32_t *path, *path_len;  // as AppendArgs
  uint8_t *k, *v;                  // device-visible pages
  long long num_pages, page_bytes;
  const int32_t *table, *ctx_len;
  int32_t* new_ctx_len;
  uint16_t *read_k, *read_v;       // [R][T][Hkv][d], nullable: the rows as the cache holds them
  int R, Hkv, T, B, NBmax;
  int tokens;                      // of a workgroup
  FastDiv by_heads;                // 2 * Hkv
};
hipError_t launch_append_q4(const AppendQ4Args& a, hipStream_t s);

struct SummaryQ4Args {
  const uint8_t* k;
  long long num_pages, page_bytes;
  const int32_t* table;
  const int32_t* prev_ctx_len;  // NULL: every candidate block
  const int32_t* ctx_len;
  int max_new;                  // with prev_ctx_len
  uint16_t *kmax, *kmin;
  int R, Hkv, B, NBmax;
  FastDiv by_hkv;
};
hipError_t launch_summaries_q4(const SummaryQ4Args& a, hipStream_t s);

struct AttnQ4Args : TreeAttnArgs {
  const uint8_t *k4, *v4;  // device-visible pages
  long long page_bytes;
  const int32_t* sel;        // [R][Hkv][k_sel]; NULL: every block
  const int32_t* sel_count;  // [R][Hkv]
  int k_sel;
};
hipError_t launch_attn_q4(const AttnQ4Args& a, hipStream_t s);

}  // namespace oasis
