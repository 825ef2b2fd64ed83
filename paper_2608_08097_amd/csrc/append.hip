// Append of a step's accepted tokens to the paged cache: row path[r][i] of the
// new keys and values goes to position ctx_len[r] + i of request r.
//
// A (token, head) entry is 256 contiguous bytes on both sides, 16 lanes of 16
// bytes; the pages may be device memory or pinned host memory (posted writes). It is a
// copy: four chunks of 8,192 tokens (268 MB both ways) 51 us, 5.3 TB/s; a batch's accepted
// rows (2.4 MB) the time of a launch. To pinned pages it runs at the link's rate: 1.2 MB of
// accepted rows 23 us, 51 GB/s; a chunk of 8,192 tokens 614 us, 55 GB/s.
#include "drafts_internal.h"

namespace oasis {
namespace {

constexpr int kAT = 256;

__global__ __launch_bounds__(kAT) void append_kernel(AppendArgs a) {
  const int r = blockIdx.y;
  const long long cap = (long long)a.NBmax * a.B;
  long long ctx = a.ctx_len[r];
  ctx = ctx < 0 ? 0 : (ctx > cap ? cap : ctx);
  int n = a.path_len ? a.path_len[r] : a.T;
  n = n < 0 ? 0 : (n > a.T ? a.T : n);
  if (n > cap - ctx) n = (int)(cap - ctx);
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.new_ctx_len) a.new_ctx_len[r] = (int)(ctx + n);
  constexpr int kPieces = kHeadDim / 8;  // of 16 bytes
  const uint32_t at = blockIdx.x * kAT + threadIdx.x;  // below 2^31 (the entry point)
  const uint32_t entry = at / kPieces;                 // K of every head of a token, then V
  const int i = a.by_hkv(entry >> 1);
  if (i >= n) return;
  int h = (int)entry - 2 * i * a.Hkv;
  const bool is_v = h >= a.Hkv;
  if (is_v) h -= a.Hkv;
  const int row = a.path ? a.path[(long long)r * a.T + i] : i;
  if (row < 0 || row >= a.T) return;
  const long long pos = ctx + i;
  const int shift = a.B == 16 ? 4 : 5;
  const int page = a.table[(long long)r * a.NBmax + (pos >> shift)];
  if (page < 0 || page >= a.num_pages) return;
  const int piece = at % kPieces * 8;
  const uint16_t* src = (is_v ? a.new_v : a.new_k) + (((long long)r * a.T + row) * a.Hkv + h) * kHeadDim + piece;
  uint16_t* dst = (is_v ? a.v : a.k) + (((long long)page * a.Hkv + h) * a.B + (pos & (a.B - 1))) * kHeadDim + piece;
  *reinterpret_cast<u32x4*>(dst) = ldg16(src);
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
  const long long threads = (long long)a.T * 2 * a.Hkv * (kHeadDim / 8);
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)((threads + kAT - 1) / kAT), (unsigned)a.R), dim3(kAT), 0, s, a);
  return hipGetLastError();
}

}  // namespace oasis
