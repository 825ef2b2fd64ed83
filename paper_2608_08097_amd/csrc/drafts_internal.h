// Internal declarations of the speculative step: attention of a drafted token
// tree, draft verification, append of accepted tokens.
#pragma once

#include "oasis_internal.h"
#include "tree_plan.h"

namespace oasis {

struct TreeAttnArgs {
  const uint16_t* q;
  const uint16_t* k;         // pages [num_pages][Hkv][B][d], or the working set's pool_k
  const uint16_t* v;         // pages as k, or pool_v [R][k_slots+1][Hkv][d][B]
  const int32_t* table;      // block table [R][NBmax], or slot_map [R][Hkv][k_slots]
  const int32_t* ctx_len;
  const uint16_t* tree_k;    // [R][T][Hkv][d]
  const uint16_t* tree_v;
  const int32_t* parent;     // [R][T]; NULL: a chain
  const int32_t* tree_len;   // [R]; NULL: T
  uint16_t* out;
  float* lse;
  float* part_o;             // [R*Hkv][nsplit][rows][d]
  float* part_ml;            // [R*Hkv][nsplit][rows][2]
  long long num_pages;
  int R, Hq, Hkv, G, T, B, NBmax, k_slots;
  float scale_log2;
  int rows, tiles, groups, nsplit;
};
hipError_t launch_tree_attn(const TreeAttnArgs& a, bool paged, hipStream_t s);

struct VerifyArgs {
  const float* target;       // [R][T] rows of V, target_stride apart
  const float* draft;        // the same, draft_stride apart; NULL: drafts without probabilities
  long long target_stride, draft_stride;
  const int32_t* tokens;
  const int32_t* parent;
  const int32_t* tree_len;
  const float* accept_u;     // [R][T]
  const float* sample_u;     // [R]
  int32_t* path;             // [R][T]
  int32_t* path_len;         // [R]
  int32_t* out_tokens;       // [R][T]
  double* part;              // [R][chunks] masses, then the walks' states
  int R, T, V, chunks;
};
constexpr int kVerifyChunk = 4096;  // vocabulary entries per workgroup
// where a request's walk ended: node, rows on the path, rejected siblings, coefficient
struct VerifyState {
  double coef;
  unsigned long long rejected;
  int node, len;
};
inline int verify_chunks(int V) { return (V + kVerifyChunk - 1) / kVerifyChunk; }
inline size_t verify_ws_bytes(long long R, int V) {
  return (size_t)R * (verify_chunks(V) * sizeof(double) + sizeof(VerifyState));
}
hipError_t launch_verify(const VerifyArgs& a, hipStream_t s);

struct AppendArgs {
  const uint16_t* new_k;     // [R][T][Hkv][d]
  const uint16_t* new_v;
  const int32_t* path;       // [R][T]; NULL: rows 0, 1, ...
  const int32_t* path_len;   // [R]; NULL: T
  uint16_t* k;               // device-visible pages [num_pages][Hkv][B][d]
  uint16_t* v;
  long long num_pages;
  const int32_t* table;
  const int32_t* ctx_len;
  int32_t* new_ctx_len;      // nullable
  int R, Hkv, T, B, NBmax;
};
hipError_t launch_append(const AppendArgs& a, hipStream_t s);

}  // namespace oasis
