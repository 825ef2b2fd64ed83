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
  float scale_log2;          // |scale| * log2(e), 1 for a scale of 0
  uint32_t q_and, q_xor;     // what makes up for that in the queries' bits
  float top;                 // most of eight probabilities, 2^(8 - tree_lift)
  int rows, tiles, groups, nsplit;
  int by_length;             // pages: the requests by length (tree_by_length)
  FastDiv by_groups, by_nsplit, by_hkv, by_g;
};
hipError_t launch_tree_attn(const TreeAttnArgs& a, bool paged, hipStream_t s);

constexpr int kVerifyBlocks = 256;  // blocks of a row at most
struct VerifyCut {
  int size, count;  // entries of a block (a multiple of 1,024), blocks
};
inline VerifyCut verify_cut(int V) {
  const int size = ((V + kVerifyBlocks - 1) / kVerifyBlocks + 1023) / 1024 * 1024;
  return VerifyCut{size, (V + size - 1) / size};
}
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
  double* part;              // [R][kVerifyBlocks] masses
  struct VerifyState* state; // [R]
  int R, T, V, groups;       // workgroups per request
  VerifyCut cut;
};
// Where a request's walk ended: coefficient, rejected siblings, node, rows on the path.
struct VerifyState {
  double coef;
  unsigned long long rejected;
  int node, len;
};
constexpr int kVerifyGroups = 16;   // workgroups per request at most
// Workgroups per request: one (a single launch), or as many as the CUs allow with
// 32 KB of the last row, or rows, for each, where that is 128 KB and more. Measured
// at 64 requests: 64 KB a request 8.0 us with one and 8.3 with two, 256 KB 11.3 and
// with four 10.8, 1 MB 24.5 and 17.9.
inline int verify_groups(long long R, long long V, bool draft) {
  const long long bytes = V * (draft ? 8 : 4);
  int g = 1;
  if (bytes >= 128 << 10)
    while (2 * g <= kVerifyGroups && R * 2 * g <= 256 && bytes / (2 * g) >= 32 << 10) g *= 2;
  return g;
}
// (the same at every size: a caller may use one workspace for calls with and without draft probabilities)
inline size_t verify_ws_bytes(long long R) { return (size_t)R * (kVerifyBlocks * sizeof(double) + sizeof(VerifyState)); }
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
  FastDiv by_hkv;
};
hipError_t launch_append(const AppendArgs& a, hipStream_t s);

}  // namespace oasis
