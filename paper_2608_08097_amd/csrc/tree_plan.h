// How a tree-attention call is cut into workgroups: host code, no HIP.
//
// The rows of a KV head (G query heads x T tree rows) are cut into groups of at
// most kTreeTiles 16-row tiles; the cached tokens of a (request, KV head) pair,
// in units of 32, are cut into nsplit runs of equal length on the device, from
// the request's own length. With several splits each leaves a partial per row
// in the workspace and a second kernel merges them.
#pragma once

#include <cstddef>

namespace oasis {

constexpr int kTreeWaves = 4;     // waves per workgroup of the form for up to two row tiles
constexpr int kTreeTiles = 16;    // 16-row tiles per workgroup at most
constexpr int kTreeMaxTokens = 64;  // a row's ancestors are one 64-bit mask
constexpr int kTreeMaxRows = 4096;  // G * T
constexpr int kTreeMaxSplits = 256;

struct TreePlan {
  int rows, tiles, groups;  // tiles per group, groups of rows
  int units;                // of 32 tokens, at capacity
  int nsplit;
  std::size_t part_o_floats, bytes;
};

// `units`: 32-token units of the longest context the caller's tables hold.
inline TreePlan tree_plan(long long pairs, int G, int T, int units) {
  TreePlan p{};
  p.rows = G * T;
  const int tiles = (p.rows + 15) / 16;
  p.groups = (tiles + kTreeTiles - 1) / kTreeTiles;
  p.tiles = (tiles + p.groups - 1) / p.groups;
  p.units = units;
  const long long items = pairs * p.groups;
  // one workgroup per CU, and up to four where each still has 64 units
  long long want = items > 0 ? 256 / items : 1;
  if (want < 1) want = 1;
  long long more = items > 0 ? 1024 / items : 1;
  if (more > units / 64) more = units / 64;
  if (want < more) want = more;
  const long long most = (units + 2 * kTreeWaves - 1) / (2 * kTreeWaves);  // two units a wave at least
  if (want > most) want = most;
  if (want > kTreeMaxSplits) want = kTreeMaxSplits;
  p.nsplit = (int)(want < 1 ? 1 : want);
  if (p.nsplit > 1) {
    p.part_o_floats = (std::size_t)pairs * p.nsplit * p.rows * 128;
    p.bytes = (std::size_t)pairs * p.nsplit * p.rows * 130 * sizeof(float);
  }
  return p;
}

}  // namespace oasis
