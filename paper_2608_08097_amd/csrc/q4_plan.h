// How an attention call over the 4-bit cache is cut into workgroups: host code, no HIP.
//
// As tree_plan.h: the rows of a KV head in groups of 16-row tiles, the cached tokens of a
// (request, KV head) pair in units of 64, these in nsplit runs.
#pragma once

#include "tree_plan.h"

namespace oasis {

constexpr int kQ4Unit = 64;   // tokens
constexpr int kQ4Waves = 4;   // of a workgroup
constexpr int kQ4RegisterTiles = 2;  // 16-row tiles up to which a wave converts for itself
constexpr int kQ4Tiles = 8;   // 16-row tiles of a workgroup at most

inline TreePlan q4_plan(long long pairs, int G, int T, int units) {
  TreePlan p{};
  p.rows = G * T;
  const int tiles = (p.rows + 15) / 16;
  p.groups = (tiles + kQ4Tiles - 1) / kQ4Tiles;
  p.tiles = (tiles + p.groups - 1) / p.groups;
  p.units = units;
  const long long items = pairs * p.groups;
  const long long slots = p.tiles > 4 ? 256 : 512;
  long long most = (units + kQ4Waves - 1) / kQ4Waves;
  if (most > kTreeMaxSplits) most = kTreeMaxSplits;
  p.nsplit = 1;
  while (items > 0 && p.nsplit * 2 <= most && items * p.nsplit < slots) p.nsplit *= 2;
  if (p.nsplit > 1) {
    p.part_o_floats = (std::size_t)pairs * p.nsplit * p.rows * 128;
    p.bytes = (std::size_t)pairs * p.nsplit * p.rows * 130 * sizeof(float);
  }
  return p;
}

}  // namespace oasis
