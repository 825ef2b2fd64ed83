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

// Calls of more than four row tiles go two by two through the form for up to two all the
// same where the row groups together read at most so many units. Measured, us with the form
// for more rows and this one (8 heads, 128 rows: pairs x units): 8 x 8 17.9 and 14.8, 8 x 32
// 18.5 and 15.6, 8 x 125 23.6 and 20.4, 16 x 125 27.5 and 29.0; 256 rows: 8 x 32 19.8 and
// 18.0, 8 x 125 26.8 and 28.9. Not measured: hundreds of pairs with a few units each, of which
// the small form's workgroups are more than the CUs hold at once.
constexpr int kQ4SmallUnits = 4700;

// `units`: 64-token units of the longest context, or of the most different blocks that a
// selection can hold. `attended`: of the most tokens that a row attends, a block as often as
// the selection lists it; the rows' references lie as far above their scores as those need
// (tree_lift).
//
// As many splits as fill the CUs, two workgroups each (one with more than four row tiles),
// but the second one only with 16 units for each workgroup: a workgroup of a few units is
// nearly all start and end. Measured, splits and us (pairs, rows, units): 64, 20, 33: 1 23.4,
// 2 19.7, 4 16.7, 8 17.8; 8, 4, 31: 1 17.0, 2 14.2, 4 11.3, 8 9.7; 8, 20, 2,048: 8 120, 16
// 68, 32 45, 64 43, 128 58; 64, 20, 2,048: 4 239, 8 197, 12 217, 16 210; 128, 72, 65: 1 84,
// 2 55, 4 62; 16, 512, 1,024: 2 555, 4 291, 8 304. Counts are powers of two, and these pairs
// divide the places evenly: where they do not (72 pairs of 128 rows: 288 workgroups on 256),
// the last round is hardly filled, and another count might end sooner. Nor are ragged
// contexts looked at: a split is a share of its own request's tokens.
inline TreePlan q4_plan(long long pairs, int G, int T, int units, int attended) {
  TreePlan p{};
  p.rows = G * T;
  const int tiles = (p.rows + 15) / 16, twos = (tiles + 1) / 2;
  const bool small = tiles > 4 && pairs * units * twos <= kQ4SmallUnits;
  p.groups = small ? twos : (tiles + kQ4Tiles - 1) / kQ4Tiles;
  p.tiles = small ? kQ4RegisterTiles : (tiles + p.groups - 1) / p.groups;
  p.units = 2 * attended;  // of 32 tokens
  const long long items = pairs * p.groups;
  const long long slots = p.tiles > 4 ? 256 : 512;
  long long most = (units + kQ4Waves - 1) / kQ4Waves;
  if (most > kTreeMaxSplits) most = kTreeMaxSplits;
  p.nsplit = 1;
  while (items > 0 && p.nsplit * 2 <= most && items * p.nsplit < slots) {
    if (items * p.nsplit * 2 > 256 && units < 16 * p.nsplit * 2) break;
    p.nsplit *= 2;
  }
  if (p.nsplit > 1) {
    p.part_o_floats = (std::size_t)pairs * p.nsplit * p.rows * 128;
    p.bytes = (std::size_t)pairs * p.nsplit * p.rows * 130 * sizeof(float);
  }
  return p;
}
inline TreePlan q4_plan(long long pairs, int G, int T, int units) { return q4_plan(pairs, G, T, units, units); }

}  // namespace oasis
