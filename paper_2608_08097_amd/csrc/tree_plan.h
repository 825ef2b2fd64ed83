// How a tree-attention call is cut into workgroups: host code, no HIP.
//
// The rows of a KV head (G query heads x T tree rows) are cut into groups of at
// most kTreeTiles 16-row tiles; the cached tokens of a (request, KV head) pair,
// in units of 32, are cut into nsplit runs of equal length on the device, from
// the request's own length. With several splits each leaves a partial per row
// in the workspace and a second kernel merges them.
#pragma once

#include <cstddef>
#include <cstdint>

#ifdef __HIP__
#define OASIS_HD __host__ __device__
#else
#define OASIS_HD
#endif

namespace oasis {

// Quotients by a divisor that a launch fixes, of any n < 2^31: a multiplication and a
// shift, where a kernel's own division takes some 30 instructions in turn, and 150 in 64
// bits, ahead of its first load. With 2^shift the next power of two, mul / 2^32 is
// 2^shift / d - 1 rounded up.
struct FastDiv {
  uint32_t mul, shift;
  OASIS_HD uint32_t operator()(uint32_t n) const {
    return ((uint32_t)(((uint64_t)n * mul) >> 32) + n) >> shift;
  }
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t shift = 0;
  while ((1ull << shift) < d) ++shift;
  return FastDiv{(uint32_t)((((1ull << shift) - d) << 32) / d + 1), shift};
}

constexpr int kTreeWaves = 4;     // waves per workgroup of the form for up to two row tiles
constexpr int kTreeRegisterTiles = 2;  // 16-row tiles up to which K and V go straight into registers
constexpr int kTreeTiles = 8;     // 16-row tiles per workgroup at most
// More row tiles than kTreeRegisterTiles go two by two through that form all the same where
// its loads, each group's own, are at most 16 KB times this: its workgroups start and end
// faster. Measured over the working set, us with the form for more rows and this one: 64
// rows, 8 pairs of 129 units (2,064 loads) 16.1 and 13.5, 64 of 33 (4,224) 19.2 and 17.3, 16
// of 257 (8,224) 23.9 and 28.3; 128 rows, 8 of 129 (4,128) 20.1 and 15.3, 16 of 129 (8,256)
// 25.5 and 24.6, 32 of 129 (16,512) 29.3 and 33.7; 256 rows, 8 of 65 (4,160) 20.2 and 15.1,
// 16 of 65 (8,320) 22.4 and 23.4, 32 of 65 (16,640) 28.4 and 34.7. And only where the CUs
// hold them at once: 256 rows, 128 pairs of 2 (1,024 workgroups) 16.3 and 23.0.
constexpr int kTreeSmallUnits = 6000;
constexpr int kTreeMaxTokens = 64;  // a row's ancestors are one 64-bit mask
constexpr int kTreeMaxRows = 4096;  // G * T
constexpr int kTreeMaxSplits = 256;

struct TreePlan {
  int rows, tiles, groups;  // tiles per group, groups of rows
  int units;                // of 32 tokens, at capacity
  int nsplit;
  std::size_t part_o_floats, bytes;
};

// How far a row's reference lies above its scores, in powers of two, in a call of at most
// `units` units of cached tokens and two of the tree: the four lanes of a row each add
// eight probabilities of a unit, at most 2^(8 - lift) together, and the sums of all of
// them shall stay below 1/2. A lift of the most tokens that any call can have (38) would
// cost values below 2^-88 their last bits; this one costs them little more than dividing
// a probability by that many tokens does.
inline int tree_lift(int units) {
  int lift = 11;
  while ((1ll << (lift - 11)) < (long long)units + 2) ++lift;
  return lift;
}

inline long long tree_slots(const TreePlan& p) {  // workgroups that the CUs hold at once
  return p.tiles > kTreeRegisterTiles ? 256 : 512;
}

// `units`: 32-token units of the longest context the caller's tables hold; `ragged`:
// the contexts may be shorter than that.
//
// The split count is the one with the least estimated time, in tenths of a
// microsecond: rounds of workgroups over the CUs, times what one of them takes, and
// the merge of their partials. A workgroup takes its start and end and its units, at
// the latency of its waves' loads or of their products, or at its share of the
// bandwidth (16 KB a unit and KV head) where that is slower. Where contexts are ragged
// the longest workgroup ends the call, so the most splits within 3 % of the least are
// taken. Measured against neighbouring counts (pairs, rows, units: count and us): 64, 20,
// 4,096: 2 840, 3 708, 4 712, 5 864, 8 722; 64, 20, 65: 1 27.3, 2 22.3, 3 20.7, 4 21.2,
// 5 25.0; 16, 512, 2,048: 3 337, 4 296, 6 404; 192, 64, up to 1,024: 1 372, 2 276, 3 276,
// 4 269, 6 290; 128, 256, 129: 1 98, 2 116; 512, 28, 65: 1 81, 2 92; 8, 8, 129: 4 17.9,
// 8 12.7, 16 11.6, 24 12.0, 33 14.8; 1, 8, 1,001: 16 28.6, 32 21.1, 64 20.5, 128 27.6.
inline TreePlan tree_plan(long long pairs, int G, int T, int units, bool ragged) {
  TreePlan p{};
  p.rows = G * T;
  const int tiles = (p.rows + 15) / 16;
  const int twos = (tiles + 1) / 2;
  const bool small =
      tiles > kTreeRegisterTiles && pairs * twos <= 512 && pairs * units * twos <= kTreeSmallUnits;
  p.groups = small ? twos : (tiles + kTreeTiles - 1) / kTreeTiles;
  p.tiles = small ? kTreeRegisterTiles : (tiles + p.groups - 1) / p.groups;
  p.units = units;
  const long long items = pairs * p.groups;
  const bool rows_form = p.tiles > kTreeRegisterTiles;
  const long long slots = tree_slots(p);
  long long most = (units + kTreeWaves - 1) / kTreeWaves;  // a unit a wave
  if (most > kTreeMaxSplits) most = kTreeMaxSplits;
  if (items > 0 && most > 4 * slots / items) most = 4 * slots / items;
  auto estimate = [&](long long n) {
    const long long u = (units + n - 1) / n;
    const long long rounds = (items * n + slots - 1) / slots;
    const long long at_once = items * n < slots ? items * n : slots;
    const long long share = u * 63 * at_once / (2560 * p.groups);  // 6.7 TB/s over 256 CUs
    long long body = rows_form ? u * 6 : (u + kTreeWaves - 1) / kTreeWaves * 16;
    if (body < share) body = share;
    // its launch, a wait for every few splits, the partials both ways at 3 TB/s
    const long long merge = n > 1 ? 30 + n * 6 / 5 + pairs * n * p.rows * 1040 / 300000 : 0;
    const long long shared = !rows_form && items * n > 256 ? 25 : 0;  // two workgroups on a CU
    return rounds * (body + (rows_form ? 110 : 70)) + shared + merge;
  };
  long long best = estimate(1);
  p.nsplit = 1;
  for (long long n = 2; n <= most; ++n) {
    const long long t = estimate(n);
    if (t < best) {
      best = t;
      p.nsplit = (int)n;
    }
  }
  if (ragged)
    for (long long n = most; n > p.nsplit; --n)
      if (estimate(n) * 100 <= best * 103) p.nsplit = (int)n;
  if (p.nsplit > 1) {
    p.part_o_floats = (std::size_t)pairs * p.nsplit * p.rows * 128;
    p.bytes = (std::size_t)pairs * p.nsplit * p.rows * 130 * sizeof(float);
  }
  return p;
}

// Workgroups of the pass over the rows of wild queries, kTreeWildRows rows each at a time.
// Calls may have 2^28 rows, of which a workgroup for every eight would be 2^33 threads: a
// launch has fewer than 2^32.
constexpr int kTreeWildRows = 8;
inline unsigned tree_wild_groups(long long rows) {
  const long long groups = (rows + kTreeWildRows - 1) / kTreeWildRows;
  return (unsigned)(groups < 1 << 14 ? groups : 1 << 14);
}

// Whether a paged call takes its requests by length, the longest first: a call of more
// workgroups than the CUs hold at once ends with the last ones it starts, so these had
// better be short. Up to 64 requests, one a lane. Measured, 64 rows, 24 requests of 1 to
// 32,768 tokens each, six draws: 311 us in order, 278 by length.
inline bool tree_by_length(const TreePlan& p, long long R, long long Hkv) {
  return R > 1 && R <= 64 && R * Hkv * p.nsplit * p.groups > tree_slots(p);
}

}  // namespace oasis
