// Verification of drafted tokens against the target's probabilities, from given
// random numbers.
//
// The walk starts at row 0. At node n with target row p and draft row q it takes
// n's children in ascending order; what the earlier ones leave is the residual
//   w = max(p - C q, 0),  mass Z      (C = 0, Z = 1 before the first)
// and child c with token x is accepted when u_c q(x) Z < w(x); a rejection adds Z
// to C and makes Z the mass of the new w. (Taking max(w - Z q, 0) child by child
// gives the same w, since what is once at 0 stays there.) Without draft
// probabilities q is 1 at x: w is p with the rejected tokens taken out, and Z loses
// their p. Where no child is accepted the next token is the first with
// cumsum(w) > u sum(w); a residual without mass gives way to p.
//
// All of it in 64 bits: a sum over a vocabulary in 32 would move the borders that
// the random numbers are held against by 1e-5 and more.
//
// The acceptance tests need scalars only, read at once, a child per lane; every
// wave walks by itself. What costs is reading rows of the vocabulary: one for the
// next token, and with draft probabilities one for each rejected child that has a
// sibling behind it. A CU reads some 120 GB/s of them, near the 64 bytes a cycle that
// it can load (finer pieces, for an even share of the waves: no gain), so a long row is
// shared by several workgroups and a second launch (verify_groups). Measured, one
// request, chain, 131,072 entries with draft probabilities (1 MB): 15.6 us with one
// workgroup, 8.3 with eight; 32,000 entries 8.9 and 7.0; 128 requests of 131,072 36 and,
// with two, 31; 48 requests, 16 rows, 50,261 entries 24.8, the passes of rejected
// siblings one after the other.
#include "drafts_internal.h"

namespace oasis {
namespace {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));  // rows of any length: 4-byte alignment

// A probability as it counts: NaN and negative ones are 0 (the median of three takes
// the smallest where one is NaN, in one instruction, which a maximum needs two for).
__device__ __forceinline__ double positive(float p) { return (double)__builtin_amdgcn_fmed3f(p, 0.f, __builtin_inff()); }

__device__ __forceinline__ double readlane_f64(double x, int l) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)b, l), hi = __builtin_amdgcn_readlane((uint32_t)(b >> 32), l);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// x of another lane of the wave over the DPP network (0 where there is none).
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_f64(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xF, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Inclusive prefix sums over the wave (steps as wave_incl_sum).
__device__ __forceinline__ double wave_prefix(double x) {
  x += dpp_f64<0x111, 0xF>(x);
  x += dpp_f64<0x112, 0xF>(x);
  x += dpp_f64<0x114, 0xF>(x);
  x += dpp_f64<0x118, 0xF>(x);
  x += dpp_f64<0x142, 0xA>(x);
  x += dpp_f64<0x143, 0xC>(x);
  return x;
}
__device__ __forceinline__ double wave_sum(double x) { return readlane_f64(wave_prefix(x), 63); }

// Where a request's walk stands.
struct Walk {
  int node, len;                        // row, rows on the path
  unsigned long long on_path, rejected;  // rejected: children of `node` (certain drafts)
  double coef;                          // C
};

__device__ __forceinline__ const float* row_of(const float* t, long long stride, int r, int T, int n) {
  return t ? t + ((long long)r * T + n) * stride : nullptr;
}

// One row's residual.
struct Residual {
  const float* p;
  const float* q;  // NULL: certain drafts
  double coef;
  unsigned long long rejected;
  int tokens;      // lane c: row c's token
  int V;
  VerifyCut cut;

  template <bool DRAFT>
  __device__ __forceinline__ double at(float pv, float qv) const {
    if constexpr (DRAFT) {
      return fmax((double)pv - coef * positive(qv), 0.0);  // a NaN or negative pv gives 0
    } else {
      return positive(pv);
    }
  }
  // w of N consecutive entries from v0 on (0 past the vocabulary)
  template <bool DRAFT, int N>
  __device__ __forceinline__ void load(int v0, double (&w)[N]) const {
    static_assert(N % 4 == 0, "quads");
    if (v0 + N <= V) {
      f32x4u pv[N / 4], qv[N / 4];
#pragma unroll
      for (int j = 0; j < N / 4; ++j) {
        pv[j] = *reinterpret_cast<const f32x4u*>(p + v0 + 4 * j);
        qv[j] = DRAFT ? *reinterpret_cast<const f32x4u*>(q + v0 + 4 * j) : f32x4u{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = at<DRAFT>(pv[j >> 2][j & 3], qv[j >> 2][j & 3]);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = v0 + j < V ? at<DRAFT>(p[v0 + j], DRAFT ? q[v0 + j] : 0.f) : 0.0;
    }
  }
  // takes the rejected tokens out of the entries [v0, v0 + N) of this lane; `first`
  // and `count` bound the whole wave's entries
  template <int N>
  __device__ __forceinline__ void take_out(int first, int count, int v0, double (&w)[N]) const {
    for (unsigned long long m = rejected; m; m &= m - 1) {
      const int x = __builtin_amdgcn_readlane(tokens, __builtin_ctzll(m));
      if ((unsigned)(x - first) >= (unsigned)count) continue;
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = x - v0 == j ? 0.0 : w[j];
    }
  }
  // The 1,024 entries from v on: 16-byte loads of 4 consecutive ones a lane; where the
  // row ends among them (0 past its end), one entry a lane and load.
  template <bool DRAFT>
  __device__ __forceinline__ void fetch(int v, int lane, f32x4u (&pv)[4], f32x4u (&qv)[4]) const {
    if (v + 1024 <= V) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        pv[j] = *reinterpret_cast<const f32x4u*>(p + v + 256 * j + 4 * lane);
        if constexpr (DRAFT) qv[j] = *reinterpret_cast<const f32x4u*>(q + v + 256 * j + 4 * lane);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int at = v + 64 * j + lane;
        pv[j >> 2][j & 3] = at < V ? p[at] : 0.f;
        if constexpr (DRAFT) qv[j >> 2][j & 3] = at < V ? q[at] : 0.f;
      }
    }
  }
  // This lane's part of the sum of those entries.
  template <bool DRAFT>
  __device__ __forceinline__ double lane_sum(int v, int lane, const f32x4u (&pv)[4], const f32x4u (&qv)[4]) const {
    double s = 0.0;
    if constexpr (DRAFT) {
#pragma unroll
      for (int j = 0; j < 16; ++j) s += at<true>(pv[j >> 2][j & 3], qv[j >> 2][j & 3]);
    } else {
      double w[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) w[j] = at<false>(pv[j >> 2][j & 3], 0.f);
      for (unsigned long long m = rejected; m; m &= m - 1) {
        const int x = __builtin_amdgcn_readlane(tokens, __builtin_ctzll(m)) - v;
        if ((unsigned)x >= 1024u) continue;
        const bool ends = v + 1024 > V;  // the order of fetch()
        const int k = ends ? x >> 6 : (x >> 8) * 4 + (x & 3), l = ends ? x & 63 : x >> 2 & 63;
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] = k == j && l == lane ? 0.0 : w[j];
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) s += w[j];
    }
    return s;
  }
};

// What lane c knows of child c: its parent, its token, its random number and both
// probabilities at its parent.
struct Child {
  int par = -1, x = -1;
  float u = 0.f;
  double px = 0.0, qx = 0.0;
};
__device__ __forceinline__ Child load_child(const VerifyArgs& a, int r, int len, int lane) {
  Child c;
  if (!a.draft) c.qx = 1.0;
  if (lane > 0 && lane < a.T) {  // read beside the length
    c.par = a.parent ? a.parent[(long long)r * a.T + lane] : lane - 1;
    c.x = a.tokens[(long long)r * a.T + lane];
    c.u = a.accept_u[(long long)r * a.T + lane];
  }
  if (lane >= len || c.par < 0 || c.par >= lane || c.x < 0 || c.x >= a.V) {
    c.par = -1;  // not a child of any row, or no token: passed over
  } else {
    c.px = positive(row_of(a.target, a.target_stride, r, a.T, c.par)[c.x]);
    if (a.draft) c.qx = positive(row_of(a.draft, a.draft_stride, r, a.T, c.par)[c.x]);
  }
  return c;
}

// The walk, alike in every wave. mass(node, C) is asked for where a sibling is left
// behind a rejected child of a drafter's row.
template <typename Mass>
__device__ __forceinline__ Walk walk(const VerifyArgs& a, const Child& ch, int len, int lane, Mass&& mass) {
  Walk w{0, len > 0 ? 1 : 0, len > 0 ? 1ull : 0ull, 0, 0.0};
  bool moved = len > 0;
  while (moved) {
    moved = false;
    w.coef = 0.0;
    w.rejected = 0;
    double z = 1.0;
    for (unsigned long long kids = __builtin_amdgcn_ballot_w64(ch.par == w.node); kids; kids &= kids - 1) {
      const int c = __builtin_ctzll(kids);
      const int xc = __builtin_amdgcn_readlane(ch.x, c);
      const double uc = (double)__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, ch.u), c));
      const double pc = readlane_f64(ch.px, c), qc = readlane_f64(ch.qx, c);
      double left;
      if (a.draft) {
        left = pc - w.coef * qc;
        left = left > 0.0 ? left : 0.0;
      } else {
        left = __builtin_amdgcn_ballot_w64((w.rejected >> lane & 1) && ch.x == xc) ? 0.0 : pc;
      }
      if (uc * qc * z < left) {
        w.node = c;
        w.on_path |= 1ull << c;
        ++w.len;
        moved = true;
        break;
      }
      if (a.draft) {
        w.coef += z;
        if (kids & (kids - 1)) z = mass(w.node, w.coef);
      } else {
        w.rejected |= 1ull << c;
        z -= left;
        z = z > 0.0 ? z : 0.0;
      }
    }
  }
  return w;
}

// The path and the emitted tokens but for the last, by one wave.
__device__ __forceinline__ void write_path(const VerifyArgs& a, int r, int lane, const Walk& w, int x) {
  // row c of the path is the path's entry number (rows of the path below c); the
  // token that leads to it is emitted one place earlier
  const int at = __popcll(w.on_path & ((1ull << lane) - 1));
  int32_t* path = a.path + (long long)r * a.T;
  int32_t* out = a.out_tokens + (long long)r * a.T;
  if (w.on_path >> lane & 1) {
    path[at] = lane;
    if (lane > 0) out[at - 1] = x;
  }
  if (lane < a.T) {
    if (lane >= w.len) path[lane] = -1;
    if (lane >= w.len) out[lane] = -1;
  }
  if (lane == 0) a.path_len[r] = w.len;
}

__device__ __forceinline__ int verify_len(const VerifyArgs& a, int r) {
  const int len = a.tree_len ? a.tree_len[r] : a.T;
  return len < 0 ? 0 : (len > a.T ? a.T : len);
}

// ---- sums over a row -------------------------------------------------------------------
//
// A row is cut into at most kVerifyBlocks blocks, which the waves of the workgroups
// that work on it take in turn; one wave then finds the block in which the border
// falls and reads it again.
constexpr int kVT = 1024;
constexpr int kWaves = kVT / 64;

// Masses of the blocks that this wave takes (number `wave` of `waves`), into
// out[block]. Two buffers of 1,024 entries in turn: one is on its way while the other
// is added up.
template <bool DRAFT>
__device__ __forceinline__ void block_masses(const Residual& res, int wave, int waves, int lane, double* out) {
  const VerifyCut bl = res.cut;
  f32x4u p0[4], q0[4], p1[4], q1[4];
  double s = 0.0;
  int b = wave, v = b * bl.size;  // v: the entries to fetch next, of block b
  if (b >= bl.count) return;
  auto step = [&]() __attribute__((always_inline)) {  // moves on (v, b) by 1,024 entries; whether there are more
    v += 1024;
    if (v >= min((b + 1) * bl.size, res.V)) {
      b += waves;
      v = b * bl.size;
    }
    return b < bl.count;
  };
  auto add = [&](int at, int block, const f32x4u (&p)[4], const f32x4u (&q)[4]) __attribute__((always_inline)) {
    s += res.lane_sum<DRAFT>(at, lane, p, q);
    if (b != block) {  // its last entries
      const double m = wave_sum(s);
      if (lane == 0) out[block] = m;
      s = 0.0;
    }
  };
  int v0 = v, v1, b0 = b, b1;
  res.fetch<DRAFT>(v0, lane, p0, q0);
  for (;;) {
    const bool more1 = step();
    v1 = v;
    b1 = b;
    if (more1) res.fetch<DRAFT>(v1, lane, p1, q1);
    add(v0, b0, p0, q0);
    if (!more1) return;
    const bool more0 = step();
    v0 = v;
    b0 = b;
    if (more0) res.fetch<DRAFT>(v0, lane, p0, q0);
    add(v1, b1, p1, q1);
    if (!more0) return;
  }
}

struct VerifyShared {
  double mass[kVerifyBlocks];
};

// The row's masses by one workgroup, into sh.mass.
template <bool DRAFT>
__device__ __forceinline__ void row_masses(const Residual& res, VerifyShared& sh) {
  __syncthreads();  // sh is free again
  block_masses<DRAFT>(res, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kWaves, threadIdx.x & 63, sh.mass);
  __syncthreads();
}

// The row's mass and the place in it where its share u is reached: the block (the
// last one of any mass where rounding leaves none, -1 where there is none) and the
// sum ahead of it. Alike in every wave, four blocks a lane.
struct BlockPick {
  double total, ahead;
  int block;
};
__device__ __forceinline__ BlockPick pick_block(const double* masses, int n, double u, int lane) {
  double m[4], mine = 0.0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m[j] = 4 * lane + j < n ? masses[4 * lane + j] : 0.0;
    mine += m[j];
  }
  const double run = wave_prefix(mine);
  const double total = readlane_f64(run, 63), border = u * total;
  const uint64_t hits = __builtin_amdgcn_ballot_w64(mine > 0.0 && run > border);
  const uint64_t some = __builtin_amdgcn_ballot_w64(mine > 0.0);
  if (!some) return BlockPick{total, 0.0, -1};
  const int who = hits ? __builtin_ctzll(hits) : 63 - __builtin_clzll(some);
  double at = run - mine, ahead = at;
  int pick = -1;
  bool done = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (m[j] > 0.0 && !done) {
      pick = 4 * lane + j;
      ahead = at;
      done = hits && at + m[j] > border;
    }
    at += m[j];
  }
  return BlockPick{total, readlane_f64(ahead, who), __builtin_amdgcn_readlane(pick, who)};
}
__device__ __forceinline__ double total_of(const double* masses, int n, int lane) {
  double mine = 0.0;
#pragma unroll
  for (int j = 0; j < 4; ++j) mine += 4 * lane + j < n ? masses[4 * lane + j] : 0.0;
  return wave_sum(mine);
}

// The token within a block at which the running sum passes its border, by one wave:
// 1,024 entries at a time, 16 consecutive ones a lane. Where rounding leaves none, the
// block's last one of any mass.
template <bool DRAFT>
__device__ __forceinline__ int pick_token(const Residual& res, const BlockPick& p, double u, int lane) {
  const VerifyCut bl = res.cut;
  const int end = min((p.block + 1) * bl.size, res.V);
  const double border = u * p.total;
  double ahead = p.ahead;
  int last = -1;
  for (int first = p.block * bl.size; first < end; first += 1024) {
    double w[16];
    const int v0 = first + 16 * lane;
    res.load<DRAFT, 16>(v0, w);
    if constexpr (!DRAFT) res.take_out<16>(first, 1024, v0, w);
    double mine = 0.0;
#pragma unroll
    for (int j = 0; j < 16; ++j) mine += w[j];
    const double run = wave_prefix(mine);
    const uint64_t hits = __builtin_amdgcn_ballot_w64(mine > 0.0 && ahead + run > border);
    const uint64_t some = __builtin_amdgcn_ballot_w64(mine > 0.0);
    if (some) {
      const int who = hits ? __builtin_ctzll(hits) : 63 - __builtin_clzll(some);
      double at = ahead + (run - mine);
      int token = -1;
      bool done = false;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        at += w[j];
        if (w[j] > 0.0 && !done) {
          token = v0 + j;
          done = hits && at > border;
        }
      }
      last = __builtin_amdgcn_readlane(token, who);
      if (hits) break;
    }
    ahead += readlane_f64(run, 63);
  }
  return last;
}

__device__ __forceinline__ Residual residual_of(const VerifyArgs& a, int r, const Child& ch, int node, double coef,
                                                unsigned long long rejected) {
  return Residual{row_of(a.target, a.target_stride, r, a.T, node), row_of(a.draft, a.draft_stride, r, a.T, node), coef,
                  rejected, ch.x, a.V, a.cut};
}

// The next token, from the block of the last row that it is in; by the workgroup (the
// first wave's is the one that counts).
template <bool DRAFT>
__device__ __forceinline__ void write_next(const VerifyArgs& a, int r, int len, Residual res, BlockPick p, double u,
                                           VerifyShared& sh) {
  const int lane = threadIdx.x & 63;
  int token = -1;
  if (p.block >= 0) {
    if (threadIdx.x >= 64) return;
    token = pick_token<DRAFT>(res, p, u, lane);
  } else {  // a residual without mass: the target's row itself
    res.rejected = 0;
    row_masses<false>(res, sh);
    p = pick_block(sh.mass, a.cut.count, u, lane);
    if (p.block >= 0) token = pick_token<false>(res, p, u, lane);
  }
  if (threadIdx.x == 0) a.out_tokens[(long long)r * a.T + len - 1] = token;
}

// The mass that the walk asks for, by the workgroup.
template <bool DRAFT>
__device__ __forceinline__ double walk_mass(const Residual& res, VerifyShared& sh) {
  row_masses<DRAFT>(res, sh);
  return total_of(sh.mass, res.cut.count, threadIdx.x & 63);
}

// One workgroup for all of a request.
template <bool DRAFT>
__global__ __launch_bounds__(kVT) void verify_kernel(VerifyArgs a) {
  __shared__ VerifyShared sh;
  const int r = blockIdx.x;
  const int lane = threadIdx.x & 63;
  const int len = verify_len(a, r);
  const Child ch = load_child(a, r, len, lane);
  const Walk w = walk(a, ch, len, lane,
                      [&](int node, double coef) { return walk_mass<DRAFT>(residual_of(a, r, ch, node, coef, 0), sh); });
  if (threadIdx.x < 64) write_path(a, r, lane, w, ch.x);
  if (len < 1) return;
  const Residual res = residual_of(a, r, ch, w.node, w.coef, w.rejected);
  const double u = (double)a.sample_u[r];
  row_masses<DRAFT>(res, sh);
  write_next<DRAFT>(a, r, w.len, res, pick_block(sh.mass, a.cut.count, u, lane), u, sh);
}

// Several workgroups for a request: each walks by itself (over whole rows where a
// mass is asked for) and takes its blocks of the last row; a second launch picks.
template <bool DRAFT>
__global__ __launch_bounds__(kVT) void verify_blocks_kernel(VerifyArgs a) {
  __shared__ VerifyShared sh;
  const int r = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int len = verify_len(a, r);
  const Child ch = load_child(a, r, len, lane);
  const Walk w = walk(a, ch, len, lane,
                      [&](int node, double coef) { return walk_mass<DRAFT>(residual_of(a, r, ch, node, coef, 0), sh); });
  if (blockIdx.x == 0 && threadIdx.x < 64) {
    write_path(a, r, lane, w, ch.x);
    if (lane == 0) a.state[r] = VerifyState{w.coef, w.rejected, w.node, w.len};
  }
  if (len < 1) return;
  block_masses<DRAFT>(residual_of(a, r, ch, w.node, w.coef, w.rejected), wave * a.groups + blockIdx.x, kWaves * a.groups,
                      lane, a.part + (long long)r * kVerifyBlocks);
}

template <bool DRAFT>
__global__ __launch_bounds__(kVT) void verify_pick_kernel(VerifyArgs a) {
  __shared__ VerifyShared sh;
  const int r = blockIdx.x;
  const int lane = threadIdx.x & 63;
  // all that is read here at once; the masses of a request without a row are not defined
  const VerifyState st = a.state[r];
  const double u = (double)a.sample_u[r];
  Child ch;
  ch.x = lane < a.T ? a.tokens[(long long)r * a.T + lane] : -1;
  const BlockPick p = pick_block(a.part + (long long)r * kVerifyBlocks, a.cut.count, u, lane);
  if (st.len < 1) return;
  write_next<DRAFT>(a, r, st.len, residual_of(a, r, ch, st.node, st.coef, st.rejected), p, u, sh);
}

template <bool DRAFT>
void launch(const VerifyArgs& a, hipStream_t s) {
  if (a.groups == 1) {
    hipLaunchKernelGGL((verify_kernel<DRAFT>), dim3((unsigned)a.R), dim3(kVT), 0, s, a);
    return;
  }
  hipLaunchKernelGGL((verify_blocks_kernel<DRAFT>), dim3((unsigned)a.groups, (unsigned)a.R), dim3(kVT), 0, s, a);
  hipLaunchKernelGGL((verify_pick_kernel<DRAFT>), dim3((unsigned)a.R), dim3(kVT), 0, s, a);
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
  a.draft ? launch<true>(a, s) : launch<false>(a, s);
  return hipGetLastError();
}

}  // namespace oasis
