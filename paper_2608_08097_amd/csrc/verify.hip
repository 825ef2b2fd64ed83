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
// The acceptance tests need scalars only, so every workgroup walks by itself, a
// child per lane, and then adds up its chunk of the last node's w; a second launch
// picks the chunk and the token in it. Both passes add a chunk in the same order.
#include "drafts_internal.h"

namespace oasis {
namespace {

constexpr int kVT = 256;                       // threads
constexpr int kVPer = kVerifyChunk / kVT;      // consecutive entries per thread

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));  // rows of any length: 4-byte alignment

__device__ __forceinline__ double positive(float p) { return p > 0.f ? (double)p : 0.0; }  // NaN counts as 0

__device__ __forceinline__ double readlane_f64(double x, int l) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)b, l), hi = __builtin_amdgcn_readlane((uint32_t)(b >> 32), l);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Sum over the workgroup, the same value in every thread.
__device__ __forceinline__ double block_sum(double x, double* s_w) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s_w[threadIdx.x >> 6] = x;
  __syncthreads();
  double t = 0.0;
  for (int w = 0; w < kVT / 64; ++w) t += s_w[w];
  return t;
}

struct Residual {
  const float* p;
  const float* q;             // NULL: drafts without probabilities
  double coef;
  const int32_t* tokens;      // of the tree
  unsigned long long rejected;  // children whose tokens are taken out (q NULL)
  int V;

  __device__ __forceinline__ double at(int v, float pv, float qv) const {
    double w = positive(pv);
    if (q) {
      w = w - coef * positive(qv);
      return w > 0.0 ? w : 0.0;
    }
    return w;
  }
  // w of the thread's kVPer entries from v0 on, their sum in order
  __device__ __forceinline__ double load(int v0, double (&w)[kVPer]) const {
    if (v0 + kVPer <= V) {
      f32x4u pv[kVPer / 4], qv[kVPer / 4];
#pragma unroll
      for (int j = 0; j < kVPer / 4; ++j) {
        pv[j] = *reinterpret_cast<const f32x4u*>(p + v0 + 4 * j);
        qv[j] = q ? *reinterpret_cast<const f32x4u*>(q + v0 + 4 * j) : f32x4u{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int j = 0; j < kVPer; ++j) w[j] = at(v0 + j, pv[j >> 2][j & 3], qv[j >> 2][j & 3]);
    } else {
#pragma unroll
      for (int j = 0; j < kVPer; ++j)
        w[j] = v0 + j < V ? at(v0 + j, p[v0 + j], q ? q[v0 + j] : 0.f) : 0.0;
    }
    for (unsigned long long m = rejected; m; m &= m - 1) {
      const int x = tokens[__builtin_ctzll(m)] - v0;
#pragma unroll
      for (int j = 0; j < kVPer; ++j) w[j] = x == j ? 0.0 : w[j];
    }
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < kVPer; ++j) s += w[j];
    return s;
  }
  // mass of the whole row, in every thread
  __device__ __forceinline__ double mass(double* s_w) const {
    double s = 0.0, w[kVPer];
    for (int v0 = threadIdx.x * kVPer; v0 < V; v0 += kVerifyChunk) s += load(v0, w);
    return block_sum(s, s_w);
  }
};

__device__ __forceinline__ const float* row_of(const float* t, long long stride, int r, int T, int n) {
  return t ? t + ((long long)r * T + n) * stride : nullptr;
}

__global__ __launch_bounds__(kVT) void verify_walk_kernel(VerifyArgs a) {
  __shared__ double s_w[kVT / 64];
  const int r = blockIdx.y;
  const int chunk = blockIdx.x;
  const int lane = threadIdx.x & 63;
  const int32_t* tokens = a.tokens + (long long)r * a.T;
  int len = a.tree_len ? a.tree_len[r] : a.T;
  len = len < 0 ? 0 : (len > a.T ? a.T : len);
  VerifyState* state = reinterpret_cast<VerifyState*>(a.part + (long long)a.R * a.chunks) + r;

  // lane c: child c's parent, token, random number, and both probabilities at its parent
  int par = -1, x = -1;
  float u = 0.f;
  double px = 0.0, qx = a.draft ? 0.0 : 1.0;
  if (lane > 0 && lane < len) {
    par = a.parent ? a.parent[(long long)r * a.T + lane] : lane - 1;
    x = tokens[lane];
    u = a.accept_u[(long long)r * a.T + lane];
    if (par < 0 || par >= lane || x < 0 || x >= a.V) {
      par = -1;  // not a child of any row, or no token: passed over
    } else {
      px = positive(row_of(a.target, a.target_stride, r, a.T, par)[x]);
      if (a.draft) qx = positive(row_of(a.draft, a.draft_stride, r, a.T, par)[x]);
    }
  }

  // every wave of every workgroup of the request walks the same way
  int node = 0, count = len > 0 ? 1 : 0;
  unsigned long long on_path = len > 0 ? 1 : 0, rejected = 0;
  double coef = 0.0, mass = 1.0;
  bool moved = len > 0;
  while (moved) {
    moved = false;
    coef = 0.0;
    mass = 1.0;
    rejected = 0;
    for (unsigned long long kids = __builtin_amdgcn_ballot_w64(par == node); kids; kids &= kids - 1) {
      const int c = __builtin_ctzll(kids);
      const int xc = __builtin_amdgcn_readlane(x, c);
      const double uc = (double)__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, u), c));
      const double pc = readlane_f64(px, c), qc = readlane_f64(qx, c);
      double w;
      if (a.draft) {
        w = pc - coef * qc;
        w = w > 0.0 ? w : 0.0;
      } else {
        w = __builtin_amdgcn_ballot_w64((rejected >> lane & 1) && x == xc) ? 0.0 : pc;
      }
      if (uc * qc * mass < w) {
        node = c;
        on_path |= 1ull << c;
        ++count;
        moved = true;
        break;
      }
      if (a.draft) {
        coef += mass;
        if (kids & (kids - 1)) {  // a sibling is left, which needs the mass
          const Residual res{row_of(a.target, a.target_stride, r, a.T, node),
                             row_of(a.draft, a.draft_stride, r, a.T, node), coef, tokens, 0, a.V};
          mass = res.mass(s_w);
        }
      } else {
        rejected |= 1ull << c;
        mass -= w;
        mass = mass > 0.0 ? mass : 0.0;
      }
    }
  }

  const Residual res{row_of(a.target, a.target_stride, r, a.T, node), row_of(a.draft, a.draft_stride, r, a.T, node),
                     coef, tokens, rejected, a.V};
  double w[kVPer];
  const int v0 = chunk * kVerifyChunk + threadIdx.x * kVPer;
  const double sum = block_sum(len > 0 && v0 < a.V ? res.load(v0, w) : 0.0, s_w);
  if (threadIdx.x == 0) a.part[(long long)r * a.chunks + chunk] = sum;
  if (chunk == 0 && threadIdx.x < 64) {
    // row c of the path is the path's entry number (rows of the path below c); the
    // token that leads to it is emitted one place earlier
    const int at = __popcll(on_path & ((1ull << lane) - 1));
    int32_t* path = a.path + (long long)r * a.T;
    int32_t* out = a.out_tokens + (long long)r * a.T;
    if (on_path >> lane & 1) {
      path[at] = lane;
      if (lane > 0) out[at - 1] = x;
    }
    if (lane < a.T) {
      if (lane >= count) path[lane] = -1;
      if (lane >= count - 1) out[lane] = -1;
    }
    if (lane == 0) {
      a.path_len[r] = count;
      *state = VerifyState{coef, rejected, node, count};
    }
  }
}

// First thread (in order) whose `hit` is set: its index, kVT if none.
__device__ __forceinline__ int first_hit(bool hit, int* s_first) {
  if (threadIdx.x == 0) *s_first = kVT;
  __syncthreads();
  if (hit) atomicMin(s_first, (int)threadIdx.x);
  __syncthreads();
  return *s_first;
}

__global__ __launch_bounds__(kVT) void verify_pick_kernel(VerifyArgs a) {
  __shared__ double s_sum[kVT + 1];
  __shared__ double s_w[kVT / 64];
  __shared__ int s_first, s_last;
  const int r = blockIdx.x;
  const VerifyState st = reinterpret_cast<const VerifyState*>(a.part + (long long)a.R * a.chunks)[r];
  if (st.len < 1) return;
  const int32_t* tokens = a.tokens + (long long)r * a.T;
  Residual res{row_of(a.target, a.target_stride, r, a.T, st.node), row_of(a.draft, a.draft_stride, r, a.T, st.node),
               st.coef, tokens, st.rejected, a.V};
  const double* part = a.part + (long long)r * a.chunks;
  // whole mass, then the first chunk whose running mass passes the border
  auto scan = [&](auto&& chunk_mass, double border, double& before) {
    double run = 0.0;
    int pick = -1, last = -1;
    before = 0.0;
    for (int s = 0; s < a.chunks; ++s) {
      const double m = chunk_mass(s);
      if (m > 0.0) {
        last = s;
        if (pick < 0 && run + m > border) {
          pick = s;
          before = run;
        }
      }
      run += m;
    }
    return pick >= 0 ? pick : last;
  };
  double total = 0.0;
  for (int s = 0; s < a.chunks; ++s) total += part[s];
  const double u = (double)a.sample_u[r];
  double before;
  int chunk;
  double w[kVPer];
  if (total > 0.0) {
    chunk = scan([&](int s) { return part[s]; }, u * total, before);
  } else {
    // a residual without mass: the target's row itself
    res.q = nullptr;
    res.rejected = 0;
    total = res.mass(s_w);
    double run = 0.0;
    chunk = -1;
    before = 0.0;
    for (int s = 0; s < a.chunks; ++s) {
      const int v0 = s * kVerifyChunk + threadIdx.x * kVPer;
      const double m = block_sum(v0 < a.V ? res.load(v0, w) : 0.0, s_w);
      if (m > 0.0) {
        chunk = s;
        before = run;
        if (run + m > u * total) break;
      }
      run += m;
    }
  }
  int token = -1;
  if (chunk >= 0) {
    const int v0 = chunk * kVerifyChunk + threadIdx.x * kVPer;
    const double mine = v0 < a.V ? res.load(v0, w) : 0.0;
    if (v0 >= a.V) {
#pragma unroll
      for (int j = 0; j < kVPer; ++j) w[j] = 0.0;
    }
    // running sums before each thread
    s_sum[threadIdx.x + 1] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
      double run = 0.0;
      s_sum[0] = 0.0;
      for (int t = 0; t < kVT; ++t) {
        run += s_sum[t + 1];
        s_sum[t + 1] = run;
      }
      s_last = -1;
    }
    __syncthreads();
    const double border = u * total - before;
    const int hit = first_hit(mine > 0.0 && s_sum[threadIdx.x + 1] > border, &s_first);
    if (mine > 0.0) atomicMax(&s_last, (int)threadIdx.x);
    __syncthreads();
    // the border may fall on the chunk's end by a rounding: its last entry then
    const int who = hit < kVT ? hit : s_last;
    if ((int)threadIdx.x == who) {
      double run = s_sum[threadIdx.x];
      int v = -1;
      bool found = false;
#pragma unroll
      for (int j = 0; j < kVPer; ++j) {
        run += w[j];
        if (w[j] > 0.0 && !found) {
          v = v0 + j;
          found = hit < kVT && run > border;
        }
      }
      a.out_tokens[(long long)r * a.T + st.len - 1] = v;
    }
    return;
  }
  if (threadIdx.x == 0) a.out_tokens[(long long)r * a.T + st.len - 1] = token;
}

}  // namespace

hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(verify_walk_kernel, dim3((unsigned)a.chunks, (unsigned)a.R), dim3(kVT), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(verify_pick_kernel, dim3((unsigned)a.R), dim3(kVT), 0, s, a);
  return hipGetLastError();
}

}  // namespace oasis
