// Reductions over a distribution, shared by the kernels that read vocabularies: the running
// top-2, log-sum-exp and non-finite flag of a thread, and their merges over a wave and a
// workgroup of four waves.
#pragma once

#include "common.hpp"
#include "kernels.hpp"

namespace spp {

struct Acc {  // running reductions
  Top2 t;
  float m, s;
  uint32_t nonfinite;
};

__device__ __forceinline__ void acc_init(Acc& a) {
  top2_init(a.t);
  a.m = -INFINITY;
  a.s = 0.f;
  a.nonfinite = 0;
}

__device__ __forceinline__ void lse_merge(float& m, float& s, float m2, float s2) {
  const float M = fmaxf(m, m2);
  if (M == -INFINITY) return;
  s = (m == -INFINITY ? 0.f : s * __expf(m - M)) + (m2 == -INFINITY ? 0.f : s2 * __expf(m2 - M));
  m = M;
}

template <bool LSE>
__device__ __forceinline__ void acc_push(Acc& a, float v, int i) {
  a.nonfinite |= !(fabsf(v) < INFINITY);
  top2_push(a.t, v, i);
  if constexpr (LSE) {
    if (fabsf(v) < INFINITY) {
      if (v > a.m) {
        a.s = a.s * __expf(a.m - v) + 1.f;
        a.m = v;
      } else {
        a.s += __expf(v - a.m);
      }
    }
  }
}

template <bool LSE>
__device__ __forceinline__ void acc_merge(Acc& a, const Acc& b) {
  top2_merge(a.t, b.t);
  if constexpr (LSE) lse_merge(a.m, a.s, b.m, b.s);
  a.nonfinite |= b.nonfinite;
}

// All 64 lanes' accumulators merged, in every lane.
template <bool LSE>
__device__ __forceinline__ Acc wave_acc(Acc a) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    Acc b = a;
    b.t.v1 = __shfl_xor(a.t.v1, o, 64);
    b.t.v2 = __shfl_xor(a.t.v2, o, 64);
    b.t.i1 = __shfl_xor(a.t.i1, o, 64);
    if constexpr (LSE) {
      b.m = __shfl_xor(a.m, o, 64);
      b.s = __shfl_xor(a.s, o, 64);
    }
    acc_merge<LSE>(a, b);
  }
  a.nonfinite = __builtin_amdgcn_ballot_w64(a.nonfinite != 0) ? 1u : 0u;
  return a;
}

__device__ __forceinline__ ScanPartial to_partial(const Acc& a) {
  return ScanPartial{a.t.v1, a.t.v2, a.t.i1, a.nonfinite, a.m, a.s, {0, 0}};
}

__device__ __forceinline__ Acc from_partial(const ScanPartial& p) {
  return Acc{Top2{p.v1, p.v2, p.i1}, p.m, p.s, p.nonfinite};
}

// Block-level: merge the 4 waves' accumulators (wave order), the result in every thread.
template <bool LSE>
__device__ __forceinline__ Acc block_acc(Acc a, ScanPartial* red) {
  a = wave_acc<LSE>(a);
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  __syncthreads();
  if (lane == 0) red[wave] = to_partial(a);
  __syncthreads();
  Acc r = from_partial(red[0]);
  for (int w = 1; w < 4; ++w) acc_merge<LSE>(r, from_partial(red[w]));
  return r;
}

}  // namespace spp
