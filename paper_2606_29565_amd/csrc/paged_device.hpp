// What the kernels over paged caches share, whatever their cells: how a sequence's cells are dealt
// out to key ranges, the queries' operands and how outputs are stored.
#pragma once

#include "common.hpp"
#include "paged.hpp"

namespace spp {
namespace {

constexpr int kWaves = 4;      // waves of an attention workgroup, each with its own key range
constexpr int kMaxSplits = 256;

// Cells of a key range: a sequence's cells dealt out evenly over at most `splits` ranges of
// whole steps of all waves.  (On the device, from the length as it is at the launch.)
__device__ __forceinline__ int range_cells(int len, int splits, int unit) {
  const int units = (len + unit - 1) / unit;
  return (units + splits - 1) / splits * unit;
}

__device__ __forceinline__ int live_cells(const PagedAttn& a, int shift, int seq) {
  const int len = a.lengths[seq], most = a.max_pages << shift;
  return len < 0 ? 0 : (len < most ? len : most);
}

__device__ __forceinline__ void store_out(const PagedAttn& a, int64_t i, float v) {
  if (a.out_mode == 0) {
    static_cast<float*>(a.out)[i] = v;
  } else if (a.out_mode == 1) {
    static_cast<bf16_t*>(a.out)[i].bits = f32_to_bf16(v);
  } else {
    store_act(static_cast<bf16_t*>(a.out), static_cast<bf16_t*>(a.out_lo), i, v);
  }
}

// Eight or four query elements in two parts of the cells' type (hi alone in fp32).
__device__ __forceinline__ void query_frag(const void* q, bool q_bf16, int64_t at, uint4& hi, uint4& lo, bf16_t) {
  if (q_bf16) {
    hi = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(q) + at);
    lo = make_uint4(0, 0, 0, 0);
    return;
  }
  const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(q) + at);
  const float4 b = *reinterpret_cast<const float4*>(static_cast<const float*>(q) + at + 4);
  split_pair(a.x, a.y, hi.x, lo.x);
  split_pair(a.z, a.w, hi.y, lo.y);
  split_pair(b.x, b.y, hi.z, lo.z);
  split_pair(b.z, b.w, hi.w, lo.w);
}
__device__ __forceinline__ void query_frag(const void* q, bool q_bf16, int64_t at, uint4& hi, uint4& lo, float) {
  if (q_bf16) {
    const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(q) + at);
    hi = make_uint4(w.x << 16, w.x & 0xFFFF0000u, w.y << 16, w.y & 0xFFFF0000u);
  } else {
    hi = *reinterpret_cast<const uint4*>(static_cast<const float*>(q) + at);
  }
  lo = make_uint4(0, 0, 0, 0);
}

}  // namespace
}  // namespace spp
