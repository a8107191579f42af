// Adjusted logits: penalties for repeated tokens, biases and an allowed set on rows of fp32
// logits, with the reductions (top-2, log-sum-exp, non-finite) of the allowed tokens.
//
//   y = x;  v in tokens: y = y > 0 ? y / rho : y * rho;  y -= alpha c;  c > 0: y -= beta
//   v in bias_tokens: y += bias;  v not allowed: y = fill
//
// Bound by memory: a row's logits are read and written once (8 bytes a token).  What each
// token needs to know of the history -- whether it occurs, and how often past the prompt -- is
// gathered per workgroup: it owns a slice of the vocabulary, reads the whole list of tokens
// (from L2 after the first workgroup; a history is a few KB against 8 bytes per token of the
// vocabulary) and counts those of its slice in LDS with integer atomics, whose order does not matter.  The
// largest index of a bias entry is kept the same way, so the last entry of a token counts.
// Nothing of the vocabulary's size besides the logits is written, cleared or read again.
#include "reduce.hpp"
#include "paged.hpp"

namespace spp {
namespace {

constexpr int kTpb = 256;

struct AdjustBatch {
  spp_adjust row[kAdjustRows];
};

// Every operation rounds by itself (no fused multiply-add), so that the result does not
// depend on how the compiler pairs them.
__device__ __forceinline__ float adjust_one(float y, const spp_adjust& r, uint32_t cnt, uint32_t bias_at,
                                            bool allowed) {
#pragma clang fp contract(off)
  if (cnt) y = y > 0.f ? y / r.repetition : y * r.repetition;
  const uint32_t c = cnt & 0x7FFFFFFFu;
  if (c) {
    y = y - r.frequency * (float)c;
    y = y - r.presence;
  }
  if (bias_at) y = y + r.bias[bias_at - 1];
  return allowed ? y : r.fill;
}

// Grid (slices, rows), UNITS * 1024 tokens a slice.  A row's tokens are cut into units of four
// at 16-byte boundaries of src (unit u holds tokens 4u - a .. 4u - a + 3, a the elements that
// src starts past such a boundary), so that all whole units are 16-byte accesses whatever the
// row's alignment; unit u of the slice belongs to thread u % 256.  LDS: a count (bit 31: seen
// in the prompt) and, with biases, a bias entry per token of the slice.
template <int UNITS>
__global__ __launch_bounds__(kTpb) void adjust_kernel(int V, AdjustBatch jobs, ScanPartial* parts) {
  constexpr int S = UNITS * 4 * kTpb;
  extern __shared__ uint32_t lds[];
  __shared__ ScanPartial red[4];
  const spp_adjust& r = jobs.row[blockIdx.y];
  const int tid = threadIdx.x;
  uint32_t* cnt = lds;
  uint32_t* bias_at = lds + S;  // (present when some row of the launch has biases)
  const int a = (int)((reinterpret_cast<uintptr_t>(r.src) & 15) / 4);
  const bool pair = ((reinterpret_cast<uintptr_t>(r.src) ^ reinterpret_cast<uintptr_t>(r.dst)) & 15) == 0;
  const int v0 = (int)blockIdx.x * S - a;  // first token of the slice (before the row: skipped)
  const bool penal = r.n_tokens > 0 && (r.repetition != 1.f || r.frequency != 0.f || r.presence != 0.f);
  const bool biased = r.n_bias > 0;

  // the slice's logits are on their way while the history is counted
  float x[UNITS][4];
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    const int t = v0 + 4 * (u * kTpb + tid);
    if (t >= 0 && t + 3 < V) {
      const float4 q = *reinterpret_cast<const float4*>(r.src + t);
      x[u][0] = q.x; x[u][1] = q.y; x[u][2] = q.z; x[u][3] = q.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[u][e] = t + e >= 0 && t + e < V ? r.src[t + e] : 0.f;
    }
  }
  if (penal)
    for (int i = tid; i < S; i += kTpb) cnt[i] = 0;
  if (biased)
    for (int i = tid; i < S; i += kTpb) bias_at[i] = 0;
  __syncthreads();
  // (a slice's tokens below 0 or from V on are none of the row's: entries there are skipped)
  const int lo = max(v0, 0), hi = min(v0 + S, V);
  if (penal)
    for (int i = tid; i < r.n_tokens; i += kTpb) {
      const int t = r.tokens[i];
      if (t >= lo && t < hi) {
        if (i < r.n_prompt)
          atomicOr(cnt + (t - v0), 0x80000000u);
        else
          atomicAdd(cnt + (t - v0), 1u);
      }
    }
  if (biased)
    for (int i = tid; i < r.n_bias; i += kTpb) {
      const int t = r.bias_tokens[i];
      if (t >= lo && t < hi) atomicMax(bias_at + (t - v0), (uint32_t)i + 1);
    }
  __syncthreads();
  Acc acc;
  acc_init(acc);
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    const int at = 4 * (u * kTpb + tid), t = v0 + at;
    if (t >= V || t + 3 < 0) continue;
    uint32_t bits = 0xFu;
    if (r.allowed) {
      const int first = max(t, 0), last = min(t + 3, V - 1);
      const uint32_t w0 = r.allowed[first >> 5], w1 = r.allowed[last >> 5];
      bits = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        bits |= (((((t + e) >> 5) == (first >> 5) ? w0 : w1) >> ((t + e) & 31)) & 1u) << e;
    }
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool ok = (bits >> e) & 1u;
      y[e] = adjust_one(x[u][e], r, penal ? cnt[at + e] : 0u, biased ? bias_at[at + e] : 0u, ok);
      if (ok && t + e >= 0 && t + e < V) acc_push<true>(acc, y[e], t + e);
    }
    if (pair && t >= 0 && t + 3 < V) {
      *reinterpret_cast<float4*>(r.dst + t) = make_float4(y[0], y[1], y[2], y[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (t + e >= 0 && t + e < V) r.dst[t + e] = y[e];
    }
  }
  if (!parts) return;
  acc = block_acc<true>(acc, red);
  if (tid == 0) parts[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = to_partial(acc);
}

// Grid (rows), one wave each: the slices' partials merged in a fixed order.
__global__ __launch_bounds__(64) void adjust_merge_kernel(int nb, const ScanPartial* parts,
                                                          spp_summary* out) {
  Acc a;
  acc_init(a);
  for (int b = threadIdx.x; b < nb; b += 64) acc_merge<true>(a, from_partial(parts[(int64_t)blockIdx.x * nb + b]));
  a = wave_acc<true>(a);
  if (threadIdx.x) return;
  const bool none = a.t.i1 == 0x7FFFFFFF;
  spp_summary s;
  s.argmax = none ? -1 : a.t.i1;
  s.top1 = a.t.v1;
  s.top2 = a.t.v2;
  s.gap = a.t.v1 - a.t.v2;
  s.lse = a.nonfinite || none ? __builtin_nanf("") : a.m + __logf(a.s);
  s.position = 0;
  s.flags = (a.nonfinite ? 1u : 0u) | (none && !a.nonfinite ? 8u : 0u);
  out[blockIdx.x] = s;
}

// Tokens of a slice: 1024 to 4096, so that a launch has about a thousand workgroups.
int slice_units(int n, int vocab) {
  const int64_t want = (int64_t)vocab * n / 1024;
  return want <= 1024 ? 1 : (want <= 2048 ? 2 : 4);
}
// Slices of a row, whatever its alignment.
int slices(int units, int vocab) { return (vocab + 3 + units * 4 * kTpb - 1) / (units * 4 * kTpb); }

}  // namespace

namespace k {

size_t adjust_work_bytes(int n, int vocab) {
  return (size_t)n * slices(slice_units(n, vocab), vocab) * sizeof(ScanPartial);
}

hipError_t adjust_logits(int n, int vocab, const spp_adjust* rows, spp_summary* summaries, void* work,
                         hipStream_t st) {
  const int units = slice_units(n, vocab), nb = slices(units, vocab);
  for (int r0 = 0; r0 < n; r0 += kAdjustRows) {
    const int m = n - r0 < kAdjustRows ? n - r0 : kAdjustRows;
    AdjustBatch b{};
    bool bias = false;
    for (int i = 0; i < m; ++i) {
      b.row[i] = rows[r0 + i];
      bias |= rows[r0 + i].n_bias > 0;
    }
    ScanPartial* parts = summaries ? static_cast<ScanPartial*>(work) + (int64_t)r0 * nb : nullptr;
    const unsigned shm = (bias ? 2u : 1u) * units * 4 * kTpb * 4;
    const dim3 grid(nb, m), block(kTpb);
    if (units == 1)
      SPP_LAUNCH(adjust_kernel<1>, grid, block, shm, st, vocab, b, parts);
    else if (units == 2)
      SPP_LAUNCH(adjust_kernel<2>, grid, block, shm, st, vocab, b, parts);
    else
      SPP_LAUNCH(adjust_kernel<4>, grid, block, shm, st, vocab, b, parts);
  }
  if (summaries)
    SPP_LAUNCH(adjust_merge_kernel, dim3(n), dim3(64), 0, st, nb, static_cast<const ScanPartial*>(work),
               summaries);
  return hipGetLastError();
}

}  // namespace k
}  // namespace spp
