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

struct Penalties {
  float repetition, frequency, presence;
};

// One token's value.  Every operation rounds by itself (no fused multiply-add), so that the
// result does not depend on how the compiler pairs them.
__device__ __forceinline__ float adjust_one(float y, const Penalties& p, uint32_t cnt, uint32_t bias_at, float bias) {
#pragma clang fp contract(off)
  const float rep = y > 0.f ? y / p.repetition : y * p.repetition;
  y = cnt ? rep : y;
  const uint32_t c = cnt & 0x7FFFFFFFu;
  const float often = p.frequency * (float)c;
  const float less = y - often;
  y = c ? less - p.presence : y;
  return bias_at ? y + bias : y;
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
  const spp_adjust r = jobs.row[blockIdx.y];
  const Penalties pen{r.repetition, r.frequency, r.presence};
  const int tid = threadIdx.x;
  uint32_t* cnt = lds;
  uint32_t* bias_at = lds + S;  // (present when some row of the launch has biases)
  const int a = (int)((reinterpret_cast<uintptr_t>(r.src) & 15) / 4);
  const bool pair = ((reinterpret_cast<uintptr_t>(r.src) ^ reinterpret_cast<uintptr_t>(r.dst)) & 15) == 0;
  const int v0 = (int)blockIdx.x * S - a;  // first token of the slice (before the row: skipped)
  const bool penal = r.n_tokens > 0 && (r.repetition != 1.f || r.frequency != 0.f || r.presence != 0.f);
  const bool biased = r.n_bias > 0, masked = r.allowed != nullptr;
  const int n_tokens = penal ? r.n_tokens : 0;

  // The lists' first entries, then the slice's logits and mask are on their way while LDS is
  // cleared: a wait for the entries, older, is not one for the logits, which keep streaming
  // while the entries are counted.  No load is in a branch of a thread's own (its registers
  // would be waited for at the branch's end): an index past the end reads the last value again.
  constexpr int AHEAD = 8;
  int tok[AHEAD], bt = 0;
  auto tokens_at = [&](int i0) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) tok[u] = r.tokens[min(i0 + u * kTpb, n_tokens - 1)];
  };
  if (n_tokens > 0) tokens_at(tid);
  if (biased) bt = r.bias_tokens[min(tid, r.n_bias - 1)];
  __builtin_amdgcn_sched_barrier(0);
  // first tokens of the row's first and last whole units (no whole unit: t_hi < t_lo)
  const int t_lo = a ? 4 - a : 0, t_hi = ((V + a) & ~3) - 4 - a;
  float x[UNITS][4];
  if (t_lo <= t_hi)
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int t = min(max(v0 + 4 * (u * kTpb + tid), t_lo), t_hi);
      const float4 q = *reinterpret_cast<const float4*>(r.src + t);
      x[u][0] = q.x; x[u][1] = q.y; x[u][2] = q.z; x[u][3] = q.w;
    }
  // the row's first and last unit, where they are not whole
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    const int t = v0 + 4 * (u * kTpb + tid);
    if ((t < t_lo || t > t_hi) && t + 3 >= 0 && t < V)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[u][e] = r.src[min(max(t + e, 0), V - 1)];
  }
  uint32_t w[UNITS][2];
  if (masked)
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      // the words of the unit's first and last token (inside the row)
      const int t = v0 + 4 * (u * kTpb + tid);
      w[u][0] = r.allowed[min(max(t, 0), V - 1) >> 5];
      w[u][1] = r.allowed[min(max(t + 3, 0), V - 1) >> 5];
    }
  const uint4 zero = make_uint4(0, 0, 0, 0);
  if (penal)
    for (int i = tid; i < S / 4; i += kTpb) reinterpret_cast<uint4*>(cnt)[i] = zero;
  if (biased)
    for (int i = tid; i < S / 4; i += kTpb) reinterpret_cast<uint4*>(bias_at)[i] = zero;
  __syncthreads();
  // (a slice's tokens below 0 or from V on are none of the row's: entries there are skipped)
  const int lo = max(v0, 0), hi = min(v0 + S, V);
  for (int i0 = tid; i0 - tid < n_tokens; i0 += AHEAD * kTpb) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (i0 + u * kTpb < n_tokens && tok[u] >= lo && tok[u] < hi) {
        if (i0 + u * kTpb < r.n_prompt)
          atomicOr(cnt + (tok[u] - v0), 0x80000000u);
        else
          atomicAdd(cnt + (tok[u] - v0), 1u);
      }
    if (i0 - tid + AHEAD * kTpb < n_tokens) tokens_at(i0 + AHEAD * kTpb);
  }
  for (int i = tid; i - tid < r.n_bias; i += kTpb) {
    if (i < r.n_bias && bt >= lo && bt < hi) atomicMax(bias_at + (bt - v0), (uint32_t)i + 1);
    if (i - tid + kTpb < r.n_bias) bt = r.bias_tokens[min(i + kTpb, r.n_bias - 1)];
  }
  __syncthreads();

  // Adjusted and stored; then x holds the allowed values, -inf elsewhere.
  uint32_t live = 0;  // a bit per value: in the row and allowed
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    const int at = 4 * (u * kTpb + tid), t = v0 + at;
    uint4 c = zero, ba = zero;
    if (penal) c = *reinterpret_cast<const uint4*>(cnt + at);
    if (biased) ba = *reinterpret_cast<const uint4*>(bias_at + at);
    if (c.x | c.y | c.z | c.w | ba.x | ba.y | ba.z | ba.w) {
      const uint32_t cs[4] = {c.x, c.y, c.z, c.w}, bs[4] = {ba.x, ba.y, ba.z, ba.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float bias = 0.f;
        if (bs[e]) bias = r.bias[bs[e] - 1];
        x[u][e] = adjust_one(x[u][e], pen, cs[e], bs[e], bias);
      }
    }
    uint32_t bits = 0xFu;
    const bool whole = t >= t_lo && t <= t_hi;
    if (!whole) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (t + e < 0 || t + e >= V) bits &= ~(1u << e);
    }
    const uint32_t in_row = bits;
    // bits t & 31 and up of the two words side by side; before the row (t < 0, bits left out
    // above) the first word is that of token 0
    if (masked)
      bits &= t >= 0 ? (uint32_t)((((uint64_t)w[u][1] << 32) | w[u][0]) >> (t & 31)) : w[u][0] << (-t & 3);
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (bits >> e) & 1u ? x[u][e] : r.fill;
    if (pair && whole) {
      *reinterpret_cast<float4*>(r.dst + t) = make_float4(y[0], y[1], y[2], y[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if ((in_row >> e) & 1u) r.dst[t + e] = y[e];
    }
    live |= bits << (4 * u);
  }
  if (!parts) return;
  // The two largest of the thread's allowed values (NaN is none), the index of the largest,
  // lowest on ties, and the sum of exponentials: the values are all there, so it needs no
  // running maximum.
  Acc acc;
  acc_init(acc);
#pragma unroll
  for (int u = 0; u < UNITS; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool ok = (live >> (4 * u + e)) & 1u;
      acc.nonfinite |= ok && !(fabsf(x[u][e]) < INFINITY);
      x[u][e] = ok ? x[u][e] : -INFINITY;
      const float y = fmaxf(x[u][e], -INFINITY);  // (NaN -> -inf)
      acc.t.i1 = y > acc.t.v1 ? v0 + 4 * (u * kTpb + tid) + e : acc.t.i1;
      acc.t.v2 = __builtin_amdgcn_fmed3f(y, acc.t.v1, acc.t.v2);
      acc.t.v1 = fmaxf(acc.t.v1, y);
    }
  if (acc.t.i1 == 0x7FFFFFFF && live) {  // nothing above -inf: the first allowed -inf
#pragma unroll
    for (int u = UNITS - 1; u >= 0; --u)
#pragma unroll
      for (int e = 3; e >= 0; --e)
        if ((live >> (4 * u + e)) & 1u && x[u][e] == x[u][e]) acc.t.i1 = v0 + 4 * (u * kTpb + tid) + e;
  }
  acc.m = acc.t.v1;
  if (acc.m > -INFINITY)
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc.s += __expf(x[u][e] - acc.m);
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
#ifdef UMAX
  if (want > 1024) return UMAX;
#endif
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
