// Adjusted logits: penalties for repeated tokens, biases and an allowed set on rows of fp32
// logits, with the reductions (top-2, log-sum-exp, non-finite) of the allowed tokens.
//
//   y = x;  v in tokens: y = y > 0 ? y / rho : y * rho;  y -= alpha c;  c > 0: y -= beta
//   v in bias_tokens: y += bias;  v not allowed: y = fill
//
// Bound by memory: a row's logits are read and written once (8 bytes a token).  What each
// token needs to know of the history -- whether it occurs, and how often past the prompt -- is
// gathered per workgroup: it owns a slice of the vocabulary, reads the whole list of tokens
// (from L2 after the first workgroup) and counts those of its slice in LDS with integer atomics,
// whose order does not matter.  That suits histories of some thousand tokens, a few KB; long ones
// outweigh the logits: 64 rows of 128256 take, from a graph, 20.0 us with 2000 tokens each, 28.7 with
// 8000 and 55 with 32768, one row 7.2 with 6000 and 14.4 with 32768.  The largest index of a bias entry is kept the same way, so the last entry of a token
// counts.  Nothing of the vocabulary's size besides the logits is written, cleared or read again.
// Measured (with the launch that merges the slices' reductions): 64 rows of 128256 with 2000 tokens
// 19.3 us through the binding, 3.4 TB/s.  One row is launches and latency: 7.2 us from a graph, 8
// through the binding.
#include "common.hpp"
#include "paged.hpp"

namespace spp {
namespace {

constexpr int kTpb = 256;

// The rows of one launch travel as its argument: one (a launch with up to about 100 bytes of
// arguments takes the host 2.8 us, with any more up to 4 KB 3.4 to 3.9) or, within 4 KB, many.
constexpr int kManyRows = 48;
template <int R>
struct AdjustBatch {
  spp_adjust row[R];
};
static_assert(sizeof(AdjustBatch<kManyRows>) + 16 <= 4096, "a kernel's argument");

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

// The allowed bits of the unit whose first token is t, from the words of its first and last token
// inside the row (before the row, t < 0, the first word is that of token 0).
__device__ __forceinline__ uint32_t mask_bits(const uint32_t (&w)[2], int t) {
  const uint32_t b = t >= 0 ? (uint32_t)((((uint64_t)w[1] << 32) | w[0]) >> (t & 31)) : w[0] << (-t & 3);
  return b & 0xFu;
}

// The reductions over a part of a row travel as four words: the largest value (NaN left out), the
// second largest, the first one's index as bits (the lowest; kNone without one), and the sum of
// exp(value - largest), NaN if a value is not finite.
constexpr int kNone = 0x7FFFFFFF;
// What the sum of a part with largest value m counts in that of a whole with largest value `all`.
__device__ __forceinline__ float part_weight(float m, float all) {
  return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - all) * 1.44269504f);
}
__device__ __forceinline__ void part_merge(float4& a, const float4& b) {
  const float m = fmaxf(a.x, b.x);
  a.y = fmaxf(fmaxf(a.y, b.y), fminf(a.x, b.x));
  const int ia = a.x == m ? __float_as_int(a.z) : kNone, ib = b.x == m ? __float_as_int(b.z) : kNone;
  a.z = __int_as_float(min(ia, ib));
  a.w = a.w * part_weight(a.x, m) + b.w * part_weight(b.x, m);
  a.x = m;
}

// Grid (slices, rows), UNITS * 1024 tokens a slice.  A row's tokens are cut into units of four
// at 16-byte boundaries of src (unit u holds tokens 4u - a .. 4u - a + 3, a the elements that
// src starts past such a boundary), so that all whole units are 16-byte accesses whatever the
// row's alignment; unit u of the slice belongs to thread u % 256.
//
// An instruction for every token of 32 rows of 128256 takes the chip 0.1 us: what counts is the
// instructions each token costs.  So
//  - the few tokens with a penalty or bias are adjusted one at a time: a thread goes over those
//    of its tokens that were counted and picks each from its registers (read again from memory,
//    with the results left where the counts were, 0.5 us longer for the 64 rows below);
//  - a slice of whole units has a path without a look at the row's ends;
//  - the reductions start from the wave's largest value (no running maximum, the index only where
//    it is), by data-parallel moves.
// 64 rows of 128256 with 2000 tokens and 100 biases, with the summaries: 19.3 us.  Before the
// stores' and the merge's own steps (then 23.1): a wave that adjusts all its tokens wherever one
// lane needs it 32.3; a list of the touched tokens made by the counting 30.4; their logits kept
// in LDS 27.0; without the last two of these points 26.3.
template <int UNITS, int R>
__global__ __launch_bounds__(kTpb) void adjust_kernel(int V, AdjustBatch<R> jobs, float4* parts) {
  constexpr int S = UNITS * 4 * kTpb;
  __shared__ __align__(16) uint32_t cnt[S];    // occurrences past the prompt; bit 31: in the prompt
  __shared__ __align__(16) uint32_t bias_at[S];  // last bias entry of the token, plus one
  __shared__ float4 red[4];
  const spp_adjust r = jobs.row[blockIdx.y];
  const Penalties pen{r.repetition, r.frequency, r.presence};
  const int tid = threadIdx.x;
  const int a = (int)((reinterpret_cast<uintptr_t>(r.src) & 15) / 4);
  const bool pair = ((reinterpret_cast<uintptr_t>(r.src) ^ reinterpret_cast<uintptr_t>(r.dst)) & 15) == 0;
  const int v0 = (int)blockIdx.x * S - a;  // first token of the slice (before the row: skipped)
  const bool penal = r.n_tokens > 0 && (r.repetition != 1.f || r.frequency != 0.f || r.presence != 0.f);
  const bool biased = r.n_bias > 0, masked = r.allowed != nullptr, sparse = penal || biased;
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
  const bool whole = v0 >= t_lo && v0 + S - 4 <= t_hi;  // the slice has no end of the row
  if (whole) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const float4 q = *reinterpret_cast<const float4*>(r.src + v0 + 4 * (u * kTpb + tid));
      x[u][0] = q.x; x[u][1] = q.y; x[u][2] = q.z; x[u][3] = q.w;
    }
  } else {
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

  constexpr uint32_t kAll = (1u << (4 * UNITS)) - 1;
  if (sparse) {
    const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      reinterpret_cast<uint4*>(cnt)[u * kTpb + tid] = zero;
      if (biased) reinterpret_cast<uint4*>(bias_at)[u * kTpb + tid] = zero;
    }
    __syncthreads();
    // (a slice's tokens below 0 or from V on are none of the row's: entries there are skipped)
    const int lo = max(v0, 0), hi = max(lo, min(v0 + S, V));  // (the last slice may be behind the row)
    for (int i0 = 0; i0 < n_tokens; i0 += AHEAD * kTpb) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const uint32_t off = (uint32_t)tok[u] - (uint32_t)lo;
        if (tid < n_tokens - i0 - u * kTpb && off < (uint32_t)(hi - lo)) {
          uint32_t* c = cnt + (lo - v0) + off;
          if (tid < r.n_prompt - i0 - u * kTpb)
            atomicOr(c, 0x80000000u);
          else
            atomicAdd(c, 1u);
        }
      }
      if (i0 + AHEAD * kTpb < n_tokens) tokens_at(i0 + AHEAD * kTpb + tid);
    }
    for (int i = tid; i - tid < r.n_bias; i += kTpb) {
      if (i < r.n_bias && bt >= lo && bt < hi) atomicMax(bias_at + (bt - v0), (uint32_t)i + 1);
      if (i - tid + kTpb < r.n_bias) bt = r.bias_tokens[min(i + kTpb, r.n_bias - 1)];
    }
    __syncthreads();
    uint32_t touched = 0;  // of the thread's own tokens, a bit each
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      uint4 c = reinterpret_cast<const uint4*>(cnt)[u * kTpb + tid];
      if (biased) {
        const uint4 b = reinterpret_cast<const uint4*>(bias_at)[u * kTpb + tid];
        c = make_uint4(c.x | b.x, c.y | b.y, c.z | b.z, c.w | b.w);
      }
      touched |= ((c.x ? 1u : 0u) | (c.y ? 2u : 0u) | (c.z ? 4u : 0u) | (c.w ? 8u : 0u)) << (4 * u);
    }
    for (uint32_t todo = touched; todo; todo &= todo - 1) {
      const int f = __ffs(todo) - 1, at = 4 * (f / 4 * kTpb + tid) + f % 4;
      const uint32_t c = cnt[at], b = biased ? bias_at[at] : 0u;
      float y = x[0][0];
#pragma unroll
      for (int k = 1; k < 4 * UNITS; ++k) y = f == k ? x[k / 4][k % 4] : y;
      y = adjust_one(y, pen, c, b, b ? r.bias[b - 1] : 0.f);
#pragma unroll
      for (int k = 0; k < 4 * UNITS; ++k) x[k / 4][k % 4] = f == k ? y : x[k / 4][k % 4];
    }
  }

  // Masked and stored; then x holds the allowed values, -inf elsewhere.  The stores pass the L2 by:
  // nothing here reads them, and lines that wait there are written back between this launch and
  // the next (64 rows of 128256 when this was chosen: 22.9 us so, 20.7 past it; loads past it too 21.8).
  uint32_t live = kAll;   // a bit per value: in the row and allowed
  float low = INFINITY;   // the smallest allowed value
  if (pair && whole) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int t = v0 + 4 * (u * kTpb + tid);
      f32x4* dst = reinterpret_cast<f32x4*>(r.dst + t);
      if (masked) {
        const uint32_t bits = mask_bits(w[u], t);
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool ok = (bits >> e) & 1u;
          y[e] = ok ? x[u][e] : r.fill;
          low = fminf(low, ok ? x[u][e] : INFINITY);
          x[u][e] = ok ? x[u][e] : -INFINITY;
        }
        __builtin_nontemporal_store(f32x4{y[0], y[1], y[2], y[3]}, dst);
        live = (live & ~(0xFu << (4 * u))) | bits << (4 * u);
      } else {
        __builtin_nontemporal_store(f32x4{x[u][0], x[u][1], x[u][2], x[u][3]}, dst);
#pragma unroll
        for (int e = 0; e < 4; ++e) low = fminf(low, x[u][e]);
      }
    }
  } else {
    live = 0;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int t = v0 + 4 * (u * kTpb + tid);
      const uint32_t bits = masked ? mask_bits(w[u], t) : 0xFu;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = t + e >= 0 && t + e < V, ok = in && ((bits >> e) & 1u);
        if (in) r.dst[t + e] = ok ? x[u][e] : r.fill;
        low = fminf(low, ok ? x[u][e] : INFINITY);
        x[u][e] = ok ? x[u][e] : -INFINITY;
        live |= (uint32_t)ok << (4 * u + e);
      }
    }
  }
  if (!parts) return;

  // The wave's part, from the largest value on: the thread's two largest (v_max and v_med
  // take NaN for none), the wave's largest, its index where a thread holds it, and the sum of
  // exponentials against it.  Of what is not finite, NaN and +inf show in that sum, -inf in `low`.
  float v1 = -INFINITY, v2 = -INFINITY;
#pragma unroll
  for (int u = 0; u < UNITS; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float y = fmaxf(x[u][e], -INFINITY);  // (NaN, a signalling one too, -> -inf)
      v2 = __builtin_amdgcn_fmed3f(y, v1, v2);
      v1 = fmaxf(v1, y);
    }
  const float m = wave_max_all(v1);
  float sum = 0.f;
  const int base = v0 + 4 * tid;
  int at = kNone;  // of the thread's value equal to the wave's largest, the lowest index
  if (m > -INFINITY) {
    int off = -1;
#pragma unroll
    for (int u = UNITS - 1; u >= 0; --u)
#pragma unroll
      for (int e = 3; e >= 0; --e) off = x[u][e] == m ? 4 * kTpb * u + e : off;
    at = off >= 0 ? base + off : at;
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((x[u][e] - m) * 1.44269504f);
    sum = wave_sum_all(sum);
  } else if (live) {  // nothing above -inf: the first allowed -inf
#pragma unroll
    for (int u = UNITS - 1; u >= 0; --u)
#pragma unroll
      for (int e = 3; e >= 0; --e)
        if ((live >> (4 * u + e)) & 1u && x[u][e] == x[u][e]) at = base + 4 * kTpb * u + e;
  }
  const int first = wave_min_all(at);
  // the second largest: among the others' largest and the holder's second
  const float next = wave_max_all(at == first ? v2 : v1);
  const bool bad = __any(low == -INFINITY) || !(sum < INFINITY) || (m == -INFINITY && __any(live != 0));
  const float4 mine = make_float4(m, next, __int_as_float(first), bad ? __builtin_nanf("") : sum);
  if ((tid & 63) == 0) red[tid >> 6] = mine;
  __syncthreads();
  if (tid == 0) {
    float4 all = red[0];
    for (int k = 1; k < kTpb / 64; ++k) part_merge(all, red[k]);
    parts[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = all;
  }
}

// Grid (rows), one wave each: the slices' parts merged in a fixed order, lanes' own first, then
// across the wave as above (merging pairs of lanes by shuffles took 1.0 to 1.4 us longer).
__global__ __launch_bounds__(64) void adjust_merge_kernel(int nb, const float4* parts, spp_summary* out) {
  parts += (int64_t)blockIdx.x * nb;
  constexpr int AHEAD = 4;
  float4 a = make_float4(-INFINITY, -INFINITY, __int_as_float(kNone), 0.f);
  for (int b0 = threadIdx.x; b0 - (int)threadIdx.x < nb; b0 += AHEAD * 64) {
    float4 p[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) p[u] = parts[min(b0 + u * 64, nb - 1)];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (b0 + u * 64 < nb) part_merge(a, p[u]);
  }
  const float m = wave_max_all(a.x);
  const float sum = wave_sum_all(a.w * part_weight(a.x, m));
  const int at = a.x == m ? __float_as_int(a.z) : kNone;
  const int first = wave_min_all(at);
  const float next = wave_max_all(at == first ? a.y : a.x);
  if (threadIdx.x) return;
  const bool none = first == kNone, bad = sum != sum;
  spp_summary s;
  s.argmax = none ? -1 : first;
  s.top1 = m;
  s.top2 = next;
  s.gap = m - next;
  s.lse = bad || none ? __builtin_nanf("") : m + __logf(sum);
  s.position = 0;
  s.flags = (bad ? 1u : 0u) | (none && !bad ? 8u : 0u);
  out[blockIdx.x] = s;
}

// Tokens of a slice: 1024 while that makes under 2048 workgroups, else 2048, which halves how
// often a history is read and the instructions of a workgroup beside its tokens' own (from a
// graph, 64 rows of 128256 with 2000 tokens each: 20.0 us, with slices of 1024 22.7, with slices of
// 4096, half as many waves to a CU, 20.0; 17 rows of 152063 with 700: 9.9, 10.7 and 10.7).
int slice_units(int n, int vocab) { return (int64_t)vocab * n <= kShortSliceTokens ? 1 : 2; }
// Slices of a row, whatever its alignment.
int slices(int units, int vocab) { return (vocab + 3 + units * 4 * kTpb - 1) / (units * 4 * kTpb); }

}  // namespace

namespace k {

size_t adjust_work_bytes(int n, int vocab) {
  return (size_t)n * slices(slice_units(n, vocab), vocab) * sizeof(float4);
}

template <int R>
void launch_rows(int units, int nb, int m, int vocab, const spp_adjust* rows, float4* parts, hipStream_t st) {
  AdjustBatch<R> b{};
  for (int i = 0; i < m; ++i) b.row[i] = rows[i];
  if (units == 1)
    SPP_LAUNCH((adjust_kernel<1, R>), dim3(nb, m), dim3(kTpb), 0, st, vocab, b, parts);
  else
    SPP_LAUNCH((adjust_kernel<2, R>), dim3(nb, m), dim3(kTpb), 0, st, vocab, b, parts);
}

hipError_t adjust_logits(int n, int vocab, const spp_adjust* rows, spp_summary* summaries, void* work,
                         hipStream_t st) {
  const int units = slice_units(n, vocab), nb = slices(units, vocab);
  // launches of like size: what is left over a multiple of kManyRows would not fill the chip (64
  // rows of 128256 from a graph: 20.4 us as 48 and 16, 20.0 as 32 and 32)
  const int launches = (n - 1) / kManyRows + 1, step = (n - 1) / launches + 1;
  for (int r0 = 0; r0 < n; r0 += step) {
    const int m = n - r0 < step ? n - r0 : step;
    float4* parts = summaries ? static_cast<float4*>(work) + (int64_t)r0 * nb : nullptr;
    if (m == 1)
      launch_rows<1>(units, nb, m, vocab, rows + r0, parts, st);
    else
      launch_rows<kManyRows>(units, nb, m, vocab, rows + r0, parts, st);
  }
  if (summaries)
    SPP_LAUNCH(adjust_merge_kernel, dim3(n), dim3(64), 0, st, nb, static_cast<const float4*>(work),
               summaries);
  return hipGetLastError();
}

}  // namespace k
}  // namespace spp
