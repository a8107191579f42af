// Log probabilities of rows of fp32 logits: of given tokens, their entropy, and the top alternatives.
//
//   m = max x,  R = sum over the others of e^(x - m),  lse = m + log(1 + R)
//   log p_t = (x_t - m) - log(1 + R),  H = log(1 + R) - (sum e^(x - m) (x - m)) / (1 + R)
// The largest logit is left out of R (one of them, where there are several) so that nothing
// cancels: a token of probability near one keeps the relative precision of its log probability, and H is a sum
// of terms of one sign.
//
// Bound by memory: a row is read once, into registers.  A workgroup takes a slice of a row, a
// second launch puts the slices together.  The alternatives go through a threshold: a wave's
// lanes hold their largest values, and a value that n_top lanes reach (found bit by bit with
// ballots, on the upper half of the bits) is reached by every one of the row's n_top largest in
// this slice; what reaches the largest of the four waves' thresholds goes to a short list, whose
// order is counted.  Ties go to the lower index: an entry of a list is the value's bits, made
// to order as unsigned integers, above the complement of the index.
#include <algorithm>

#include "common.hpp"
#include "paged.hpp"

namespace spp {
namespace {

constexpr int kTpb = 256;
constexpr int kUnits = 8;                       // 16-byte units a thread
constexpr int kSlice = kUnits * 4 * kTpb;       // tokens of a slice
constexpr int kList = 1024;                     // entries of the short list
constexpr int kRows = 96;                       // rows of a launch, within 4 KB of arguments
template <int R>
struct LogprobBatch {
  spp_logprob_row row[R];
};
static_assert(sizeof(LogprobBatch<kRows>) + 64 <= 4096, "a kernel's argument");

// A slice's (or wave's) sums: m, R and sum e^(x - m) (x - m); m -inf without a value above it.
struct Sums {
  float m, r, t;
};
constexpr float kLog2e = 1.44269504f;

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
// What a part adds to the sums of the whole, whose largest value M its own is below (or equal to that
// of an earlier part).
__device__ __forceinline__ void add_part(Sums& a, const Sums& p, float M) {
  const bool none = p.m == -INFINITY && p.r == p.r;  // (a NaN in r stays)
  const float d = p.m - M, w = exp_of(d);
  a.r += none ? 0.f : w * (1.f + p.r);
  a.t += none ? 0.f : w * (p.t + (1.f + p.r) * (w > 0.f ? d : 0.f));
}

// Values in an order of unsigned integers (0: NaN and -inf, which are no alternatives).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);  // (-0 is 0)
  const uint32_t u = b ^ ((int32_t)b < 0 ? ~0u : 0x80000000u);
  return x > -INFINITY ? u : 0u;
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ uint64_t entry(uint32_t u, int index) { return (uint64_t)u << 32 | (uint32_t)~index; }

// The entries of `list` in order, the first `top` to out (0 behind the last).  All of the workgroup.
__device__ __forceinline__ void store_top(const uint64_t* list, int n, int top, uint64_t* out) {
  for (int i = threadIdx.x; i < n; i += kTpb) {
    const uint64_t e = list[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += list[j] > e;
    if (rank < top) out[rank] = e;
  }
  for (int i = n + (int)threadIdx.x; i < top; i += kTpb) out[i] = 0;
}

// Grid (slices, rows).  Units of four tokens at 16-byte boundaries of the row, whatever its
// alignment, unit u of the slice to thread u % 256 (as adjust_kernel).
template <int R>
__global__ __launch_bounds__(kTpb) void logprob_slice_kernel(int V, LogprobBatch<R> jobs, int top, Sums* parts,
                                                             uint64_t* lists) {
  __shared__ Sums wave_sums[4];
  __shared__ uint32_t wave_floor[4];
  __shared__ uint64_t list[kList];
  __shared__ uint64_t best[4];
  __shared__ int count;
  const float* src = jobs.row[blockIdx.y].logits;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int a = (int)((reinterpret_cast<uintptr_t>(src) & 15) / 4);
  const int v0 = (int)blockIdx.x * kSlice - a;  // first token of the slice (before the row: none)
  float x[kUnits][4];
  const int t_lo = a ? 4 - a : 0, t_hi = ((V + a) & ~3) - 4 - a;  // the row's first and last whole unit
  if (v0 >= t_lo && v0 + kSlice - 4 <= t_hi) {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const float4 q = *reinterpret_cast<const float4*>(src + v0 + 4 * (u * kTpb + tid));
      x[u][0] = q.x; x[u][1] = q.y; x[u][2] = q.z; x[u][3] = q.w;
    }
  } else {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int t = v0 + 4 * (u * kTpb + tid);
      float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
      if (t >= t_lo && t <= t_hi) {
        q = *reinterpret_cast<const float4*>(src + t);
      } else if (t + 3 >= 0 && t < V) {
        q.x = src[min(max(t, 0), V - 1)];
        q.y = src[min(max(t + 1, 0), V - 1)];
        q.z = src[min(max(t + 2, 0), V - 1)];
        q.w = src[min(max(t + 3, 0), V - 1)];
      }
      const float f[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) x[u][e] = t + e >= 0 && t + e < V ? f[e] : -INFINITY;
    }
  }

  float mine = -INFINITY;
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) mine = fmaxf(mine, x[u][e]);  // (NaN left out)
  const float m = wave_max_all(mine), mu = m == -INFINITY ? 0.f : m;
  float r = 0.f, t = 0.f;
  int same = 0;
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float d = x[u][e] - mu;
      const bool is = x[u][e] == m;
      const float w = is ? 0.f : exp_of(d);
      same += is;
      r += w;
      t += w * fmaxf(d, -1e4f);  // (of -inf: nothing)
    }
  r = wave_sum_all(r);
  t = wave_sum_all(t);
  const float more = wave_sum_all((float)same) - 1.f;
  if (lane == 0) wave_sums[wave] = Sums{m, m == -INFINITY ? r : r + more, t};
  if (top > 0) {
    const uint32_t u = ordered(mine);
    uint32_t floor = 0;
    for (int b = 31; b >= 16; --b) {
      const uint32_t next = floor | 1u << b;
      floor = __popcll(__ballot(u >= next)) >= top ? next : floor;
    }
    if (lane == 0) wave_floor[wave] = floor;
    if (tid == 0) count = 0;
  }
  __syncthreads();
  const int64_t part = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (tid == 0) {
    float M = -INFINITY;
    int p = 0;
    for (int k = 0; k < 4; ++k)
      if (wave_sums[k].m > M) M = wave_sums[k].m, p = k;
    Sums all = wave_sums[p];
    for (int k = 0; k < 4; ++k)
      if (k != p) add_part(all, wave_sums[k], M);
    parts[part] = all;
  }
  if (top == 0) return;
  uint64_t* out = lists + part * top;
  const uint32_t floor = max(max(max(wave_floor[0], wave_floor[1]), max(wave_floor[2], wave_floor[3])), 1u);
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t o = ordered(x[u][e]);
      if (o >= floor) {
        const int at = atomicAdd(&count, 1);
        if (at < kList) list[at] = entry(o, v0 + 4 * (u * kTpb + tid) + e);
      }
    }
  __syncthreads();
  const int n = count;
  if (n <= kList) {
    store_top(list, n, top, out);
    return;
  }
  // Too many (a row of the same value over and over): one after the other, each the largest below
  // the last.
  uint64_t last = ~0ull;
  for (int i = 0; i < top; ++i) {
    uint64_t b = 0;
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t o = ordered(x[u][e]);
        const uint64_t c = o ? entry(o, v0 + 4 * (u * kTpb + tid) + e) : 0;
        b = c < last && c > b ? c : b;
      }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t c = (uint64_t)__shfl_xor((unsigned long long)b, o, 64);
      b = c > b ? c : b;
    }
    if (lane == 0) best[wave] = b;
    __syncthreads();
    last = max(max(best[0], best[1]), max(best[2], best[3]));
    __syncthreads();
    if (tid == 0) out[i] = last;
  }
}

// Grid (rows): the slices of a row put together, in their order; then the tokens' log probabilities.
template <int R>
__global__ __launch_bounds__(kTpb) void logprob_merge_kernel(int V, LogprobBatch<R> jobs, int slices, int top,
                                                             const Sums* parts, const uint64_t* lists, float* lse,
                                                             float* entropy, int32_t* top_tokens, float* top_logprobs) {
  __shared__ float red[4];
  __shared__ float red_r[4], red_t[4];
  __shared__ int red_p[4];
  __shared__ uint64_t red_floor[4];
  __shared__ uint64_t list[2048];
  __shared__ uint64_t sorted[64];
  __shared__ int count;
  const spp_logprob_row job = jobs.row[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  parts += (int64_t)blockIdx.x * slices;
  float m = -INFINITY;
  int at = 0x7FFFFFFF;
  for (int s = tid; s < slices; s += kTpb) {
    const float v = parts[s].m;
    if (v > m) m = v, at = s;
  }
  const float wm = wave_max_all(m);
  const int wp = wave_min_all(m == wm ? at : 0x7FFFFFFF);
  if (lane == 0) red[wave] = wm, red_p[wave] = wp;
  if (tid == 0) count = 0;
  __syncthreads();
  const float M = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  int p = 0x7FFFFFFF;
  for (int k = 0; k < 4; ++k)
    if (red[k] == M) p = min(p, red_p[k]);
  Sums a{M, 0.f, 0.f};
  for (int s = tid; s < slices; s += kTpb) {
    const Sums v = parts[s];
    if (s == p) {
      a.r += v.r;
      a.t += v.t;
    } else {
      add_part(a, v, M);
    }
  }
  a.r = wave_sum_all(a.r);
  a.t = wave_sum_all(a.t);
  if (lane == 0) red_r[wave] = a.r, red_t[wave] = a.t;
  __syncthreads();
  const float r = red_r[0] + red_r[1] + red_r[2] + red_r[3], t = red_t[0] + red_t[1] + red_t[2] + red_t[3];
  // without a finite largest value nothing has a probability
  const bool none = M == -INFINITY && r == r, bad = !(M > -INFINITY && M < INFINITY) && !none;
  const float rest = bad ? __builtin_nanf("") : log1pf(r);
  if (tid == 0) {
    if (lse) lse[blockIdx.x] = none ? -INFINITY : M + rest;
    if (entropy) entropy[blockIdx.x] = none ? __builtin_nanf("") : rest - t / (1.f + r);
  }
  auto logprob = [&](float x) { return none ? __builtin_nanf("") : (x - M) - rest; };
  for (int i = tid; i < job.n_tokens; i += kTpb) {
    const int v = job.tokens[i];
    job.logprobs[i] = (unsigned)v < (unsigned)V ? logprob(job.logits[v]) : __builtin_nanf("");
  }
  if (top == 0) return;
  // Every slice's list is in order; what is below the last entry of any of them is not among the
  // first `top`.
  lists += (int64_t)blockIdx.x * slices * top;
  uint64_t floor = 1;
  for (int s = tid; s < slices; s += kTpb) floor = max(floor, lists[(int64_t)s * top + top - 1]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) floor = max(floor, (uint64_t)__shfl_xor((unsigned long long)floor, o, 64));
  if (lane == 0) red_floor[wave] = floor;
  __syncthreads();
  floor = max(max(red_floor[0], red_floor[1]), max(red_floor[2], red_floor[3]));
  for (int64_t i = tid; i < (int64_t)slices * top; i += kTpb) {
    const uint64_t e = lists[i];
    if (e >= floor) {
      const int k = atomicAdd(&count, 1);
      if (k < 2048) list[k] = e;
    }
  }
  __syncthreads();
  const int n = count;
  if (n <= 2048) {
    store_top(list, n, top, sorted);
  } else {  // (over 32 slices whose lists interleave: one after the other)
    uint64_t last = ~0ull;
    for (int i = 0; i < top; ++i) {
      uint64_t b = 0;
      for (int64_t k = tid; k < (int64_t)slices * top; k += kTpb) {
        const uint64_t e = lists[k];
        b = e < last && e > b ? e : b;
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) b = max(b, (uint64_t)__shfl_xor((unsigned long long)b, o, 64));
      if (lane == 0) red_floor[wave] = b;
      __syncthreads();
      last = max(max(red_floor[0], red_floor[1]), max(red_floor[2], red_floor[3]));
      __syncthreads();
      if (tid == 0) sorted[i] = last;
    }
  }
  __syncthreads();
  for (int i = tid; i < top; i += kTpb) {
    const uint64_t e = sorted[i];
    top_tokens[(int64_t)blockIdx.x * top + i] = e ? (int32_t)~(uint32_t)e : -1;
    top_logprobs[(int64_t)blockIdx.x * top + i] = e ? logprob(unordered((uint32_t)(e >> 32))) : -INFINITY;
  }
}

int slices_of(int vocab) { return (vocab + 3 + kSlice - 1) / kSlice; }  // whatever the row's alignment

template <int R>
void launch_rows(int m, int vocab, const spp_logprob_row* rows, int top, Sums* parts, uint64_t* lists, float* lse,
                 float* entropy, int32_t* top_tokens, float* top_logprobs, hipStream_t st) {
  LogprobBatch<R> b{};
  std::copy_n(rows, m, b.row);
  const int slices = slices_of(vocab);
  SPP_LAUNCH((logprob_slice_kernel<R>), dim3(slices, m), dim3(kTpb), 0, st, vocab, b, top, parts, lists);
  SPP_LAUNCH((logprob_merge_kernel<R>), dim3(m), dim3(kTpb), 0, st, vocab, b, slices, top, parts, lists, lse, entropy,
             top_tokens, top_logprobs);
}

}  // namespace

namespace k {

size_t logprob_work_bytes(int n, int vocab, int top) {
  const size_t slices = (size_t)n * slices_of(vocab);
  return (slices * sizeof(Sums) + 15) / 16 * 16 + slices * top * sizeof(uint64_t);
}

hipError_t logprobs(int n, int vocab, const spp_logprob_row* rows, int top, int32_t* top_tokens, float* top_logprobs,
                    float* lse, float* entropy, void* work, hipStream_t st) {
  const int slices = slices_of(vocab);
  Sums* parts = static_cast<Sums*>(work);
  uint64_t* lists = reinterpret_cast<uint64_t*>(static_cast<char*>(work) +
                                                ((size_t)n * slices * sizeof(Sums) + 15) / 16 * 16);
  const int launches = (n - 1) / kRows + 1, step = (n - 1) / launches + 1;  // (of like size)
  for (int r0 = 0; r0 < n; r0 += step) {
    const int m = std::min(step, n - r0);
    const int64_t p = (int64_t)r0 * slices, t = (int64_t)r0 * top;
    (m == 1 ? launch_rows<1> : launch_rows<kRows>)(m, vocab, rows + r0, top, parts + p, lists + p * top,
                                                   lse ? lse + r0 : nullptr, entropy ? entropy + r0 : nullptr,
                                                   top_tokens + t, top_logprobs + t, st);
  }
  return hipGetLastError();
}

}  // namespace k
}  // namespace spp
