// Log probabilities of rows of fp32 logits: of given tokens, their entropy, and the top alternatives.
//
//   m = max x,  R = sum over the others of e^(x - m),  lse = m + log(1 + R)
//   log p_t = (x_t - m) - log(1 + R),  H = log(1 + R) - (sum e^(x - m) (x - m)) / (1 + R)
// The largest logit is left out of R (one of them, where there are several) so that nothing
// cancels: a token of probability near one keeps the relative precision of its log probability, and H is a sum
// of terms of one sign.
//
// Bound by memory: a row is read once, into registers.  A workgroup takes a slice of a row, a
// second launch puts the slices together (a row of one slice is done in the first).
//
// The alternatives go through a floor that all of them reach.  The lanes of a wave hold their
// largest values; the largest value that c of them reach is found bit by bit with ballots, on the upper half
// of the bits.  With c a quarter of n_top the least of the four waves' is a floor of the slice, with
// c = n_top each wave's is (the floor where a wave has too few values).  What reaches it goes to a short
// list, whose order is counted.  Ties go to the lower index: an entry of a list is the value's bits,
// made to order as unsigned integers, above the complement of the index.
#include <algorithm>

#include "common.hpp"
#include "paged.hpp"

namespace spp {
namespace {

constexpr int kTpb = 256;
constexpr int kList = 1024;                     // entries of a slice's short list
constexpr int kMergeList = 2048;                // entries of all lists of a row that are merged in LDS
constexpr int kRows = 96;                       // rows of a launch, within 4 KB of arguments
template <int R>
struct LogprobBatch {
  spp_logprob_row row[R];
};
static_assert(sizeof(LogprobBatch<kRows>) + 96 <= 4096, "a kernel's argument");

// Where the results go, and what the slices leave for the merge.
struct LogprobOut {
  int32_t* top_tokens;
  float* top_logprobs;
  float *lse, *entropy;
};

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

// The largest value, lower half zero, that c lanes of the wave reach (0: so many have none).
__device__ __forceinline__ uint32_t wave_floor(uint32_t u, int c) {
  uint32_t floor = 0;
#pragma unroll
  for (int b = 31; b >= 16; --b) {
    const uint32_t next = floor | 1u << b;
    floor = __popcll(__ballot(u >= next)) >= c ? next : floor;
  }
  return floor;
}

// The entries of `list` in order, the first `top` to out (0 behind the last).  All of the workgroup.
__device__ __forceinline__ void store_top(const uint64_t* list, int n, int top, uint64_t* out) {
  for (int i = threadIdx.x; i < n; i += kTpb) {
    const uint64_t e = list[i];
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) rank += list[j] > e;
    if (rank < top) out[rank] = e;
  }
  for (int i = n + (int)threadIdx.x; i < top; i += kTpb) out[i] = 0;
}

__device__ __forceinline__ uint64_t wave_most(uint64_t b) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) b = max(b, (uint64_t)__shfl_xor((unsigned long long)b, o, 64));
  return b;
}

// The first of a thread's tokens and its logit, on their way while the rest is computed.
struct Given {
  int token;
  float logit;
};
__device__ __forceinline__ Given first_given(const spp_logprob_row& job, int V) {
  Given g{-1, 0.f};
  if (job.n_tokens > 0) {
    g.token = job.tokens[min((int)threadIdx.x, job.n_tokens - 1)];
    g.logit = job.logits[min(max(g.token, 0), V - 1)];
  }
  return g;
}

// A row's results from its sums and its alternatives in order.  All of the workgroup.
__device__ __forceinline__ void finish_row(const spp_logprob_row& job, int64_t row, int V, const Sums& a, Given g,
                                           const uint64_t* sorted, int top, const LogprobOut& out) {
  // without a finite largest value nothing has a probability
  const bool none = a.m == -INFINITY && a.r == a.r, bad = !(a.m > -INFINITY && a.m < INFINITY) && !none;
  const float nan = __builtin_nanf("");
  const float rest = bad ? nan : log1pf(a.r);
  const int tid = threadIdx.x;
  if (tid == 0) {
    if (out.lse) out.lse[row] = none ? -INFINITY : a.m + rest;
    if (out.entropy) out.entropy[row] = none ? nan : rest - a.t / (1.f + a.r);
  }
  auto logprob = [&](float x) { return none ? nan : (x - a.m) - rest; };
  for (int i = tid; i < job.n_tokens; i += kTpb) {
    job.logprobs[i] = (unsigned)g.token < (unsigned)V ? logprob(g.logit) : nan;
    if (i + kTpb < job.n_tokens) {
      g.token = job.tokens[i + kTpb];
      g.logit = job.logits[min(max(g.token, 0), V - 1)];
    }
  }
  for (int i = tid; i < top; i += kTpb) {
    const uint64_t e = sorted[i];
    out.top_tokens[row * top + i] = e ? (int32_t)~(uint32_t)e : -1;
    out.top_logprobs[row * top + i] = e ? logprob(unordered((uint32_t)(e >> 32))) : -INFINITY;
  }
}

// Grid (slices, rows), UNITS * 1024 tokens a slice.  Units of four tokens at 16-byte boundaries of the
// row, whatever its alignment, unit u of the slice to thread u % 256 (as adjust_kernel).
template <int UNITS, int R>
__global__ __launch_bounds__(kTpb) void logprob_slice_kernel(int V, LogprobBatch<R> jobs, int top, Sums* parts,
                                                             uint64_t* lists, LogprobOut out) {
  constexpr int S = UNITS * 4 * kTpb;
  __shared__ Sums wave_sums[4];
  __shared__ uint32_t floors[2][4];
  __shared__ uint64_t list[kList];
  __shared__ uint64_t sorted[SPP_MAX_TOP];
  __shared__ uint64_t best[4];
  __shared__ int count;
  const spp_logprob_row job = jobs.row[blockIdx.y];
  const float* src = job.logits;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int a = (int)((reinterpret_cast<uintptr_t>(src) & 15) / 4);
  const int v0 = (int)blockIdx.x * S - a;  // first token of the slice (before the row: none)
  float x[UNITS][4];
  const int t_lo = a ? 4 - a : 0, t_hi = ((V + a) & ~3) - 4 - a;  // the row's first and last whole unit
  if (v0 >= t_lo && v0 + S - 4 <= t_hi) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const float4 q = *reinterpret_cast<const float4*>(src + v0 + 4 * (u * kTpb + tid));
      x[u][0] = q.x; x[u][1] = q.y; x[u][2] = q.z; x[u][3] = q.w;
    }
  } else {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
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

  const bool solo = gridDim.x == 1;
  Given given{-1, 0.f};
  if (solo) given = first_given(job, V);
  float of[UNITS], mine = -INFINITY;  // largest values of a unit and of all, NaN left out
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    of[u] = fmaxf(fmaxf(x[u][0], x[u][1]), fmaxf(x[u][2], x[u][3]));
    mine = fmaxf(mine, of[u]);
  }
  const float m = wave_max_all(mine), mu = m == -INFINITY ? 0.f : m;
  // All terms, the largest one's 1 among them; where it outweighs the others it is left out
  // instead of taken off.
  float r = 0.f, t = 0.f;
#pragma unroll
  for (int u = 0; u < UNITS; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float d = x[u][e] - mu, w = exp_of(d);
      r += w;
      t += w * fmaxf(d, -1e4f);  // (of -inf: nothing)
    }
  r = wave_sum_all(r);
  t = wave_sum_all(t);
  if (m == -INFINITY) {
    // (no term, or NaN)
  } else if (r >= 2.f) {
    r -= 1.f;
  } else {
    float rest = 0.f, same = 0.f;
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool is = x[u][e] == m;
        same += is ? 1.f : 0.f;
        rest += is ? 0.f : exp_of(x[u][e] - m);
      }
    r = wave_sum_all(rest) + (wave_sum_all(same) - 1.f);
  }
  if (lane == 0) wave_sums[wave] = Sums{m, r, t};
  if (top > 0) {
    const uint32_t f = wave_floor(ordered(mine), (top + 3) / 4);
    if (lane == 0) floors[0][wave] = f;
    if (tid == 0) count = 0;
  }
  __syncthreads();
  Sums all;
  {
    float M = -INFINITY;
    int p = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (wave_sums[k].m > M) M = wave_sums[k].m, p = k;
    all = wave_sums[p];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k != p) add_part(all, wave_sums[k], M);
  }
  const int64_t part = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (!solo && tid == 0) parts[part] = all;
  uint64_t* to = solo ? sorted : lists + part * top;
  if (top > 0) {
    uint32_t floor = min(min(floors[0][0], floors[0][1]), min(floors[0][2], floors[0][3]));
    if (floor == 0) {  // (a wave with few values: a mask, or the row's end)
      const uint32_t f = wave_floor(ordered(mine), top);
      if (lane == 0) floors[1][wave] = f;
      __syncthreads();
      floor = max(max(floors[1][0], floors[1][1]), max(floors[1][2], floors[1][3]));
    }
    // (as a number to compare with; NaN compares false, -inf has to)
    const float least = floor ? unordered(floor) : -3.402823466e38f;
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
      if (of[u] >= least) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (x[u][e] >= least) {
            const int at = atomicAdd(&count, 1);
            if (at < kList) list[at] = entry(ordered(x[u][e]), v0 + 4 * (u * kTpb + tid) + e);
          }
      }
    __syncthreads();
    const int n = count;
    if (n <= kList) {
      store_top(list, n, top, to);
    } else {
      // Too many (a row of the same value over and over): one after the other, each the largest
      // below the last.
      uint64_t last = ~0ull;
      for (int i = 0; i < top; ++i) {
        uint64_t b = 0;
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t o = ordered(x[u][e]);
            const uint64_t c = o ? entry(o, v0 + 4 * (u * kTpb + tid) + e) : 0;
            b = c < last && c > b ? c : b;
          }
        b = wave_most(b);
        if (lane == 0) best[wave] = b;
        __syncthreads();
        last = max(max(best[0], best[1]), max(best[2], best[3]));
        __syncthreads();
        if (tid == 0) to[i] = last;
      }
    }
  }
  if (!solo) return;
  __syncthreads();
  finish_row(job, blockIdx.y, V, all, given, sorted, top, out);
}

// Grid (rows): the slices of a row put together, in their order.
//
// Every slice's list is in order, so j lists whose entry number p (from 0) reaches a value have j (p + 1)
// entries that do: the largest value that ceil(top / (p + 1)) of the lists' entries p reach is a floor of the
// alternatives, for every p, and the highest of those tried counts.
template <int R>
__global__ __launch_bounds__(kTpb) void logprob_merge_kernel(int V, LogprobBatch<R> jobs, int slices, int top,
                                                             const Sums* parts, const uint64_t* lists, LogprobOut out) {
  __shared__ float red[4];
  __shared__ float red_r[4], red_t[4];
  __shared__ int red_p[4];
  __shared__ uint64_t red_most[4];
  __shared__ uint64_t all[kMergeList], list[kMergeList];
  __shared__ uint64_t sorted[SPP_MAX_TOP];
  __shared__ int count;
  const spp_logprob_row job = jobs.row[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int entries = min((int64_t)slices * top, (int64_t)kMergeList + 1);
  parts += (int64_t)blockIdx.x * slices;
  lists += (int64_t)blockIdx.x * slices * top;
  // All loads go out together: a first slice and token a thread, and the lists.
  const Given given = first_given(job, V);
  Sums own{-INFINITY, 0.f, 0.f};
  if (tid < slices) own = parts[tid];
  const bool fits = top > 0 && entries <= kMergeList;
  if (fits) {
    constexpr int N = kMergeList / kTpb;
    uint64_t e[N];
#pragma unroll
    for (int j = 0; j < N; ++j) e[j] = lists[min(tid + j * kTpb, entries - 1)];
#pragma unroll
    for (int j = 0; j < N; ++j) all[tid + j * kTpb] = e[j];
  }
  float m = own.m;
  int at = m > -INFINITY ? tid : 0x7FFFFFFF;
  for (int s = tid + kTpb; s < slices; s += kTpb) {
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
    const Sums v = s == tid ? own : parts[s];
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
  uint64_t most = 1;
  if (fits) {
    // entries p of about thrice a list's share, and the last
    const int ps = min(top, 3 * top / slices + 2);
    for (int i = tid; i < slices * ps; i += kTpb) {
      const int s0 = i / ps, k = i % ps + 1 == ps ? top - 1 : i % ps, need = (top + k) / (k + 1);
      const uint64_t e = all[s0 * top + k];
      int reach = 0;
#pragma unroll 8
      for (int s = 0; s < slices; ++s) reach += all[s * top + k] >= e;
      if (reach >= need) most = max(most, e);
    }
  }
  most = wave_most(most);
  if (lane == 0) red_most[wave] = most;
  __syncthreads();
  a.r = red_r[0] + red_r[1] + red_r[2] + red_r[3];
  a.t = red_t[0] + red_t[1] + red_t[2] + red_t[3];
  if (fits) {
    const uint64_t floor = max(max(red_most[0], red_most[1]), max(red_most[2], red_most[3]));
    for (int i = tid; i < entries; i += kTpb)
      if (all[i] >= floor) list[atomicAdd(&count, 1)] = all[i];
    __syncthreads();
    store_top(list, count, top, sorted);
  } else {  // (more than fit: one after the other, each the largest below the last)
    uint64_t last = ~0ull;
    for (int i = 0; i < top; ++i) {
      uint64_t b = 0;
      for (int64_t k = tid; k < (int64_t)slices * top; k += kTpb) {
        const uint64_t e = lists[k];
        b = e < last && e > b ? e : b;
      }
      b = wave_most(b);
      __syncthreads();
      if (lane == 0) red_most[wave] = b;
      __syncthreads();
      last = max(max(red_most[0], red_most[1]), max(red_most[2], red_most[3]));
      if (tid == 0) sorted[i] = last;
    }
  }
  __syncthreads();
  finish_row(job, blockIdx.x, V, a, given, sorted, top, out);
}

// Tokens of a slice: 8192 where that makes one of a row, which is then done in one launch; else 2048
// while that makes no more than 1024 workgroups, else 8192.
int slice_units(int n, int vocab) {
  return vocab + 3 > 8 * 4 * kTpb && (int64_t)vocab * n <= kShortSliceTokens ? 2 : 8;
}
int slices_of(int units, int vocab) {  // whatever the row's alignment
  return (vocab + 3 + units * 4 * kTpb - 1) / (units * 4 * kTpb);
}
size_t work_of(int units, int n, int vocab, int top) {
  const size_t slices = (size_t)n * slices_of(units, vocab);
  return (slices * sizeof(Sums) + 15) / 16 * 16 + slices * top * sizeof(uint64_t);
}

template <int UNITS, int R>
void launch_rows(int m, int vocab, const spp_logprob_row* rows, int top, Sums* parts, uint64_t* lists, LogprobOut out,
                 hipStream_t st) {
  LogprobBatch<R> b{};
  std::copy_n(rows, m, b.row);
  const int slices = slices_of(UNITS, vocab);
  SPP_LAUNCH((logprob_slice_kernel<UNITS, R>), dim3(slices, m), dim3(kTpb), 0, st, vocab, b, top, parts, lists, out);
  if (slices > 1)
    SPP_LAUNCH((logprob_merge_kernel<R>), dim3(m), dim3(kTpb), 0, st, vocab, b, slices, top, parts, lists, out);
}

}  // namespace

namespace k {

size_t logprob_work_bytes(int n, int vocab, int top) { return work_of(slice_units(n, vocab), n, vocab, top); }

hipError_t logprobs(int n, int vocab, const spp_logprob_row* rows, int top, int32_t* top_tokens, float* top_logprobs,
                    float* lse, float* entropy, void* work, hipStream_t st) {
  const int units = slice_units(n, vocab), slices = slices_of(units, vocab);
  Sums* parts = static_cast<Sums*>(work);
  uint64_t* lists = reinterpret_cast<uint64_t*>(static_cast<char*>(work) +
                                                ((size_t)n * slices * sizeof(Sums) + 15) / 16 * 16);
  const int launches = (n - 1) / kRows + 1, step = (n - 1) / launches + 1;  // (of like size)
  for (int r0 = 0; r0 < n; r0 += step) {
    const int m = std::min(step, n - r0);
    const int64_t p = (int64_t)r0 * slices, t = (int64_t)r0 * top;
    const LogprobOut out{top_tokens + t, top_logprobs + t, lse ? lse + r0 : nullptr, entropy ? entropy + r0 : nullptr};
    const auto launch = units == 2 ? (m == 1 ? launch_rows<2, 1> : launch_rows<2, kRows>)
                                   : (m == 1 ? launch_rows<8, 1> : launch_rows<8, kRows>);
    launch(m, vocab, rows + r0, top, parts + p, lists + p * top, out, st);
  }
  return hipGetLastError();
}

}  // namespace k
}  // namespace spp
