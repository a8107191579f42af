// Log probabilities of rows of fp32 logits: of given tokens, their entropy, and the top alternatives.
//
//   m = max x,  R = sum over the others of e^(x - m),  lse = m + log(1 + R)
//   log p_t = (x_t - m) - log(1 + R),  H = log(1 + R) - (sum e^(x - m) (x - m)) / (1 + R)
// The largest logit is left out of R (one of them, where there are several) so that nothing
// cancels: a token of probability near one keeps the relative precision of its log probability, and H is a sum
// of terms of one sign.  (Terms below 2^-126, the smallest normal number, may be lost.)
//
// Bound by memory: a row is read once, into registers, a slice of it to a workgroup; a second launch puts
// the slices together (a row of one slice is done in the first).
//
// The alternatives go through a floor that all of them reach: where n_top groups of tokens have largest
// values that reach a number, so do the n_top largest.  A slice leaves the largest value of
// every group of 32 tokens, a 32nd of what it reads, with no work on alternatives of its own; the merge finds the
// floor, reads again the few groups that reach it, and counts the order of the few values that do.  Ties go to the
// lower index: an entry of that list is the value's bits, made to order as unsigned integers, above
// the complement of the index.  (With a list in order from every slice instead: 64 rows of 128256 with 8
// alternatives 11.8 us and 4.6 of merge, with 50 14.2 and 6.1, one row with 50 6.6 and 77; without any 7.8 and 3.3.)
//
// Measured: 64 rows of 128256, 33 MB, read in 8.0 us (4.1 TB/s) and merged in 6.7 with 8 alternatives; 17 rows of
// 152063, half of each masked, 4.7 and 9.1 with 50; one row 3.1 and 6.0 with 20; one of 4096, one launch, 4.2.  The merge is
// a chain of waits (two loads, five barriers, a few LDS round trips and 700 instructions a wave: 13000 cycles), and
// what it waits for is not the fetch of its code: a part run twice in a row takes as long again.
#include <algorithm>

#include "common.hpp"
#include "floors.hpp"
#include "paged.hpp"

namespace spp {
namespace {

constexpr int kTpb = 256;
constexpr int kMergeTpb = 1024;                 // of the merge: few instructions a thread between its waits
constexpr int kGroup = 32;                      // tokens of a group: 8 units
// Entries of the list of alternatives, and groups they are in.  The values of fewer than n_top groups always fit,
// and more entries than that are of more than n_top groups.
constexpr int kList = 2048;
static_assert(kList / kGroup >= SPP_MAX_TOP, "the values of n_top groups");
constexpr int kHeld = 8;                        // groups a thread of the merge keeps in registers,
constexpr int kNear = 5;                        // of which the last three are of rows over 163840 tokens
constexpr int kRows = 96;                       // rows of a launch, within 4 KB of arguments
template <int R>
struct LogprobBatch {
  spp_logprob_row row[R];
};
static_assert(sizeof(LogprobBatch<kRows>) + 96 <= 4096, "a kernel's argument");

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

// A number that c lanes of the wave reach, and of values that differ few more, whatever their size and spread (0: so many
// have no value); hi: the wave's largest.
__device__ __forceinline__ uint32_t wave_floor(uint32_t u, uint32_t hi, int c) {
  if (__popcll(__ballot(u != 0)) < c) return 0;
  const int least = wave_min_all((int)((u ? u : ~0u) ^ 0x80000000u));  // (the order of signed integers)
  return narrow_floor((uint32_t)least ^ 0x80000000u, __builtin_amdgcn_readfirstlane(hi), c,
                      [&](uint32_t m) { return __popcll(__ballot(u >= m)); });
}

// A number that `top` of the workgroup's threads' values reach, W <= 16 waves: with c a Wth of `top`, what
// top / c of the waves' floors of c reach, or, where so many waves have too few values (a mask, or the row's
// end), the largest of their floors of `top`, or the lowest number.  All of the workgroup; `lds` 2 W words.
template <int W>
__device__ __forceinline__ float workgroup_floor(float mine, float wave_most, int top, uint32_t* lds) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int c = (top + W - 1) / W, need = (top + c - 1) / c;
  const uint32_t u = ordered(mine), hi = ordered(wave_most), f = c == 1 ? hi : wave_floor(u, hi, c);
  if (lane == 0) lds[wave] = f;
  __syncthreads();
  // the floor that has need - 1 others above it (equal ones in order)
  const uint32_t own = lds[lane % W];
  int above = 0;
#pragma unroll
  for (int k = 0; k < W; ++k) {
    const uint32_t o = lds[k];
    above += o > own || (o == own && k < lane % W);
  }
  const int at = __ffsll((unsigned long long)__ballot(above == need - 1)) - 1;
  uint32_t floor = (uint32_t)__builtin_amdgcn_readlane((int)own, at);
  if (floor == 0) {
    const uint32_t g = wave_floor(u, hi, top);
    if (lane == 0) lds[W + wave] = g;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < W; ++k) floor = max(floor, lds[W + k]);
  }
  return floor >= 0x00800000u ? unordered(floor) : -3.402823466e38f;
}

// Sum over the four lanes of a quad.
__device__ __forceinline__ int quad_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, true);  // lanes 1 0 3 2
  return v + __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, true);  // lanes 2 3 0 1
}
// The first `top` entries of `list` in order to out (0 behind the last): four threads count how many are
// above an entry.  All of the workgroup.
__device__ __forceinline__ void store_top(const uint64_t* list, int n, int top, uint64_t* out) {
  const int part = threadIdx.x & 3;
  for (int i0 = 0; i0 < n; i0 += blockDim.x / 4) {
    const int i = i0 + (threadIdx.x >> 2);
    const uint64_t e = list[min(i, n - 1)];
    int rank = 0;
    for (int j0 = part; j0 - part < n; j0 += 32) {  // (eight reads on their way together)
      uint64_t o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = list[min(j0 + 4 * k, kList - 1)];
#pragma unroll
      for (int k = 0; k < 8; ++k) rank += j0 + 4 * k < n && o[k] > e;
    }
    rank = quad_sum(rank);
    if (i < n && part == 0 && rank < top) out[rank] = e;
  }
  for (int i = n + (int)threadIdx.x; i < top; i += blockDim.x) out[i] = 0;
}

// The wave's lanes append item(j) to a list of `cap` entries for every j of N with has(j): one addition to
// its length for all.  (Over `cap` the length still grows.)
template <int N, typename H, typename F>
__device__ __forceinline__ void append(int* length, int cap, H has, F put) {
  uint64_t who[N];
  int total = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    who[j] = __ballot(has(j));
    total += __popcll(who[j]);
  }
  if (total == 0) return;
  int at = 0;
  if ((threadIdx.x & 63) == 0) at = atomicAdd(length, total);
  at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (who[j]) {
      const int mine = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(who[j] >> 32),
                                                      __builtin_amdgcn_mbcnt_lo((uint32_t)who[j], 0u));
      if (has(j) && mine < cap) put(j, mine);
      at += __popcll(who[j]);
    }
}

// Where a row starts against 16-byte boundaries: unit u of four tokens starts at token 4 u - a, the
// whole ones from lo to hi (none: hi < lo).
struct RowUnits {
  const float* src;
  int V, a, lo, hi;
  __device__ __forceinline__ RowUnits(const float* s, int v) : src(s), V(v) {
    a = (int)((reinterpret_cast<uintptr_t>(s) & 15) / 4);
    lo = a ? 4 - a : 0;
    hi = ((V + a) & ~3) - 4 - a;
  }
  // The same of a row that has a whole unit: one load whatever t is, and others only at the row's ends.
  __device__ __forceinline__ void load_long(int t, float (&x)[4]) const {
    const float4 q = *reinterpret_cast<const float4*>(src + min(max(t, lo), hi));
    x[0] = q.x; x[1] = q.y; x[2] = q.z; x[3] = q.w;
    if (t < lo || t > hi) load(t, x);
  }
  // The unit that starts at token t; -inf outside the row.
  __device__ __forceinline__ void load(int t, float (&x)[4]) const {
    float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
    if (t >= lo && t <= hi) {
      q = *reinterpret_cast<const float4*>(src + t);
    } else if (t + 3 >= 0 && t < V) {
      q.x = src[min(max(t, 0), V - 1)];
      q.y = src[min(max(t + 1, 0), V - 1)];
      q.z = src[min(max(t + 2, 0), V - 1)];
      q.w = src[min(max(t + 3, 0), V - 1)];
    }
    const float f[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = t + e >= 0 && t + e < V ? f[e] : -INFINITY;
  }
};

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

// What every log probability of a row is formed from: log p = (x - m) - rest.
struct RowLog {
  float m, rest;
  __device__ __forceinline__ float operator()(float x) const { return (x - m) - rest; }
};

// A row's sums, and its tokens' log probabilities.  All of the workgroup.
__device__ __forceinline__ RowLog finish_sums(const spp_logprob_row& job, int64_t row, int V, const Sums& a, Given g,
                                              const LogprobOut& out) {
  // without a finite largest value nothing has a probability
  const bool none = a.m == -INFINITY && a.r == a.r, bad = !(a.m > -INFINITY && a.m < INFINITY);
  const float nan = __builtin_nanf("");
  const RowLog log{a.m, bad ? nan : log1pf(a.r)};
  const int tid = threadIdx.x, step = blockDim.x;
  if (tid == 0) {
    if (out.lse) out.lse[row] = none ? -INFINITY : a.m + log.rest;
    if (out.entropy) out.entropy[row] = log.rest - a.t / (1.f + a.r);
  }
  for (int i = tid; i < job.n_tokens; i += step) {
    job.logprobs[i] = (unsigned)g.token < (unsigned)V ? log(g.logit) : nan;
    if (i + step < job.n_tokens) {
      g.token = job.tokens[i + step];
      g.logit = job.logits[min(max(g.token, 0), V - 1)];
    }
  }
  return log;
}
// Its alternatives, in order.
__device__ __forceinline__ void finish_top(int64_t row, const RowLog& log, const uint64_t* sorted, int top,
                                           const LogprobOut& out) {
  for (int i = threadIdx.x; i < top; i += blockDim.x) {
    const uint64_t e = sorted[i];
    out.top_tokens[row * top + i] = e ? (int32_t)~(uint32_t)e : -1;
    out.top_logprobs[row * top + i] = e ? log(unordered((uint32_t)(e >> 32))) : -INFINITY;
  }
}

// Rows in which too many values reach the floor (the same value over and over, as behind a mask's finite
// fill): the largest number that `top` values reach, bit by bit.  count(u): how many of the wave's values reach
// u.  All of the workgroup; `lds` 2 W numbers.  (A row of 128256, 20 alternatives: 24 us in all, 46 where the equals
// begin in its middle; 252 and 556 by bins of eight bits over the whole row.)
template <int W, typename C>
__device__ __forceinline__ uint32_t exact_floor(int top, int* lds, C count) {
  uint32_t v = 0;
  for (int b = 31; b >= 0; --b) {
    const uint32_t next = v | 1u << b;
    const int mine = count(next);
    int* at = lds + (b & 1) * W;  // (the other half may still be read)
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = mine;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) all += at[k];
    if (all >= top) v = next;
  }
  return v;
}
// The first `need` tokens whose value is v, as entries of the list from `at` on: the row in order, until they
// are found.  All of the workgroup; `lds` 2 W numbers.
template <int W>
__device__ void append_equal(const RowUnits& row, uint32_t v, int need, uint64_t* list, int at, int* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int had = 0;
  for (int i0 = 0, k = 0; 4 * i0 - row.a < row.V && had < need; i0 += 64 * W, k ^= 1) {
    const int t = 4 * (i0 + (int)threadIdx.x) - row.a;
    float x[4];
    row.load(t, x);
    int before = 0, mine = 0, all = 0;  // equals in lanes below, of the lane, of the wave
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool is = ordered(x[e]) == v;
      const uint64_t who = __ballot(is);
      before += __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
      all += __popcll(who);
      mine |= is ? 1 << e : 0;
    }
    if (lane == 0) lds[k * W + wave] = all;  // (the other half may still be read)
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const int n = lds[k * W + j];
      before += j < wave ? n : 0;
      total += n;
    }
    before += had;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (mine >> e & 1) {
        if (before < need) list[at + before] = entry(v, t + e);
        ++before;
      }
    had += total;
  }
}

// The slice's tokens into registers.
template <int UNITS>
__device__ __forceinline__ void load_slice(const RowUnits& row, int v0, float (&x)[UNITS][4]) {
  const int tid = threadIdx.x;
  if (v0 >= row.lo && v0 + UNITS * 4 * kTpb - 4 <= row.hi) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const float4 q = *reinterpret_cast<const float4*>(row.src + v0 + 4 * (u * kTpb + tid));
      x[u][0] = q.x; x[u][1] = q.y; x[u][2] = q.z; x[u][3] = q.w;
    }
  } else {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) row.load(v0 + 4 * (u * kTpb + tid), x[u]);
  }
}

// The slice's sums, in every thread; `mine` is the thread's largest value, wave_most the wave's.
//
// A thread's own sums are against its largest value so far, eight tokens at a time: they are formed while
// the later loads are on their way, with nothing to wait for in other lanes.
template <int UNITS>
__device__ __forceinline__ Sums slice_sums(const float (&x)[UNITS][4], float& mine, float& wave_most, Sums* wave_sums) {
  mine = -INFINITY;  // (NaN left out)
  float r = 0.f, t = 0.f;
#pragma unroll
  for (int u0 = 0; u0 < UNITS; u0 += 2) {
    float most = mine;
#pragma unroll
    for (int u = u0; u < u0 + 2; ++u)
      most = fmaxf(most, fmaxf(fmaxf(x[u][0], x[u][1]), fmaxf(x[u][2], x[u][3])));
    const float mu = most == -INFINITY ? 0.f : most;
    if (u0) {
      const float back = mine - mu, w = exp_of(back);
      t = w * (t + r * fmaxf(back, -1e4f));
      r *= w;
    }
    mine = most;
#pragma unroll
    for (int u = u0; u < u0 + 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float d = x[u][e] - mu, w = exp_of(d);
        r += w;
        t += w * fmaxf(d, -1e4f);  // (of -inf: nothing)
      }
  }
  // The wave's: all terms, the largest one's 1 among them; where it outweighs the others it is left
  // out instead of taken off.
  const float m = wave_max_all(mine), mu = m == -INFINITY ? 0.f : m;
  wave_most = m;
  {
    const float back = mine - mu, w = exp_of(back);
    t = wave_sum_all(w * (t + r * fmaxf(back, -1e4f)));
    r = wave_sum_all(w * r);
  }
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
  if ((threadIdx.x & 63) == 0) wave_sums[threadIdx.x >> 6] = Sums{m, r, t};
  __syncthreads();
  float M = -INFINITY;
  int p = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (wave_sums[k].m > M) M = wave_sums[k].m, p = k;
  Sums all = wave_sums[p];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k != p) add_part(all, wave_sums[k], M);
  return all;
}

// Grid (slices, rows), UNITS * 1024 tokens a slice: unit u of the slice to thread u % 256.  Leaves the
// slice's sums and, with `maxima`, the largest values of its groups: of 8 units a thread's, of 2 those
// of four neighbours.
template <int UNITS, int R>
__global__ __launch_bounds__(kTpb) void logprob_slice_kernel(int V, LogprobBatch<R> jobs, Sums* parts, float* maxima) {
  static_assert(UNITS == 8 || UNITS == 2, "groups of 8 units");
  constexpr int S = UNITS * 4 * kTpb, GROUPS = S / kGroup;
  __shared__ Sums wave_sums[4];
  const RowUnits row(jobs.row[blockIdx.y].logits, V);
  const int tid = threadIdx.x;
  const int64_t part = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  float x[UNITS][4], mine, most;
  load_slice<UNITS>(row, (int)blockIdx.x * S - row.a, x);
  const Sums all = slice_sums<UNITS>(x, mine, most, wave_sums);
  if (tid == 0) parts[part] = all;
  if (!maxima) return;
  maxima += part * GROUPS;
  if constexpr (UNITS == 8) {
    maxima[tid] = mine;
  } else {
    mine = fmaxf(mine, __shfl_xor(mine, 1, 64));
    mine = fmaxf(mine, __shfl_xor(mine, 2, 64));
    if (tid % 4 == 0) maxima[tid / 4] = mine;
  }
}
// The first token of unit j of group g of a row.
template <int UNITS>
__device__ __forceinline__ int group_token(int a, int g, int j) {
  constexpr int GROUPS = UNITS * 4 * kTpb / kGroup;
  const int slice = g / GROUPS, k = g % GROUPS;
  const int unit = UNITS == 8 ? j * kTpb + k : (j >> 2) * kTpb + 4 * k + (j & 3);
  return slice * (UNITS * 4 * kTpb) - a + 4 * unit;
}

// Grid (rows): a row of one slice, start to end.
template <int R>
__global__ __launch_bounds__(kTpb) void logprob_row_kernel(int V, LogprobBatch<R> jobs, int top, LogprobOut out) {
  constexpr int UNITS = 8, W = kTpb / 64;
  __shared__ Sums wave_sums[W];
  __shared__ uint32_t floors[2 * W];
  __shared__ uint64_t list[kList], sorted[SPP_MAX_TOP];
  __shared__ int count, counts[2 * W];
  const spp_logprob_row job = jobs.row[blockIdx.x];
  const RowUnits row(job.logits, V);
  const int tid = threadIdx.x;
  float x[UNITS][4], mine, most;
  load_slice<UNITS>(row, -row.a, x);
  const Given given = first_given(job, V);
  if (tid == 0) count = 0;
  const Sums all = slice_sums<UNITS>(x, mine, most, wave_sums);
  if (top > 0) {
    // the values above `least`, or that and more (NaN and -inf compare false)
    auto list_from = [&](auto above) {
#pragma unroll
      for (int u = 0; u < UNITS; u += 2)
        append<8>(
            &count, kList, [&](int j) { return above(x[u + j / 4][j % 4]); },
            [&](int j, int at) {
              list[at] = entry(ordered(x[u + j / 4][j % 4]), 4 * ((u + j / 4) * kTpb + tid) + j % 4 - row.a);
            });
      __syncthreads();
    };
    const float least = workgroup_floor<W>(mine, most, top, floors);
    list_from([&](float y) { return y >= least; });
    int n = count;
    if (n > kList) {
      const uint32_t v = exact_floor<W>(top, counts, [&](uint32_t u) {
        int c = 0;
#pragma unroll
        for (int k = 0; k < UNITS; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) c += __popcll(__ballot(ordered(x[k][e]) >= u));
        return c;
      });
      if (tid == 0) count = 0;
      __syncthreads();
      list_from([&](float y) { return ordered(y) > v; });
      n = count;  // (below top)
      append_equal<W>(row, v, top - n, list, n, counts);
      n = top;
      __syncthreads();
    }
    store_top(list, n, top, sorted);
    __syncthreads();
  }
  finish_top(blockIdx.x, finish_sums(job, blockIdx.x, V, all, given, out), sorted, top, out);
}

// Grid (rows): the slices of a row put together, in their order, and its alternatives found.  What it
// takes is the waits of its steps for each other.
template <int UNITS, int R>
__global__ __launch_bounds__(kMergeTpb) void logprob_merge_kernel(int V, LogprobBatch<R> jobs, int slices, int top,
                                                                  const Sums* parts, const float* maxima,
                                                                  LogprobOut out) {
  constexpr int W = kMergeTpb / 64, GROUPS = UNITS * 4 * kTpb / kGroup;
  __shared__ float red[W], red_r[W], red_t[W];
  __shared__ int red_p[W], count[2], counts[2 * W], groups[kList];
  __shared__ uint32_t floors[2 * W];
  __shared__ uint64_t list[kList], sorted[SPP_MAX_TOP];
  const spp_logprob_row job = jobs.row[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n_groups = slices * GROUPS;
  parts += (int64_t)blockIdx.x * slices;
  maxima += (int64_t)blockIdx.x * n_groups;

  // All loads go out together: a slice and a token a thread, and the groups' largest values.
  Sums own{-INFINITY, 0.f, 0.f};
  if (tid < slices) own = parts[tid];
  const bool more = n_groups > kNear * kMergeTpb;
  float held[kHeld], mine = -INFINITY;
  if (top > 0) {
#pragma unroll
    for (int j = 0; j < kNear; ++j) held[j] = maxima[min(j * kMergeTpb + tid, n_groups - 1)];
    if (more)
#pragma unroll
      for (int j = kNear; j < kHeld; ++j) held[j] = maxima[min(j * kMergeTpb + tid, n_groups - 1)];
  }
  const Given given = first_given(job, V);
  if (tid < 2) count[tid] = 0;

  float m = own.m;
  for (int s = tid + kMergeTpb; s < slices; s += kMergeTpb) m = fmaxf(m, parts[s].m);
  const float wm = wave_max_all(m);
  if (lane == 0) red[wave] = wm;
  float least = 0.f;
  if (top > 0) {
    auto most_of = [&](int h, int to) {
#pragma unroll
      for (int j = h; j < to; ++j) {
        held[j] = j * kMergeTpb + tid < n_groups ? held[j] : -INFINITY;
        mine = fmaxf(mine, held[j]);
      }
    };
    most_of(0, kNear);
    if (more) most_of(kNear, kHeld);
    for (int g = kHeld * kMergeTpb + tid; g < n_groups; g += kMergeTpb) mine = fmaxf(mine, maxima[g]);
    least = workgroup_floor<W>(mine, wave_max_all(mine), top, floors);
  } else {
    __syncthreads();
  }
  float M = red[0];
#pragma unroll
  for (int k = 1; k < W; ++k) M = fmaxf(M, red[k]);
  // (every term, the largest one's among them)
  Sums a{M, 0.f, 0.f};
  if (tid < slices) add_part(a, own, M);
  for (int s = tid + kMergeTpb; s < slices; s += kMergeTpb) add_part(a, parts[s], M);
  a.r = wave_sum_all(a.r);
  a.t = wave_sum_all(a.t);
  if (lane == 0) red_r[wave] = a.r, red_t[wave] = a.t;
  auto groups_from = [&](auto above) {
    append<kNear>(
        count + 1, kList, [&](int j) { return above(held[j]); },
        [&](int j, int at) { groups[at] = j * kMergeTpb + tid; });
    if (more)
      append<kHeld - kNear>(
          count + 1, kList, [&](int j) { return above(held[kNear + j]); },
          [&](int j, int at) { groups[at] = (kNear + j) * kMergeTpb + tid; });
    for (int g0 = kHeld * kMergeTpb; g0 < n_groups; g0 += kMergeTpb) {
      const int g = g0 + tid;
      const float y = g < n_groups ? maxima[g] : -INFINITY;
      append<1>(
          count + 1, kList, [&](int) { return above(y); }, [&](int, int at) { groups[at] = g; });
    }
  };
  if (top > 0) {
    groups_from([&](float y) { return y >= least; });
  }
  __syncthreads();
  const RowUnits row(job.logits, V);
  int n = top > 0 ? 8 * min(count[1], kList + 1) : 0;  // units of the groups
  const bool listed = n <= 8 * kList;
  float x[4];
  int t = 0;
  auto unit_at = [&](int i) {
    t = i < n ? group_token<UNITS>(row.a, groups[min(i, n - 1) >> 3], i & 7) : V;
    row.load_long(t, x);
  };
  // (the first units are on their way already)
  auto list_from = [&](auto above) {
    for (int i0 = 0; i0 < n; i0 += kMergeTpb) {
      append<4>(
          count, kList, [&](int j) { return above(x[j]); },
          [&](int j, int at) { list[at] = entry(ordered(x[j]), t + j); });
      if (i0 + kMergeTpb < n) unit_at(i0 + kMergeTpb + tid);
    }
    __syncthreads();
  };
  if (top > 0 && listed) unit_at(tid);
  a.r = red_r[0];
  a.t = red_t[0];
#pragma unroll
  for (int k = 1; k < W; ++k) a.r += red_r[k], a.t += red_t[k];
  if (a.m == -INFINITY) {
    // (no term, or NaN)
  } else if (a.r >= 2.f) {
    a.r -= 1.f;
  } else {
    // The largest term outweighs the others: the first slice that has it gives its R as it is.
    int at = tid < slices && own.m == M ? tid : 0x7FFFFFFF;
    for (int s = tid + kMergeTpb; s < slices; s += kMergeTpb)
      if (parts[s].m == M) at = min(at, s);
    at = wave_min_all(at);
    if (lane == 0) red_p[wave] = at;
    __syncthreads();
    int p = red_p[0];
#pragma unroll
    for (int k = 1; k < W; ++k) p = min(p, red_p[k]);
    Sums b{M, 0.f, 0.f};
    for (int s = tid; s < slices; s += kMergeTpb) {
      if (s == p)
        b.r += parts[s].r;
      else
        add_part(b, parts[s], M);
    }
    b.r = wave_sum_all(b.r);
    if (lane == 0) red[wave] = b.r;
    __syncthreads();
    a.r = red[0];
#pragma unroll
    for (int k = 1; k < W; ++k) a.r += red[k];
  }
  const RowLog log = finish_sums(job, blockIdx.x, V, a, given, out);
  if (top == 0) return;
  if (listed) list_from([&](float y) { return y >= least; });
  int found = count[0];
  if (!listed || found > kList) {
    // The groups' n_top-th largest value exactly: fewer groups are above it, so what they have above it
    // fits, and where that is not enough the rest are its equals.
    const uint32_t v = exact_floor<W>(top, counts, [&](uint32_t u) {
      int c = 0;
#pragma unroll
      for (int j = 0; j < kNear; ++j) c += __popcll(__ballot(ordered(held[j]) >= u));
      if (more)
#pragma unroll
        for (int j = kNear; j < kHeld; ++j) c += __popcll(__ballot(ordered(held[j]) >= u));
      for (int g0 = kHeld * kMergeTpb; g0 < n_groups; g0 += kMergeTpb)
        c += __popcll(__ballot(g0 + tid < n_groups && ordered(maxima[g0 + tid]) >= u));
      return c;
    });
    if (tid < 2) count[tid] = 0;
    __syncthreads();
    groups_from([&](float y) { return ordered(y) > v; });
    __syncthreads();
    n = 8 * count[1];
    if (n > 0) unit_at(tid);
    list_from([&](float y) { return ordered(y) > v; });
    found = count[0];
    if (found < top) {
      append_equal<W>(row, v, top - found, list, found, counts);
      found = top;
      __syncthreads();
    }
  }
  store_top(list, found, top, sorted);
  __syncthreads();
  finish_top(blockIdx.x, log, sorted, top, out);
}

// Tokens of a slice: 8192 where that makes one of a row, which is then done in one launch (from a graph, a row of
// 4096 with 8 alternatives 5.9 us, in two slices 8.1); else 2048 while that makes no more than 1024 workgroups (one
// row of 128256 with 20 9.1, in slices of 8192 10.0; 8 rows 9.8 and 10.5), else 8192, a quarter of the parts (64 rows
// with 8 13.3 and 13.6).
int slice_units(int n, int vocab) {
  return vocab + 3 > 8 * 4 * kTpb && (int64_t)vocab * n <= kShortSliceTokens ? 2 : 8;
}
int slices_of(int units, int vocab) {  // whatever the row's alignment
  return (vocab + 3 + units * 4 * kTpb - 1) / (units * 4 * kTpb);
}

template <int UNITS, int R>
void launch_rows(int m, int vocab, const spp_logprob_row* rows, int top, Sums* parts, float* maxima,
                 const LogprobOut& out, hipStream_t st) {
  LogprobBatch<R> b{};
  std::copy_n(rows, m, b.row);
  const int slices = slices_of(UNITS, vocab);
  if (slices == 1) {
    SPP_LAUNCH((logprob_row_kernel<R>), dim3(m), dim3(kTpb), 0, st, vocab, b, top, out);
    return;
  }
  SPP_LAUNCH((logprob_slice_kernel<UNITS, R>), dim3(slices, m), dim3(kTpb), 0, st, vocab, b, parts,
             top > 0 ? maxima : nullptr);
  SPP_LAUNCH((logprob_merge_kernel<UNITS, R>), dim3(m), dim3(kMergeTpb), 0, st, vocab, b, slices, top, parts, maxima, out);
}

size_t parts_bytes(int n, int slices) { return ((size_t)n * slices * sizeof(Sums) + 15) / 16 * 16; }

}  // namespace

namespace k {

size_t logprob_work_bytes(int n, int vocab, int top) {
  const int units = slice_units(n, vocab), slices = slices_of(units, vocab);
  return parts_bytes(n, slices) + (top ? (size_t)n * slices * (units * 4 * kTpb / kGroup) * sizeof(float) : 0);
}

hipError_t logprobs(int n, int vocab, const spp_logprob_row* rows, int top, int32_t* top_tokens, float* top_logprobs,
                    float* lse, float* entropy, void* work, hipStream_t st) {
  const int units = slice_units(n, vocab), slices = slices_of(units, vocab);
  Sums* parts = static_cast<Sums*>(work);
  float* maxima = reinterpret_cast<float*>(static_cast<char*>(work) + parts_bytes(n, slices));
  const int launches = (n - 1) / kRows + 1, step = (n - 1) / launches + 1;  // (of like size)
  for (int r0 = 0; r0 < n; r0 += step) {
    const int m = std::min(step, n - r0);
    const int64_t p = (int64_t)r0 * slices, t = (int64_t)r0 * top;
    const LogprobOut out{top_tokens + t, top_logprobs + t, lse ? lse + r0 : nullptr, entropy ? entropy + r0 : nullptr};
    const auto launch = units == 2 ? (m == 1 ? launch_rows<2, 1> : launch_rows<2, kRows>)
                                   : (m == 1 ? launch_rows<8, 1> : launch_rows<8, kRows>);
    launch(m, vocab, rows + r0, top, parts + p, maxima + p * (units * 4 * kTpb / kGroup), out, st);
  }
  return hipGetLastError();
}

}  // namespace k
}  // namespace spp
