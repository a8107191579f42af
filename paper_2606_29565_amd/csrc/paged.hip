// Paged caches: attention of one new token per sequence, the copies of pages, and the QKV
// epilogue that writes into them.
//
// Attention.  For a sequence and kv head with G query heads, over its live cells j:
//   o = sum_j p_j v_j / l,  l = sum_j p_j,  p_j = 2^(s_j - m),  s_j = scale log2(e) q.k_j,
// in one pass with the running maximum m (the sums so far are scaled by 2^(m_old - m) when it
// grows).  Each cell's key and value are read once (2 dh elements) and used by G heads: 4 G
// operations a pair of bytes in bf16, so HBM bounds it and the matrix cores, a sixteenth or
// more of whose columns are in use, keep up many times over.
//
// Both products are turned over so that nothing is exchanged between lanes but the maximum:
//   S^T = K Q^T: A = 16 keys, B = the heads' queries (16 columns, G in use);
//   O^T = V^T P^T: A = 16 dims of V^T, B = the probabilities.
// Lane (i, g) of S^T's result holds rows 4g .. 4g+3 of column i, and as the operand B of
// the second product it has to hold the E keys of reduction group g (E = 8 in bf16, 4 in
// fp32) of column i.  With row r of key tile t standing for key E (r / 4) + 4 t + r % 4 of the
// step these are the same keys: a lane's scores become its operand in place.  A step is 4 E
// keys (E / 4 tiles); every load is 16 bytes of a key's row or of E consecutive cells of a
// V^T row, straight from the page to the operand's registers: no LDS, no barrier.  E divides the
// page, so a lane finds one page for its keys and one for its values of such a step.
//
// A trip of the loop takes two of these steps (64 keys in bf16, 32 in fp32): a V^T row of a page
// of 64 cells or more is then read in whole 128-byte lines.  (One step a trip read each line in
// two halves, a trip apart, with as many cells in flight on an XCD as its L2 holds: 231 us for 64 sequences
// of U[1024, 8192] cells, 8 heads of 128, 1.14 GB, against 220, and 289 against 259 with
// loads that bypass the L2.)
// The next trip's keys are loaded once this trip's scores are formed, its values once this
// trip's sums are: one register set of each (236, with fp32 queries 252, of the 256 that two waves a SIMD have), and
// always one of the two in flight.
#include <algorithm>
#include <cmath>

#include "paged_device.hpp"

namespace spp {
namespace {

template <typename T>
constexpr int step_keys() { return 8 * Elem<T>::kPerFrag; }

// The first n of a unit's elements (E of T), the others zero.
__device__ __forceinline__ uint4 keep_first(const uint4& v, int n, bf16_t) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = n >= 2 * i + 2 ? w[i] : (n == 2 * i + 1 ? w[i] & 0xFFFFu : 0u);
  return make_uint4(o[0], o[1], o[2], o[3]);
}
__device__ __forceinline__ uint4 keep_first(const uint4& v, int n, float) {
  return make_uint4(n > 0 ? v.x : 0u, n > 1 ? v.y : 0u, n > 2 ? v.z : 0u, n > 3 ? v.w : 0u);
}

// Grid (key ranges, kv heads * head tiles, sequences).  A workgroup's range is cut among its
// waves, each of which keeps (m, l, O^T) of its own; they are merged through LDS in wave
// order, and the workgroup writes the sequence's output when its range is the only one, else
// its (unnormalized) sums and (m, l) for paged_join_kernel.
template <typename T, int DH, bool QLO>
__global__ __launch_bounds__(64 * kWaves, 2) void paged_attn_kernel(PageView v, int64_t layer_off, PagedAttn a,
                                                                 float scale2, int tiles, float* o_part,
                                                                 float2* ml_part) {
  constexpr int E = Elem<T>::kPerFrag, KT = 4 * E, KS = 2 * KT, NT = E / 4, NC = DH / (4 * E), ND = DH / 16;
  constexpr int OS = DH + 4;  // row stride of the merge buffer (its 16-byte stores hit all banks)
  __shared__ float o_lds[kWaves * 16 * OS];
  __shared__ float2 ml_lds[kWaves * 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int split = blockIdx.x, splits = gridDim.x, seq = blockIdx.z;
  const int head = blockIdx.y / tiles, tile = blockIdx.y % tiles;
  const int G = a.n_q / v.n_kv, q0 = head * G + tile * 16, nh = min(16, G - tile * 16);

  const int len = live_cells(a, v.shift, seq);
  const int range = range_cells(len, splits, KS * kWaves);
  const int r0 = split * range;
  if (r0 >= len && split > 0) return;  // (the join counts the ranges alike)
  const int r1 = min(len, r0 + range), share = range / kWaves;
  const int k_begin = r0 + wave * share, k_end = min(r1, k_begin + share);
  const bool solo = range >= len;  // (an empty sequence: range 0, this writes its zeros)

  // (a row past the last repeats that: its sums are this lane's alone and go nowhere)
  uint4 qh[NC], ql[NC];
  const int64_t q_at = (int64_t)seq * a.q_stride + (int64_t)(q0 + min(i, nh - 1)) * DH + g * E;
#pragma unroll
  for (int c = 0; c < NC; ++c) query_frag(a.q, a.q_bf16, q_at + c * KT, qh[c], ql[c], T{});
  float m = -INFINITY, l = 0.f;
  f32x4 acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int P1 = (1 << v.shift) - 1;
  const int32_t* tab = a.table + (int64_t)seq * a.table_stride;
  const int64_t page_bytes = v.page(), half = v.half();
  // this head's keys and values inside a page of this layer
  const char* kbase = v.base + layer_off + ((int64_t)head * DH << v.shift) * Elem<T>::kBytes;
  const char* vbase = kbase + half;
  const int last_page = (len - 1) >> v.shift;
  const int trips = k_begin < k_end ? (k_end - k_begin + KS - 1) / KS : 0;

  // Page numbers (not yet checked) of this lane's keys and values, by step half.
  int kp[2], vp[2], vq[2];  // next step's; and the values' of the step whose keys are issued
  auto pages = [&](int k) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int k0 = k_begin + k * KS + u * KT;
      kp[u] = tab[min((k0 + E * (i >> 2)) >> v.shift, last_page)];
      vp[u] = tab[min((k0 + E * g) >> v.shift, last_page)];
    }
  };
  uint4 kf[2][NT][NC], vf[2][ND];
  // The loads of step k's keys, after those of the next step's page numbers: so the wait for
  // these, a step on, is not one for the cells.  (A page that is not listed: page 0 is read,
  // and left out by the mask.)
  auto issue_keys = [&](int k) {
    const char* kr[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int kb = k_begin + k * KS + u * KT + E * (i >> 2);
      kr[u] = kbase + ((unsigned)kp[u] < (unsigned)v.n_pages ? kp[u] : 0) * page_bytes +
              ((kb & P1) + (i & 3)) * (DH * Elem<T>::kBytes) + g * 16;
      vq[u] = vp[u];
    }
    pages(k + 1);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < NC; ++c) kf[u][t][c] = ld_global(kr[u] + t * 4 * DH * Elem<T>::kBytes + c * 64);
  };
  int nl[2];  // live keys of this lane's blocks
  auto issue_values = [&](int k) {
    const char* vr[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int vb = k_begin + k * KS + u * KT + E * g;
      const bool ok = (unsigned)vq[u] < (unsigned)v.n_pages;
      nl[u] = ok ? min(k_end - vb, E) : 0;
      vr[u] = vbase + (ok ? vq[u] : 0) * page_bytes + (((int64_t)i << v.shift) + (vb & P1)) * Elem<T>::kBytes;
    }
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int u = 0; u < 2; ++u) vf[u][d] = ld_global(vr[u] + (((int64_t)d * 16) << v.shift) * Elem<T>::kBytes);
  };
  float s[2][E];
  auto scores = [&]() {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        f32x4 d = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          d = mma_frag(kf[u][t][c], qh[c], d, T{});
          if constexpr (QLO) d = mma_frag(kf[u][t][c], ql[c], d, T{});
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) s[u][4 * t + j] = d[j];
      }
  };
  auto fold = [&]() {
    const bool whole = __all(nl[0] == E && nl[1] == E);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < E; ++j) s[u][j] = whole || j < nl[u] ? s[u][j] * scale2 : -INFINITY;
    float top = s[0][0];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < E; ++j) top = fmaxf(top, s[u][j]);
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float mn = fmaxf(m, top);
    const float mu = mn == -INFINITY ? 0.f : mn;  // nothing live yet
    const float alpha = __builtin_amdgcn_exp2f(m - mu);
    m = mn;
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int j = 0; j < E; ++j) {
        s[u][j] = __builtin_amdgcn_exp2f(s[u][j] - mu);
        sum += s[u][j];
      }
    l = l * alpha + sum;
    if (!__all(alpha == 1.f)) {
#pragma unroll
      for (int d = 0; d < ND; ++d) acc[d] *= alpha;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint4 ph, pl;
      if constexpr (E == 8) {
        split_pair(s[u][0], s[u][1], ph.x, pl.x);
        split_pair(s[u][2], s[u][3], ph.y, pl.y);
        split_pair(s[u][4], s[u][5], ph.z, pl.z);
        split_pair(s[u][6], s[u][7], ph.w, pl.w);
      } else {
        ph = make_uint4(__float_as_uint(s[u][0]), __float_as_uint(s[u][1]), __float_as_uint(s[u][2]),
                        __float_as_uint(s[u][3]));
      }
      if (!whole) {
#pragma unroll
        for (int d = 0; d < ND; ++d) vf[u][d] = keep_first(vf[u][d], nl[u], T{});
      }
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        acc[d] = mma_frag(vf[u][d], ph, acc[d], T{});
        if constexpr (E == 8) acc[d] = mma_frag(vf[u][d], pl, acc[d], T{});
      }
    }
  };
  // The next step's keys are on their way from the moment this step's scores are formed, its
  // values from the end of this step's sums: one set of registers each.
  if (trips > 0) {
    pages(0);
    issue_keys(0);
    issue_values(0);
    for (int k = 0; k + 1 < trips; ++k) {
      scores();
      __builtin_amdgcn_sched_barrier(0);
      issue_keys(k + 1);
      __builtin_amdgcn_sched_barrier(0);
      fold();
      __builtin_amdgcn_sched_barrier(0);
      issue_values(k + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    scores();
    fold();
  }
  // l over the key groups of the step
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (g == 0) ml_lds[wave * 16 + i] = make_float2(m, l);
#pragma unroll
  for (int d = 0; d < ND; ++d)
    *reinterpret_cast<float4*>(o_lds + (wave * 16 + i) * OS + d * 16 + g * 4) =
        make_float4(acc[d][0], acc[d][1], acc[d][2], acc[d][3]);
  __syncthreads();
  for (int e = tid; e < nh * DH; e += 64 * kWaves) {
    const int h = e / DH, d = e % DH;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, ml_lds[w * 16 + h].x);
    const float mu = M == -INFINITY ? 0.f : M;
    float o = 0.f, L = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 ml = ml_lds[w * 16 + h];
      const float f = __builtin_amdgcn_exp2f(ml.x - mu);
      o += f * o_lds[(w * 16 + h) * OS + d];
      L += f * ml.y;
    }
    if (solo) {
      store_out(a, (int64_t)seq * a.out_stride + (int64_t)(q0 + h) * DH + d, L == 0.f ? 0.f : o / L);
    } else {
      const int64_t at = ((int64_t)seq * a.n_q + q0 + h) * splits + split;
      o_part[at * DH + d] = o;
      if (d == 0) ml_part[at] = make_float2(M, L);
    }
  }
}

// Grid (query heads, sequences), 256 threads: the ranges of one head joined.  Thread s first
// takes range s's factor; then DH / 4 threads cover the row and the groups of so many threads
// take the ranges in turn, four of a thread's loads in flight; the groups' sums are added in
// order.  Latency bounds it: no load waits for another.  (64 ranges of 32 heads of 128: one thread a
// column and every range in a row 20.7 us, the groups 4.2; with the length, the factors and
// the sums loaded one after the other and reductions by shuffles, 0.7 us longer than this.)
template <int DH>
__global__ __launch_bounds__(kMaxSplits) void paged_join_kernel(PagedAttn a, int shift, int splits, int unit,
                                                                const float* o_part, const float2* ml_part) {
  constexpr int COLS = DH / 4, GRPS = kMaxSplits / COLS;
  __shared__ float f_lds[kMaxSplits], w_max[4], w_sum[4];
  __shared__ float4 o_lds[GRPS][COLS];
  const int h = blockIdx.x, seq = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = tid % COLS, grp = tid / COLS;
  const int64_t at = ((int64_t)seq * a.n_q + h) * splits;
  // The length, the factors and the first sums are on their way together: of a range that the
  // length does not reach, whatever the workspace holds is loaded and left out.
  const float4* op = reinterpret_cast<const float4*>(o_part + at * DH) + col;
  float2 ml = ml_part[at + min(tid, splits - 1)];
  float4 v[4];
  auto sums = [&](int s0) {
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = op[(int64_t)min(s0 + u * GRPS, splits - 1) * COLS];
  };
  sums(grp);
  const int len = live_cells(a, shift, seq);
  const int range = range_cells(len, splits, unit);
  if (range >= len) return;  // one range: its workgroup has written the output
  const int n = (len + range - 1) / range;
  ml = tid < n ? ml : make_float2(-INFINITY, 0.f);
  float M = wave_max_all(ml.x);
  if (lane == 0) w_max[wave] = M;
  __syncthreads();
  M = fmaxf(fmaxf(w_max[0], w_max[1]), fmaxf(w_max[2], w_max[3]));
  const float f = __builtin_amdgcn_exp2f(ml.x - (M == -INFINITY ? 0.f : M));
  f_lds[tid] = f;
  const float part = wave_sum_all(f * ml.y);
  if (lane == 0) w_sum[wave] = part;
  __syncthreads();
  const float L = w_sum[0] + w_sum[1] + w_sum[2] + w_sum[3];
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = grp; s0 - grp < n; s0 += 4 * GRPS) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (s0 + u * GRPS < n) {
        const float w = f_lds[s0 + u * GRPS];
        o = make_float4(o.x + w * v[u].x, o.y + w * v[u].y, o.z + w * v[u].z, o.w + w * v[u].w);
      }
    if (s0 - grp + 4 * GRPS < n) sums(s0 + 4 * GRPS);
  }
  o_lds[grp][col] = o;
  __syncthreads();
  if (tid < DH) {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < GRPS; ++k) sum += reinterpret_cast<const float*>(o_lds[k])[tid];
    store_out(a, (int64_t)seq * a.out_stride + (int64_t)h * DH + tid, L == 0.f ? 0.f : sum / L);
  }
}

// One wave per (row, head) of the fused QKV output of a step whose rows are one token of one
// sequence each: as qkv_epilogue_kernel, with the cells written into the sequence's page.
template <typename T>
__global__ __launch_bounds__(64) void paged_epilogue_kernel(Shape s, StepView sv, int M, int64_t layer_off,
                                                            PageView v, const int32_t* table, int64_t table_stride,
                                                            const float* P, int splits, const float* ss, int nb,
                                                            const float2* rope, float* q_out) {
  const int r = blockIdx.x, hh = blockIdx.y;
  const int dh = s.dh, half = dh / 2;
  const int N = (s.n_q + 2 * s.n_kv) * dh;
  const int64_t split_stride = (int64_t)M * N;
  const int64_t pr = (int64_t)r * N + (int64_t)hh * dh;
  const int kind = hh < s.n_q ? 0 : (hh < s.n_q + s.n_kv ? 1 : 2);
  const int pos = sv.row[r].pos;
  T* cells = nullptr;  // this layer's K of the row's page
  if (kind) {
    const int page = table[(int64_t)r * table_stride + (pos >> v.shift)];
    cells = reinterpret_cast<T*>(v.base + page * v.page() + layer_off);
  }
  const int cell = pos & ((1 << v.shift) - 1);
  const float inv = row_inv(ss, r, nb, s.d, s.eps);
  for (int i = threadIdx.x; i < half; i += 64) {
    float a = add_splits(0.f, P, split_stride, splits, pr + i) * inv;
    float b = add_splits(0.f, P, split_stride, splits, pr + i + half) * inv;
    if (kind < 2) {
      const float2 cs = rope[(int64_t)r * half + i];
      const float a2 = a * cs.x - b * cs.y;
      const float b2 = a * cs.y + b * cs.x;
      a = a2;
      b = b2;
    }
    if (kind == 0) {
      q_out[((int64_t)r * s.n_q + hh) * dh + i] = a;
      q_out[((int64_t)r * s.n_q + hh) * dh + i + half] = b;
    } else if (kind == 1) {
      T* k = cells + (((int64_t)(hh - s.n_q) << v.shift) + cell) * dh;
      store_elem(k, i, a);
      store_elem(k, i + half, b);
    } else {
      T* vt = cells + v.half() / Elem<T>::kBytes + ((int64_t)(hh - s.n_q - s.n_kv) * dh << v.shift) + cell;
      store_elem(vt, (int64_t)i << v.shift, a);
      store_elem(vt, (int64_t)(i + half) << v.shift, b);
    }
  }
}

// The pages of a copy for one or a few sequences: a launch with up to about 100 bytes of
// arguments takes the host 2.8 us, with any more 3.4 to 3.9 (5 forks written and compacted,
// two such copies: 24.4 us with the long list, 21.8 so).
constexpr int kFewPages = 6;
struct FewPages {
  int32_t a[kFewPages], b[kFewPages];
};

// Grid (blocks, pages of the list): page b[y] = page a[y], an equal stretch for each block, four
// 16-byte units of a thread in flight.  No load is in a branch (past the end the last unit is
// read again), so none is waited for by itself.  (One page of 2 MiB to 64 others 25 us, 5.4 TB/s of
// writes; 16 pages moved 11.5 us, 5.8 TB/s.  Units dealt to the blocks in turn 24 and 15.5;
// with branches around the loads 44 and 21.)
template <typename L>
__global__ __launch_bounds__(256) void page_copy_kernel(PageView v, L l) {
  const int64_t bytes = v.page(), units = bytes / 16;
  const u32x4* src = reinterpret_cast<const u32x4*>(v.base + l.a[blockIdx.y] * bytes);
  u32x4* dst = reinterpret_cast<u32x4*>(v.base + l.b[blockIdx.y] * bytes);
  const int64_t per = (units + gridDim.x - 1) / gridDim.x, u0 = blockIdx.x * per, u1 = min(u0 + per, units);
  for (int64_t u = u0 + threadIdx.x; u < u1; u += 4 * 256) {
    u32x4 w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = src[min(u + k * 256, u1 - 1)];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (u + k * 256 < u1) dst[u + k * 256] = w[k];
  }
}

// Grid (pages of the list, fastest, times layers * 2 * kv heads): one head's keys or values of one
// page, to or from the session's buffer, in 16-byte units.  Of the last page only the live
// cells move.  (Neighbouring workgroups take neighbouring pages, so that the pieces of a V^T row
// are read close in time: 8100 cells of 4 layers of the 8B shape, 265 MB, into pages of 64 in 55.9 us;
// heads fastest 64.5.  Several pages to a workgroup: no shorter.  The loads pass the L2 by, where
// lines read once would only make room among the stores': 46.1 us, 5.8 TB/s, and 41.0 the other
// way, 42.8 before.  Stores that pass it too: both ways together 97.5 us for 94.9.)
template <typename T, bool TO_PAGES>
__global__ __launch_bounds__(256) void page_session_kernel(PageView v, PageList l, int n_pages, T* kv, int64_t cap,
                                                           int64_t c0, int cells) {
  constexpr int E = Elem<T>::kPerFrag;
  const int P = 1 << v.shift, dh = v.dh;
  const int pg = blockIdx.x % n_pages, hd = blockIdx.x / n_pages;
  const int head = hd % v.n_kv, which = hd / v.n_kv % 2, layer = hd / v.n_kv / 2;
  const int64_t at = c0 + (int64_t)pg * P;                 // first cell of the page
  const int live = min(P, cells - pg * P);            // its live cells
  T* page = reinterpret_cast<T*>(v.base + l.a[pg] * v.page() + (2 * layer + which) * v.half()) +
            ((int64_t)head * dh << v.shift);
  T* sess = kv + ((int64_t)(2 * layer + which) * v.n_kv + head) * cap * dh;
  if (which == 0) {  // rows of a cell: [cell][dim] on both sides
    T* s0 = sess + at * dh;
    const int n = live * dh / E;
    const u32x4* src = reinterpret_cast<const u32x4*>(TO_PAGES ? s0 : page);
    u32x4* dst = reinterpret_cast<u32x4*>(TO_PAGES ? page : s0);
    for (int u0 = threadIdx.x; u0 < n; u0 += 4 * 256) {
      u32x4 w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = __builtin_nontemporal_load(src + min(u0 + k * 256, n - 1));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (u0 + k * 256 < n) dst[u0 + k * 256] = w[k];
    }
    return;
  }
  // rows of a dim: P cells of the page, cap of the session; the live whole units, then what the
  // last unit holds of live cells (the cells past the last stay as they are)
  const int full = live / E, rs = v.shift - (E == 8 ? 3 : 2);  // 1 << rs units a row
  for (int u0 = threadIdx.x; full && u0 < dh << rs; u0 += 4 * 256) {
    u32x4 w[4];
    T *p[4], *s[4];
    bool ok[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int u = u0 + k * 256, d = u >> rs, c = u & ((1 << rs) - 1);
      ok[k] = d < dh && c < full;
      p[k] = page + (ok[k] ? ((d << v.shift) + c * E) : 0);
      s[k] = sess + at + (ok[k] ? d * cap + c * E : 0);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      w[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(TO_PAGES ? s[k] : p[k]));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (ok[k]) *reinterpret_cast<u32x4*>(TO_PAGES ? p[k] : s[k]) = w[k];
  }
  if (live % E)
    for (int d = threadIdx.x; d < dh; d += 256)
      for (int c = full * E; c < live; ++c) {
        T* p = page + ((int64_t)d << v.shift) + c;
        T* s = sess + d * cap + at + c;
        if (TO_PAGES) *p = *s; else *s = *p;
      }
}

template <typename T, int DH>
hipError_t launch_attn(const PageView& v, int64_t layer_off, const PagedAttn& a, int splits, void* work,
                       hipStream_t st) {
  const int G = a.n_q / v.n_kv, tiles = (G + 15) / 16;
  const float scale = a.scale != 0.f ? a.scale : (float)(1.0 / std::sqrt((double)DH));
  const float scale2 = (float)(scale * 1.4426950408889634);
  float* o_part = static_cast<float*>(work);
  float2* ml_part = reinterpret_cast<float2*>(o_part + (int64_t)a.n * a.n_q * splits * DH);
  const dim3 grid(splits, v.n_kv * tiles, a.n);
  if (Elem<T>::kBytes == 2 && !a.q_bf16)
    SPP_LAUNCH((paged_attn_kernel<T, DH, Elem<T>::kBytes == 2>), grid, dim3(64 * kWaves), 0, st, v, layer_off, a,
               scale2, tiles, o_part, ml_part);
  else
    SPP_LAUNCH((paged_attn_kernel<T, DH, false>), grid, dim3(64 * kWaves), 0, st, v, layer_off, a, scale2, tiles,
               o_part, ml_part);
  if (splits > 1) return k::paged_join(v, a, splits, step_keys<T>() * kWaves, o_part, ml_part, st);
  return hipGetLastError();
}

}  // namespace

namespace k {

hipError_t paged_join(const PageView& v, const PagedAttn& a, int splits, int unit, const float* o_part,
                      const float2* ml_part, hipStream_t st) {
  const dim3 grid(a.n_q, a.n), block(kMaxSplits);
  if (v.dh == 128)
    SPP_LAUNCH((paged_join_kernel<128>), grid, block, 0, st, a, v.shift, splits, unit, o_part, ml_part);
  else
    SPP_LAUNCH((paged_join_kernel<64>), grid, block, 0, st, a, v.shift, splits, unit, o_part, ml_part);
  return hipGetLastError();
}

// Ranges of a sequence and kv head.  A range is at least one step of its workgroup's waves (256
// cells in bf16, 128 in fp32).
//  - A table of two such steps at most: one range, without the second launch (a sequence of 256
//    cells, 4 heads of 64 in fp32: 6.5 us, in two ranges 7.7), and one of four where
//    the sequences and heads are 128 workgroups already (32 sequences of 1000 cells, 8 heads of
//    128 in bf16, 256 workgroups: 27.8 us, in four ranges 32.9; 16 of them 19.1 and 17.4, of 700
//    cells 14.5 and 16.0; one of them 17.7 and 9.8).  Of 8-bit codes, whose steps are shorter,
//    one range of three steps as well where heads are 64, half the bytes a step: i8, from a graph, 1 / 8 / 64 sequences
//    of 600 cells, 2 heads of 64, 6.3 / 6.4 / 6.5 us, in three ranges 6.5 / 6.7 / 8.0 (e4m3 5.6 / 5.7 / 5.9 and 6.2 / 6.4 / 7.4);
//    but 8 heads of 128, 1 / 8 / 16 of them 9.3 / 9.5 / 9.6, in three ranges 7.9 / 8.3 / 10.5 (e4m3 8.3 / 8.5 / 8.6 and
//    7.5 / 7.9 / 9.9).
//  - Else about 1024 workgroups over all, two rounds of two to a CU (three sequences of 32749
//    cells, 8 heads of 128: 77 us; aiming at 2048 83, at 4096 89), but up to four ranges of eight
//    steps or more each, which even out sequences of unequal lengths (64 of U[1024, 8192] cells,
//    8 heads of 128: 220 us; two ranges each 230, three 225, eight 219; ranges of 1024 cells at
//    most, however many, 263; 128 of up to 2000 cells: one range 125 us, two 134, four 142).
int paged_splits(const PageView& v, int n, int n_q, int max_pages) {
  const int tiles = (n_q / v.n_kv + 15) / 16;
  const int unit = (v.code ? kCodeStep : v.elem == 2 ? step_keys<bf16_t>() : step_keys<float>()) * kWaves;
  const int64_t most = (((int64_t)max_pages << v.shift) + unit - 1) / unit, wgs = (int64_t)n * v.n_kv * tiles;
  if (most <= (wgs >= 128 ? 4 : v.code && v.dh == 64 ? 3 : 2)) return 1;
  const int64_t want = std::max<int64_t>(std::min<int64_t>(4, most / 8), kSplitWorkgroups / wgs);
  return (int)std::max<int64_t>(1, std::min<int64_t>({want, most, (int64_t)kMaxSplits}));
}

size_t paged_work_bytes(const PageView& v, int n, int n_q, int max_pages) {
  const int splits = paged_splits(v, n, n_q, max_pages);
  return splits == 1 ? 0 : (size_t)n * n_q * splits * (v.dh + 2) * 4;
}

hipError_t paged_attention(const PageView& v, int layer, const PagedAttn& a, void* work, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  const int splits = paged_splits(v, a.n, a.n_q, a.max_pages);
  if (v.code) return code_attention(v, layer, a, splits, work, st);
  const int64_t off = v.layer() * layer;
  if (v.elem == 2)
    return v.dh == 128 ? launch_attn<bf16_t, 128>(v, off, a, splits, work, st)
                       : launch_attn<bf16_t, 64>(v, off, a, splits, work, st);
  return v.dh == 128 ? launch_attn<float, 128>(v, off, a, splits, work, st)
                     : launch_attn<float, 64>(v, off, a, splits, work, st);
}

hipError_t page_copy(const PageView& v, const PageList& l, int n, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  if (n > kPageBatch) return hipErrorInvalidValue;
  // 4 units a thread, at most 64 workgroups a page and about 4096 in all
  const int64_t blocks = (v.page() / 16 + 1023) / 1024;
  const int per = (int)std::min<int64_t>(blocks, std::max(64, 4096 / n));
  if (n <= kFewPages) {
    FewPages f{};
    std::copy_n(l.a, n, f.a);
    std::copy_n(l.b, n, f.b);
    SPP_LAUNCH((page_copy_kernel<FewPages>), dim3(per, n), dim3(256), 0, st, v, f);
  } else {
    SPP_LAUNCH((page_copy_kernel<PageList>), dim3(per, n), dim3(256), 0, st, v, l);
  }
  return hipGetLastError();
}

hipError_t page_session(const PageView& v, const PageList& l, int n, void* kv, int64_t cap, int64_t c0, int cells,
                        bool to_pages, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  if (n > kPageBatch) return hipErrorInvalidValue;
  if (v.code) return code_session(v, l, n, kv, cap, c0, cells, to_pages, st);
  const dim3 grid(v.n_layers * 2 * v.n_kv * n), block(256);
#define SPP_SESSION(T, D) \
  SPP_LAUNCH((page_session_kernel<T, D>), grid, block, 0, st, v, l, n, static_cast<T*>(kv), cap, c0, cells)
  if (v.elem == 2) {
    if (to_pages) SPP_SESSION(bf16_t, true); else SPP_SESSION(bf16_t, false);
  } else {
    if (to_pages) SPP_SESSION(float, true); else SPP_SESSION(float, false);
  }
#undef SPP_SESSION
  return hipGetLastError();
}

hipError_t paged_epilogue(const Shape& s, const StepView& sv, int n_rows, int layer, const PageView& v,
                          const int32_t* table, int64_t table_stride, const float* partials, int splits,
                          const float* ss, const float2* rope, float* q_out, hipStream_t st) {
  if (v.code)
    return code_epilogue(s, sv, n_rows, layer, v, table, table_stride, partials, splits, ss, rope, q_out, st);
  const dim3 grid(n_rows, s.n_q + 2 * s.n_kv);
  const int64_t off = v.layer() * layer;
  if (s.bf16)
    SPP_LAUNCH((paged_epilogue_kernel<bf16_t>), grid, dim3(64), 0, st, s, sv, n_rows, off, v, table, table_stride,
               partials, splits, ss, res_blocks(s), rope, q_out);
  else
    SPP_LAUNCH((paged_epilogue_kernel<float>), grid, dim3(64), 0, st, s, sv, n_rows, off, v, table, table_stride,
               partials, splits, ss, res_blocks(s), rope, q_out);
  return hipGetLastError();
}

}  // namespace k
}  // namespace spp
