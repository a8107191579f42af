// Paged caches of 8-bit codes: cells written and read back, a session's cells copied in and out,
// the QKV epilogue that appends, and attention of one new token per sequence.
//
// An element is a code times the scale of its block, 16 cells of one head (keys and values apart):
//   s = the smallest power of two with max |x| / s <= Q, at least 2^-100;  code = x / s rounded
// to the nearest, ties to even, Q = 127 (signed integers) or 448 (e4m3 floats).  Cells appended to a
// block that holds cells already keep s at least what it was, and where it grows the codes there
// are rounded to the new one.  That s is a power of two makes all of this exact but the
// rounding to a code; a scale that grows at least doubles, so the roundings of a cell that is
// kept sum to less than one step of the last scale, however often it grew; and a code of at most 8
// significant bits times its scale is exact in bf16.  A block that is given an infinity or a NaN
// has the scale NaN, and so reads.
#include <algorithm>
#include <cmath>

#include "paged_device.hpp"

namespace spp {
namespace {

// Code formats: int8 (SPP_CELLS_I8) and e4m3 (SPP_CELLS_E4M3).
constexpr bool is_i8(int code) { return code == SPP_CELLS_I8; }

constexpr uint32_t kInfBits = 0x7F800000u;

// The scale that values of at most |x| need, from the bits of |x|.
template <int CODE>
__device__ __forceinline__ float scale_for(uint32_t top) {
  // x = 1.f 2^(E - 127): x / 2^(E - 133) < 128 and x / 2^(E - 135) < 512, at most Q up to a fraction
  // of 127 / 64 - 1 (of 448 / 256 - 1), else the next power of two
  constexpr uint32_t most = is_i8(CODE) ? 0x7E0000u : 0x600000u;
  constexpr int below = is_i8(CODE) ? 6 : 8;
  const int e = (int)(top >> 23) - below + ((top & 0x7FFFFFu) > most ? 1 : 0);
  return top >= kInfBits ? __builtin_nanf("") : __uint_as_float((uint32_t)max(e, 27) << 23);
}
// 1 / s of a power of two from 2^-100 to 2^122 (NaN for NaN).
__device__ __forceinline__ float inverse(float s) {
  const uint32_t e = __float_as_uint(s) >> 23;
  return e >= 255 ? __builtin_nanf("") : __uint_as_float((254u - e) << 23);
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Four values, already divided by the scale, as codes (the first in the low byte).
template <int CODE>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  if constexpr (is_i8(CODE)) {
    const uint32_t lo = __builtin_amdgcn_perm((uint32_t)(int)__builtin_rintf(b), (uint32_t)(int)__builtin_rintf(a), 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm((uint32_t)(int)__builtin_rintf(d), (uint32_t)(int)__builtin_rintf(c), 0x0C0C0400u);
    return lo | hi << 16;
  } else {
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
  }
}
template <int CODE>
__device__ __forceinline__ void decode4(uint32_t w, float (&x)[4]) {
  if constexpr (is_i8(CODE)) {
    x[0] = (float)(int8_t)w;
    x[1] = (float)(int8_t)(w >> 8);
    x[2] = (float)(int8_t)(w >> 16);
    x[3] = (float)(int8_t)(w >> 24);
  } else {
    x[0] = __builtin_amdgcn_cvt_f32_fp8(w, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8(w, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8(w, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8(w, 3);
  }
}
// Codes of a scale that grew, at the new one (ratio = old / new).
template <int CODE>
__device__ __forceinline__ uint32_t shrink4(uint32_t w, float ratio) {
  float x[4];
  decode4<CODE>(w, x);
  return encode4<CODE>(x[0] * ratio, x[1] * ratio, x[2] * ratio, x[3] * ratio);
}
// Four codes as values, two bf16 pairs or four floats.
template <int CODE>
__device__ __forceinline__ void values4(uint32_t w, float scale, bf16_t* out) {
  float x[4];
  decode4<CODE>(w, x);
  uint2 o;  // (exact: the upper halves)
  o.x = __builtin_amdgcn_perm(__float_as_uint(x[1] * scale), __float_as_uint(x[0] * scale), 0x07060302u);
  o.y = __builtin_amdgcn_perm(__float_as_uint(x[3] * scale), __float_as_uint(x[2] * scale), 0x07060302u);
  *reinterpret_cast<uint2*>(out) = o;
}
template <int CODE>
__device__ __forceinline__ void values4(uint32_t w, float scale, float* out) {
  float x[4];
  decode4<CODE>(w, x);
  *reinterpret_cast<float4*>(out) = make_float4(x[0] * scale, x[1] * scale, x[2] * scale, x[3] * scale);
}

// The largest magnitude of the wave (below 2^31: in the order of integers, which ~ turns over).
__device__ __forceinline__ uint32_t wave_top(uint32_t v) { return (uint32_t)~wave_min_all((int)~v); }

// Where a head's block is: its codes (K: the block's first cell, V: its first cell of dim 0) and scale.
struct BlockAt {
  uint8_t* codes;
  float* scale;
};
__device__ __forceinline__ BlockAt block_at(const PageView& v, int64_t layer_off, int page, int which, int head,
                                            int cell) {
  char* layer = v.base + page * v.page() + layer_off;
  char* codes = layer + which * v.half() + ((int64_t)head * v.dh << v.shift) + (which ? cell : cell * v.dh);
  float* scales = reinterpret_cast<float*>(layer + 2 * v.half()) + (which * v.n_kv + head) * v.blocks();
  return BlockAt{reinterpret_cast<uint8_t*>(codes), scales + cell / kBlockCells};
}

// The scale of a block that keeps its first `kept` cells and is given values of at most |top|.
template <int CODE>
__device__ __forceinline__ float grown(float old, int kept, uint32_t top) {
  const float need = scale_for<CODE>(top);
  if (kept == 0) return need;
  return need != need || old != old ? __builtin_nanf("") : fmaxf(need, old);
}

// The codes of a key block's first `kept` cells at a scale that grew: the wave's 4-byte words.
template <int CODE>
__device__ __forceinline__ void shrink_keys(uint8_t* codes, int kept, int dh, float ratio, int lane) {
  uint32_t* w = reinterpret_cast<uint32_t*>(codes);
  for (int i = lane; i < kept * dh / 4; i += 64) w[i] = shrink4<CODE>(w[i], ratio);
}

// 16 codes of one dim of a value block: the first `kept` as they are (at a scale that grew if
// `grew`), those from there on of `fresh`.
template <int CODE>
__device__ __forceinline__ uint4 merge_values(uint4 was, uint4 fresh, int kept, bool grew, float ratio) {
  uint32_t o[4], w[4] = {was.x, was.y, was.z, was.w}, f[4] = {fresh.x, fresh.y, fresh.z, fresh.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (grew) w[j] = shrink4<CODE>(w[j], ratio);
    const int n = kept - 4 * j;  // codes of this word that are kept
    const uint32_t mask = n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
    o[j] = (w[j] & mask) | (f[j] & ~mask);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// A write or read as its kernel takes it: within 100 bytes, as a launch with more takes the host 0.6 us
// longer (3.4 instead of 2.8).
struct RowsArg {
  char* layer;                   // the layer in page 0
  int64_t page;                  // bytes between pages
  const int32_t *table, *first, *rows;
  void *k, *v;
  uint32_t k_stride8, v_stride8;  // elements between rows, by eight
  int32_t table_stride, max_pages, n_pages, n_rows, max_cells;
  uint16_t shift, heads2;        // log2 of a page's cells; kv heads, keys and values apart
};
static_assert(sizeof(RowsArg) <= 96, "a short launch");
// What a wave of a write or a read has: a block of one head's keys or values, and the rows of the
// caller that are its cells lo .. hi - 1.
struct BlockRows {
  bool any;
  int which, head;
  int page, cell, lo, hi;  // the block's first cell in its page; lo: cells before it are kept
  int64_t row;             // of cell 0 of the block (before the sequence's first row for cells < lo)
};
__device__ __forceinline__ BlockRows block_rows(const RowsArg& c, int wave, int seq) {
  BlockRows r{};
  const int blocks = row_blocks(c.max_cells, c.shift), job = (int)blockIdx.x * 4 + wave, hw = job / blocks;
  if (hw >= c.heads2) return r;
  r.which = hw & 1;
  r.head = hw >> 1;
  const int first = c.first[seq], r0 = c.rows[seq], r1 = min(max(c.rows[seq + 1], 0), c.n_rows);
  if (first < 0 || r0 < 0) return r;
  const int count = min(min(r1 - r0, c.max_cells), (c.max_pages << c.shift) - first);
  if (count <= 0) return r;  // (so first is below 2^30)
  const int at = (first & -row_span(c.max_cells, c.shift)) + kBlockCells * (job % blocks);
  if (at >= first + count || at + kBlockCells <= first) return r;
  r.any = true;
  r.page = c.table[(int64_t)seq * c.table_stride + (at >> c.shift)];
  r.cell = at & ((1 << c.shift) - 1);
  r.lo = max(first - at, 0);
  r.hi = min(first + count - at, kBlockCells);
  r.row = (int64_t)r0 + at - first;
  return r;
}
template <int DH>
__device__ __forceinline__ BlockAt block_at(const RowsArg& c, const BlockRows& b, int page) {
  const int heads = c.heads2 >> 1;
  const int64_t half = (int64_t)heads * DH << c.shift;
  char* layer = c.layer + page * c.page;
  char* codes = layer + b.which * half + ((int64_t)b.head * DH << c.shift) + (b.which ? b.cell : b.cell * DH);
  float* scales = reinterpret_cast<float*>(layer + 2 * half) + ((b.which * heads + b.head) << (c.shift - 4));
  return BlockAt{reinterpret_cast<uint8_t*>(codes), scales + b.cell / kBlockCells};
}

// A wave's rows of 16 cells of one head: lane l has unit l % UPR (16 bytes, E dims) of the C cells from
// C (l / UPR) on.
template <typename T, int DH>
struct RowMap {
  static constexpr int E = Elem<T>::kPerFrag, UPR = DH / E, C = kBlockCells * UPR / 64, D = DH / 64;
  // Where a dim's 16 codes are in the wave's LDS: 16 bytes more every E dims, so that the lanes of a
  // row write other banks.
  static constexpr int kBytes = DH * 16 + DH / E * 16;
  static __device__ __forceinline__ int at(int dim) { return dim * 16 + dim / E * 16; }
};
template <typename T>
__device__ __forceinline__ void unit_values(const uint4& x, float* f) {
  if constexpr (Elem<T>::kPerFrag == 8) frag_to_f32(x, reinterpret_cast<float(&)[8]>(*f));
  else frag_to_f32(x, reinterpret_cast<float(&)[4]>(*f));
}
// What the wave's lanes have written to LDS is there for its lanes to read.
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Grid (blocks of a sequence, fastest, times K and V of each head, four to a workgroup; sequences), a
// wave to a block.  Values change from rows of dims to rows of cells in LDS.
//
// Bound by memory: 12844 cells of 5 prompts, 8 heads of 128, 79 MB from bf16 rows to e4m3 cells in 16.5 us
// (4.8 TB/s) and back in 14.2 (5.6); 19.4 and 16.2 by any four blocks to a workgroup, and then, with values loaded a dim
// or two of all 16 cells a lane and stored as they come, 26.9 and 21.2.  fp32 rows, 131 MB, 25.3 (5.2) and 21.4.  One
// token: what is looked up one after the other (the rows, the page, what the block keeps), 2.7 us and 2.8
// for one sequence of 4 heads of 64, 5.1 and 4.0 for 64 of 8 heads of 128.
template <typename T, int CODE, int DH>
__global__ __launch_bounds__(256) void write_kernel(RowsArg c) {
  using M = RowMap<T, DH>;
  __shared__ __align__(16) uint8_t lds[4 * M::kBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const BlockRows b = block_rows(c, wave, blockIdx.y);
  if (!b.any) return;
  const int64_t stride = 8ll * (b.which ? c.v_stride8 : c.k_stride8);
  const int unit = lane % M::UPR, cell0 = lane / M::UPR * M::C;
  const T* src = static_cast<const T*>(b.which ? c.v : c.k) + b.head * DH + unit * M::E;
  uint4 x[M::C];  // (rows outside [lo, hi) repeat one inside)
#pragma unroll
  for (int p = 0; p < M::C; ++p)
    x[p] = *reinterpret_cast<const uint4*>(src + (b.row + min(max(cell0 + p, b.lo), b.hi - 1)) * stride);
  __builtin_amdgcn_sched_barrier(0);  // (the rows are on their way before the page's number is looked at)
  if ((unsigned)b.page >= (unsigned)c.n_pages) return;
  const BlockAt to = block_at<DH>(c, b, b.page);
  // what the block keeps: its scale, and of values the lane's dims
  float old = 0.f;
  uint4 was[M::D];
  if (b.lo) {
    old = *to.scale;
    if (b.which)
#pragma unroll
      for (int d = 0; d < M::D; ++d) was[d] = *reinterpret_cast<const uint4*>(to.codes + ((lane + 64 * d) << c.shift));
  }
  float f[M::C][M::E];
  uint32_t top = 0;
#pragma unroll
  for (int p = 0; p < M::C; ++p) {
    unit_values<T>(x[p], f[p]);
#pragma unroll
    for (int e = 0; e < M::E; ++e) top = max(top, magnitude(f[p][e]));
  }
  top = wave_top(top);
  const float scale = grown<CODE>(old, b.lo, top), inv = inverse(scale);
  if (lane == 0) *to.scale = scale;
  if (b.which == 0) {
    if (b.lo && scale > old) shrink_keys<CODE>(to.codes, b.lo, DH, old * inv, lane);
#pragma unroll
    for (int p = 0; p < M::C; ++p) {
      const int cell = cell0 + p;
      if (cell < b.lo || cell >= b.hi) continue;
      uint32_t* dst = reinterpret_cast<uint32_t*>(to.codes + cell * DH + unit * M::E);
      const uint32_t w0 = encode4<CODE>(f[p][0] * inv, f[p][1] * inv, f[p][2] * inv, f[p][3] * inv);
      if constexpr (M::E == 8)
        *reinterpret_cast<uint2*>(dst) =
            make_uint2(w0, encode4<CODE>(f[p][4] * inv, f[p][5] * inv, f[p][6] * inv, f[p][7] * inv));
      else
        *dst = w0;
    }
    return;
  }
  uint8_t* mine = lds + wave * M::kBytes;
#pragma unroll
  for (int e = 0; e < M::E; ++e) {
    uint8_t* at = mine + M::at(unit * M::E + e) + cell0;
    if constexpr (M::C == 2) {
      *reinterpret_cast<uint16_t*>(at) = (uint16_t)encode4<CODE>(f[0][e] * inv, f[1][e] * inv, 0.f, 0.f);
    } else {
#pragma unroll
      for (int p = 0; p < M::C; p += 4)
        *reinterpret_cast<uint32_t*>(at + p) =
            encode4<CODE>(f[p][e] * inv, f[p + 1][e] * inv, f[p + 2][e] * inv, f[p + 3][e] * inv);
    }
  }
  wave_lds_sync();
#pragma unroll
  for (int d = 0; d < M::D; ++d) {
    const int dim = lane + 64 * d;
    uint4* dst = reinterpret_cast<uint4*>(to.codes + (dim << c.shift));
    uint4 o = *reinterpret_cast<const uint4*>(mine + M::at(dim));
    if (b.lo) o = merge_values<CODE>(was[d], o, b.lo, scale > old, old * inv);
    *dst = o;
  }
}

// The same grid: cells as values into the caller's rows; zeros where the page is not listed.
template <typename T, int CODE, int DH>
__global__ __launch_bounds__(256) void read_kernel(RowsArg c) {
  using M = RowMap<T, DH>;
  __shared__ __align__(16) uint8_t lds[4 * M::kBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const BlockRows b = block_rows(c, wave, blockIdx.y);
  if (!b.any) return;
  const int64_t stride = 8ll * (b.which ? c.v_stride8 : c.k_stride8);
  const bool listed = (unsigned)b.page < (unsigned)c.n_pages;
  const BlockAt at = block_at<DH>(c, b, listed ? b.page : 0);
  const float held = *at.scale, scale = listed ? held : 0.f;
  const int unit = lane % M::UPR, cell0 = lane / M::UPR * M::C;
  T* dst = static_cast<T*>(b.which ? c.v : c.k) + b.head * DH + unit * M::E;
  uint32_t w[M::C][M::E / 4];  // codes of the lane's dims, cell by cell
  if (b.which == 0) {
#pragma unroll
    for (int p = 0; p < M::C; ++p) {
      const uint32_t* src = reinterpret_cast<const uint32_t*>(at.codes + (cell0 + p) * DH + unit * M::E);
#pragma unroll
      for (int k = 0; k < M::E / 4; ++k) w[p][k] = src[k];
    }
  } else {
    uint8_t* mine = lds + wave * M::kBytes;
#pragma unroll
    for (int d = 0; d < M::D; ++d) {
      const int dim = lane + 64 * d;
      *reinterpret_cast<uint4*>(mine + M::at(dim)) = *reinterpret_cast<const uint4*>(at.codes + (dim << c.shift));
    }
    wave_lds_sync();
#pragma unroll
    for (int k = 0; k < M::E / 4; ++k) {
#pragma unroll
      for (int p = 0; p < M::C; ++p) w[p][k] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint8_t* from = mine + M::at(unit * M::E + 4 * k + e) + cell0;
        uint32_t q[(M::C + 3) / 4];
        if constexpr (M::C == 2) {
          q[0] = *reinterpret_cast<const uint16_t*>(from);
        } else {
#pragma unroll
          for (int p = 0; p < M::C / 4; ++p) q[p] = *reinterpret_cast<const uint32_t*>(from + 4 * p);
        }
#pragma unroll
        for (int p = 0; p < M::C; ++p) w[p][k] |= (q[p / 4] >> (8 * (p % 4)) & 0xFFu) << (8 * e);
      }
    }
  }
#pragma unroll
  for (int p = 0; p < M::C; ++p) {
    const int cell = cell0 + p;
    float x[M::E];
#pragma unroll
    for (int k = 0; k < M::E / 4; ++k) decode4<CODE>(listed ? w[p][k] : 0u, reinterpret_cast<float(&)[4]>(x[4 * k]));
    if (cell < b.lo || cell >= b.hi) continue;
    uint32_t o[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (M::E == 8)  // (exact: the upper halves)
        o[k] = __builtin_amdgcn_perm(__float_as_uint(x[2 * k + 1] * scale), __float_as_uint(x[2 * k] * scale), 0x07060302u);
      else
        o[k] = __float_as_uint(x[k] * scale);
    }
    *reinterpret_cast<uint4*>(dst + (b.row + cell) * stride) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// Grid (64 cells of the copy, fastest, times layers * 2 * kv heads): four blocks of one head's keys or values,
// between a session's buffer and their pages.  Keys: a wave to a block, rows of dims on both sides.  Values:
// rows of cells on both sides, read and written 16 bytes of the session's at a time, UPR lanes to a row of 64
// cells, so that whole lines move; a block's largest value is put together over the workgroup.  Only live
// cells move; the cells of the session past the last stay as they are.  The loads pass the L2 by (they are
// read once).
// Bound by memory: 8100 cells of 4 layers of the 8B shape, 199 MB, in 36.5 us (5.5 TB/s) and out in 34.4; with 32
// bytes of a row of cells to a wave 58 both ways.
template <typename T, int CODE, int DH, bool TO_PAGES>
__global__ __launch_bounds__(256) void session_kernel(PageView v, PageList l, int groups, T* kv, int64_t cap,
                                                      int64_t c0, int cells) {
  constexpr int E = Elem<T>::kPerFrag;
  __shared__ uint32_t tops[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int base = blockIdx.x % groups * 64;  // of the cells that are copied
  const int hd = blockIdx.x / groups, head = hd % v.n_kv, which = hd / v.n_kv % 2, layer = hd / v.n_kv / 2;
  const int64_t layer_off = v.layer() * layer;
  T* sess = kv + ((int64_t)(2 * layer + which) * v.n_kv + head) * cap * DH;
  auto load = [](const void* p) {
    const u32x4 q = __builtin_nontemporal_load(static_cast<const u32x4*>(p));
    return make_uint4(q.x, q.y, q.z, q.w);
  };
  if (which == 0) {
    const int at = base + wave * kBlockCells, live = min(kBlockCells, cells - at);
    if (live <= 0) return;
    const BlockAt page = block_at(v, layer_off, l.a[at >> v.shift], 0, head, at & ((1 << v.shift) - 1));
    sess += (c0 + at) * DH;
    constexpr int N = kBlockCells * DH / E / 64;
    const int units = live * (DH / E);
    if constexpr (TO_PAGES) {
      uint4 x[N];
#pragma unroll
      for (int p = 0; p < N; ++p) x[p] = load(sess + (int64_t)min(p * 64 + lane, units - 1) * E);
      float f[N][E];
      uint32_t top = 0;
#pragma unroll
      for (int p = 0; p < N; ++p) {
        unit_values<T>(x[p], f[p]);
#pragma unroll
        for (int e = 0; e < E; ++e) top = max(top, magnitude(f[p][e]));
      }
      const float scale = scale_for<CODE>(wave_top(top)), inv = inverse(scale);
#pragma unroll
      for (int p = 0; p < N; ++p) {
        const int u = p * 64 + lane;
        if (u >= units) continue;
        uint32_t* dst = reinterpret_cast<uint32_t*>(page.codes + u * E);
        const uint32_t w0 = encode4<CODE>(f[p][0] * inv, f[p][1] * inv, f[p][2] * inv, f[p][3] * inv);
        if constexpr (E == 8)
          *reinterpret_cast<uint2*>(dst) =
              make_uint2(w0, encode4<CODE>(f[p][4] * inv, f[p][5] * inv, f[p][6] * inv, f[p][7] * inv));
        else
          *dst = w0;
      }
      if (lane == 0) *page.scale = scale;
    } else {
      const float scale = *page.scale;
      uint32_t w[N][E / 4];
#pragma unroll
      for (int p = 0; p < N; ++p) {
        const uint32_t* src = reinterpret_cast<const uint32_t*>(page.codes + min(p * 64 + lane, units - 1) * E);
#pragma unroll
        for (int k = 0; k < E / 4; ++k) w[p][k] = __builtin_nontemporal_load(src + k);
      }
#pragma unroll
      for (int p = 0; p < N; ++p) {
        const int u = p * 64 + lane;
        if (u < units)
#pragma unroll
          for (int k = 0; k < E / 4; ++k) values4<CODE>(w[p][k], scale, sess + u * E + 4 * k);
      }
    }
    return;
  }
  // Thread: unit `unit` of the rows of dims d0, d0 + ROWS ...; the unit's cells are of one block.
  constexpr int UPR = 64 / E, ROWS = 256 / UPR, N = DH / ROWS;
  const int unit = tid % UPR, d0 = tid / UPR, at = base + unit * E, block = unit * E / kBlockCells;
  const bool any = at - at % kBlockCells < cells;  // (a block without a cell may have no page)
  const int live = min(max(cells - at, 0), E);     // of the unit
  const int cell = at & ((1 << v.shift) - 1), inner = cell % kBlockCells;
  const BlockAt page = block_at(v, layer_off, any ? l.a[at >> v.shift] : l.a[0], 1, head, any ? cell - inner : 0);
  sess += c0 + at;
  if constexpr (TO_PAGES) {
    if (tid < 4) tops[tid] = 0;
    uint4 x[N];  // (the session's rows hold whole blocks of 64 cells)
#pragma unroll
    for (int p = 0; p < N; ++p) x[p] = load(sess + (int64_t)(d0 + p * ROWS) * cap);
    float f[N][E];
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < N; ++p) {
      unit_values<T>(x[p], f[p]);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (e >= live) f[p][e] = 0.f;  // (whatever lies behind the last cell)
        top = max(top, magnitude(f[p][e]));
      }
    }
    __syncthreads();
    // over the wave's lanes of the block: those of its other rows, and of its other units
#pragma unroll
    for (int o = 32; o >= UPR; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
#pragma unroll
    for (int o = kBlockCells / E / 2; o >= 1; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    if (lane < UPR && inner == 0) atomicMax(&tops[block], top);
    __syncthreads();
    const float scale = scale_for<CODE>(tops[block]), inv = inverse(scale);
    if (!any) return;
#pragma unroll
    for (int p = 0; p < N; ++p) {
      uint32_t* dst = reinterpret_cast<uint32_t*>(page.codes + ((d0 + p * ROWS) << v.shift) + inner);
      const uint32_t w0 = encode4<CODE>(f[p][0] * inv, f[p][1] * inv, f[p][2] * inv, f[p][3] * inv);
      if constexpr (E == 8)
        *reinterpret_cast<uint2*>(dst) =
            make_uint2(w0, encode4<CODE>(f[p][4] * inv, f[p][5] * inv, f[p][6] * inv, f[p][7] * inv));
      else
        *dst = w0;
    }
    if (d0 == 0 && inner == 0) *page.scale = scale;
  } else {
    if (live == 0) return;
    const float scale = *page.scale;
    uint32_t w[N][E / 4];
#pragma unroll
    for (int p = 0; p < N; ++p) {
      const uint32_t* src = reinterpret_cast<const uint32_t*>(page.codes + ((d0 + p * ROWS) << v.shift) + inner);
#pragma unroll
      for (int k = 0; k < E / 4; ++k) w[p][k] = __builtin_nontemporal_load(src + k);
    }
#pragma unroll
    for (int p = 0; p < N; ++p) {
      T* o = sess + (int64_t)(d0 + p * ROWS) * cap;
#pragma unroll
      for (int k = 0; k < E / 4; ++k) {
        if (live == E) {
          values4<CODE>(w[p][k], scale, o + 4 * k);
        } else {
          float x[4];
          decode4<CODE>(w[p][k], x);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (4 * k + e < live) store_elem(o, 4 * k + e, x[e] * scale);
        }
      }
    }
  }
}

// One wave per (row, head) of the fused QKV output of a step whose rows are one token of one
// sequence each, as paged_epilogue_kernel: a key or value joins the block at the sequence's end.
template <int CODE>
__global__ __launch_bounds__(64) void code_epilogue_kernel(Shape s, StepView sv, int M, int64_t layer_off, PageView v,
                                                           const int32_t* table, int64_t table_stride, const float* P,
                                                           int splits, const float* ss, int nb, const float2* rope,
                                                           float* q_out) {
  const int r = blockIdx.x, hh = blockIdx.y, i = threadIdx.x;
  const int dh = s.dh, half = dh / 2;
  const int N = (s.n_q + 2 * s.n_kv) * dh;
  const int64_t split_stride = (int64_t)M * N;
  const int64_t pr = (int64_t)r * N + (int64_t)hh * dh;
  const int kind = hh < s.n_q ? 0 : (hh < s.n_q + s.n_kv ? 1 : 2);
  const int pos = sv.row[r].pos;
  const float inv_rms = row_inv(ss, r, nb, s.d, s.eps);
  float a = 0.f, b = 0.f;  // of dims i and i + half (lanes past the half, dh 64: none)
  const bool in = i < half;
  if (in) {
    a = add_splits(0.f, P, split_stride, splits, pr + i) * inv_rms;
    b = add_splits(0.f, P, split_stride, splits, pr + i + half) * inv_rms;
    if (kind < 2) {
      const float2 cs = rope[(int64_t)r * half + i];
      const float a2 = a * cs.x - b * cs.y;
      const float b2 = a * cs.y + b * cs.x;
      a = a2;
      b = b2;
    }
  }
  if (kind == 0) {
    if (in) {
      q_out[((int64_t)r * s.n_q + hh) * dh + i] = a;
      q_out[((int64_t)r * s.n_q + hh) * dh + i + half] = b;
    }
    return;
  }
  const int page = table[(int64_t)r * table_stride + (pos >> v.shift)];
  const int which = kind - 1, head = hh - s.n_q - which * s.n_kv, cell = pos & ((1 << v.shift) - 1);
  const int kept = cell % kBlockCells;
  const BlockAt to = block_at(v, layer_off, page, which, head, cell - kept);
  const float old = kept ? *to.scale : 0.f;
  const uint32_t top = wave_top(max(magnitude(a), magnitude(b)));
  const float scale = grown<CODE>(old, kept, top), inv = inverse(scale);
  const bool grew = kept && scale > old;
  const uint32_t codes = encode4<CODE>(a * inv, b * inv, 0.f, 0.f);
  if (which == 0) {
    if (grew) shrink_keys<CODE>(to.codes, kept, dh, old * inv, i);
    if (in) {
      to.codes[kept * dh + i] = (uint8_t)codes;
      to.codes[kept * dh + i + half] = (uint8_t)(codes >> 8);
    }
  } else if (in) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint4* dst = reinterpret_cast<uint4*>(to.codes + ((i + k * half) << v.shift));
      const uint32_t w = (codes >> (8 * k) & 0xFFu) * 0x01010101u;  // (behind the last cell: anything)
      uint4 o = make_uint4(w, w, w, w);
      if (kept) o = merge_values<CODE>(*dst, o, kept, grew, old * inv);
      *dst = o;
    }
  }
  if (i == 0) *to.scale = scale;
}

// ---- attention ----------------------------------------------------------------------------

// Eight codes as eight bf16, exactly: the operand of a 16x16x32 product.
template <int CODE>
__device__ __forceinline__ uint4 code_frag(uint32_t w0, uint32_t w1) {
  const uint32_t w[2] = {w0, w1};
  uint32_t o[4];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if constexpr (is_i8(CODE)) {
      float x[4];
      decode4<CODE>(w[j], x);
      o[2 * j] = __builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u);
      o[2 * j + 1] = __builtin_amdgcn_perm(__float_as_uint(x[3]), __float_as_uint(x[2]), 0x07060302u);
    } else {
      o[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[j], 1.f, false));
      o[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[j], 1.f, true));
    }
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// The first n of 16 codes, the others zero.
__device__ __forceinline__ uint4 keep_codes(const uint4& v, int n) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t o[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int k = n - 4 * j;
    o[j] = k >= 4 ? w[j] : k <= 0 ? 0u : w[j] & ((1u << (8 * k)) - 1);
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// Attention over codes: the plan of paged_attn_kernel (both products turned over, nothing
// exchanged between lanes but the maximum, cells straight from the page to the operands), with a
// step of 64 keys whose lane group g holds the scores and values of block g of 16 cells.  So a lane
// has one scale for its 16 scores and one for its 16 probabilities, applied in fp32 outside the
// products:
//   s_j = scale log2(e) sk q.ck_j,   o = sum_j (p_j sv) cv_j / sum_j p_j.
// Row r of key tile t stands for key 16 (r / 4) + 4 t + r % 4.  A 16-byte load of a key's row is 16
// dims, two operands of the 16x16x32 products; the queries are laid out alike.
// Codes are exact in bf16; what multiplies them, p_j sv and queries in fp32, goes in two bf16 parts each, which leave 2^-17
// of it (one part would leave 2^-8 of a weight, more than a bf16 output's own rounding where values cancel).  Scores, maxima,
// the sums of p and of the output are fp32.  The query's second part, half as many products again: 121 us against 115 for
// the 64 sequences below, 7.8 against 6.8 for the one.
// HBM bounds it: a cell is 2 (dh + 1/4) bytes and 4 G dh operations.  64 sequences of U[1024, 8192] cells, 8
// heads of 128, 569 MB: 114-117 us, 5.0 TB/s, where bf16 cells take 212-221; three of 32749 in e4m3 43.5 (4.6 TB/s);
// one of 8192 6.6.  A step is 744 vector instructions, half of them an integer's way to bf16 by fp32, a third of the
// time.  That is not what it waits for: with both products on operands that cost less (q as integers of two
// 7-bit parts on 16x16x64 integer products, probabilities and values in fp16) it took 116, and 7.9 for one sequence.
// Two steps a trip, 204 registers: 156 where this took 127 (both with a graph's own time); three workgroups to a CU 127 and
// one 125, against 116.  Waves with a stretch of the range each: 151 against 140 in pages of 128 cells, 162 against 147 of
// 256, 129 against 127 of 64.
template <int CODE, int DH, bool QLO>
__global__ __launch_bounds__(64 * kWaves, 2) void code_attn_kernel(PageView v, int64_t layer_off, PagedAttn a,
                                                                float scale2, int tiles, float* o_part,
                                                                float2* ml_part) {
  constexpr int KT = kCodeStep, NT = 4, NK = DH / 64, ND = DH / 16, B = kBlockCells;
  constexpr int OS = DH + 4;
  __shared__ float o_lds[kWaves * 16 * OS];
  __shared__ float2 ml_lds[kWaves * 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int split = blockIdx.x, splits = gridDim.x, seq = blockIdx.z;
  const int head = blockIdx.y / tiles, tile = blockIdx.y % tiles;
  const int G = a.n_q / v.n_kv, q0 = head * G + tile * 16, nh = min(16, G - tile * 16);

  const int len = live_cells(a, v.shift, seq);
  const int range = range_cells(len, splits, KT * kWaves);
  const int r0 = split * range;
  if (r0 >= len && split > 0) return;  // (the join counts the ranges alike)
  // The waves take the steps of the range in turn, so that the halves of a line of V^T (pages of 128 cells
  // and more) are read by neighbours at about the same time.
  const int r1 = min(len, r0 + range), k_begin = r0 + wave * KT, k_end = r1;
  constexpr int STEP = KT * kWaves;
  const bool solo = range >= len;  // (an empty sequence: range 0, this writes its zeros)

  uint4 qh[2 * NK], ql[2 * NK];
  const int64_t q_at = (int64_t)seq * a.q_stride + (int64_t)(q0 + min(i, nh - 1)) * DH + g * 16;
#pragma unroll
  for (int c = 0; c < 2 * NK; ++c)
    query_frag(a.q, a.q_bf16, q_at + c / 2 * 64 + c % 2 * 8, qh[c], ql[c], bf16_t{});
  float m = -INFINITY, l = 0.f;
  f32x4 acc[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int P1 = (1 << v.shift) - 1;
  const int32_t* tab = a.table + (int64_t)seq * a.table_stride;
  const int64_t page_bytes = v.page(), half = v.half();
  const char* kbase = v.base + layer_off + ((int64_t)head * DH << v.shift);
  const char* vbase = kbase + half;
  const char* sbase = v.base + layer_off + 2 * half + (int64_t)head * v.blocks() * 4;
  const int64_t v_scales = (int64_t)v.n_kv * v.blocks() * 4;
  const int last_page = (len - 1) >> v.shift;
  const int trips = k_begin < k_end ? (k_end - k_begin + STEP - 1) / STEP : 0;

  int kp, vp, vq;
  auto pages = [&](int k) {
    const int k0 = k_begin + k * STEP;
    kp = tab[min((k0 + B * (i >> 2)) >> v.shift, last_page)];
    vp = tab[min((k0 + B * g) >> v.shift, last_page)];
  };
  uint4 kf[NT][NK], vf[ND];
  float ks, vs;
  int nl;
  auto issue_keys = [&](int k) {
    const int kb = k_begin + k * STEP + B * (i >> 2);
    const char* kr = kbase + ((unsigned)kp < (unsigned)v.n_pages ? kp : 0) * page_bytes +
                     ((kb & P1) + (i & 3)) * DH + g * 16;
    vq = vp;
    pages(k + 1);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < NK; ++c) kf[t][c] = ld_global(kr + t * 4 * DH + c * 64);
  };
  auto issue_values = [&](int k) {
    const int vb = k_begin + k * STEP + B * g;
    const bool ok = (unsigned)vq < (unsigned)v.n_pages;
    nl = ok ? min(k_end - vb, B) : 0;
    const int64_t page = (ok ? vq : 0) * page_bytes;
    const char* vr = vbase + page + (((int64_t)i << v.shift) + (vb & P1));
    const char* sr = sbase + page + (vb & P1) / B * 4;
    ks = __uint_as_float(ld_global_u32(sr));
    vs = __uint_as_float(ld_global_u32(sr + v_scales));
#pragma unroll
    for (int d = 0; d < ND; ++d) vf[d] = ld_global(vr + (((int64_t)d * 16) << v.shift));
  };
  float s[B];
  auto scores = [&]() {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4 d = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        const uint4 k0 = code_frag<CODE>(kf[t][c].x, kf[t][c].y), k1 = code_frag<CODE>(kf[t][c].z, kf[t][c].w);
        d = mma_frag(k0, qh[2 * c], d, bf16_t{});
        d = mma_frag(k1, qh[2 * c + 1], d, bf16_t{});
        if constexpr (QLO) {
          d = mma_frag(k0, ql[2 * c], d, bf16_t{});
          d = mma_frag(k1, ql[2 * c + 1], d, bf16_t{});
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) s[4 * t + j] = d[j];
    }
  };
  auto fold = [&]() {
    const bool whole = __all(nl == B);
    const float f = ks * scale2;
#pragma unroll
    for (int j = 0; j < B; ++j) s[j] = whole || j < nl ? s[j] * f : -INFINITY;
    float top = s[0];
#pragma unroll
    for (int j = 1; j < B; ++j) top = fmaxf(top, s[j]);
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float mn = fmaxf(m, top);
    const float mu = mn == -INFINITY ? 0.f : mn;  // nothing live yet
    const float alpha = __builtin_amdgcn_exp2f(m - mu);
    m = mn;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < B; ++j) {
      s[j] = __builtin_amdgcn_exp2f(s[j] - mu);
      sum += s[j];
    }
    l = l * alpha + sum;
    if (!__all(alpha == 1.f)) {
#pragma unroll
      for (int d = 0; d < ND; ++d) acc[d] *= alpha;
    }
    const float w = nl > 0 ? vs : 0.f;
#pragma unroll
    for (int j = 0; j < B; ++j) s[j] *= w;
    uint4 ph[2], pl[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      split_pair(s[8 * u], s[8 * u + 1], ph[u].x, pl[u].x);
      split_pair(s[8 * u + 2], s[8 * u + 3], ph[u].y, pl[u].y);
      split_pair(s[8 * u + 4], s[8 * u + 5], ph[u].z, pl[u].z);
      split_pair(s[8 * u + 6], s[8 * u + 7], ph[u].w, pl[u].w);
    }
    if (!whole) {
#pragma unroll
      for (int d = 0; d < ND; ++d) vf[d] = keep_codes(vf[d], nl);
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const uint4 v0 = code_frag<CODE>(vf[d].x, vf[d].y), v1 = code_frag<CODE>(vf[d].z, vf[d].w);
      acc[d] = mma_frag(v0, ph[0], acc[d], bf16_t{});
      acc[d] = mma_frag(v0, pl[0], acc[d], bf16_t{});
      acc[d] = mma_frag(v1, ph[1], acc[d], bf16_t{});
      acc[d] = mma_frag(v1, pl[1], acc[d], bf16_t{});
    }
  };
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

template <int CODE, int DH>
hipError_t launch_attn(const PageView& v, int64_t layer_off, const PagedAttn& a, int splits, void* work,
                       hipStream_t st) {
  const int G = a.n_q / v.n_kv, tiles = (G + 15) / 16;
  const float scale = a.scale != 0.f ? a.scale : (float)(1.0 / std::sqrt((double)DH));
  const float scale2 = (float)(scale * 1.4426950408889634);
  float* o_part = static_cast<float*>(work);
  float2* ml_part = reinterpret_cast<float2*>(o_part + (int64_t)a.n * a.n_q * splits * DH);
  const dim3 grid(splits, v.n_kv * tiles, a.n), block(64 * kWaves);
  if (a.q_bf16)
    SPP_LAUNCH((code_attn_kernel<CODE, DH, false>), grid, block, 0, st, v, layer_off, a, scale2, tiles, o_part, ml_part);
  else
    SPP_LAUNCH((code_attn_kernel<CODE, DH, true>), grid, block, 0, st, v, layer_off, a, scale2, tiles, o_part, ml_part);
  if (splits > 1) return k::paged_join(v, a, splits, kCodeStep * kWaves, o_part, ml_part, st);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t launch_session(const PageView& v, const PageList& l, void* kv, int64_t cap, int64_t c0, int cells,
                          bool to_pages, hipStream_t st) {
  const int groups = (cells + 63) / 64;
  const dim3 grid(groups * 2 * v.n_kv * v.n_layers), block(256);
#define SPP_SESSION(C, W) \
  SPP_LAUNCH((session_kernel<T, C, DH, W>), grid, block, 0, st, v, l, groups, static_cast<T*>(kv), cap, c0, cells)
  if (v.code == SPP_CELLS_I8) {
    if (to_pages) SPP_SESSION(SPP_CELLS_I8, true); else SPP_SESSION(SPP_CELLS_I8, false);
  } else {
    if (to_pages) SPP_SESSION(SPP_CELLS_E4M3, true); else SPP_SESSION(SPP_CELLS_E4M3, false);
  }
#undef SPP_SESSION
  return hipGetLastError();
}

RowsArg rows_arg(const PageView& v, int layer, const CellRows& c) {
  return RowsArg{v.base + v.layer() * layer, v.page(), c.table, c.first, c.rows, c.k, c.v,
                 (uint32_t)(c.k_stride / 8), (uint32_t)(c.v_stride / 8), (int32_t)c.table_stride, c.max_pages,
                 v.n_pages, c.n_rows, c.max_cells, (uint16_t)v.shift, (uint16_t)(2 * v.n_kv)};
}
dim3 rows_grid(const PageView& v, const CellRows& c) { return dim3((unsigned)row_workgroups(v, c.max_cells), c.n); }
template <typename T, int CODE, int DH>
hipError_t launch_write(const PageView& v, int layer, const CellRows& c, hipStream_t st) {
  SPP_LAUNCH((write_kernel<T, CODE, DH>), rows_grid(v, c), dim3(256), 0, st, rows_arg(v, layer, c));
  return hipGetLastError();
}
template <typename T, int CODE, int DH>
hipError_t launch_read(const PageView& v, int layer, const CellRows& c, hipStream_t st) {
  SPP_LAUNCH((read_kernel<T, CODE, DH>), rows_grid(v, c), dim3(256), 0, st, rows_arg(v, layer, c));
  return hipGetLastError();
}

}  // namespace

namespace k {

hipError_t code_attention(const PageView& v, int layer, const PagedAttn& a, int splits, void* work, hipStream_t st) {
  const int64_t off = v.layer() * layer;
  if (v.code == SPP_CELLS_I8)
    return v.dh == 128 ? launch_attn<SPP_CELLS_I8, 128>(v, off, a, splits, work, st)
                       : launch_attn<SPP_CELLS_I8, 64>(v, off, a, splits, work, st);
  return v.dh == 128 ? launch_attn<SPP_CELLS_E4M3, 128>(v, off, a, splits, work, st)
                     : launch_attn<SPP_CELLS_E4M3, 64>(v, off, a, splits, work, st);
}

hipError_t code_session(const PageView& v, const PageList& l, int n, void* kv, int64_t cap, int64_t c0, int cells,
                        bool to_pages, hipStream_t st) {
  (void)n;  // (the cells say how many pages)
  if (v.given == 4)  // (fp32 models have heads of 64)
    return v.dh == 64 ? launch_session<float, 64>(v, l, kv, cap, c0, cells, to_pages, st) : hipErrorInvalidValue;
  return v.dh == 128 ? launch_session<bf16_t, 128>(v, l, kv, cap, c0, cells, to_pages, st)
                     : launch_session<bf16_t, 64>(v, l, kv, cap, c0, cells, to_pages, st);
}

hipError_t code_epilogue(const Shape& s, const StepView& sv, int n_rows, int layer, const PageView& v,
                         const int32_t* table, int64_t table_stride, const float* partials, int splits,
                         const float* ss, const float2* rope, float* q_out, hipStream_t st) {
  const dim3 grid(n_rows, s.n_q + 2 * s.n_kv), block(64);
  const int64_t off = v.layer() * layer;
  if (v.code == SPP_CELLS_I8)
    SPP_LAUNCH((code_epilogue_kernel<SPP_CELLS_I8>), grid, block, 0, st, s, sv, n_rows, off, v, table, table_stride,
               partials, splits, ss, res_blocks(s), rope, q_out);
  else
    SPP_LAUNCH((code_epilogue_kernel<SPP_CELLS_E4M3>), grid, block, 0, st, s, sv, n_rows, off, v, table, table_stride,
               partials, splits, ss, res_blocks(s), rope, q_out);
  return hipGetLastError();
}

hipError_t code_write(const PageView& v, int layer, const CellRows& c, hipStream_t st) {
  const bool i8 = v.code == SPP_CELLS_I8;
  if (v.dh == 128)
    return c.bf16 ? (i8 ? launch_write<bf16_t, SPP_CELLS_I8, 128> : launch_write<bf16_t, SPP_CELLS_E4M3, 128>)(v, layer, c, st)
                  : (i8 ? launch_write<float, SPP_CELLS_I8, 128> : launch_write<float, SPP_CELLS_E4M3, 128>)(v, layer, c, st);
  return c.bf16 ? (i8 ? launch_write<bf16_t, SPP_CELLS_I8, 64> : launch_write<bf16_t, SPP_CELLS_E4M3, 64>)(v, layer, c, st)
                : (i8 ? launch_write<float, SPP_CELLS_I8, 64> : launch_write<float, SPP_CELLS_E4M3, 64>)(v, layer, c, st);
}

hipError_t code_read(const PageView& v, int layer, const CellRows& c, hipStream_t st) {
  const bool i8 = v.code == SPP_CELLS_I8;
  if (v.dh == 128)
    return c.bf16 ? (i8 ? launch_read<bf16_t, SPP_CELLS_I8, 128> : launch_read<bf16_t, SPP_CELLS_E4M3, 128>)(v, layer, c, st)
                  : (i8 ? launch_read<float, SPP_CELLS_I8, 128> : launch_read<float, SPP_CELLS_E4M3, 128>)(v, layer, c, st);
  return c.bf16 ? (i8 ? launch_read<bf16_t, SPP_CELLS_I8, 64> : launch_read<bf16_t, SPP_CELLS_E4M3, 64>)(v, layer, c, st)
                : (i8 ? launch_read<float, SPP_CELLS_I8, 64> : launch_read<float, SPP_CELLS_E4M3, 64>)(v, layer, c, st);
}

}  // namespace k
}  // namespace spp
