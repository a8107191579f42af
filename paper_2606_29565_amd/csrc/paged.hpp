// Internal interface of the kernels over paged caches and adjusted logits.
#pragma once

#include "kernels.hpp"
#include "spp.h"

namespace spp {

// A pool's pages as the kernels see them: [page][layer][K, V][n_kv * page_cells * dh], K as
// [head][cell][dim], V as [head][dim][cell].
struct PageView {
  char* base;
  int32_t n_pages, n_layers, n_kv, dh, shift;  // 1 << shift cells per page
  int32_t elem;                                // bytes of an element
  __host__ __device__ int64_t half() const { return ((int64_t)n_kv * dh << shift) * elem; }  // bytes of K (or V) of a layer
  __host__ __device__ int64_t page() const { return 2 * half() * n_layers; }
};

// One attention call: tables and lengths on the device.
struct PagedAttn {
  const void* q;             // [n][n_q][dh], rows q_stride elements apart
  int64_t q_stride;
  int32_t q_bf16;
  int32_t n, n_q;
  const int32_t* table;
  int64_t table_stride;
  int32_t max_pages;
  const int32_t* lengths;
  float scale;
  void* out;                 // as q; out_mode 2: the low halves of a (hi, lo) pair go to out_lo
  void* out_lo;
  int64_t out_stride;
  int32_t out_mode;          // 0 fp32, 1 bf16, 2 bf16 pair
};

// Pages copied in one launch travel as a kernel argument.
constexpr int kPageBatch = 256;
struct PageList {
  int32_t a[kPageBatch], b[kPageBatch];
};

// Workgroups of an attention call that its ranges make up to: as many sequences or more get no
// more ranges each for being fewer.
constexpr int kSplitWorkgroups = 1024;
// Tokens of all rows up to which adjusted logits are cut into the shorter slices.
constexpr int kShortSliceTokens = 2048 * 1024;

namespace k {

// Key ranges per sequence and kv head of a call: a rule on n, the heads and the table's width.
int paged_splits(const PageView& v, int n, int n_q, int max_pages);
// Workspace of this very call (of fewer sequences it may be more, see kSplitWorkgroups).
size_t paged_work_bytes(const PageView& v, int n, int n_q, int max_pages);
hipError_t paged_attention(const PageView& v, int layer, const PagedAttn& a, void* work,
                           hipStream_t st);

// dst page b[i] = src page a[i], i < n <= kPageBatch; no page is both.
hipError_t page_copy(const PageView& v, const PageList& l, int n, hipStream_t st);
// Cells [c0, c0 + cells) of every layer between a session's buffer (cap cells a layer) and
// the pages a[i] of those cells; c0 a multiple of the page.  to_pages: which way.
hipError_t page_session(const PageView& v, const PageList& l, int n, void* kv, int64_t cap,
                        int64_t c0, int cells, bool to_pages, hipStream_t st);

// The QKV epilogue of a step of one-token rows over pages: as qkv_epilogue, with q out in
// fp32 (not scaled) and the cells of row r written at position sv.row[r].pos of sequence r's
// table.
hipError_t paged_epilogue(const Shape& s, const StepView& sv, int n_rows, int layer,
                          const PageView& v, const int32_t* table, int64_t table_stride,
                          const float* partials, int splits, const float* ss, const float2* rope,
                          float* q_out, hipStream_t st);

// Workspace of this very call (of fewer rows it may be more, see kShortSliceTokens).
size_t adjust_work_bytes(int n, int vocab);
hipError_t adjust_logits(int n, int vocab, const spp_adjust* rows, spp_summary* summaries,
                         void* work, hipStream_t st);

}  // namespace k
}  // namespace spp
