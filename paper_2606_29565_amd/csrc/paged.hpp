// Internal interface of the kernels over paged caches, adjusted logits and log probabilities.
#pragma once

#include "kernels.hpp"
#include "spp.h"

namespace spp {

constexpr int kBlockCells = 16;  // cells of a head that share a scale in a cache of 8-bit codes

// A pool's pages as the kernels see them: [page][layer][K, V][n_kv * page_cells * dh], K as
// [head][cell][dim], V as [head][dim][cell].  Where the elements are 8-bit codes, each layer ends with
// their fp32 scales, [K, V][head][block of 16 cells], filled up to 128 bytes.
struct PageView {
  char* base;
  int32_t n_pages, n_layers, n_kv, dh, shift;  // 1 << shift cells per page
  int32_t elem;                                // bytes of an element
  int32_t code = 0;                            // spp_cell_codes, or 0: the elements are values
  int32_t given = 0;                           // code: bytes of an element of the session that is copied
  __host__ __device__ int64_t half() const { return ((int64_t)n_kv * dh << shift) * elem; }  // bytes of K (or V) of a layer
  __host__ __device__ int blocks() const { return (1 << shift) / kBlockCells; }
  __host__ __device__ int64_t scales() const { return code ? (8ll * n_kv * blocks() + 127) / 128 * 128 : 0; }
  __host__ __device__ int64_t layer() const { return 2 * half() + scales(); }
  __host__ __device__ int64_t page() const { return layer() * n_layers; }
};
// The pages of a pool and its device.
const PageView& pool_view(spp_pool_t pool, int* device);

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

// Rows [rows[i], rows[i+1]) of k and v are cells first[i] .. of sequence i.
struct CellRows {
  int32_t n;
  const int32_t* table;
  int64_t table_stride;
  int32_t max_pages;
  const int32_t *first, *rows;
  int32_t n_rows, max_cells;
  int32_t bf16;
  void* k;                   // [n_rows][n_kv][dh], rows k_stride elements apart
  int64_t k_stride;
  void* v;
  int64_t v_stride;
};

// A workgroup has the four blocks of 64 cells of one head, so that the rows of V^T that it shares lines of are its
// own, where sequences are long and a page's rows are not blocks themselves; else any four.  An odd number of such
// groups to a head: those past the last cell are of other XCDs for each head.  Written and read in groups / by any
// four, us, 8 heads of 128: pages of 64, 5 sequences of 4096 cells 21.2 and 20.8 / 25.6 and 23.6, 64 of 512 32.7 and
// 32.0 / 40.3 and 36.6, of 400 26.1 and 25.9 / 29.1 and 29.3, of 300 21.0 and 20.8 / 20.4 and 19.8, of 80 10.3 and 9.5 /
// 8.1 and 7.4; pages of 16, 64 of 512 33.8 and 34.9 / 31.4 and 31.5 (the last three with even numbers of groups too,
// in an order turned by one for each head).
__host__ __device__ inline int row_span(int max_cells, int shift) {
  return shift > 4 && max_cells >= 384 ? 64 : kBlockCells;
}
__host__ __device__ inline int row_blocks(int max_cells, int shift) {
  const int span = row_span(max_cells, shift), spans = (max_cells + span - 2) / span + 1;
  return span == kBlockCells ? spans : (spans | 1) * (span / kBlockCells);
}
// Workgroups of a write or a read for each of its sequences: two sides of every head's blocks, four to one.
inline int64_t row_workgroups(const PageView& v, int max_cells) {
  return (2ll * v.n_kv * row_blocks(max_cells, v.shift) + 3) / 4;
}

// Keys of a step of a wave of the attention over 8-bit codes.
constexpr int kCodeStep = 64;

// Pages copied in one launch travel as a kernel argument.
constexpr int kPageBatch = 256;
struct PageList {
  int32_t a[kPageBatch], b[kPageBatch];
};

// Workgroups of an attention call that its ranges make up to: as many sequences or more get no
// more ranges each for being fewer.
constexpr int kSplitWorkgroups = 1024;
// Tokens of all rows up to which adjusted logits and log probabilities are cut into the shorter slices.
constexpr int kShortSliceTokens = 2048 * 1024;

namespace k {

// Key ranges per sequence and kv head of a call: a rule on n, the heads and the table's width.
int paged_splits(const PageView& v, int n, int n_q, int max_pages);
// Workspace of this very call (of fewer sequences it may be more, see kSplitWorkgroups).
size_t paged_work_bytes(const PageView& v, int n, int n_q, int max_pages);
hipError_t paged_attention(const PageView& v, int layer, const PagedAttn& a, void* work,
                           hipStream_t st);

// The ranges of a call joined into its outputs (unit: the cells that ranges are multiples of).
hipError_t paged_join(const PageView& v, const PagedAttn& a, int splits, int unit, const float* o_part,
                      const float2* ml_part, hipStream_t st);

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

// The same over pages of 8-bit codes (their callers are the three above).
hipError_t code_attention(const PageView& v, int layer, const PagedAttn& a, int splits, void* work,
                          hipStream_t st);
hipError_t code_session(const PageView& v, const PageList& l, int n, void* kv, int64_t cap, int64_t c0,
                        int cells, bool to_pages, hipStream_t st);
hipError_t code_epilogue(const Shape& s, const StepView& sv, int n_rows, int layer, const PageView& v,
                         const int32_t* table, int64_t table_stride, const float* partials, int splits,
                         const float* ss, const float2* rope, float* q_out, hipStream_t st);

// Rows of a caller into cells of 8-bit codes, and such cells into rows.
hipError_t code_write(const PageView& v, int layer, const CellRows& c, hipStream_t st);
hipError_t code_read(const PageView& v, int layer, const CellRows& c, hipStream_t st);

// Workspace of this very call (of fewer rows it may be more, see kShortSliceTokens).
size_t adjust_work_bytes(int n, int vocab);
hipError_t adjust_logits(int n, int vocab, const spp_adjust* rows, spp_summary* summaries,
                         void* work, hipStream_t st);

// Workspace of this very call (of fewer rows it may be more, see kShortSliceTokens).
size_t logprob_work_bytes(int n, int vocab, int top);
hipError_t logprobs(int n, int vocab, const spp_logprob_row* rows, int top, int32_t* top_tokens,
                    float* top_logprobs, float* lse, float* entropy, void* work, hipStream_t st);

}  // namespace k
}  // namespace spp
