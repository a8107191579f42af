// Host stand-ins for the kernels over paged caches and adjusted logits (paged.hpp), for the CPU
// build of the runtime with pool.cpp.  Test infrastructure only.  The copies move the bytes the
// kernels move; the epilogue of a decode step writes the row's token into every element of its
// cell, where a wrong table, page or position shows.
#include <cstring>

#include "paged.hpp"

namespace spp {
namespace k {

int paged_splits(const PageView&, int, int, int) { return 2; }
size_t paged_work_bytes(const PageView&, int n, int n_q, int) { return (size_t)n * n_q * 16; }
hipError_t paged_attention(const PageView&, int, const PagedAttn& a, void* work, hipStream_t st) {
  const PagedAttn c = a;
  stub::enqueue(st, [c, work] {  // reads the tables and writes the workspace it asked for
    volatile int32_t sum = 0;
    for (int i = 0; i < c.n; ++i) {
      sum = sum + c.lengths[i];
      for (int j = 0; j < c.max_pages; ++j) sum = sum + c.table[i * c.table_stride + j];
    }
    std::memset(work, 1, (size_t)c.n * c.n_q * 16);
  });
  return hipSuccess;
}

hipError_t page_copy(const PageView& v, const PageList& l, int n, hipStream_t st) {
  if (n > kPageBatch) return hipErrorInvalidValue;
  stub::enqueue(st, [=] {
    for (int i = 0; i < n; ++i) std::memcpy(v.base + l.b[i] * v.page(), v.base + l.a[i] * v.page(), v.page());
  });
  return hipSuccess;
}

hipError_t page_session(const PageView& v, const PageList& l, int n, void* kv, int64_t cap, int64_t c0, int cells,
                        bool to_pages, hipStream_t st) {
  if (n > kPageBatch) return hipErrorInvalidValue;
  stub::enqueue(st, [=] {
    const int64_t P = 1 << v.shift, e = v.elem;
    for (int64_t c = 0; c < cells; ++c)
      for (int64_t lay = 0; lay < v.n_layers; ++lay)
        for (int64_t h = 0; h < v.n_kv; ++h)
          for (int64_t d = 0; d < v.dh; ++d) {
            char* pk = v.base + l.a[c / P] * v.page() + 2 * lay * v.half() + ((h * P + c % P) * v.dh + d) * e;
            char* pv = v.base + l.a[c / P] * v.page() + (2 * lay + 1) * v.half() + ((h * v.dh + d) * P + c % P) * e;
            char* s = static_cast<char*>(kv);
            char* sk = s + ((2 * lay * v.n_kv + h) * cap * v.dh + (c0 + c) * v.dh + d) * e;
            char* sv = s + (((2 * lay + 1) * v.n_kv + h) * cap * v.dh + d * cap + c0 + c) * e;
            if (to_pages) {
              std::memcpy(pk, sk, e);
              std::memcpy(pv, sv, e);
            } else {
              std::memcpy(sk, pk, e);
              std::memcpy(sv, pv, e);
            }
          }
  });
  return hipSuccess;
}

hipError_t paged_epilogue(const Shape&, const StepView& sv, int n_rows, int layer, const PageView& v,
                          const int32_t* table, int64_t table_stride, const float*, int, const float*,
                          const float2*, float*, hipStream_t st) {
  stub::enqueue(st, [=] {
    const int64_t P = 1 << v.shift;
    for (int r = 0; r < n_rows; ++r) {
      const int pos = sv.row[r].pos;
      char* page = v.base + table[r * table_stride + pos / P] * v.page() + 2 * layer * v.half();
      const uint16_t tag = (uint16_t)sv.token[r];
      for (int64_t h = 0; h < v.n_kv; ++h)
        for (int64_t d = 0; d < v.dh; ++d) {
          std::memcpy(page + ((h * P + pos % P) * v.dh + d) * v.elem, &tag, 2);
          std::memcpy(page + v.half() + ((h * v.dh + d) * P + pos % P) * v.elem, &tag, 2);
        }
    }
  });
  return hipSuccess;
}

size_t adjust_work_bytes(int n, int) { return (size_t)n * 32; }
hipError_t adjust_logits(int n, int vocab, const spp_adjust* rows, spp_summary*, void*, hipStream_t st) {
  for (int i = 0; i < n; ++i) {
    const spp_adjust r = rows[i];  // (the caller's array is read during the call)
    stub::enqueue(st, [=] {
      for (int v = 0; v < vocab; ++v) r.dst[v] = r.src[v];
    });
  }
  return hipSuccess;
}

}  // namespace k
}  // namespace spp
