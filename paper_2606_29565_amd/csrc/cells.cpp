// Rows of a caller into cells of 8-bit codes and back, behind the C ABI (include/spp.h).
#include "paged.hpp"
#include "runtime.hpp"

using namespace spp;

namespace {

bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

spp_status check_cells(const spp_paged_cells* a, const PageView** view, int* device) {
  if (!a || !a->pool) return fail(SPP_E_INVALID_ARG, "null argument");
  const PageView& v = pool_view(a->pool, device);
  *view = &v;
  if (!v.code) return fail(SPP_E_INVALID_ARG, "the pool's cells are no 8-bit codes");
  if (a->n_seqs < 0 || a->n_seqs > 65535) return fail(SPP_E_INVALID_ARG, "n_seqs outside [0, 65535]");
  if (a->layer < 0 || a->layer >= v.n_layers) return fail(SPP_E_INVALID_ARG, "layer %d", a->layer);
  if (a->max_pages < 1 || ((int64_t)a->max_pages << v.shift) > (1 << 30))
    return fail(SPP_E_INVALID_ARG, "max_pages < 1 or over 2^30 cells");
  if (a->max_cells < 1 || a->max_cells > (1 << 24)) return fail(SPP_E_INVALID_ARG, "max_cells outside [1, 2^24]");
  if (a->io_dtype != SPP_DTYPE_BF16 && a->io_dtype != SPP_DTYPE_F32) return fail(SPP_E_INVALID_ARG, "io_dtype");
  // (a launch has fewer than 2^32 threads along the blocks, 128 for each of a head: row_workgroups)
  if (v.n_kv > 32767 || (int64_t)a->max_cells * v.n_kv > 63ll << 23)
    return fail(SPP_E_INVALID_ARG, "%d kv heads (at most 32767, times max_cells at most 63 * 2^23)", v.n_kv);
  if (a->n_rows < 0) return fail(SPP_E_INVALID_ARG, "n_rows < 0");
  if (a->n_seqs == 0) return SPP_OK;
  if (!a->table || !a->first || !a->rows || (a->n_rows && (!a->k || !a->v)))
    return fail(SPP_E_INVALID_ARG, "null pointer");
  const int64_t row = (int64_t)v.n_kv * v.dh;
  constexpr int64_t most = 8ll * UINT32_MAX;  // (the kernels' form of a stride)
  const auto bad = [&](int64_t stride) { return stride < row || stride > most || stride % 8; };
  if (bad(a->k_stride) || bad(a->v_stride) || !aligned(a->k, 16) || !aligned(a->v, 16))
    return fail(SPP_E_INVALID_ARG, "rows of k and v: %lld elements at least, multiples of 8, 16-byte aligned",
                (long long)row);
  if (a->table_stride < a->max_pages || a->table_stride > INT32_MAX)
    return fail(SPP_E_INVALID_ARG, "table_stride below max_pages or over 2^31 - 1");
  if (!aligned(a->table, 4) || !aligned(a->first, 4) || !aligned(a->rows, 4))
    return fail(SPP_E_INVALID_ARG, "table, first and rows are 4-byte aligned");
  return SPP_OK;
}

using Launch = hipError_t (*)(const PageView&, int, const CellRows&, hipStream_t);

spp_status run_cells(const spp_paged_cells* a, Launch launch, const char* what, void* stream) {
  const PageView* v = nullptr;
  int device = 0;
  if (const spp_status rc = check_cells(a, &v, &device); rc != SPP_OK) return rc;
  if (a->n_seqs == 0 || a->n_rows == 0) return SPP_OK;
  const CellRows c{a->n_seqs, a->table, a->table_stride, a->max_pages, a->first, a->rows, a->n_rows, a->max_cells,
                   a->io_dtype == SPP_DTYPE_BF16, a->k, a->k_stride, a->v, a->v_stride};
  hipSetDevice(device);
  const hipError_t e = launch(*v, a->layer, c, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(SPP_E_HIP, "%s: %s", what, hipGetErrorString(e));
  return SPP_OK;
}

}  // namespace

extern "C" {

spp_status spp_paged_write(const spp_paged_cells* a, void* stream) {
  return run_cells(a, k::code_write, "paged write", stream);
}

spp_status spp_paged_read(const spp_paged_cells* a, void* stream) {
  return run_cells(a, k::code_read, "paged read", stream);
}

}  // extern "C"
