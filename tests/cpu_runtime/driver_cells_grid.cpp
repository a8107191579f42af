// Writes and reads of cells of 8-bit codes (cells.cpp) whose launch is as large as it gets, over host stand-ins for HIP
// and the kernels: a call that is accepted has fewer than 2^32 threads in its grid's first extent, as a dispatch
// holds no more, for kv heads and most cells about every border; what is past that is refused before any launch.
// Prints "OK" and exits 0 when every check holds.
#include <cstdio>
#include <vector>

#include <hip/hip_runtime.h>

#include "paged.hpp"
#include "spp.h"

namespace {
int64_t g_workgroups = -1;  // of the last launch, for each sequence
int g_fail = 0;
}  // namespace

namespace spp {
namespace k {

hipError_t code_write(const PageView& v, int, const CellRows& c, hipStream_t) {
  g_workgroups = row_workgroups(v, c.max_cells);
  return hipSuccess;
}
hipError_t code_read(const PageView& v, int layer, const CellRows& c, hipStream_t st) { return code_write(v, layer, c, st); }

}  // namespace k
}  // namespace spp

int main() {
  constexpr int64_t kMost = 63ll << 23;
  const auto check = [](bool ok, const char* what, int heads, int page, int64_t cells) {
    if (ok) return;
    if (++g_fail < 20)
      std::fprintf(stderr, "%s: %d kv heads, pages of %d, %lld cells, %lld workgroups\n", what, heads, page, (long long)cells,
                   (long long)g_workgroups);
  };
  int accepted = 0, refused = 0;
  alignas(16) static char x[64];
  static int32_t table[1], first[1], rows[2] = {0, 1};
  for (int heads : {1, 2, 3, 8, 31, 32, 33, 64, 127, 128, 1000, 4096, 16383, 32767})
    for (int page : {16, 64}) {
      spp_pool_config cfg{1, heads, 64, SPP_CELLS_I8, page, 1, 1};
      std::vector<char> pages(spp_pool_bytes(&cfg));
      spp_pool_t pool = nullptr;
      if (spp_pool_create(&cfg, pages.data(), pages.size(), &pool) != SPP_OK) {
        check(false, spp_last_error(), heads, page, 0);
        continue;
      }
      const int64_t border = kMost / heads;
      for (int64_t cells : {(int64_t)1, (int64_t)383, (int64_t)384, border / 2, border - 200, border - 1, border, border + 1,
                            border + 17, border + 65, border + 1000, 2 * border, (int64_t)1 << 24}) {
        if (cells < 1 || cells > 1 << 24) continue;
        const int64_t row = (int64_t)heads * 64;
        const spp_paged_cells a{pool, 0, 1, table, 1, 1, first, rows, 1, (int32_t)cells, SPP_DTYPE_F32, x, row, x, row};
        for (const auto call : {spp_paged_write, spp_paged_read}) {
          g_workgroups = -1;
          const spp_status rc = call(&a, nullptr);
          if (cells * heads <= kMost) {
            check(rc == SPP_OK, "refused", heads, page, cells);
            check(g_workgroups > 0 && g_workgroups * 256 < (1ll << 32), "too many threads", heads, page, cells);
            ++accepted;
          } else {
            check(rc == SPP_E_INVALID_ARG && g_workgroups < 0, "launched", heads, page, cells);
            ++refused;
          }
        }
      }
      spp_pool_destroy(pool);
    }
  check(accepted > 100 && refused > 100, "cases", accepted, refused, 0);
  if (g_fail) return 1;
  std::printf("OK\n");
  return 0;
}
