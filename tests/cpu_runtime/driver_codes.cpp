// Scenarios for pools of 8-bit codes (pool.cpp, cells.cpp, logprobs.cpp) over host stand-ins for HIP and the
// kernels, run under AddressSanitizer and ThreadSanitizer by tests/test_codes_host.py:
//   1. sessions of models of either dtype go in and out, and the kernels are told their element's size;
//   2. copies on write and compaction carry a page's scales;
//   3. what spp_paged_write and spp_paged_read refuse, and what they hand on;
//   4. the checks of spp_logprobs, and what it hands on;
//   5. several threads write, fork and reserve.
// Prints "OK" and exits 0 when every check holds.
#include <atomic>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <thread>
#include <vector>

#include <hip/hip_runtime.h>

#include "paged.hpp"
#include "spp.h"

namespace {
std::mutex g_mu;
int g_given = 0;                        // of the last session copy
std::vector<spp::CellRows> g_calls;     // writes and reads
int g_layer = -1, g_rows = 0;
}  // namespace

namespace spp {
namespace k {

int paged_splits(const PageView&, int, int, int) { return 1; }
size_t paged_work_bytes(const PageView&, int, int, int) { return 0; }
hipError_t paged_attention(const PageView&, int, const PagedAttn&, void*, hipStream_t) { return hipSuccess; }
hipError_t page_copy(const PageView& v, const PageList& l, int n, hipStream_t st) {
  stub::enqueue(st, [=] {
    for (int i = 0; i < n; ++i) std::memcpy(v.base + l.b[i] * v.page(), v.base + l.a[i] * v.page(), v.page());
  });
  return hipSuccess;
}
hipError_t page_session(const PageView& v, const PageList&, int, void* kv, int64_t, int64_t, int, bool to_pages,
                        hipStream_t st) {
  std::lock_guard<std::mutex> lk(g_mu);
  g_given = v.given;
  stub::enqueue(st, [=] {
    if (to_pages) *v.base = *static_cast<char*>(kv);
  });
  return hipSuccess;
}
hipError_t paged_epilogue(const Shape&, const StepView&, int, int, const PageView&, const int32_t*, int64_t,
                          const float*, int, const float*, const float2*, float*, hipStream_t) {
  return hipSuccess;
}
size_t adjust_work_bytes(int n, int) { return (size_t)n * 16; }
hipError_t adjust_logits(int, int, const spp_adjust*, spp_summary*, void*, hipStream_t) { return hipSuccess; }

hipError_t code_write(const PageView& v, int layer, const CellRows& c, hipStream_t) {
  std::lock_guard<std::mutex> lk(g_mu);
  g_calls.push_back(c);
  g_layer = layer;
  return v.code ? hipSuccess : hipErrorInvalidValue;
}
hipError_t code_read(const PageView& v, int layer, const CellRows& c, hipStream_t st) {
  return code_write(v, layer, c, st);
}
size_t logprob_work_bytes(int n, int, int top) { return (size_t)n * (16 + 8 * top); }
hipError_t logprobs(int n, int, const spp_logprob_row* rows, int, int32_t*, float*, float*, float*, void*, hipStream_t) {
  for (int i = 0; i < n; ++i) g_rows += rows[i].n_tokens;
  return hipSuccess;
}

}  // namespace k
}  // namespace spp

namespace {

std::atomic<int> g_fail{0};
#define CHECK(c)                                                                     \
  do {                                                                               \
    if (!(c)) {                                                                      \
      std::fprintf(stderr, "%s:%d: check failed: %s (%s)\n", __FILE__, __LINE__, #c, \
                   spp_last_error());                                                \
      ++g_fail;                                                                      \
    }                                                                                \
  } while (0)

constexpr int kLayers = 2, kD = 64, kNq = 2, kNkv = 1, kDh = 64, kF = 64, kV = 512;

struct Model {
  std::vector<void*> bufs;
  std::vector<const void*> per[9];
  spp_model_t m = nullptr;
  void* dev(size_t n) {
    void* p = nullptr;
    hipMalloc(&p, n);
    bufs.push_back(p);
    return p;
  }
  explicit Model(int dtype, int kv = kNkv) {
    spp_weights w{};
    w.embed = dev((size_t)kV * kD * 4);
    w.final_norm = dev(kD * 4);
    w.lm_head = dev((size_t)kV * kD * 4);
    for (auto& p : per)
      for (int l = 0; l < kLayers; ++l) p.push_back(dev((size_t)kNq * kDh * kD * 4));
    w.attn_norm = per[0].data();
    w.wq = per[1].data();
    w.wk = per[2].data();
    w.wv = per[3].data();
    w.wo = per[4].data();
    w.mlp_norm = per[5].data();
    w.w_gate = per[6].data();
    w.w_up = per[7].data();
    w.w_down = per[8].data();
    spp_model_config c{};
    c.n_layers = kLayers;
    c.d_model = kD;
    c.n_q_heads = kNq;
    c.n_kv_heads = kv;
    c.head_dim = kDh;
    c.ffn_dim = kF;
    c.vocab = kV;
    c.rms_eps = 1e-5f;
    c.rope_base = 1e4;
    c.dtype = dtype;
    c.max_tokens = 16;
    c.max_sessions = 4;
    CHECK(spp_model_create(&c, &w, &m) == SPP_OK);
  }
  ~Model() {
    spp_model_destroy(m);
    for (void* p : bufs) hipFree(p);
  }
};

struct Session {
  void* kv = nullptr;
  spp_session_t s = nullptr;
  Session(Model& m, int cells) {
    const size_t n = spp_session_kv_bytes(m.m, cells);
    hipMalloc(&kv, n);
    std::memset(kv, 0x5A, n);
    const spp_session_config c{cells, 0};
    CHECK(spp_session_create(m.m, &c, kv, n, &s) == SPP_OK);
  }
  ~Session() {
    hipDeviceSynchronize();
    spp_session_destroy(s);
    hipFree(kv);
  }
};

struct Pool {
  spp_pool_config cfg{kLayers, kNkv, kDh, 0, 16, 0, 16};
  spp_page_layout lay{};
  char* pages = nullptr;
  spp_pool_t p = nullptr;
  Pool(int dtype, int n_pages) {
    cfg.dtype = dtype;
    cfg.n_pages = n_pages;
    hipMalloc((void**)&pages, spp_pool_bytes(&cfg));
    CHECK(spp_pool_page_layout(&cfg, &lay) == SPP_OK);
    CHECK(spp_pool_create(&cfg, pages, spp_pool_bytes(&cfg), &p) == SPP_OK);
  }
  ~Pool() {
    spp_pool_destroy(p);
    hipFree(pages);
  }
  std::vector<int32_t> table(int seq) {
    int32_t n = 0;
    CHECK(spp_seq_table(p, seq, nullptr, 0, &n) == SPP_OK);
    std::vector<int32_t> t(n);
    CHECK(spp_seq_table(p, seq, t.data(), n, &n) == SPP_OK);
    return t;
  }
};

void sessions() {
  for (int code : {SPP_CELLS_I8, SPP_CELLS_E4M3})
    for (int dtype : {SPP_DTYPE_F32, SPP_DTYPE_BF16}) {
      Model m(dtype);
      Pool pool(code, 8);
      Session sess(m, 64);
      CHECK(spp_session_restore(sess.s, 40) == SPP_OK);
      int32_t q = -1;
      CHECK(spp_seq_create(pool.p, 0, &q) == SPP_OK);
      g_given = 0;
      CHECK(spp_seq_import(pool.p, q, sess.s, nullptr) == SPP_OK);
      CHECK(g_given == (dtype == SPP_DTYPE_F32 ? 4 : 2));
      CHECK(pool.table(q).size() == 3);
      CHECK(spp_seq_export(pool.p, q, sess.s, nullptr) == SPP_OK);
      // a decode step of a model of either dtype
      std::vector<float> d(kV);
      float* dist = d.data();
      const int32_t tok = 3;
      CHECK(spp_decode_batch(pool.p, m.m, 1, &q, &tok, &dist, nullptr) == SPP_OK);
      hipDeviceSynchronize();
      spp_seq_info_t info;
      CHECK(spp_seq_info(pool.p, q, &info) == SPP_OK && info.n_cells == 41);
    }
  // other shapes, and pools of values, keep their checks
  Model f32(SPP_DTYPE_F32), two(SPP_DTYPE_BF16, 2);
  Pool codes(SPP_CELLS_I8, 8), values(SPP_DTYPE_BF16, 8);
  Session a(f32, 64), b(two, 64);
  spp_session_restore(a.s, 10);
  spp_session_restore(b.s, 10);
  int32_t q = -1, v = -1;
  CHECK(spp_seq_create(codes.p, 0, &q) == SPP_OK && spp_seq_create(values.p, 0, &v) == SPP_OK);
  CHECK(spp_seq_import(codes.p, q, b.s, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_import(values.p, v, a.s, nullptr) == SPP_E_INVALID_ARG);
}

void copies() {
  Pool pool(SPP_CELLS_E4M3, 12);
  std::memset(pool.pages, 0, pool.lay.page_stride * 12);
  spp_scale_layout sc;
  CHECK(spp_pool_scale_layout(&pool.cfg, &sc) == SPP_OK);
  int32_t base = -1, forks[3];
  CHECK(spp_seq_create(pool.p, 37, &base) == SPP_OK);
  auto scale = [&](int page, int layer, bool v) {
    return reinterpret_cast<float*>(pool.pages + page * pool.lay.page_stride + layer * pool.lay.layer_stride +
                                    (v ? sc.v_offset : sc.k_offset));
  };
  for (int page : pool.table(base))
    for (int l = 0; l < kLayers; ++l)
      for (int v = 0; v < 2; ++v) *scale(page, l, v) = 1.f + page + 10 * l + 100 * v;
  CHECK(spp_seq_fork(pool.p, base, 3, forks) == SPP_OK);
  CHECK(spp_seq_reserve(pool.p, 3, forks, 1, nullptr) == SPP_OK);
  hipDeviceSynchronize();
  auto same = [&](int seq) {
    const int page = pool.table(seq)[2];
    for (int l = 0; l < kLayers; ++l)
      for (int v = 0; v < 2; ++v)
        if (*scale(page, l, v) != 3.f + 10 * l + 100 * v) return false;
    return true;
  };
  for (int32_t f : forks) CHECK(pool.table(f)[2] != pool.table(base)[2] && same(f));
  CHECK(spp_seq_free(pool.p, forks[0]) == SPP_OK);
  int32_t moved = 0;
  CHECK(spp_pool_compact(pool.p, nullptr, &moved) == SPP_OK && moved == 1);
  hipDeviceSynchronize();
  CHECK(same(forks[1]) && same(forks[2]) && same(base));
}

void cells() {
  Pool pool(SPP_CELLS_I8, 8), values(SPP_DTYPE_BF16, 8);
  char* x = nullptr;
  hipMalloc((void**)&x, 1 << 16);
  int32_t tab[8] = {}, first[2] = {}, rows[3] = {};
  const spp_paged_cells good{pool.p, 1, 2, tab, 4, 4, first, rows, 5, 3, SPP_DTYPE_BF16, x, 64, x, 72};
  CHECK(spp_paged_write(&good, nullptr) == SPP_OK && spp_paged_read(&good, nullptr) == SPP_OK);
  CHECK(g_calls.size() == 2 && g_layer == 1);
  const spp::CellRows c = g_calls[0];
  CHECK(c.n == 2 && c.table == tab && c.table_stride == 4 && c.max_pages == 4 && c.first == first && c.rows == rows &&
        c.n_rows == 5 && c.max_cells == 3 && c.bf16 == 1 && c.k == x && c.k_stride == 64 && c.v_stride == 72);
  g_calls.clear();
  CHECK(spp_paged_write(nullptr, nullptr) == SPP_E_INVALID_ARG);
  for (int bad = 0; bad < 25; ++bad) {
    spp_paged_cells b = good;
    switch (bad) {
      case 0: b.pool = nullptr; break;
      case 1: b.pool = values.p; break;
      case 2: b.layer = kLayers; break;
      case 3: b.layer = -1; break;
      case 4: b.n_seqs = -1; break;
      case 5: b.n_seqs = 65536; break;
      case 6: b.table = nullptr; break;
      case 7: b.table_stride = 3; break;
      case 8: b.max_pages = 0; break;
      case 9: b.max_pages = (1 << 26) + 1; b.table_stride = 1 << 27; break;
      case 10: b.first = nullptr; break;
      case 11: b.rows = nullptr; break;
      case 12: b.n_rows = -1; break;
      case 13: b.max_cells = 0; break;
      case 14: b.max_cells = (1 << 24) + 1; break;
      case 15: b.io_dtype = SPP_CELLS_I8; break;
      case 16: b.k = nullptr; break;
      case 17: b.v = nullptr; break;
      case 18: b.k = x + 8; break;
      case 19: b.v = x + 2; break;
      case 20: b.k_stride = 56; break;
      case 21: b.v_stride = 68; break;
      case 22: b.table = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(tab) + 2); break;
      case 23: b.first = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(first) + 1); break;
      case 24: b.rows = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(rows) + 3); break;
    }
    CHECK(spp_paged_write(&b, nullptr) == SPP_E_INVALID_ARG);
    CHECK(spp_paged_read(&b, nullptr) == SPP_E_INVALID_ARG);
  }
  spp_paged_cells none = good;  // nothing to do: no launch
  none.n_seqs = 0;
  none.table = nullptr;
  CHECK(spp_paged_write(&none, nullptr) == SPP_OK);
  none = good;
  none.n_rows = 0;
  none.k = none.v = nullptr;
  CHECK(spp_paged_read(&none, nullptr) == SPP_OK);
  CHECK(g_calls.empty());
  // attention over such a pool is the same call
  int32_t len[1] = {5};
  const spp_paged_attn a{pool.p, 0, 1, 2, SPP_DTYPE_F32, x, 128, tab, 4, 4, len, 0.f, x, 128};
  CHECK(spp_paged_attention(&a, nullptr, 0, nullptr) == SPP_OK);
  hipFree(x);
}

void logprobs() {
  float x[64];
  int32_t t[4];
  alignas(16) char work[256];
  spp_logprob_row rows[2] = {{x, t, x, 3}, {x, nullptr, nullptr, 0}};
  CHECK(spp_logprobs_work_bytes(2, 10, 1) == 48);
  CHECK(spp_logprobs(2, 10, rows, 1, t, x, x, nullptr, work, 48, nullptr) == SPP_OK && g_rows == 3);
  CHECK(spp_logprobs(2, 10, rows, 0, nullptr, nullptr, nullptr, x, work, 48, nullptr) == SPP_OK && g_rows == 6);
  CHECK(spp_logprobs(2, 10, rows, 1, t, x, x, x, work, 47, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_logprobs(2, 10, rows, 1, t, x, x, x, work + 4, 200, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_logprobs(2, 10, rows, 1, nullptr, x, x, x, work, 48, nullptr) == SPP_E_INVALID_ARG);
  rows[1].n_tokens = 1;
  CHECK(spp_logprobs(2, 10, rows, 1, t, x, x, x, work, 48, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_logprobs(0, 10, nullptr, 0, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr) == SPP_OK);
  CHECK(g_rows == 6);
}

void threads() {
  Pool pool(SPP_CELLS_I8, 64);
  std::memset(pool.pages, 0, pool.lay.page_stride * 64);
  char* x = nullptr;
  hipMalloc((void**)&x, 1 << 12);
  int32_t tab[4] = {}, first[1] = {}, rows[2] = {};
  const spp_paged_cells call{pool.p, 0, 1, tab, 4, 4, first, rows, 1, 1, SPP_DTYPE_BF16, x, 64, x, 64};
  std::vector<std::thread> ts;
  for (int k = 0; k < 4; ++k)
    ts.emplace_back([&] {
      for (int i = 0; i < 50; ++i) {
        int32_t q = -1, f[2];
        CHECK(spp_seq_create(pool.p, 20, &q) == SPP_OK);
        CHECK(spp_seq_fork(pool.p, q, 1, f) == SPP_OK);
        CHECK(spp_seq_reserve(pool.p, 1, f, 1, nullptr) == SPP_OK);
        CHECK(spp_paged_write(&call, nullptr) == SPP_OK);
        CHECK(spp_seq_commit(pool.p, f[0], 1) == SPP_OK);
        CHECK(spp_seq_free(pool.p, f[0]) == SPP_OK && spp_seq_free(pool.p, q) == SPP_OK);
      }
    });
  for (auto& t : ts) t.join();
  hipDeviceSynchronize();
  spp_pool_info_t info;
  CHECK(spp_pool_info(pool.p, &info) == SPP_OK && info.used_pages == 0);
  hipFree(x);
}

}  // namespace

int main() {
  sessions();
  copies();
  cells();
  logprobs();
  threads();
  if (g_fail) return 1;
  std::printf("OK\n");
  return 0;
}
