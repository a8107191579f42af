// Scenarios for the order of a pool's device work (pool.cpp) over host stand-ins for HIP and the
// kernels, run under AddressSanitizer and ThreadSanitizer by tests/test_pool_line.py, one to a
// process: the name of the scenario is the argument.  Prints "OK" and exits 0 when every check
// holds.  The stand-ins of the paged kernels are here: a copy moves its bytes when its stream
// comes to it, and one may be told to fail.
#include <atomic>
#include <chrono>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <thread>
#include <vector>

#include <hip/hip_runtime.h>

#include "paged.hpp"
#include "spp.h"

namespace {
int g_launches_left = -1;  // copies that still start (-1: all)
bool launch_fails() { return g_launches_left == 0 || (g_launches_left > 0 && g_launches_left-- == 0); }
}  // namespace

namespace spp {
namespace k {

int paged_splits(const PageView&, int, int, int) { return 1; }
size_t paged_work_bytes(const PageView&, int n, int n_q, int max_pages) {  // (falls, as a rule on n may)
  return n >= 16 && max_pages < 100 ? 0 : (size_t)n_q * max_pages * (n >= 5 ? n : 2 * n);
}
hipError_t paged_attention(const PageView&, int, const PagedAttn&, void*, hipStream_t) { return hipSuccess; }

hipError_t page_copy(const PageView& v, const PageList& l, int n, hipStream_t st) {
  if (launch_fails()) return hipErrorInvalidValue;
  stub::enqueue(st, [=] {
    for (int i = 0; i < n; ++i) std::memcpy(v.base + l.b[i] * v.page(), v.base + l.a[i] * v.page(), v.page());
  });
  return hipSuccess;
}

hipError_t page_session(const PageView& v, const PageList& l, int n, void* kv, int64_t, int64_t, int, bool to_pages,
                        hipStream_t st) {
  if (launch_fails()) return hipErrorInvalidValue;
  stub::enqueue(st, [=] {  // (a byte of each page stands for its cells)
    for (int i = 0; i < n; ++i) {
      char *p = v.base + l.a[i] * v.page(), *s = static_cast<char*>(kv);
      if (to_pages) *p = *s; else *s = *p;
    }
  });
  return hipSuccess;
}

hipError_t paged_epilogue(const Shape&, const StepView&, int, int, const PageView&, const int32_t*, int64_t,
                          const float*, int, const float*, const float2*, float*, hipStream_t) {
  return hipSuccess;
}
size_t adjust_work_bytes(int n, int) { return (size_t)n * 16; }
hipError_t adjust_logits(int, int, const spp_adjust*, spp_summary*, void*, hipStream_t) { return hipSuccess; }

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

constexpr int kLayers = 2, kD = 64, kDh = 64, kV = 512, kPage = 16;

struct Pool {
  spp_pool_config cfg{};
  spp_page_layout lay{};
  char* pages = nullptr;
  spp_pool_t p = nullptr;
  Pool(int n_pages, int max_seqs) {
    cfg.n_layers = kLayers;
    cfg.n_kv_heads = 1;
    cfg.head_dim = kDh;
    cfg.dtype = SPP_DTYPE_BF16;
    cfg.page_cells = kPage;
    cfg.n_pages = n_pages;
    cfg.max_seqs = max_seqs;
    hipMalloc((void**)&pages, spp_pool_bytes(&cfg));
    CHECK(spp_pool_page_layout(&cfg, &lay) == SPP_OK);
    CHECK(spp_pool_create(&cfg, pages, spp_pool_bytes(&cfg), &p) == SPP_OK);
  }
  ~Pool() {
    spp_pool_destroy(p);
    hipFree(pages);
  }
  int create(int cells) {
    int32_t q = -1;
    CHECK(spp_seq_create(p, cells, &q) == SPP_OK);
    return q;
  }
  std::vector<int32_t> table(int seq) {
    int32_t n = 0;
    CHECK(spp_seq_table(p, seq, nullptr, 0, &n) == SPP_OK);
    std::vector<int32_t> t(n);
    CHECK(spp_seq_table(p, seq, t.data(), n, &n) == SPP_OK);
    return t;
  }
  char* page(int i) { return pages + i * lay.page_stride; }
  void fill(int i, int tag) { std::memset(page(i), tag, lay.page_stride); }
  bool holds(int i, int tag) {
    for (int64_t b = 0; b < lay.page_stride; ++b)
      if (page(i)[b] != (char)tag) return false;
    return true;
  }
};

struct Streams {
  hipStream_t st[2];
  Streams() {
    for (hipStream_t& s : st) hipStreamCreate(&s);
  }
  ~Streams() {
    for (hipStream_t s : st) hipStreamDestroy(s);
  }
  hipStream_t operator[](int i) const { return st[i]; }
};

// Work that keeps a stream for a while.
void busy(hipStream_t st) {
  stub::enqueue(st, [] { std::this_thread::sleep_for(std::chrono::milliseconds(30)); });
}

// A page that a compaction is still reading is free on the host: a reserve that copies nothing may
// hand it out, and what its caller then writes on the reserve's stream comes after that read.
void reserve_orders() {
  Streams st;
  Pool pool(8, 4);
  const int a = pool.create(kPage), b = pool.create(kPage), c = pool.create(0);
  pool.fill(0, 1);
  pool.fill(1, 2);
  CHECK(spp_seq_free(pool.p, a) == SPP_OK);
  busy(st[0]);
  int32_t moved = 0;
  CHECK(spp_pool_compact(pool.p, st[0], &moved) == SPP_OK && moved == 1);
  CHECK(spp_seq_reserve(pool.p, 1, &c, 1, st[1]) == SPP_OK);
  CHECK(pool.table(b) == std::vector<int32_t>{0} && pool.table(c) == std::vector<int32_t>{1});
  stub::enqueue(st[1], [&] { pool.fill(1, 9); });
  hipDeviceSynchronize();
  CHECK(pool.holds(0, 2) && pool.holds(1, 9));
}

// A copy on write of more pages than one launch lists, whose second launch fails: the first one's
// target pages are free again, and who takes them comes after it.
void failed_page_copy() {
  constexpr int kForks = 300;
  Streams st;
  Pool pool(2 + 2 * kForks, kForks + 2);
  const int a = pool.create(5), d = pool.create(0);
  pool.fill(0, 7);
  std::vector<int32_t> forks(kForks);
  CHECK(spp_seq_fork(pool.p, a, kForks, forks.data()) == SPP_OK);
  busy(st[0]);
  g_launches_left = 1;
  CHECK(spp_seq_reserve(pool.p, kForks, forks.data(), 1, st[0]) == SPP_E_HIP);
  g_launches_left = -1;
  spp_pool_info_t i;
  CHECK(spp_pool_info(pool.p, &i) == SPP_OK && i.used_pages == 1 && i.shared_pages == 1);
  for (int32_t f : forks) CHECK(pool.table(f) == std::vector<int32_t>{0});
  CHECK(spp_seq_reserve(pool.p, 1, &d, 1, st[1]) == SPP_OK && pool.table(d) == std::vector<int32_t>{1});
  stub::enqueue(st[1], [&] { pool.fill(1, 9); });
  hipDeviceSynchronize();
  CHECK(pool.holds(0, 7) && pool.holds(1, 9));
}

// A reserve that fails gives back the pages it added to the tables too, shared ones copied or not.
void failed_reserve_changes_nothing() {
  Streams st;
  Pool pool(20, 6);
  const int a = pool.create(5), b = pool.create(kPage), c = pool.create(0), e = pool.create(3);
  int32_t f = -1;
  CHECK(spp_seq_fork(pool.p, a, 1, &f) == SPP_OK);
  CHECK(spp_seq_reserve(pool.p, 1, &e, 2 * kPage, st[0]) == SPP_OK);  // (an earlier reserve stays)
  spp_pool_info_t was, now;
  CHECK(spp_pool_info(pool.p, &was) == SPP_OK);
  std::map<int, std::vector<int32_t>> tables;
  for (int q : {a, b, c, e, f}) tables[q] = pool.table(q);
  const int32_t all[] = {b, f, c, e, a};
  for (int cells : {1, kPage, 3 * kPage}) {
    g_launches_left = 0;
    CHECK(spp_seq_reserve(pool.p, 5, all, cells, st[1]) == SPP_E_HIP);
    g_launches_left = -1;
    CHECK(spp_pool_info(pool.p, &now) == SPP_OK && std::memcmp(&was, &now, sizeof now) == 0);
    for (int q : {a, b, c, e, f}) CHECK(pool.table(q) == tables[q]);
  }
  CHECK(spp_seq_reserve(pool.p, 5, all, kPage, st[1]) == SPP_OK);
  CHECK(spp_pool_info(pool.p, &now) == SPP_OK && now.shared_pages == 0);
  hipDeviceSynchronize();
}

struct Model {
  std::vector<void*> bufs;
  std::vector<const void*> layers;
  spp_model_t m = nullptr;
  spp_session_t s = nullptr;
  void* kv = nullptr;
  void* dev(size_t n) {
    void* p = nullptr;
    hipMalloc(&p, n);
    bufs.push_back(p);
    return p;
  }
  explicit Model(int cells) {  // and a session of it with so many cells
    spp_weights w{};
    w.embed = dev((size_t)kV * kD * 2);
    w.final_norm = dev(kD * 2);
    w.lm_head = dev((size_t)kV * kD * 2);
    layers.assign(kLayers, dev((size_t)kD * kD * 2));  // (one buffer is every matrix: all are 64 x 64)
    for (const void* const** p : {&w.attn_norm, &w.wq, &w.wk, &w.wv, &w.wo, &w.mlp_norm, &w.w_gate, &w.w_up, &w.w_down})
      *p = layers.data();
    spp_model_config c{};
    c.n_layers = kLayers;
    c.d_model = kD;
    c.n_q_heads = c.n_kv_heads = 1;
    c.head_dim = kDh;
    c.ffn_dim = kD;
    c.vocab = kV;
    c.rms_eps = 1e-5f;
    c.rope_base = 1e4;
    c.dtype = SPP_DTYPE_BF16;
    c.max_tokens = 16;
    c.max_sessions = 1;
    CHECK(spp_model_create(&c, &w, &m) == SPP_OK);
    kv = dev(spp_session_kv_bytes(m, cells + 64));
    const spp_session_config sc{cells + 64, 0};
    CHECK(spp_session_create(m, &sc, kv, spp_session_kv_bytes(m, cells + 64), &s) == SPP_OK);
    CHECK(spp_session_restore(s, cells) == SPP_OK);
  }
  ~Model() {
    spp_session_destroy(s);
    spp_model_destroy(m);
    for (void* p : bufs) hipFree(p);
  }
};

// An import and an export of more pages than one launch lists, whose second launch fails: what
// the first launch reads and writes is used by the model's next step, and by the pool's next
// work, after it.
void failed_session_copy() {
  for (int it = 0; it < 4; ++it) {
    Streams st;
    Pool pool(300, 4);
    Model model(257 * kPage);
    const int q = pool.create(it & 1 ? 257 * kPage : 0), c = pool.create(0);
    bool first = false, seen = false;
    busy(st[0]);
    stub::enqueue(st[0], [&] { first = true; });
    g_launches_left = 1;
    CHECK((it & 1 ? spp_seq_export : spp_seq_import)(pool.p, q, model.s, st[0]) == SPP_E_HIP);
    g_launches_left = -1;
    const int32_t tok = 3;
    if (it & 2)
      CHECK(spp_kv_append_delta(model.s, &tok, 1, st[1]) == SPP_OK);
    else
      CHECK(spp_seq_reserve(pool.p, 1, &c, 1, st[1]) == SPP_OK);
    stub::enqueue(st[1], [&] { seen = first; });
    hipDeviceSynchronize();
    CHECK(seen);
    spp_seq_info_t i;  // what a failed copy leaves is no state
    spp_session_info_t si;
    CHECK(spp_seq_info(pool.p, q, &i) == SPP_OK && spp_session_info(model.s, &si) == SPP_OK);
    if (it & 1)
      CHECK(si.n_committed == (it & 2 ? 1 : 0) && i.n_cells == 257 * kPage);
    else
      CHECK(i.n_cells == 0);
  }
}

// A workspace for a call serves every smaller one, whatever the rule does with their number; a
// call is held to what itself needs.
void workspace_of_smaller_calls() {
  Pool pool(4, 4);
  std::vector<int32_t> tab(4096, 0), len(64, 1);
  alignas(16) static char io[64 * 4 * kDh * 2], work[1 << 16];
  const auto call = [&](int n, int max_pages) {
    return spp_paged_attn{pool.p, 0, n, 4, SPP_DTYPE_BF16, io, 4 * kDh, tab.data(), max_pages, max_pages, len.data(),
                          0.f, io, 4 * kDh};
  };
  for (int max_pages : {1, 60}) {
    size_t most = 0;
    for (int n = 1; n <= 40; ++n) {
      const spp_paged_attn a = call(n, max_pages), less = call(n, max_pages / 2 + 1);
      const size_t bytes = spp_paged_attention_work_bytes(&a);
      CHECK(bytes >= most && bytes >= spp_paged_attention_work_bytes(&less));
      most = bytes;
    }
    CHECK(most == (size_t)4 * max_pages * 15);
    for (int n = 1; n <= 40; ++n) {
      const spp_paged_attn a = call(n, max_pages);
      CHECK(spp_paged_attention(&a, work, most, nullptr) == SPP_OK);
      CHECK(spp_paged_attention(&a, nullptr, 0, nullptr) == (n >= 16 ? SPP_OK : SPP_E_INVALID_ARG));
    }
  }
}

// A model's step waits for the copies of its sessions' cells, and for nothing that the pool does
// after them: later work of the pool that waits for that step (here for what follows it on its
// stream) gets to see it.  Two pools take turns at the model, so that every copy has one before it.
void later_work_holds_no_step() {
  Streams st;
  Pool pool(16, 6), other(16, 6);
  Model model(20);
  for (int it = 0; it < 12; ++it) {
    Pool& p = it % 3 == 2 ? other : pool;
    const int low = p.create(kPage), q = p.create(0);
    std::atomic<bool> copied{false}, stepped{false};
    bool in_order = false, seen = false;
    busy(st[0]);
    stub::enqueue(st[0], [&] { copied = true; });
    CHECK(spp_seq_import(p.p, q, model.s, st[0]) == SPP_OK);
    if (it & 1) CHECK(spp_seq_export(p.p, q, model.s, st[0]) == SPP_OK);
    CHECK(spp_seq_free(p.p, low) == SPP_OK);
    stub::enqueue(st[0], [&] {
      for (int ms = 0; ms < 3000 && !stepped; ++ms) std::this_thread::sleep_for(std::chrono::milliseconds(1));
      seen = stepped;
    });
    int32_t moved = 0;
    CHECK(spp_pool_compact(p.p, st[0], &moved) == SPP_OK && moved == 1);
    const int32_t tok = 3;
    if (it & 2)
      CHECK(spp_shift(model.s, 1, st[1]) == SPP_OK);
    else
      CHECK(spp_kv_append_delta(model.s, &tok, 1, st[1]) == SPP_OK);
    stub::enqueue(st[1], [&] {
      in_order = copied;
      stepped = true;
    });
    hipDeviceSynchronize();
    CHECK(in_order && seen);
    CHECK(spp_seq_free(p.p, q) == SPP_OK && spp_session_restore(model.s, 20) == SPP_OK);
    if (g_fail) return;
  }
}

// More models wait for copies of one pool than it has events: each still comes after its own copy,
// with the pool's later work in between or not, and when it has waited its event is the pool's again.
void more_models_than_events() {
  constexpr int kModels = 6;
  Streams st;
  Pool pool(64, 8);
  Model models[kModels] = {Model(20), Model(20), Model(20), Model(20), Model(20), Model(20)};
  for (int round = 0; round < 4; ++round) {
    std::atomic<bool> copied[kModels] = {};
    bool after[kModels] = {};
    std::vector<int> seqs;
    for (int i = 0; i < kModels; ++i) {
      seqs.push_back(pool.create(0));
      stub::enqueue(st[0], [&, i] {
        std::this_thread::sleep_for(std::chrono::milliseconds(3));
        copied[i] = true;
      });
      CHECK(spp_seq_import(pool.p, seqs[i], models[i].s, st[0]) == SPP_OK);
      int32_t f = -1;
      if (i & 1) {
        CHECK(spp_seq_fork(pool.p, seqs[i], 1, &f) == SPP_OK && spp_seq_reserve(pool.p, 1, &f, 1, st[0]) == SPP_OK);
        CHECK(spp_seq_free(pool.p, f) == SPP_OK);
      }
    }
    for (int i = 0; i < kModels; ++i) {
      if (round == 1 && i % 2) continue;  // (these keep waiting for theirs)
      CHECK(spp_shift(models[i].s, 1, st[1]) == SPP_OK);
      stub::enqueue(st[1], [&, i] { after[i] = copied[i]; });
    }
    hipDeviceSynchronize();
    for (int i = 0; i < kModels; ++i) {
      CHECK(after[i] || (round == 1 && i % 2));
      CHECK(spp_seq_free(pool.p, seqs[i]) == SPP_OK && spp_session_restore(models[i].s, 20) == SPP_OK);
    }
  }
}

}  // namespace

int main(int argc, char** argv) {
  const std::map<std::string, void (*)()> scenarios = {
      {"reserve_orders", reserve_orders},
      {"failed_page_copy", failed_page_copy},
      {"failed_session_copy", failed_session_copy},
      {"failed_reserve_changes_nothing", failed_reserve_changes_nothing},
      {"workspace_of_smaller_calls", workspace_of_smaller_calls},
      {"later_work_holds_no_step", later_work_holds_no_step},
      {"more_models_than_events", more_models_than_events},
  };
  const auto it = argc > 1 ? scenarios.find(argv[1]) : scenarios.end();
  if (it == scenarios.end()) return 2;
  it->second();
  CHECK(stub::live_allocations() == 0);
  stub::shutdown();
  if (g_fail) return 1;
  std::puts("OK");
  return 0;
}
