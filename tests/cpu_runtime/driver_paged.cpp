// Scenarios for the paged sequences (pool.cpp) over host stand-ins for HIP and the kernels, run
// under AddressSanitizer and ThreadSanitizer by tests/test_paged_host.py:
//   1. random creates, forks, reserves, decode steps, truncations, frees, compactions, imports
//      and exports, each sequence's cells compared with a plain list of what they hold, the
//      page counts with the tables, on two streams in turn;
//   2. calls that are refused leave everything as it was;
//   3. several threads share a pool and a model;
//   4. the checks of the stand-alone calls;
//   5. a model's steps come after the copies of its sessions' cells, whatever streams and pools.
// Prints "OK" and exits 0 when every check holds.
#include <algorithm>
#include <atomic>
#include <chrono>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <memory>
#include <random>
#include <set>
#include <thread>
#include <vector>

#include <hip/hip_runtime.h>

#include "spp.h"

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
  explicit Model(int max_sessions, int layers = kLayers) {
    spp_weights w{};
    w.embed = dev((size_t)kV * kD * 2);
    w.final_norm = dev(kD * 2);
    w.lm_head = dev((size_t)kV * kD * 2);
    for (int k = 0; k < 9; ++k)
      for (int l = 0; l < layers; ++l) per[k].push_back(dev((size_t)kNq * kDh * kD * 2));
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
    c.n_layers = layers;
    c.d_model = kD;
    c.n_q_heads = kNq;
    c.n_kv_heads = kNkv;
    c.head_dim = kDh;
    c.ffn_dim = kF;
    c.vocab = kV;
    c.rms_eps = 1e-5f;
    c.rope_base = 1e4;
    c.dtype = SPP_DTYPE_BF16;
    c.max_tokens = 16;
    c.max_sessions = max_sessions;
    CHECK(spp_model_create(&c, &w, &m) == SPP_OK);
  }
  ~Model() {
    spp_model_destroy(m);
    for (void* p : bufs) hipFree(p);
  }
};

spp_pool_config pool_config(int page, int n_pages, int max_seqs) {
  spp_pool_config c{};
  c.n_layers = kLayers;
  c.n_kv_heads = kNkv;
  c.head_dim = kDh;
  c.dtype = SPP_DTYPE_BF16;
  c.page_cells = page;
  c.n_pages = n_pages;
  c.max_seqs = max_seqs;
  return c;
}

struct Pool {
  spp_pool_config cfg;
  spp_page_layout lay{};
  char* pages = nullptr;
  spp_pool_t p = nullptr;
  Pool(int page, int n_pages, int max_seqs) : cfg(pool_config(page, n_pages, max_seqs)) {
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
  uint16_t* at(int page, int layer, bool v, int cell, int d) {
    const int64_t* s = v ? lay.v_stride : lay.k_stride;
    return reinterpret_cast<uint16_t*>(pages + page * lay.page_stride + layer * lay.layer_stride +
                                       (v ? lay.v_offset : 0)) +
           cell * s[1] + d * s[2];
  }
  void write(int seq, int cell, uint16_t tag) {
    const auto t = table(seq);
    for (int l = 0; l < kLayers; ++l)
      for (int v = 0; v < 2; ++v)
        for (int d = 0; d < kDh; ++d) *at(t[cell / cfg.page_cells], l, v, cell % cfg.page_cells, d) = tag;
  }
  bool holds(int seq, const std::vector<uint16_t>& want) {
    spp_seq_info_t info;
    if (spp_seq_info(p, seq, &info) != SPP_OK || info.n_cells != (int)want.size()) return false;
    const auto t = table(seq);
    for (size_t c = 0; c < want.size(); ++c)
      for (int l = 0; l < kLayers; ++l)
        for (int v = 0; v < 2; ++v)
          for (int d = 0; d < kDh; d += 21)
            if (*at(t[c / cfg.page_cells], l, v, (int)c % cfg.page_cells, d) != want[c]) return false;
    return true;
  }
};

struct Sess {
  void* kv = nullptr;
  spp_session_t s = nullptr;
  spp_model_t m;
  int cap;
  Sess(spp_model_t model, int capacity) : m(model), cap(capacity) {
    hipMalloc(&kv, spp_session_kv_bytes(m, cap));
    spp_session_config c{cap, 0};
    CHECK(spp_session_create(m, &c, kv, spp_session_kv_bytes(m, cap), &s) == SPP_OK);
  }
  ~Sess() {
    spp_session_destroy(s);
    hipFree(kv);
  }
  uint16_t* at(int l, bool v, int cell, int d) {
    spp_kv_layout y;
    spp_session_kv_layout(m, cap, l, &y);
    const int64_t* st = v ? y.v_stride : y.k_stride;
    return reinterpret_cast<uint16_t*>(static_cast<char*>(kv) + (v ? y.v_offset : y.k_offset)) + cell * st[1] +
           d * st[2];
  }
  void fill(const std::vector<uint16_t>& w) {
    for (size_t c = 0; c < w.size(); ++c)
      for (int l = 0; l < kLayers; ++l)
        for (int v = 0; v < 2; ++v)
          for (int d = 0; d < kDh; ++d) *at(l, v, (int)c, d) = w[c];
    CHECK(spp_session_restore(s, (int)w.size()) == SPP_OK);
  }
  bool holds(const std::vector<uint16_t>& w) {
    spp_session_info_t i;
    if (spp_session_info(s, &i) != SPP_OK || i.n_committed != (int)w.size() || i.valid) return false;
    for (size_t c = 0; c < w.size(); ++c)
      for (int l = 0; l < kLayers; ++l)
        for (int v = 0; v < 2; ++v)
          for (int d = 0; d < kDh; d += 13)
            if (*at(l, v, (int)c, d) != w[c]) return false;
    return true;
  }
};

void random_calls(unsigned seed, int page, int n_pages) {
  std::mt19937 rng(seed);
  auto below = [&](int n) { return (int)(rng() % (unsigned)std::max(1, n)); };
  Model model(4);
  hipStream_t st[2];
  hipStreamCreate(&st[0]);
  hipStreamCreate(&st[1]);
  {
    Pool pool(page, n_pages, 12);
    Sess sess(model.m, 300), into(model.m, 300);
    std::vector<float> dist(12 * kV);
    std::map<int, std::vector<uint16_t>> have;  // what each sequence should hold
    auto pick = [&] { return std::next(have.begin(), below((int)have.size()))->first; };
    for (int step = 0; step < 400; ++step) {
      hipStream_t s = st[below(2)];
      const int op = have.empty() ? 0 : below(10);
      if (op == 0) {
        const int n = below(4 * page);
        int32_t q = -1;
        const spp_status rc = spp_seq_create(pool.p, n, &q);
        CHECK(rc == SPP_OK || rc == SPP_E_CAPACITY);
        if (rc == SPP_OK) {
          CHECK(!have.count(q));
          hipDeviceSynchronize();
          for (int c = 0; c < n; ++c) {
            have[q].push_back((uint16_t)(seed * 31 + step * 7 + c));
            pool.write(q, c, have[q].back());
          }
          have[q];
        }
      } else if (op == 1 || op == 2) {
        const int src = pick(), n = 1 + below(4);
        int32_t q[4];
        const spp_status rc = spp_seq_fork(pool.p, src, n, q);
        CHECK(rc == (n <= 12 - (int)have.size() ? SPP_OK : SPP_E_CAPACITY));
        if (rc == SPP_OK)
          for (int i = 0; i < n; ++i) {
            CHECK(!have.count(q[i]));
            have[q[i]] = have[src];
          }
      } else if (op <= 5) {  // a decode step of some of them
        std::vector<int32_t> qs, toks;
        std::vector<float*> ds;
        for (auto& h : have)
          if (below(2)) {
            qs.push_back(h.first);
            toks.push_back(below(kV));
            ds.push_back(&dist[h.first * kV]);
          }
        if (qs.empty()) continue;
        std::shuffle(qs.begin(), qs.end(), rng);
        const spp_status rc = spp_decode_batch(pool.p, model.m, (int)qs.size(), qs.data(), toks.data(), ds.data(), s);
        CHECK(rc == SPP_OK || rc == SPP_E_CAPACITY);
        if (rc == SPP_OK) {
          for (size_t i = 0; i < qs.size(); ++i) have[qs[i]].push_back((uint16_t)toks[i]);
          std::vector<spp_summary> sum(qs.size());
          CHECK(spp_seq_summaries(pool.p, (int)qs.size(), qs.data(), sum.data()) == SPP_OK);
          for (size_t i = 0; i < qs.size(); ++i) CHECK(sum[i].position == (int)have[qs[i]].size());
        }
      } else if (op == 6) {  // cells that the caller writes
        const int q = pick(), n = 1 + below(2 * page);
        const int32_t qq = q;
        const spp_status rc = spp_seq_reserve(pool.p, 1, &qq, n, s);
        CHECK(rc == SPP_OK || rc == SPP_E_CAPACITY);
        if (rc == SPP_OK) {
          hipDeviceSynchronize();
          const int w = 1 + below(n), at = (int)have[q].size();
          for (int c = 0; c < w; ++c) {
            have[q].push_back((uint16_t)(step + 1000 * c));
            pool.write(q, at + c, have[q].back());
          }
          CHECK(spp_seq_commit(pool.p, q, w) == SPP_OK);
        }
      } else if (op == 7) {
        const int q = pick();
        if (below(2)) {
          CHECK(spp_seq_free(pool.p, q) == SPP_OK);
          CHECK(spp_seq_free(pool.p, q) == SPP_E_INVALID_ARG);
          have.erase(q);
        } else {
          const int n = below((int)have[q].size() + 3);
          CHECK(spp_seq_truncate(pool.p, q, n) == SPP_OK);
          if (n < (int)have[q].size()) have[q].resize(n);
        }
      } else if (op == 8) {
        int32_t moved = -1;
        CHECK(spp_pool_compact(pool.p, s, &moved) == SPP_OK && moved >= 0);
        spp_pool_info_t i;
        CHECK(spp_pool_info(pool.p, &i) == SPP_OK);
        for (auto& h : have)
          for (int32_t pg : pool.table(h.first)) CHECK(pg < i.used_pages);
        CHECK(spp_pool_compact(pool.p, s, &moved) == SPP_OK && moved == 0);
      } else {
        const int q = pick();
        if (below(2)) {
          std::vector<uint16_t> w(below(5 * page));
          for (size_t c = 0; c < w.size(); ++c) w[c] = (uint16_t)(step * 3 + c);
          hipDeviceSynchronize();
          sess.fill(w);
          const spp_status rc = spp_seq_import(pool.p, q, sess.s, s);
          CHECK(rc == SPP_OK || rc == SPP_E_CAPACITY);
          if (rc == SPP_OK) have[q] = w;
        } else {
          const spp_status rc = spp_seq_export(pool.p, q, into.s, s);
          CHECK(rc == ((int)have[q].size() <= into.cap ? SPP_OK : SPP_E_CAPACITY));
          hipDeviceSynchronize();
          if (rc == SPP_OK) CHECK(into.holds(have[q]));
        }
      }
      hipDeviceSynchronize();
      std::map<int, int> refs;
      for (auto& h : have) {
        CHECK(pool.holds(h.first, h.second));
        for (int32_t pg : pool.table(h.first)) ++refs[pg];
      }
      spp_pool_info_t i;
      CHECK(spp_pool_info(pool.p, &i) == SPP_OK);
      int shared = 0;
      for (auto& r : refs) shared += r.second > 1;
      CHECK(i.used_pages == (int)refs.size() && i.shared_pages == shared && i.n_seqs == (int)have.size());
      if (g_fail) return;
    }
  }
  hipStreamDestroy(st[0]);
  hipStreamDestroy(st[1]);
}

void refusals() {
  Model model(2), other(2, 1);
  Pool pool(16, 6, 3);
  spp_pool_t none = nullptr;
  for (int bad = 0; bad < 12; ++bad) {
    spp_pool_config c = pool_config(16, 6, 3);
    if (bad == 0) c.page_cells = 24;
    if (bad == 1) c.page_cells = 8;
    if (bad == 2) c.page_cells = 512;
    if (bad == 3) c.head_dim = 96;
    if (bad == 4) c.dtype = 2;
    if (bad == 5) c.n_layers = 0;
    if (bad == 6) c.n_kv_heads = 0;
    if (bad == 7) c.n_pages = 0;
    if (bad == 8) c.max_seqs = 0;
    if (bad == 9) c.max_seqs = 65537;
    if (bad == 10) c.n_layers = 1 << 20;
    if (bad == 11) c.n_kv_heads = 1 << 24;
    CHECK(spp_pool_bytes(&c) == 0);
    CHECK(spp_pool_create(&c, pool.pages, (size_t)1 << 40, &none) == SPP_E_INVALID_ARG && !none);
  }
  CHECK(spp_pool_create(&pool.cfg, pool.pages, spp_pool_bytes(&pool.cfg) - 1, &none) == SPP_E_INVALID_ARG);
  CHECK(spp_pool_create(&pool.cfg, pool.pages + 8, (size_t)1 << 40, &none) == SPP_E_INVALID_ARG);
  CHECK(spp_pool_create(&pool.cfg, nullptr, (size_t)1 << 40, &none) == SPP_E_INVALID_ARG);
  CHECK(spp_pool_bytes(nullptr) == 0 && spp_pool_destroy(nullptr) == SPP_OK);

  int32_t a = -1, b = -1, q[3], n = 0;
  CHECK(spp_seq_create(pool.p, 16 * 6 + 1, &a) == SPP_E_CAPACITY && a == -1);
  CHECK(spp_seq_create(pool.p, 2147483647, &a) == SPP_E_CAPACITY);
  CHECK(spp_seq_create(pool.p, -1, &a) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_create(pool.p, 20, &a) == SPP_OK && spp_seq_create(pool.p, 48, &b) == SPP_OK);
  int32_t t[1];
  CHECK(spp_seq_table(pool.p, a, t, 1, &n) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_fork(pool.p, a, 2, q) == SPP_E_CAPACITY);
  CHECK(spp_seq_fork(pool.p, a, 0, q) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_fork(pool.p, 2, 1, q) == SPP_E_INVALID_ARG && spp_seq_fork(pool.p, -1, 1, q) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_fork(pool.p, 99, 1, q) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_fork(pool.p, a, 1, q) == SPP_OK);
  // one free page: a and its fork may each take one cell (one of them copies), not seventeen
  const int32_t both[2] = {a, q[0]}, twice[2] = {a, a};
  CHECK(spp_seq_reserve(pool.p, 2, both, 17, nullptr) == SPP_E_CAPACITY);
  CHECK(spp_seq_reserve(pool.p, 2, twice, 1, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_reserve(pool.p, 0, both, 1, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_reserve(pool.p, 1, both, 0, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_reserve(pool.p, 1, nullptr, 1, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_reserve(pool.p, 1, both, 2147483647, nullptr) == SPP_E_CAPACITY);
  CHECK(spp_seq_commit(pool.p, a, 1) == SPP_E_STATE);  // its page is shared
  CHECK(spp_seq_reserve(pool.p, 2, both, 1, nullptr) == SPP_OK);
  CHECK(spp_seq_commit(pool.p, a, 12) == SPP_OK && spp_seq_commit(pool.p, a, 1) == SPP_E_STATE);
  CHECK(spp_seq_commit(pool.p, a, -1) == SPP_E_INVALID_ARG && spp_seq_commit(pool.p, a, 2147483647) == SPP_E_STATE);
  CHECK(spp_seq_truncate(pool.p, a, -1) == SPP_E_INVALID_ARG);
  spp_seq_info_t si;
  CHECK(spp_seq_info(pool.p, a, &si) == SPP_OK && si.n_cells == 32 && si.n_pages == 2 && !si.decoded);

  std::vector<float> d(3 * kV);
  float* ds[3] = {d.data(), d.data() + kV, nullptr};
  int32_t tok[3] = {1, 2, 3};
  CHECK(spp_decode_batch(pool.p, other.m, 1, &a, tok, ds, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_decode_batch(pool.p, nullptr, 1, &a, tok, ds, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_decode_batch(pool.p, model.m, 1, &a, nullptr, ds, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_decode_batch(pool.p, model.m, 1, &a, tok, ds + 2, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_decode_batch(pool.p, model.m, 2, twice, tok, ds, nullptr) == SPP_E_INVALID_ARG);
  tok[0] = kV;
  CHECK(spp_decode_batch(pool.p, model.m, 1, &a, tok, ds, nullptr) == SPP_E_INVALID_ARG);
  tok[0] = 1;
  CHECK(spp_decode_batch(pool.p, model.m, 1, &a, tok, ds, nullptr) == SPP_E_CAPACITY);  // page 3 of a
  spp_summary sum[2];
  CHECK(spp_seq_summaries(pool.p, 1, &a, sum) == SPP_E_STATE);
  CHECK(spp_decode_batch(pool.p, model.m, 1, q, tok, ds, nullptr) == SPP_OK);
  CHECK(spp_seq_summaries(pool.p, 1, q, sum) == SPP_OK && sum[0].argmax == 7 && sum[0].position == 21);
  CHECK(spp_seq_summaries(pool.p, 2, both, sum) == SPP_E_STATE);
  spp_pool_info_t pi;
  CHECK(spp_pool_info(pool.p, &pi) == SPP_OK && pi.used_pages == 6 && pi.n_seqs == 3);

  Sess sess(model.m, 40), wrong(other.m, 40);
  CHECK(spp_session_restore(sess.s, 40) == SPP_OK);
  CHECK(spp_seq_import(pool.p, q[0], sess.s, nullptr) == SPP_E_CAPACITY);   // 3 pages; 1 of its own
  CHECK(spp_seq_import(pool.p, a, wrong.s, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_export(pool.p, a, wrong.s, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_import(pool.p, 7, sess.s, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_seq_export(pool.p, b, sess.s, nullptr) == SPP_E_CAPACITY);      // 48 cells into 40
  spp_session_info_t ssi;
  CHECK(spp_session_info(sess.s, &ssi) == SPP_OK && ssi.n_committed == 40);
  CHECK(spp_seq_info(pool.p, q[0], &si) == SPP_OK && si.n_cells == 21 && si.decoded);
  // an export invalidates the session's ready record; its handle is stale
  spp_ready_t ready;
  CHECK(spp_session_restore(sess.s, 2) == SPP_OK);
  CHECK(spp_preposition(sess.s, tok, 2, d.data(), nullptr, nullptr, &ready) == SPP_OK);
  CHECK(spp_seq_export(pool.p, a, sess.s, nullptr) == SPP_OK);
  hipDeviceSynchronize();
  int32_t token;
  spp_gate_outcome out;
  CHECK(spp_gate(ready, 0.f, nullptr, nullptr, 0, nullptr, &token, &out, nullptr) == SPP_OK && out == SPP_FALL_INVALID);

  // the stand-alone calls' checks
  void* x = nullptr;
  hipMalloc(&x, 1 << 16);
  int32_t tab[4] = {0, 1, 2, 3}, len[1] = {5};
  const spp_paged_attn good{pool.p, 0, 1, 2, SPP_DTYPE_BF16, x, 128, tab, 4, 4, len, 0.f, x, 128};
  const size_t need = spp_paged_attention_work_bytes(&good);
  CHECK(need == 32 && spp_paged_attention(&good, x, need, nullptr) == SPP_OK);
  CHECK(spp_paged_attention(&good, x, need - 1, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_paged_attention(&good, nullptr, need, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_paged_attention(&good, (char*)x + 4, need, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_paged_attention(nullptr, x, need, nullptr) == SPP_E_INVALID_ARG);
  for (int bad = 0; bad < 20; ++bad) {
    spp_paged_attn c = good;
    switch (bad) {
      case 0: c.pool = nullptr; break;
      case 1: c.layer = kLayers; break;
      case 2: c.layer = -1; break;
      case 3: c.n_seqs = -1; break;
      case 4: c.n_seqs = 65536; break;
      case 5: c.n_q_heads = 0; break;
      case 6: c.io_dtype = 5; break;
      case 7: c.q = nullptr; break;
      case 8: c.q_stride = 127; break;
      case 9: c.out_stride = 132; break;
      case 10: c.table = nullptr; break;
      case 11: c.table_stride = 3; break;
      case 12: c.max_pages = 0; break;
      case 13: c.max_pages = (1 << 26) + 1; c.table_stride = 1 << 27; break;
      case 14: c.lengths = nullptr; break;
      case 15: c.scale = INFINITY; break;
      case 16: c.out = (char*)x + 2; break;
      case 18: c.table = (const int32_t*)((const char*)tab + 2); break;
      case 19: c.lengths = (const int32_t*)((const char*)len + 1); break;
      case 17: c.n_q_heads = 65536; c.q_stride = c.out_stride = 1 << 23; break;
    }
    CHECK(spp_paged_attention_work_bytes(&c) == 0);
    CHECK(spp_paged_attention(&c, x, 1 << 16, nullptr) == SPP_E_INVALID_ARG);
  }
  spp_paged_attn empty = good;
  empty.n_seqs = 0;
  empty.q = nullptr;
  CHECK(spp_paged_attention(&empty, nullptr, 0, nullptr) == SPP_OK);
  spp_adjust row{};
  row.src = row.dst = d.data();
  row.repetition = 1.f;
  CHECK(spp_adjust_logits(1, kV, &row, nullptr, nullptr, 0, nullptr) == SPP_OK);
  CHECK(spp_adjust_logits(0, kV, nullptr, nullptr, nullptr, 0, nullptr) == SPP_OK);
  CHECK(spp_adjust_logits(1, 0, &row, nullptr, nullptr, 0, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_adjust_logits(1, (1 << 24) + 1, &row, nullptr, nullptr, 0, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_adjust_logits(-1, kV, &row, nullptr, nullptr, 0, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_adjust_logits(1, kV, nullptr, nullptr, nullptr, 0, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_adjust_logits(1, kV, &row, sum, nullptr, 0, nullptr) == SPP_E_INVALID_ARG);
  CHECK(spp_adjust_logits_work_bytes(0, kV) == 0 && spp_adjust_logits_work_bytes(1, -5) == 0);
  for (int bad = 0; bad < 15; ++bad) {
    spp_adjust r = row;
    switch (bad) {
      case 0: r.src = nullptr; break;
      case 1: r.dst = nullptr; break;
      case 2: r.n_tokens = -1; break;
      case 3: r.n_tokens = 1; break;
      case 4: r.tokens = tab; r.n_tokens = 2; r.n_prompt = 3; break;
      case 5: r.n_prompt = -1; break;
      case 6: r.n_bias = 1; break;
      case 7: r.n_bias = 1; r.bias_tokens = tab; break;
      case 8: r.repetition = 0.f; break;
      case 9: r.frequency = NAN; break;
      case 10: r.presence = INFINITY; break;
      case 11: r.fill = NAN; break;
      case 12: r.src = (const float*)((const char*)r.src + 2); break;
      case 13: r.allowed = (const uint32_t*)((const char*)tab + 1); break;
      case 14: r.tokens = tab; r.n_tokens = (1 << 30) + 1; break;
    }
    CHECK(spp_adjust_logits(1, kV, &r, nullptr, nullptr, 0, nullptr) == SPP_E_INVALID_ARG);
  }
  hipDeviceSynchronize();
  hipFree(x);
}

// Threads with sequences of their own on one pool and model, another that compacts.
void threads() {
  Model model(4);
  Pool pool(16, 200, 64);
  std::vector<std::thread> ts;
  for (int k = 0; k < 4; ++k)
    ts.emplace_back([&, k] {
      hipStream_t st;
      hipStreamCreate(&st);
      Sess sess(model.m, 100);
      sess.fill(std::vector<uint16_t>(30 + k, (uint16_t)(100 + k)));
      std::vector<float> d(3 * kV);
      float* ds[3] = {d.data(), d.data() + kV, d.data() + 2 * kV};
      for (int it = 0; it < 12; ++it) {
        int32_t q[3];
        CHECK(spp_seq_create(pool.p, 0, &q[0]) == SPP_OK);
        CHECK(spp_seq_import(pool.p, q[0], sess.s, st) == SPP_OK);
        CHECK(spp_seq_fork(pool.p, q[0], 2, q + 1) == SPP_OK);
        const int32_t tok[3] = {k, k + 10, k + 20};
        for (int s = 0; s < 3; ++s) CHECK(spp_decode_batch(pool.p, model.m, 3, q, tok, ds, st) == SPP_OK);
        spp_summary sum[3];
        CHECK(spp_seq_summaries(pool.p, 3, q, sum) == SPP_OK && sum[2].position == 33 + k);
        CHECK(spp_seq_export(pool.p, q[1], sess.s, st) == SPP_OK);
        hipStreamSynchronize(st);
        std::vector<uint16_t> want(30 + k, (uint16_t)(100 + k));
        want.resize(33 + k, (uint16_t)(k + 10));
        CHECK(sess.holds(want));
        want.resize(30 + k);
        sess.fill(want);
        for (int i = 0; i < 3; ++i) CHECK(spp_seq_free(pool.p, q[i]) == SPP_OK);
      }
      hipStreamDestroy(st);
    });
  ts.emplace_back([&] {
    hipStream_t st;
    hipStreamCreate(&st);
    for (int it = 0; it < 30; ++it) {
      spp_pool_info_t i;
      CHECK(spp_pool_compact(pool.p, st, nullptr) == SPP_OK && spp_pool_info(pool.p, &i) == SPP_OK);
    }
    hipStreamSynchronize(st);
    hipStreamDestroy(st);
  });
  for (auto& t : ts) t.join();
  spp_pool_info_t i;
  CHECK(spp_pool_info(pool.p, &i) == SPP_OK && i.used_pages == 0 && i.n_seqs == 0);
}

// Copies on two streams by two pools, then a step of the model on a third: what is enqueued behind
// the step sees all of it done.  A pool or the model may end first.
void copies_then_steps() {
  hipStream_t st[3];
  for (hipStream_t& s : st) hipStreamCreate(&s);
  for (int it = 0; it < 8; ++it) {
    auto pool = std::make_unique<Pool>(16, 8, 2), other = std::make_unique<Pool>(32, 8, 2);
    auto model = std::make_unique<Model>(1);
    auto sess = std::make_unique<Sess>(model->m, 100);
    sess->fill(std::vector<uint16_t>(40, 5));
    int32_t q = -1, r = -1;
    CHECK(spp_seq_create(pool->p, 0, &q) == SPP_OK && spp_seq_create(other->p, 0, &r) == SPP_OK);
    int first = 0, second = 0;
    bool seen = false, again = false;
    const auto late = [](int* done) {
      std::this_thread::sleep_for(std::chrono::milliseconds(5));
      *done = 1;
    };
    stub::enqueue(st[0], [&] { late(&first); });
    CHECK(spp_seq_import(pool->p, q, sess->s, st[0]) == SPP_OK);
    if (it & 1) {  // the second pool's copy comes after the first's
      CHECK(spp_seq_import(other->p, r, sess->s, st[1]) == SPP_OK);
      stub::enqueue(st[1], [&] { again = first; });
    }
    stub::enqueue(st[1], [&] { late(&second); });
    CHECK(spp_seq_export(it & 2 ? other->p : pool->p, it & 2 ? r : q, sess->s, st[1]) == SPP_OK);
    if (it & 2 && !(it & 1)) CHECK(spp_session_restore(sess->s, 40) == SPP_OK);  // (r was empty)
    const int32_t tok = 7;
    if (it & 4)
      CHECK(spp_shift(sess->s, 1, st[2]) == SPP_OK);
    else
      CHECK(spp_kv_append_delta(sess->s, &tok, 1, st[2]) == SPP_OK);
    const bool empty = it & 2 && !(it & 1);  // (an export of no cells copies nothing)
    stub::enqueue(st[2], [&] { seen = first && (empty || second); });
    hipDeviceSynchronize();
    CHECK(seen && again == (bool)(it & 1));
    // once more behind that step, on the first stream
    bool last = false;
    stub::enqueue(st[2], [&] { late(&second); last = true; });
    CHECK(spp_shift(sess->s, 1, st[2]) == SPP_OK);
    CHECK(spp_seq_import(pool->p, q, sess->s, st[0]) == SPP_OK);
    bool behind = false;
    stub::enqueue(st[0], [&] { behind = last; });
    hipDeviceSynchronize();
    CHECK(behind);
    sess.reset();
    if (it & 1) model.reset();
    pool.reset();
    other.reset();
  }
  for (hipStream_t s : st) hipStreamDestroy(s);
}

}  // namespace

int main() {
  refusals();
  random_calls(1, 16, 40);
  random_calls(2, 16, 14);
  random_calls(3, 32, 300);
  threads();
  copies_then_steps();
  CHECK(stub::live_allocations() == 0);
  stub::shutdown();
  if (g_fail) return 1;
  std::puts("OK");
  return 0;
}
