// Paged caches and adjusted logits behind the C ABI (include/spp.h): the pages of a pool --
// tables, references, free pages, copies on write, compaction --, the decode step of many paged
// sequences, and the calls of the stand-alone operators.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <functional>
#include <new>
#include <queue>
#include <vector>

#include "paged.hpp"
#include "runtime.hpp"

using namespace spp;

namespace {

struct Seq {
  bool live = false;
  int n = 0;                    // cells
  std::vector<int32_t> pages;   // at least those of its cells; pages past them are its own
  int summary_at = -1;          // length after the decode step whose summary is kept (-1: none)
};

using Lowest = std::priority_queue<int32_t, std::vector<int32_t>, std::greater<int32_t>>;

}  // namespace

struct spp_pool_s {
  spp_pool_config cfg{};
  PageView v{};
  int device = 0;
  std::vector<int32_t> refs;     // sequences that list a page
  Lowest free_pages;          // lowest first
  std::vector<Seq> seqs;
  Lowest free_seqs;           // sequence numbers, lowest first
  int n_seqs = 0, n_shared = 0;
  ScanResult* summary = nullptr;  // device, one slot per sequence
  // The pool's device work so far is events[done].  An event that a model has to wait for
  // (Model::copied) is not recorded again while it has: two would do for one model.
  std::shared_ptr<Event> events[4];
  int done = 0;
  bool recorded = false;
  std::mutex mu;                  // taken before a session's and a model's
  ~spp_pool_s() {
    if (recorded) hipEventSynchronize(events[done]->ev);
    if (summary) hipFree(summary);
  }
};

namespace {

spp_status check_pool_config(const spp_pool_config& c) {
  if (c.n_layers < 1 || c.n_kv_heads < 1 || (c.head_dim != 64 && c.head_dim != 128) ||
      (c.dtype != SPP_DTYPE_BF16 && c.dtype != SPP_DTYPE_F32))
    return fail(SPP_E_INVALID_ARG, "n_layers and n_kv_heads >= 1, head_dim 64 or 128, dtype F32 or BF16");
  const int p = c.page_cells;
  if (p != 16 && p != 32 && p != 64 && p != 128 && p != 256)
    return fail(SPP_E_INVALID_ARG, "page_cells must be 16, 32, 64, 128 or 256");
  if (c.n_pages < 1 || c.max_seqs < 1 || c.max_seqs > 65536)
    return fail(SPP_E_INVALID_ARG, "n_pages >= 1 and 1 <= max_seqs <= 65536");
  // bytes of a page below 2^31: kernels address inside one with 32 bits
  const double page = 2.0 * c.n_layers * c.n_kv_heads * c.head_dim * p * (c.dtype == SPP_DTYPE_BF16 ? 2 : 4);
  if (page >= 2147483648.0) return fail(SPP_E_INVALID_ARG, "a page of %g bytes (2 GiB is too many)", page);
  return SPP_OK;
}

PageView view_of(const spp_pool_config& c, void* base) {
  int shift = 4;
  while ((1 << shift) < c.page_cells) ++shift;
  return PageView{static_cast<char*>(base), c.n_pages, c.n_layers, c.n_kv_heads, c.head_dim, shift,
                  c.dtype == SPP_DTYPE_BF16 ? 2 : 4};
}

// Pages that hold `cells` cells.
int pages_for(const spp_pool_s& p, int64_t cells) { return (int)((cells + p.cfg.page_cells - 1) >> p.v.shift); }

spp_status check_seq(const spp_pool_s& p, int32_t seq) {
  if (seq < 0 || seq >= p.cfg.max_seqs || !p.seqs[seq].live)
    return fail(SPP_E_INVALID_ARG, "no sequence %d", seq);
  return SPP_OK;
}

// Distinct live sequences.
spp_status check_seqs(const spp_pool_s& p, int32_t n, const int32_t* seqs) {
  if (n < 1 || !seqs) return fail(SPP_E_INVALID_ARG, "null argument or n < 1");
  std::vector<int32_t> order(seqs, seqs + n);
  std::sort(order.begin(), order.end());
  for (int i = 0; i < n; ++i) {
    if (const spp_status rc = check_seq(p, order[i]); rc != SPP_OK) return rc;
    if (i && order[i] == order[i - 1]) return fail(SPP_E_INVALID_ARG, "sequence %d is listed twice", order[i]);
  }
  return SPP_OK;
}

// Takes the lowest free page (the caller has counted that there is one).
int32_t take_page(spp_pool_s& p) {
  const int32_t pg = p.free_pages.top();
  p.free_pages.pop();
  p.refs[pg] = 1;
  return pg;
}

void drop_page(spp_pool_s& p, int32_t pg) {
  const int32_t left = --p.refs[pg];
  if (left == 1) --p.n_shared;
  if (left == 0) p.free_pages.push(pg);
}

void drop_pages_from(spp_pool_s& p, Seq& s, size_t first) {
  for (size_t i = first; i < s.pages.size(); ++i) drop_page(p, s.pages[i]);
  if (s.pages.size() > first) s.pages.resize(first);
}

// Takes the lowest free sequence number (the caller has counted that there is one).
int32_t take_seq(spp_pool_s& p) {
  const int32_t q = p.free_seqs.top();
  p.free_seqs.pop();
  p.seqs[q].live = true;
  ++p.n_seqs;
  return q;
}

// The pool's device work is one line: `st` continues after all of it, and note_work marks
// what was enqueued since as its new end.
spp_status order_after(spp_pool_s& p, hipStream_t st) {
  hipSetDevice(p.device);
  if (p.recorded) HIPCHK(hipStreamWaitEvent(st, p.events[p.done]->ev, 0));
  return SPP_OK;
}
spp_status note_work(spp_pool_s& p, hipStream_t st) {
  // an event of the pool's alone, the last one if it is (each held by a model: the last one, and
  // that model waits for what follows too)
  constexpr int n = sizeof(p.events) / sizeof(p.events[0]);
  int at = p.done;
  for (int i = 0; i < n && p.events[at].use_count() > 1; ++i) at = (at + 1) % n;
  HIPCHK(hipEventRecord(p.events[at]->ev, st));
  p.done = at;
  p.recorded = true;
  return SPP_OK;
}
// The same at the end of work that came to rc: launches before a failed one are in the line too.
spp_status end_work(spp_pool_s& p, hipStream_t st, spp_status rc) {
  const spp_status noted = note_work(p, st);
  return rc != SPP_OK ? rc : noted;
}

// Copies pages: (source, destination) pairs, no page both; batches travel as launch arguments.
// `st` already continues the pool's line.
spp_status copy_pages(spp_pool_s& p, const std::vector<std::pair<int32_t, int32_t>>& moves, hipStream_t st) {
  if (moves.empty()) return SPP_OK;
  const auto copy = [&](size_t at) -> spp_status {
    PageList l;
    const int n = (int)std::min<size_t>(kPageBatch, moves.size() - at);
    for (int i = 0; i < n; ++i) {
      l.a[i] = moves[at + i].first;
      l.b[i] = moves[at + i].second;
    }
    HIPCHK(k::page_copy(p.v, l, n, st));
    return SPP_OK;
  };
  spp_status rc = SPP_OK;
  for (size_t at = 0; at < moves.size() && rc == SPP_OK; at += kPageBatch) rc = copy(at);
  return end_work(p, st, rc);
}

// Makes the next `cells` cells of the sequences writable (spp_seq_reserve).  Nothing changes
// unless the pages suffice.  `st` continues after the pool's work also where nothing is copied:
// earlier work may still read a page that is handed out here.
spp_status reserve(spp_pool_s& p, int32_t n, const int32_t* seqs, int32_t cells, hipStream_t st) {
  int64_t need = 0;
  // a shared page is copied by each of its writers but the last reference's
  std::vector<std::pair<int32_t, int>> shared;  // (page, sequences of this call that write it)
  for (int i = 0; i < n; ++i) {
    const Seq& s = p.seqs[seqs[i]];
    if ((int64_t)s.n + cells > SPP_MAX_CAPACITY)
      return fail(SPP_E_CAPACITY, "sequence %d of %d cells is at its longest", seqs[i], s.n);
    need += std::max<int64_t>(0, pages_for(p, (int64_t)s.n + cells) - (int64_t)s.pages.size());
    if (s.n % p.cfg.page_cells) {
      const int32_t pg = s.pages[s.n >> p.v.shift];
      if (p.refs[pg] > 1) shared.push_back({pg, 1});
    }
  }
  std::sort(shared.begin(), shared.end());
  for (size_t i = 0; i < shared.size();) {
    size_t j = i;
    while (j < shared.size() && shared[j].first == shared[i].first) ++j;
    need += std::min<int64_t>((int64_t)(j - i), p.refs[shared[i].first] - 1);
    i = j;
  }
  if (need > (int64_t)p.free_pages.size())
    return fail(SPP_E_CAPACITY, "%lld pages needed, %zu free", (long long)need, p.free_pages.size());
  std::vector<std::pair<int32_t, int32_t>> moves;
  std::vector<int32_t*> moved;  // the table entries of the moves
  moves.reserve(n);  // (what can throw comes before the first change)
  moved.reserve(n);
  std::vector<size_t> had(n);   // pages of the tables before
  for (int i = 0; i < n; ++i) {
    Seq& s = p.seqs[seqs[i]];
    had[i] = s.pages.size();
    s.pages.reserve(pages_for(p, (int64_t)s.n + cells));
  }
  if (const spp_status rc = order_after(p, st); rc != SPP_OK) return rc;
  for (int i = 0; i < n; ++i) {
    Seq& s = p.seqs[seqs[i]];
    if (s.n % p.cfg.page_cells) {
      int32_t& pg = s.pages[s.n >> p.v.shift];
      if (p.refs[pg] > 1) {
        const int32_t own = take_page(p);
        moves.push_back({pg, own});
        moved.push_back(&pg);
        drop_page(p, pg);
        pg = own;
      }
    }
    const int want = pages_for(p, (int64_t)s.n + cells);
    while ((int)s.pages.size() < want) s.pages.push_back(take_page(p));
  }
  const spp_status rc = copy_pages(p, moves, st);
  if (rc != SPP_OK) {  // the pages stay shared (each still has the reference of another), the tables as they were
    for (size_t i = 0; i < moves.size(); ++i) {
      drop_page(p, moves[i].second);
      if (p.refs[moves[i].first]++ == 1) ++p.n_shared;
      *moved[i] = moves[i].first;
    }
    for (int i = 0; i < n; ++i) drop_pages_from(p, p.seqs[seqs[i]], had[i]);
  }
  return rc;
}

spp_status check_model(const spp_pool_s& p, const Model& m) {
  if (m.s.n_layers != p.cfg.n_layers || m.s.n_kv != p.cfg.n_kv_heads || m.s.dh != p.cfg.head_dim ||
      m.cfg.dtype != p.cfg.dtype || m.device != p.device)
    return fail(SPP_E_INVALID_ARG, "the model's layers, kv heads, head_dim, dtype or device are not the pool's");
  return SPP_OK;
}

// Copies cells [0, n) between a session's buffer and pages, ordered after and before the
// device work of the pool and of the session's model.  The caller holds the pool's and the
// session's mutexes.
spp_status copy_session(spp_pool_s& p, const std::vector<int32_t>& pages, int n, Session& s, bool to_pages,
                        hipStream_t st) {
  if (n == 0) return SPP_OK;
  Model& m = *s.m;
  std::lock_guard<std::mutex> mk(m.mu);
  if (const spp_status rc = order_after(p, st); rc != SPP_OK) return rc;
  if (const spp_status rc = after_steps(m, st); rc != SPP_OK) return rc;
  const int count = pages_for(p, n);
  const auto copy = [&](int at) -> spp_status {
    PageList l;
    const int c = std::min(kPageBatch, count - at);
    std::copy_n(pages.begin() + at, c, l.a);
    const int64_t c0 = (int64_t)at << p.v.shift;
    HIPCHK(k::page_session(p.v, l, c, s.kv, s.cap_stride, c0, (int)std::min<int64_t>(n - c0, (int64_t)c << p.v.shift),
                           to_pages, st));
    return SPP_OK;
  };
  spp_status rc = SPP_OK;
  for (int at = 0; at < count && rc == SPP_OK; at += kPageBatch) rc = copy(at);
  rc = end_work(p, st, rc);
  // the model's next step waits for the pool's work up to here, which holds this copy and what
  // the model waited for so far
  m.copied = p.events[p.done];
  return rc;
}

// The cells of a decode step's rows: row r is the new token of seqs[r], at its length.
struct PagedStep : StepCache {
  const spp_pool_s& p;
  const Model& m;
  const int32_t* seqs;
  int n, width = 1;
  const int32_t *table = nullptr, *lengths = nullptr;  // device
  PagedStep(const spp_pool_s& pool, const Model& model, const int32_t* list, int count)
      : p(pool), m(model), seqs(list), n(count) {
    for (int i = 0; i < n; ++i) width = std::max(width, pages_for(p, (int64_t)p.seqs[seqs[i]].n + 1));
  }
  size_t record_bytes() const override { return ((size_t)n * width + n) * 4; }
  size_t part_bytes() const override {
    return std::max<size_t>(16, k::paged_work_bytes(p.v, n, m.s.n_q, width));
  }
  void fill(char* host, char* dev) override {
    int32_t* t = reinterpret_cast<int32_t*>(host);
    for (int i = 0; i < n; ++i) {
      const Seq& s = p.seqs[seqs[i]];
      const int have = pages_for(p, (int64_t)s.n + 1);
      std::copy_n(s.pages.begin(), have, t + (size_t)i * width);
      std::fill(t + (size_t)i * width + have, t + (size_t)(i + 1) * width, -1);
      t[(size_t)n * width + i] = s.n + 1;
    }
    table = reinterpret_cast<const int32_t*>(dev);
    lengths = table + (size_t)n * width;
  }
  hipError_t epilogue(const StepView& v, int rows, int layer, const float* partials, int splits,
                      const float* ss, const float2* rope, float* q, hipStream_t st) override {
    return k::paged_epilogue(m.s, v, rows, layer, p.v, table, width, partials, splits, ss, rope, q, st);
  }
  hipError_t attention(int layer, const float* q, void* part, void* out, void* out_lo, hipStream_t st) override {
    const int64_t stride = (int64_t)m.s.n_q * m.s.dh;
    const PagedAttn a{q, stride, 0, n, m.s.n_q, table, width, width, lengths, 0.f, out, out_lo, stride,
                      m.s.bf16 ? 2 : 0};
    return k::paged_attention(p.v, layer, a, part, st);
  }
};

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool aligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

spp_status check_attn(const spp_paged_attn* a) {
  if (!a || !a->pool) return fail(SPP_E_INVALID_ARG, "null argument");
  const spp_pool_config& c = a->pool->cfg;
  if (a->n_seqs < 0 || a->n_seqs > 65535) return fail(SPP_E_INVALID_ARG, "n_seqs outside [0, 65535]");
  if (a->n_q_heads < 1 || a->n_q_heads % c.n_kv_heads || a->n_q_heads > 65535)
    return fail(SPP_E_INVALID_ARG, "n_q_heads %d is no multiple of %d kv heads", a->n_q_heads, c.n_kv_heads);
  if (a->max_pages < 1 || (int64_t)a->max_pages * c.page_cells > (1 << 30))
    return fail(SPP_E_INVALID_ARG, "max_pages < 1 or over 2^30 cells");
  if (a->layer < 0 || a->layer >= c.n_layers) return fail(SPP_E_INVALID_ARG, "layer %d", a->layer);
  if (a->io_dtype != SPP_DTYPE_BF16 && a->io_dtype != SPP_DTYPE_F32) return fail(SPP_E_INVALID_ARG, "io_dtype");
  if (!std::isfinite(a->scale)) return fail(SPP_E_INVALID_ARG, "scale is not finite");
  if (a->n_seqs == 0) return SPP_OK;
  if (!a->q || !a->table || !a->lengths || !a->out) return fail(SPP_E_INVALID_ARG, "null pointer");
  const int64_t row = (int64_t)a->n_q_heads * c.head_dim;
  if (a->q_stride < row || a->out_stride < row || a->q_stride % 8 || a->out_stride % 8 || !aligned16(a->q) ||
      !aligned16(a->out))
    return fail(SPP_E_INVALID_ARG, "rows of q and out: %lld elements at least, multiples of 8, 16-byte aligned",
                (long long)row);
  if (a->table_stride < a->max_pages) return fail(SPP_E_INVALID_ARG, "table_stride < max_pages");
  if (!aligned4(a->table) || !aligned4(a->lengths))
    return fail(SPP_E_INVALID_ARG, "table and lengths are 4-byte aligned");
  return SPP_OK;
}

// No C++ exception crosses the boundary: the bookkeeping allocates.
template <typename F>
spp_status guarded(F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail(SPP_E_NOMEM, "out of host memory");
  } catch (...) {
    return fail(SPP_E_STATE, "unexpected exception");
  }
}

}  // namespace

extern "C" {

size_t spp_pool_bytes(const spp_pool_config* cfg) {
  if (!cfg || check_pool_config(*cfg) != SPP_OK) return 0;
  return (size_t)view_of(*cfg, nullptr).page() * cfg->n_pages;
}

spp_status spp_pool_page_layout(const spp_pool_config* cfg, spp_page_layout* out) {
  if (!cfg || !out) return fail(SPP_E_INVALID_ARG, "null argument");
  if (const spp_status rc = check_pool_config(*cfg); rc != SPP_OK) return rc;
  const PageView v = view_of(*cfg, nullptr);
  const int64_t P = cfg->page_cells, dh = cfg->head_dim;
  *out = spp_page_layout{v.page(), 2 * v.half(), v.half(), {P * dh, dh, 1}, {P * dh, 1, P}, v.elem};
  return SPP_OK;
}

spp_status spp_pool_create(const spp_pool_config* cfg, void* pages, size_t bytes, spp_pool_t* out) {
  if (!cfg || !pages || !out) return fail(SPP_E_INVALID_ARG, "null argument");
  *out = nullptr;
  if (const spp_status rc = check_pool_config(*cfg); rc != SPP_OK) return rc;
  if (bytes < spp_pool_bytes(cfg))
    return fail(SPP_E_INVALID_ARG, "pages of %zu bytes, need %zu", bytes, spp_pool_bytes(cfg));
  if (!aligned16(pages)) return fail(SPP_E_INVALID_ARG, "pages not 16-byte aligned");
  return guarded([&] {
    std::unique_ptr<spp_pool_s> p(new spp_pool_s);
    p->cfg = *cfg;
    p->v = view_of(*cfg, pages);
    hipGetDevice(&p->device);
    p->refs.assign(cfg->n_pages, 0);
    std::vector<int32_t> all(cfg->n_pages);
    for (int32_t i = 0; i < cfg->n_pages; ++i) all[i] = i;
    p->free_pages = Lowest(std::greater<int32_t>(), std::move(all));
    p->seqs.resize(cfg->max_seqs);
    std::vector<int32_t> numbers(cfg->max_seqs);
    for (int32_t i = 0; i < cfg->max_seqs; ++i) numbers[i] = i;
    p->free_seqs = Lowest(std::greater<int32_t>(), std::move(numbers));
    for (auto& e : p->events) {
      e = std::make_shared<Event>();
      if (hipEventCreateWithFlags(&e->ev, hipEventDisableTiming) != hipSuccess)
        return fail(SPP_E_NOMEM, "pool resources");
    }
    if (hipMalloc((void**)&p->summary, sizeof(ScanResult) * cfg->max_seqs) != hipSuccess)
      return fail(SPP_E_NOMEM, "pool resources");
    *out = p.release();
    return SPP_OK;
  });
}

spp_status spp_pool_destroy(spp_pool_t p) {
  delete p;
  return SPP_OK;
}

spp_status spp_pool_info(spp_pool_t p, spp_pool_info_t* out) {
  if (!p || !out) return fail(SPP_E_INVALID_ARG, "null argument");
  std::lock_guard<std::mutex> lk(p->mu);
  out->n_pages = p->cfg.n_pages;
  out->used_pages = p->cfg.n_pages - (int32_t)p->free_pages.size();
  out->shared_pages = p->n_shared;
  out->n_seqs = p->n_seqs;
  out->max_seqs = p->cfg.max_seqs;
  return SPP_OK;
}

spp_status spp_seq_create(spp_pool_t p, int32_t n_cells, int32_t* seq_out) {
  if (!p || !seq_out || n_cells < 0) return fail(SPP_E_INVALID_ARG, "null argument or n_cells < 0");
  if (n_cells > SPP_MAX_CAPACITY) return fail(SPP_E_CAPACITY, "%d cells (at most %d)", n_cells, SPP_MAX_CAPACITY);
  return guarded([&] {
    std::lock_guard<std::mutex> lk(p->mu);
    const int want = pages_for(*p, n_cells);
    if (want > (int)p->free_pages.size())
      return fail(SPP_E_CAPACITY, "%d pages needed, %zu free", want, p->free_pages.size());
    if (p->n_seqs >= p->cfg.max_seqs) return fail(SPP_E_CAPACITY, "%d sequences already", p->n_seqs);
    std::vector<int32_t> pages(want);
    const int32_t q = take_seq(*p);
    for (int32_t& pg : pages) pg = take_page(*p);
    p->seqs[q].n = n_cells;
    p->seqs[q].pages = std::move(pages);
    *seq_out = q;
    return SPP_OK;
  });
}

spp_status spp_seq_free(spp_pool_t p, int32_t seq) {
  if (!p) return fail(SPP_E_INVALID_ARG, "null pool");
  return guarded([&] {
    std::lock_guard<std::mutex> lk(p->mu);
    if (const spp_status rc = check_seq(*p, seq); rc != SPP_OK) return rc;
    drop_pages_from(*p, p->seqs[seq], 0);
    p->seqs[seq] = Seq{};
    p->free_seqs.push(seq);
    --p->n_seqs;
    return SPP_OK;
  });
}

spp_status spp_seq_info(spp_pool_t p, int32_t seq, spp_seq_info_t* out) {
  if (!p || !out) return fail(SPP_E_INVALID_ARG, "null argument");
  std::lock_guard<std::mutex> lk(p->mu);
  if (const spp_status rc = check_seq(*p, seq); rc != SPP_OK) return rc;
  const Seq& s = p->seqs[seq];
  *out = spp_seq_info_t{s.n, (int32_t)s.pages.size(), s.summary_at >= 0 ? 1 : 0};
  return SPP_OK;
}

spp_status spp_seq_table(spp_pool_t p, int32_t seq, int32_t* table, int32_t cap, int32_t* n_out) {
  if (!p || !n_out) return fail(SPP_E_INVALID_ARG, "null argument");
  std::lock_guard<std::mutex> lk(p->mu);
  if (const spp_status rc = check_seq(*p, seq); rc != SPP_OK) return rc;
  const std::vector<int32_t>& pages = p->seqs[seq].pages;
  if (table && cap < (int)pages.size())
    return fail(SPP_E_INVALID_ARG, "table of %d entries, %zu pages", cap, pages.size());
  if (table) std::copy(pages.begin(), pages.end(), table);
  *n_out = (int32_t)pages.size();
  return SPP_OK;
}

spp_status spp_seq_fork(spp_pool_t p, int32_t src, int32_t n, int32_t* seqs_out) {
  if (!p || !seqs_out || n < 1) return fail(SPP_E_INVALID_ARG, "null argument or n < 1");
  return guarded([&] {
    std::lock_guard<std::mutex> lk(p->mu);
    if (const spp_status rc = check_seq(*p, src); rc != SPP_OK) return rc;
    if (n > p->cfg.max_seqs - p->n_seqs)
      return fail(SPP_E_CAPACITY, "%d of %d sequences already", p->n_seqs, p->cfg.max_seqs);
    // the pages that hold cells; reserved ones past them stay the source's own
    const int held = pages_for(*p, p->seqs[src].n);
    std::vector<std::vector<int32_t>> tables(
        n, std::vector<int32_t>(p->seqs[src].pages.begin(), p->seqs[src].pages.begin() + held));
    for (int i = 0; i < n; ++i) {
      const int32_t q = take_seq(*p);
      p->seqs[q].n = p->seqs[src].n;
      p->seqs[q].pages = std::move(tables[i]);
      seqs_out[i] = q;
    }
    for (int j = 0; j < held; ++j) {
      int32_t& r = p->refs[p->seqs[src].pages[j]];
      if (r == 1) ++p->n_shared;
      r += n;
    }
    return SPP_OK;
  });
}

spp_status spp_seq_reserve(spp_pool_t p, int32_t n, const int32_t* seqs, int32_t cells, void* stream) {
  if (!p || cells < 1) return fail(SPP_E_INVALID_ARG, "null pool or cells < 1");
  return guarded([&] {
    std::lock_guard<std::mutex> lk(p->mu);
    if (const spp_status rc = check_seqs(*p, n, seqs); rc != SPP_OK) return rc;
    return reserve(*p, n, seqs, cells, static_cast<hipStream_t>(stream));
  });
}

spp_status spp_seq_commit(spp_pool_t p, int32_t seq, int32_t cells) {
  if (!p || cells < 0) return fail(SPP_E_INVALID_ARG, "null pool or cells < 0");
  std::lock_guard<std::mutex> lk(p->mu);
  if (const spp_status rc = check_seq(*p, seq); rc != SPP_OK) return rc;
  Seq& s = p->seqs[seq];
  if (cells == 0) return SPP_OK;
  const bool shared = s.n % p->cfg.page_cells && p->refs[s.pages[s.n >> p->v.shift]] > 1;
  if (shared || ((int64_t)s.pages.size() << p->v.shift) < (int64_t)s.n + cells)
    return fail(SPP_E_STATE, "%d cells after %d are not reserved", cells, s.n);
  s.n += cells;
  s.summary_at = -1;
  return SPP_OK;
}

spp_status spp_seq_truncate(spp_pool_t p, int32_t seq, int32_t n) {
  if (!p || n < 0) return fail(SPP_E_INVALID_ARG, "null pool or n < 0");
  return guarded([&] {
    std::lock_guard<std::mutex> lk(p->mu);
    if (const spp_status rc = check_seq(*p, seq); rc != SPP_OK) return rc;
    Seq& s = p->seqs[seq];
    if (n < s.n) {
      s.n = n;
      s.summary_at = -1;
    }
    drop_pages_from(*p, s, pages_for(*p, s.n));
    return SPP_OK;
  });
}

spp_status spp_seq_import(spp_pool_t p, int32_t seq, spp_session_t s, void* stream) {
  if (!p || !s) return fail(SPP_E_INVALID_ARG, "null argument");
  return guarded([&] {
    std::lock_guard<std::mutex> lk(p->mu);
    if (spp_status rc = check_seq(*p, seq); rc != SPP_OK) return rc;
    if (spp_status rc = check_model(*p, *s->m); rc != SPP_OK) return rc;
    std::lock_guard<std::mutex> sk(s->mu);
    const int want = pages_for(*p, s->n_s);
    Seq& q = p->seqs[seq];
    // pages that its former cells give back
    int64_t back = 0;
    for (int32_t pg : q.pages) back += p->refs[pg] == 1;
    if (want > (int64_t)p->free_pages.size() + back)
      return fail(SPP_E_CAPACITY, "%d pages needed, %lld free", want, (long long)(p->free_pages.size() + back));
    q.pages.reserve(want);
    drop_pages_from(*p, q, 0);
    while ((int)q.pages.size() < want) q.pages.push_back(take_page(*p));
    q.n = s->n_s;
    q.summary_at = -1;
    const spp_status rc = copy_session(*p, q.pages, q.n, *s, true, static_cast<hipStream_t>(stream));
    if (rc != SPP_OK) q.n = 0;  // (what a failed copy leaves are no cells)
    return rc;
  });
}

spp_status spp_seq_export(spp_pool_t p, int32_t seq, spp_session_t s, void* stream) {
  if (!p || !s) return fail(SPP_E_INVALID_ARG, "null argument");
  return guarded([&] {
    std::lock_guard<std::mutex> lk(p->mu);
    if (spp_status rc = check_seq(*p, seq); rc != SPP_OK) return rc;
    if (spp_status rc = check_model(*p, *s->m); rc != SPP_OK) return rc;
    std::lock_guard<std::mutex> sk(s->mu);
    const Seq& q = p->seqs[seq];
    if (q.n > s->capacity) return fail(SPP_E_CAPACITY, "%d cells exceed capacity %d", q.n, s->capacity);
    invalidate(*s);  // Sec. 3.6: in the same call as the mutation
    s->n_s = 0;      // (what a failed copy leaves is no state)
    const spp_status rc = copy_session(*p, q.pages, q.n, *s, false, static_cast<hipStream_t>(stream));
    if (rc == SPP_OK) s->n_s = q.n;
    return rc;
  });
}

spp_status spp_pool_compact(spp_pool_t p, void* stream, int32_t* n_moved) {
  if (!p) return fail(SPP_E_INVALID_ARG, "null pool");
  return guarded([&] {
    std::lock_guard<std::mutex> lk(p->mu);
    const int32_t used = p->cfg.n_pages - (int32_t)p->free_pages.size();
    std::vector<std::pair<int32_t, int32_t>> moves;
    std::vector<int32_t> to(p->cfg.n_pages);
    int32_t hole = 0;
    for (int32_t pg = 0; pg < p->cfg.n_pages; ++pg) {
      to[pg] = pg;
      if (pg < used || !p->refs[pg]) continue;
      while (p->refs[hole]) ++hole;  // (as many holes below `used` as pages in use above it)
      to[pg] = hole++;
      moves.push_back({pg, to[pg]});
    }
    std::vector<int32_t> rest;
    rest.reserve(p->cfg.n_pages);  // (giving pages back never allocates)
    for (int32_t pg = used; pg < p->cfg.n_pages; ++pg) rest.push_back(pg);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (!moves.empty())
      if (const spp_status rc = order_after(*p, st); rc != SPP_OK) return rc;
    if (const spp_status rc = copy_pages(*p, moves, st); rc != SPP_OK) return rc;
    for (Seq& s : p->seqs)
      for (int32_t& pg : s.pages) pg = to[pg];
    for (const auto& mv : moves) std::swap(p->refs[mv.first], p->refs[mv.second]);
    p->free_pages = Lowest(std::greater<int32_t>(), std::move(rest));
    if (n_moved) *n_moved = (int32_t)moves.size();
    return SPP_OK;
  });
}

spp_status spp_decode_batch(spp_pool_t p, spp_model_t m, int32_t n, const int32_t* seqs, const int32_t* tokens,
                            float* const* dists, void* stream) {
  if (!p || !m || !dists) return fail(SPP_E_INVALID_ARG, "null argument");
  return guarded([&] {
    std::lock_guard<std::mutex> lk(p->mu);
    spp_status rc = check_seqs(*p, n, seqs);
    if (rc == SPP_OK) rc = check_model(*p, *m);
    if (rc == SPP_OK) rc = check_tokens(*m, tokens, n);
    if (rc != SPP_OK) return rc;
    for (int i = 0; i < n; ++i)
      if (!dists[i]) return fail(SPP_E_INVALID_ARG, "null dist %d", i);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if ((rc = reserve(*p, n, seqs, 1, st)) != SPP_OK) return rc;  // (st follows the pool's work from here)
    std::lock_guard<std::mutex> mk(m->mu);
    const int per = std::min({(int)k::kScanMax, (int)m->cfg.max_sessions, (int)m->cfg.max_tokens});
    for (int at = 0; at < n; at += per) {
      const int c = std::min(per, n - at);
      std::vector<SegReq> segs(c);
      for (int i = 0; i < c; ++i)
        segs[i] = SegReq{nullptr, tokens + at + i, 1, p->seqs[seqs[at + i]].n, dists[at + i], nullptr,
                         p->summary + seqs[at + i]};
      PagedStep cache(*p, *m, seqs + at, c);
      if ((rc = run_step(*m, segs.data(), c, true, st, nullptr, nullptr, &cache)) != SPP_OK) break;
      for (int i = 0; i < c; ++i) {
        Seq& s = p->seqs[seqs[at + i]];
        s.summary_at = ++s.n;
      }
    }
    return end_work(*p, st, rc);
  });
}

spp_status spp_seq_summaries(spp_pool_t p, int32_t n, const int32_t* seqs, spp_summary* out) {
  if (!p || !seqs || !out || n < 1) return fail(SPP_E_INVALID_ARG, "null argument or n < 1");
  return guarded([&] {
    std::lock_guard<std::mutex> lk(p->mu);
    int lo = p->cfg.max_seqs, hi = -1;
    for (int i = 0; i < n; ++i) {
      if (const spp_status rc = check_seq(*p, seqs[i]); rc != SPP_OK) return rc;
      if (p->seqs[seqs[i]].summary_at < 0) return fail(SPP_E_STATE, "sequence %d has no summary", seqs[i]);
      lo = std::min(lo, (int)seqs[i]);
      hi = std::max(hi, (int)seqs[i]);
    }
    std::vector<ScanResult> r(hi - lo + 1);
    HIPCHK(hipEventSynchronize(p->events[p->done]->ev));
    HIPCHK(hipMemcpy(r.data(), p->summary + lo, r.size() * sizeof(ScanResult), hipMemcpyDeviceToHost));
    for (int i = 0; i < n; ++i) fill_summary(r[seqs[i] - lo], p->seqs[seqs[i]].summary_at, out + i);
    return SPP_OK;
  });
}

size_t spp_paged_attention_work_bytes(const spp_paged_attn* a) {
  if (check_attn(a) != SPP_OK || a->n_seqs == 0) return 0;
  // fewer sequences may take more ranges each: the most that any number of them up to n_seqs takes
  // (what one takes never falls with max_pages)
  size_t most = k::paged_work_bytes(a->pool->v, a->n_seqs, a->n_q_heads, a->max_pages);
  for (int n = std::min(a->n_seqs, kSplitWorkgroups); n >= 1; --n)
    most = std::max(most, k::paged_work_bytes(a->pool->v, n, a->n_q_heads, a->max_pages));
  return most;
}

spp_status spp_paged_attention(const spp_paged_attn* a, void* work, size_t work_bytes, void* stream) {
  if (const spp_status rc = check_attn(a); rc != SPP_OK) return rc;
  if (a->n_seqs == 0) return SPP_OK;
  const spp_pool_s& p = *a->pool;
  const size_t need = k::paged_work_bytes(p.v, a->n_seqs, a->n_q_heads, a->max_pages);
  if (need && (!work || work_bytes < need || !aligned16(work)))
    return fail(SPP_E_INVALID_ARG, "workspace of %zu bytes, need %zu, 16-byte aligned", work ? work_bytes : 0, need);
  const PagedAttn c{a->q, a->q_stride, a->io_dtype == SPP_DTYPE_BF16, a->n_seqs, a->n_q_heads, a->table,
                    a->table_stride, a->max_pages, a->lengths, a->scale, a->out, nullptr, a->out_stride,
                    a->io_dtype == SPP_DTYPE_BF16 ? 1 : 0};
  hipSetDevice(p.device);
  const hipError_t e = k::paged_attention(p.v, a->layer, c, work, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(SPP_E_HIP, "paged attention: %s", hipGetErrorString(e));
  return SPP_OK;
}

size_t spp_adjust_logits_work_bytes(int32_t n, int32_t vocab) {
  if (n < 1 || vocab < 1 || vocab > (1 << 24)) return 0;
  // the most rows that are cut into the shorter slices may take more than n rows
  const int few = std::min(n, kShortSliceTokens / vocab);
  return std::max(k::adjust_work_bytes(n, vocab), few ? k::adjust_work_bytes(few, vocab) : 0);
}

spp_status spp_adjust_logits(int32_t n, int32_t vocab, const spp_adjust* rows, spp_summary* summaries, void* work,
                             size_t work_bytes, void* stream) {
  if (n < 0 || (n > 0 && !rows)) return fail(SPP_E_INVALID_ARG, "null rows or n < 0");
  if (vocab < 1 || vocab > (1 << 24)) return fail(SPP_E_INVALID_ARG, "vocab outside [1, 2^24]");
  for (int i = 0; i < n; ++i) {
    const spp_adjust& r = rows[i];
    if (!r.src || !r.dst || r.n_tokens < 0 || r.n_bias < 0 || (r.n_tokens && !r.tokens) ||
        (r.n_bias && (!r.bias_tokens || !r.bias)))
      return fail(SPP_E_INVALID_ARG, "row %d: null pointer or negative count", i);
    if (!aligned4(r.src) || !aligned4(r.dst) || !aligned4(r.tokens) || !aligned4(r.bias_tokens) ||
        !aligned4(r.bias) || !aligned4(r.allowed))
      return fail(SPP_E_INVALID_ARG, "row %d: pointers are 4-byte aligned", i);
    if (r.n_tokens > (1 << 30) || r.n_bias > (1 << 30)) return fail(SPP_E_INVALID_ARG, "row %d: a list over 2^30", i);
    if (r.n_prompt < 0 || r.n_prompt > r.n_tokens) return fail(SPP_E_INVALID_ARG, "row %d: n_prompt", i);
    if (!(r.repetition > 0.f) || !std::isfinite(r.repetition) || !std::isfinite(r.frequency) ||
        !std::isfinite(r.presence) || std::isnan(r.fill))
      return fail(SPP_E_INVALID_ARG, "row %d: repetition must be > 0, penalties finite, fill a number", i);
  }
  if (n == 0) return SPP_OK;
  if (!aligned4(summaries)) return fail(SPP_E_INVALID_ARG, "summaries are 4-byte aligned");
  const size_t need = summaries ? k::adjust_work_bytes(n, vocab) : 0;
  if (need && (!work || work_bytes < need || !aligned16(work)))
    return fail(SPP_E_INVALID_ARG, "workspace of %zu bytes, need %zu, 16-byte aligned", work ? work_bytes : 0, need);
  const hipError_t e = k::adjust_logits(n, vocab, rows, summaries, work, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(SPP_E_HIP, "adjust logits: %s", hipGetErrorString(e));
  return SPP_OK;
}

}  // extern "C"
