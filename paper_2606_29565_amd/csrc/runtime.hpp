// What the parts of the host runtime share: the model and session objects and the device
// step over packed rows (runtime.cpp), which the paged sequences of pool.cpp take too.
#pragma once

#include "spp.h"

#include <hip/hip_runtime.h>

#include <memory>
#include <mutex>
#include <vector>

#include "kernels.hpp"

namespace spp {

// Records the calling thread's error text and returns `st`.
spp_status fail(spp_status st, const char* fmt, ...);

#define HIPCHK(expr)                                                                     \
  do {                                                                                   \
    hipError_t e_ = (expr);                                                              \
    if (e_ != hipSuccess) return fail(SPP_E_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

inline int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

// A device buffer that grows on demand.  Growing frees the old block, so the caller
// must make sure no queued work still uses it.
struct DevBuf {
  void* p = nullptr;
  size_t bytes = 0;
};

// An event that lives as long as one of those who wait for it.
struct Event {
  hipEvent_t ev = nullptr;
  Event() = default;
  Event(const Event&) = delete;
  Event& operator=(const Event&) = delete;
  ~Event() {
    if (ev) hipEventDestroy(ev);
  }
};

// Per-kernel timing for spp_profile_preposition (dispatch events, see LaunchRecorder).
using Prof = LaunchRecorder;

struct Model {
  spp_model_config cfg{};
  Shape s{};
  int device = 0;
  int n_cu = 256;                     // compute units of the device (attention work sizing)
  size_t elem = 2;
  const void* embed = nullptr;
  const void* final_norm = nullptr;
  const void* lm_head = nullptr;
  const float* lm_bias = nullptr;
  std::vector<const void*> attn_norm, wq, wk, wv, wo, mlp_norm, wg, wu, wd;  // wq..wd tiled
  bool fp4 = false;                   // wq..wd are MXFP4 codes (tiled), scales in wsc
  std::vector<const void*> wsc[7];    // tiled e8m0 scales per spp_weight_kind (MXFP4)
  std::vector<void*> owned;           // library-owned packed copies (weights_packed == 0)
  void* lm_tiled = nullptr;           // packed LM head for the batched path (max_sessions > 1)
  int slab[5] = {1, 1, 1, 1, 1};      // tiled-layout slab (K-steps) of QKV, O, gate/up, down, LM head
  // work buffers
  float* x = nullptr;
  void* h = nullptr;
  void* q = nullptr;
  void* att = nullptr;
  void* act = nullptr;
  float* part = nullptr;
  size_t part_elems = 0;              // floats of `part`
  char* small = nullptr;              // one allocation: the scan buffers, ss, range, rope and z
  float* ss = nullptr;                // row sums of squares [max_tokens][res_blocks]
  uint32_t* range = nullptr;          // the step's fp16 range word per segment [kMaxSegments]
  float2* rope = nullptr;
  void* z = nullptr;
  float* logits_rows = nullptr;
  ScanPartial* gate_parts = nullptr; // two scan buffers of k::kScanBufBytes, side by side
  ScanPartial* lm_parts = nullptr;
  ScanResult* gate_host = nullptr;   // pinned, device-mapped [64] results, then the done word
  ScanResult* gate_dev = nullptr;
  uint32_t gate_seq = 0;
  uint32_t gate_late = 0;            // a scan that its call gave up on and that may still run (0: none)
  DevBuf o_part, ml_part, params_dev;
  char* params_host = nullptr;
  size_t params_host_bytes = 0;
  hipEvent_t params_free = nullptr;  // the last params upload has been consumed
  hipEvent_t step_done = nullptr;    // the last step has finished with the work buffers
  hipEvent_t chunk_end[2] = {};      // ends of the last two layer chunks of a yielding pass
  bool step_recorded = false;
  std::shared_ptr<Event> copied;      // a pool has copied a session's cells since (null: none has)
  std::mutex mu;       // one step at a time per model (work buffers)
  std::mutex gate_mu;  // one gate scan at a time per model (gate buffers)
};

struct Session {
  Model* m = nullptr;
  int id = 0;
  int capacity = 0, cap_stride = 0, budget = 0;
  void* kv = nullptr;
  size_t kv_bytes = 0;
  std::mutex mu;
  int n_s = 0;
  std::vector<int32_t> entry;  // the pre-positioned entry (speculative cells n_s..)
  bool valid = false;
  uint64_t epoch = 0;
  int position = -1;
  float* dist = nullptr;
  hipEvent_t done = nullptr;
  uint64_t decoded_epoch = ~0ull;  // epoch whose device work was seen finished
  ScanResult* summary = nullptr;  // device slot written by the LM head
  // Released with the last reference: a gate that looked the session up by its id keeps
  // it alive until it returns, even when spp_session_destroy runs meanwhile.
  ~Session() {
    if (done) {
      hipEventSynchronize(done);
      hipEventDestroy(done);
    }
    if (summary) hipFree(summary);
  }
};

// One segment of a step: `len` tokens at position n_past of a session, or of a paged sequence
// (then s is null).
struct SegReq {
  Session* s;
  const int32_t* tok;
  int len;
  int n_past;
  float* dist;
  const uint32_t* bitmap;
  ScanResult* summary;  // where the LM head's reductions go
};

// Cooperative yield of an idle-window pass (Sec. 3.1): the layers are enqueued in chunks,
// at most two chunks ahead of the device, and before each chunk the caller's flag is read;
// once it is set, nothing more is enqueued and the pass ends when the device has drained.
struct YieldCtl {
  const volatile uint32_t* flag;
  int chunk;       // layers per chunk
  bool yielded;
};

// Where the cells of a step's rows are, if not in the sessions' buffers: the step's record
// carries what the cache needs, and its epilogue and attention replace the sessions' own.
struct StepCache {
  virtual ~StepCache() = default;
  virtual size_t record_bytes() const = 0;          // appended to the step's record
  virtual size_t part_bytes() const = 0;            // workspace of the attention
  virtual void fill(char* host, char* dev) = 0;     // writes the record; keeps its device address
  virtual hipError_t epilogue(const StepView& v, int rows, int layer, const float* partials, int splits,
                              const float* ss, const float2* rope, float* q, hipStream_t st) = 0;
  virtual hipError_t attention(int layer, const float* q, void* part, void* out, void* out_lo,
                               hipStream_t st) = 0;
};

// What touches the cells of a model's sessions is one line: `st` continues after all of it, and
// note_step marks what was enqueued since as its new end.  (Copies of a pool mark it with the
// event that the pool records anyway, and does not record again while it is `copied`: a second
// record in a row costs the device 4 us.)  The caller holds m.mu.
inline spp_status after_steps(Model& m, hipStream_t st) {
  if (m.step_recorded) HIPCHK(hipStreamWaitEvent(st, m.step_done, 0));
  if (m.copied) HIPCHK(hipStreamWaitEvent(st, m.copied->ev, 0));
  return SPP_OK;
}
inline spp_status note_step(Model& m, hipStream_t st) {
  HIPCHK(hipEventRecord(m.step_done, st));
  m.step_recorded = true;
  m.copied.reset();
  return SPP_OK;
}

spp_status run_step(Model& m, const SegReq* segs, int nseg, bool logits, hipStream_t st, Prof* prof,
                    YieldCtl* y = nullptr, StepCache* cache = nullptr);
spp_status check_tokens(const Model& m, const int32_t* t, int n);
// Invalidates a session's ready record (Sec. 3.6); the caller holds its mutex.
void invalidate(Session& s);
void fill_summary(const ScanResult& r, int position, spp_summary* out);

}  // namespace spp

struct spp_model_s : spp::Model {};
struct spp_session_s : spp::Session {};
