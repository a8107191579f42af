// Log probabilities of rows of logits behind the C ABI (include/spp.h).
#include <algorithm>

#include "paged.hpp"
#include "runtime.hpp"

using namespace spp;

namespace {

bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

bool shape_ok(int32_t n, int32_t vocab, int32_t n_top) {
  return n >= 0 && n <= (1 << 20) && vocab >= 1 && vocab <= (1 << 24) && n_top >= 0 && n_top <= SPP_MAX_TOP;
}

}  // namespace

extern "C" {

size_t spp_logprobs_work_bytes(int32_t n, int32_t vocab, int32_t n_top) {
  if (n < 1 || !shape_ok(n, vocab, n_top)) return 0;
  // the most rows that are cut into the shorter slices may take more than n rows
  const int few = std::min(n, kShortSliceTokens / vocab);
  return std::max(k::logprob_work_bytes(n, vocab, n_top), few ? k::logprob_work_bytes(few, vocab, n_top) : 0);
}

spp_status spp_logprobs(int32_t n, int32_t vocab, const spp_logprob_row* rows, int32_t n_top, int32_t* top_tokens,
                        float* top_logprobs, float* lse, float* entropy, void* work, size_t work_bytes,
                        void* stream) {
  if (!shape_ok(n, vocab, n_top))
    return fail(SPP_E_INVALID_ARG, "n outside [0, 2^20], vocab outside [1, 2^24] or n_top outside [0, %d]", SPP_MAX_TOP);
  if (n == 0) return SPP_OK;
  if (!rows || (n_top && (!top_tokens || !top_logprobs))) return fail(SPP_E_INVALID_ARG, "null argument");
  if (!aligned(top_tokens, 4) || !aligned(top_logprobs, 4) || !aligned(lse, 4) || !aligned(entropy, 4))
    return fail(SPP_E_INVALID_ARG, "results are 4-byte aligned");
  for (int i = 0; i < n; ++i) {
    const spp_logprob_row& r = rows[i];
    if (!r.logits || r.n_tokens < 0 || (r.n_tokens && (!r.tokens || !r.logprobs)))
      return fail(SPP_E_INVALID_ARG, "row %d: null pointer or negative count", i);
    if (r.n_tokens > (1 << 30)) return fail(SPP_E_INVALID_ARG, "row %d: a list over 2^30", i);
    if (!aligned(r.logits, 4) || !aligned(r.tokens, 4) || !aligned(r.logprobs, 4))
      return fail(SPP_E_INVALID_ARG, "row %d: pointers are 4-byte aligned", i);
  }
  const size_t need = k::logprob_work_bytes(n, vocab, n_top);
  if (!work || work_bytes < need || !aligned(work, 16))
    return fail(SPP_E_INVALID_ARG, "workspace of %zu bytes, need %zu, 16-byte aligned", work ? work_bytes : 0, need);
  const hipError_t e = k::logprobs(n, vocab, rows, n_top, top_tokens, top_logprobs, lse, entropy, work,
                                   static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(SPP_E_HIP, "logprobs: %s", hipGetErrorString(e));
  return SPP_OK;
}

}  // extern "C"
