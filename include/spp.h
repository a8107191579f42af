/* spp.h -- speculative pre-positioning on one MI355X (gfx950): the C ABI.
 *
 * A stateful session keeps a persistent KV cache of n_s committed tokens
 * (Sec. 2 of the paper).  In the idle window after a state update the caller
 * runs a PRE-POSITION step (Alg. 1): the entry tokens (query prefix plus
 * assistant header, or a post-tool-call envelope) are appended at the live end
 * n_s and one forward pass runs over the entry only, against the resident
 * cells.  The logits at the last entry token -- the decision point
 * p = n_s + L_entry of Eq. (decision-point) -- are the READY DISTRIBUTION
 * (Sec. 2.1, Sec. 3.3).  When a request arrives, the GATE (Alg. 2, Eq. (gate))
 * scans that cached distribution: it serves the argmax token iff the top-1 to
 * top-2 logit gap (Eq. (gap)) is strictly greater than tau and the token is in
 * the fast-answer set; otherwise the request falls through.  Any mutation of
 * the state invalidates the cached distribution in the same call (Sec. 3.6).
 *
 * Conventions for every entry point:
 *   - Return value: spp_status.  0 = SPP_OK, > 0 = an informational outcome,
 *     < 0 = an error; spp_last_error() then describes it (thread-local string).
 *     No C++ exception crosses this boundary.
 *   - Device memory holding weights, KV cells, distributions and fast-answer
 *     bitmaps is allocated and owned by the caller and must outlive every model
 *     and session that points at it.  The library owns its own work buffers
 *     (allocated at model creation) and the opaque model / session objects.
 *   - `stream` is a hipStream_t (NULL = the default stream).  Device work is
 *     enqueued on it in order; calls marked "asynchronous" return before the
 *     device finishes.
 *   - Matrices are row-major.  A projection weight W of a layer y = x W^T is
 *     stored [out_features][in_features].  Element type is the model dtype:
 *     SPP_DTYPE_BF16 (16-bit bf16 patterns) or SPP_DTYPE_F32.
 *   - One thread at a time per session for mutating calls; spp_gate may run
 *     concurrently with a pending pre-position of the same session.
 */
#ifndef SPP_H
#define SPP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SPP_OK = 0,
  SPP_SKIPPED_BUDGET = 1,   /* Alg. 1: L_entry > cell-budget headroom B; nothing touched  */
  SPP_YIELDED = 2,          /* Sec. 3.1: an idle-window pass gave way to a request       */
  SPP_E_INVALID_ARG = -1,   /* null pointer, bad size, token outside [0, vocab), tau < 0 */
  SPP_E_CAPACITY = -2,      /* committed tokens would exceed the session's KV capacity  */
  SPP_E_HIP = -3,           /* a HIP runtime call failed                                 */
  SPP_E_STATE = -4,         /* call not allowed in the current state                     */
  SPP_E_NOMEM = -5          /* the library could not allocate its work buffers          */
} spp_status;

/* Alg. 2 outcomes.  The paper's "fall through" is split by its cause. */
typedef enum {
  SPP_SERVED = 0,           /* gate fired: *token_out is the cached argmax                */
  SPP_FALL_INVALID = 1,     /* no valid ready distribution, stale handle, or not decoded */
  SPP_FALL_INELIGIBLE = 2,  /* realized entry differs from the pre-positioned entry      */
  SPP_FALL_GAP = 3,         /* gap <= tau                                                */
  SPP_FALL_NOT_IN_SET = 4,  /* argmax not in the fast-answer set                         */
  SPP_FALL_NONFINITE = 5    /* the distribution holds NaN or +-inf (never served)        */
} spp_gate_outcome;

/* State mutations of Sec. 3.6. */
typedef enum {
  SPP_MUT_SHIFT = 0,        /* sliding-window shift done by the caller: invalidates only
                               (spp_shift relocates the cells itself)                    */
  SPP_MUT_ROLLBACK = 1,     /* discard committed tokens: n_s <- min(arg, n_s)            */
  SPP_MUT_UPDATE = 2        /* a fresh update was committed elsewhere: invalidate only   */
} spp_mutation;

typedef enum { SPP_DTYPE_F32 = 0, SPP_DTYPE_BF16 = 1 } spp_dtype;

/* Cells of a pool in 8 bits an element: a code (a signed integer, or a float of 4 exponent and 3
 * mantissa bits, largest 448) times the scale of its block.  See "caches of 8-bit codes". */
typedef enum { SPP_CELLS_I8 = 8, SPP_CELLS_E4M3 = 9 } spp_cell_codes;

/* Storage of the projection weights wq..w_down.  MXFP4 is the OCP microscaling format
 * (the 4-bit weight-only variant of the 70B-class headline model, Sec. 4): every weight
 * is a 4-bit e2m1 code (bit 3 sign, bits 2..1 exponent, bit 0 mantissa: magnitudes
 * 0, 0.5, 1, 1.5, 2, 3, 4, 6), and every 32 consecutive weights of a row share one
 * 8-bit e8m0 scale E, w = 2^(E - 127) * e2m1(code), E in [1, 254].  Row-major storage:
 * codes [rows][cols/2] bytes with the even column in the low nibble, scales
 * [rows][cols/32] bytes.  Activations, KV cells, embedding and LM head stay bf16. */
typedef enum { SPP_WFMT_DTYPE = 0, SPP_WFMT_MXFP4 = 1 } spp_weight_format;

typedef struct spp_model_s* spp_model_t;
typedef struct spp_session_s* spp_session_t;

/* Decoder shape.  Pre-norm decoder: RMSNorm (rms_eps), rotate-half RoPE
 * (rope_base), grouped-query attention where q head h reads kv head
 * h / (n_q_heads / n_kv_heads), SwiGLU MLP, untied LM head with optional bias. */
typedef struct {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, ffn_dim, vocab;
  float rms_eps;
  double rope_base;
  int32_t dtype;            /* spp_dtype of weights, KV cells and matrix-core operands  */
  int32_t max_tokens;       /* most tokens one call processes (sizes the work buffers)  */
  int32_t max_sessions;     /* most sessions one batched call covers (1..64)            */
  int32_t weights_packed;   /* 1: wq..w_down are already in the tiled layout written by
                               spp_pack_weight; 0: they are row-major and the library keeps
                               tiled copies (it does not read the caller's projection
                               weights after spp_model_create returns)                    */
  int32_t weight_format;    /* spp_weight_format of wq..w_down (MXFP4: bf16 models only)  */
} spp_model_config;

/* Device pointers to the weights (caller-owned).  The per-layer members are HOST
 * arrays of n_layers device pointers; the library copies the arrays.  The projection
 * weights wq..w_down are row-major or tiled (spp_model_config.weights_packed); the
 * embedding, norms and LM head are always row-major. */
typedef struct {
  const void* embed;                 /* [vocab][d_model]                               */
  const void* final_norm;            /* [d_model]                                      */
  const void* lm_head;               /* [vocab][d_model]                               */
  const float* lm_bias;              /* [vocab] fp32, or NULL for no bias              */
  const void* const* attn_norm;      /* [d_model]                                      */
  const void* const* wq;             /* [n_q_heads*head_dim][d_model]                  */
  const void* const* wk;             /* [n_kv_heads*head_dim][d_model]                 */
  const void* const* wv;             /* [n_kv_heads*head_dim][d_model]                 */
  const void* const* wo;             /* [d_model][n_q_heads*head_dim]                  */
  const void* const* mlp_norm;       /* [d_model]                                      */
  const void* const* w_gate;         /* [ffn_dim][d_model]                             */
  const void* const* w_up;           /* [ffn_dim][d_model]                             */
  const void* const* w_down;         /* [d_model][ffn_dim]                             */
  /* MXFP4 models only (else ignored): scales[kind], kind an spp_weight_kind, is a HOST
   * array of n_layers device pointers to that projection's e8m0 scales -- row-major
   * [rows][cols/32] bytes, or tiled by spp_pack_weight_mxfp4 when weights_packed = 1.
   * The projection members above then point at the 4-bit codes. */
  const void* const* scales[7];
} spp_weights;

typedef struct {
  int32_t capacity;         /* KV cells the caller's buffer holds per layer              */
  int32_t budget;           /* the session's cell budget (0 = capacity): pre-positions
                               need L_entry <= budget - n_s (Alg. 1's headroom B)         */
} spp_session_config;

/* Where cell (head, position, dim) of layer `layer` lives inside a session's KV
 * buffer: byte offset of K element = k_offset + (head*k_stride[0] +
 * position*k_stride[1] + dim*k_stride[2]) * elem_bytes, likewise for V. */
typedef struct {
  int64_t k_offset, v_offset;        /* bytes                                          */
  int64_t k_stride[3], v_stride[3];  /* elements, for (head, position, dim)            */
  int32_t elem_bytes;
} spp_kv_layout;

/* Handle to a ready distribution: a value, nothing to free.  It names the
 * session and the epoch of the pre-position; once any mutation (or a newer
 * pre-position) bumps the session's epoch, the handle is stale and the gate
 * returns SPP_FALL_INVALID (Sec. 3.6: a stale answer is never served). */
typedef struct {
  int32_t session_id;
  int32_t reserved;
  uint64_t epoch;
} spp_ready_t;

/* The reductions over a ready distribution (Eq. (gap)): argmax (ties -> lowest
 * index), the two largest logits (a duplicated maximum gives gap 0), the gap,
 * log-sum-exp (NaN when any logit is NaN or +-inf), and the flags.
 *
 * Flag bit 2 (bf16 models): the forward pass met an attention input outside the range
 * of fp16, in which the attention of bf16 models multiplies -- a query scaled by
 * log2(e)/sqrt(head_dim), or a K or V cell, of magnitude above 65504.  Precondition of
 * the bf16 path: every K/V cell and every scaled query stays within +-65504 (magnitudes
 * below 2^-14 are kept to fp16's absolute resolution, 2^-24).  A flagged distribution
 * is never served: the gate answers SPP_FALL_NONFINITE. */
typedef struct {
  int32_t argmax;
  float top1, top2, gap, lse;
  int32_t position;         /* decision point p = n_s + L_entry                         */
  uint32_t flags;           /* bit 0: nonfinite logits; bit 1: argmax in the default set;
                               bit 2: an attention input beyond the fp16 range          */
} spp_summary;

/* The fields Alg. 1 records on the session (decision-point position, a decoded flag and
 * a validity flag for the cached distribution), with the cell accounting behind its
 * budget check and the epoch that invalidation bumps (Sec. 3.6). */
typedef struct {
  int32_t n_committed;      /* n_s                                                      */
  int32_t used_cells;       /* n_s + entry cells of the current pre-position            */
  int32_t capacity, budget;
  int32_t position;         /* last recorded decision point (-1 = none)                 */
  int32_t valid;            /* 1 while the ready distribution is current               */
  int32_t decoded;          /* 1 once the pre-position's device work has finished      */
  int32_t entry_len;
  uint64_t epoch;
} spp_session_info_t;

/* ---- models ---------------------------------------------------------------------- */

/* The target model whose single forward pass over the entry is Alg. 1's Forward(E) (the
 * paper's engine serves one decoder on one accelerator, Sec. 4; its architecture is not
 * given there and follows spp_model_config).
 * Validates the shape (head_dim 64 or 128 for bf16, 64 for fp32; n_q_heads a multiple of
 * n_kv_heads; d_model, ffn_dim and n_q_heads*head_dim multiples of 64 (bf16) or 32
 * (fp32); d_model a width the LM-head kernel covers: ceil(d_model / 512) (bf16) or
 * ceil(d_model / 256) (fp32) in {1, 2, 4, 8, 10, 16}; with MXFP4 weights also d_model,
 * ffn_dim and n_q_heads*head_dim multiples of 128), copies the weight pointers and
 * allocates the work buffers on the current HIP device.  SPP_E_INVALID_ARG on a bad
 * shape or null pointer. */
spp_status spp_model_create(const spp_model_config* cfg, const spp_weights* weights,
                            spp_model_t* out);
spp_status spp_model_destroy(spp_model_t model);

/* Which projection weight of a layer spp_pack_weight rearranges; the shape follows
 * from the model configuration. */
typedef enum {
  SPP_W_Q = 0,     /* [n_q_heads*head_dim][d_model]  */
  SPP_W_K = 1,     /* [n_kv_heads*head_dim][d_model] */
  SPP_W_V = 2,     /* [n_kv_heads*head_dim][d_model] */
  SPP_W_O = 3,     /* [d_model][n_q_heads*head_dim]  */
  SPP_W_GATE = 4,  /* [ffn_dim][d_model]             */
  SPP_W_UP = 5,    /* [ffn_dim][d_model]             */
  SPP_W_DOWN = 6   /* [d_model][ffn_dim]             */
} spp_weight_kind;

/* Rearranges one row-major projection weight of a model with configuration `cfg`
 * (device memory, model dtype) into the tiled layout the projection kernels stream:
 * every 16 rows x 128 bytes of columns become one 2 KB block in the order a 64-lane
 * wave loads it, and the blocks are ordered so that the workgroups of a projection
 * launch read adjacent blocks at the same moment (the order depends on the projection
 * and the configuration, hence both arguments).  src and dst are distinct device
 * buffers of rows*cols elements.  The result is what spp_model_create expects with
 * weights_packed = 1 for the same configuration.  Asynchronous on `stream`.
 * SPP_E_INVALID_ARG for a bad configuration, unknown `which` or null pointer. */
spp_status spp_pack_weight(const spp_model_config* cfg, int32_t which, const void* src, void* dst,
                           void* stream);

/* MXFP4 counterpart of spp_pack_weight: rearranges one projection's row-major codes
 * ([rows][cols/2] bytes) and scales ([rows][cols/32] bytes) into the tiled layout of the
 * 4-bit projection kernels: per 16 rows x 128 columns, a 1 KB code block in the order
 * the 64 lanes of a wave feed the matrix cores and a 64-byte scale block, ordered like
 * the bf16 tiles.  cfg->weight_format must be SPP_WFMT_MXFP4 and cols a multiple of 128.
 * Destinations are distinct device buffers of the same sizes as the sources.
 * Asynchronous on `stream`.  SPP_E_INVALID_ARG for a bad configuration, unknown `which`
 * or null pointer. */
spp_status spp_pack_weight_mxfp4(const spp_model_config* cfg, int32_t which,
                                 const void* codes_src, const void* scales_src, void* codes_dst,
                                 void* scales_dst, void* stream);

/* ---- sessions -------------------------------------------------------------------- */

/* Largest KV capacity of a session in cells per layer (2^24 - 64: the attention kernels
 * address one kv head's keys and values with 32-bit byte offsets). */
#define SPP_MAX_CAPACITY (16777216 - 64)

/* Bytes of device memory a session of `capacity` cells needs for its KV buffer. */
size_t spp_session_kv_bytes(spp_model_t model, int32_t capacity);
spp_status spp_session_kv_layout(spp_model_t model, int32_t capacity, int32_t layer,
                                 spp_kv_layout* out);

/* A stateful session (Sec. 2: one persistent KV cache of n_s accumulated tokens that
 * survives across requests and advances incrementally) over a caller-owned KV buffer of
 * kv_bytes >= spp_session_kv_bytes(), 16-byte aligned, laid out as
 * spp_session_kv_layout describes.  cfg->capacity is the cells per layer the buffer
 * holds, at most SPP_MAX_CAPACITY; cfg->budget (0 = capacity) bounds n_s plus the entry
 * of a pre-position, the cell budget of Alg. 1.  Starts with n_s = 0 and no ready
 * distribution.  SPP_E_INVALID_ARG on a null pointer, capacity outside
 * [1, SPP_MAX_CAPACITY], budget outside [0, capacity], a short or misaligned buffer; SPP_E_NOMEM if the session's small device record cannot
 * be allocated.  The session is named by a process-unique id (spp_session_id), which
 * ready handles carry. */
spp_status spp_session_create(spp_model_t model, const spp_session_config* cfg, void* kv_dev,
                              size_t kv_bytes, spp_session_t* out);
/* Removes the session from the id registry and invalidates its record: a gate still
 * holding a handle of it falls through as SPP_FALL_INVALID; a gate or summary already
 * inside the session finishes first, and the session's resources are released when the
 * last such call returns.  SPP_E_INVALID_ARG for a session destroyed before. */
spp_status spp_session_destroy(spp_session_t session);
int32_t spp_session_id(spp_session_t session);

/* Metadata-only restore (the paper's constant-time T_restore): declare that cells
 * [0, n_tokens) of every layer already hold committed state the caller wrote (see
 * spp_session_kv_layout).  Invalidates any ready distribution. */
spp_status spp_session_restore(spp_session_t session, int32_t n_tokens);

/* Commit a delta (a data batch, a tool result): drops the speculative entry cells,
 * invalidates the ready distribution (Sec. 3.6), then appends `n` tokens (host
 * array) at n_s with one forward pass and advances n_s.  Asynchronous.
 * SPP_E_CAPACITY if n_s + n > capacity; SPP_E_INVALID_ARG on a token outside
 * [0, vocab) or n outside [1, max_tokens]. */
spp_status spp_kv_append_delta(spp_session_t session, const int32_t* tokens, int32_t n,
                               void* stream);

/* Alg. 1.  If L_entry > B (B = budget - n_s): invalidates, touches no cell and
 * returns SPP_SKIPPED_BUDGET.  Otherwise appends the entry (host array) at n_s, runs
 * one forward pass over it, writes the fp32 logits of the last entry token to
 * dist_dev[vocab] (caller-owned device memory), records p = n_s + L_entry, bumps
 * the epoch, marks the session valid, and returns the handle in *out.  The entry
 * cells stay speculative (n_s does not move).  `default_bitmap_dev` (nullable,
 * ceil(vocab/32) words, bit t&31 of word t>>5) sets summary flag bit 1.
 * Asynchronous: the gate treats the distribution as not decoded until the device
 * work has finished. */
spp_status spp_preposition(spp_session_t session, const int32_t* entry, int32_t L_entry,
                           float* dist_dev, const uint32_t* default_bitmap_dev, void* stream,
                           spp_ready_t* out);

/* The idle-window pre-position (Sec. 3.1: speculative work runs only while the session
 * is idle and gives way at once to an arriving request; Alg. 1).  Computes what
 * spp_preposition computes, but enqueues the forward pass in chunks of `chunk_layers`
 * layers, at most two chunks ahead of the device, and reads *yield_flag (caller-owned
 * host memory; a serving thread sets it nonzero when a request arrives) before each
 * chunk.  Blocking: returns when the pass has finished (SPP_OK: the ready record is in
 * place and decoded) or, once the flag is seen set, when the chunks already enqueued
 * have drained (SPP_YIELDED: nothing more was enqueued, no logits were made, the
 * session has no ready record and n_s is unchanged; the entry cells written so far are
 * uncommitted).  A flag already set at the call yields before any device work.  The
 * wait after a set flag is bounded by two chunks of layers (plus the LM head if the
 * last chunk was already enqueued).  Stream priorities are not used: the yield is the
 * library's own.  While the pass runs it holds the model's step lock, so a forward pass
 * of any session of the same model (resume, append, another pre-position) waits for it:
 * a serving thread sets the flag first, then makes its call.  Gates of other sessions
 * do not wait; a gate of this session waits for the yield and then falls through as
 * SPP_FALL_INVALID.  Budget, argument errors and the handle as in
 * spp_preposition; SPP_E_INVALID_ARG for a null flag or chunk_layers < 1. */
spp_status spp_preposition_idle(spp_session_t session, const int32_t* entry, int32_t L_entry,
                                float* dist_dev, const uint32_t* default_bitmap_dev,
                                const volatile uint32_t* yield_flag, int32_t chunk_layers,
                                void* stream, spp_ready_t* out);

/* Fall-through resume (Eq. (fallthrough); Sec. 3.5): the arriving request extends the
 * pre-positioned entry by `delta` (n >= 1 tokens, host array).  The entry's cells stay
 * where the pre-position wrote them (the constant-time restore) and are committed
 * together with the delta: n_s <- n_s + L_entry + n.  Forward passes over the delta
 * alone (max_tokens rows each) write its cells, and the last one writes the fp32 logits
 * at the new end to dist_dev[vocab], recorded as the session's new ready state (position
 * n_s, epoch bumped, so earlier handles go stale; entry_len 0, so only the relaxed gate
 * with realized = NULL can serve it).  With no entry present (never pre-positioned,
 * skipped, or dropped by a mutation) the delta is appended after the committed cells,
 * which is the cold path.  A one-token delta is one decode step.  Unlike a pre-position,
 * a resume is on the critical path: it is bounded by the session's capacity, not by its
 * idle-window budget, and SPP_E_CAPACITY (nothing changed) if the cells do not fit.
 * Asynchronous on `stream`; default_bitmap_dev as in spp_preposition. */
spp_status spp_resume(spp_session_t session, const int32_t* delta, int32_t n, float* dist_dev,
                      const uint32_t* default_bitmap_dev, void* stream, spp_ready_t* out);

/* The reductions the LM head computed over the ready distribution of `ready` (Eq. (gap):
 * argmax, top-1 and top-2 logits, their gap; Sec. 3.3: under the gate the cache may
 * hold only the argmax and the gap), with the log-sum-exp and the flags.  Blocks until
 * the pre-position behind `ready` has finished.  SPP_E_STATE if the handle is stale or
 * its session is gone; SPP_E_INVALID_ARG for a null `out`. */
spp_status spp_ready_summary(spp_ready_t ready, spp_summary* out);

/* Alg. 2.  Checks, in this order: handle current and session valid and device work
 * finished (else SPP_FALL_INVALID); the realized entry (host array, NULL = relaxed
 * streaming mode of Sec. 3.4) equal to the pre-positioned entry (else
 * SPP_FALL_INELIGIBLE).  Then one scan of the cached distribution on `stream`
 * computes the argmax, the two largest logits and the set bit; the call waits for
 * it and decides: nonfinite -> SPP_FALL_NONFINITE; gap > tau is false ->
 * SPP_FALL_GAP; argmax not in the set (fast_bitmap_dev, device, ceil(vocab/32)
 * words; NULL = empty set) -> SPP_FALL_NOT_IN_SET; else SPP_SERVED with
 * *token_out = argmax (otherwise *token_out = -1).  Synchronous.  Read-only: the
 * distribution keeps serving repeated requests.  SPP_E_INVALID_ARG for tau < 0 or
 * NaN; SPP_E_HIP if the scan has not finished after 20 s.  Until that scan has, the next
 * gates of the model (spp_gate_batch too, on whatever stream) wait as long for it and
 * return the same error, with no scan of their own.  `scan_out` (nullable) receives the
 * scan's summary. */
spp_status spp_gate(spp_ready_t ready, float tau, const uint32_t* fast_bitmap_dev,
                    const int32_t* realized_entry, int32_t n_realized, void* stream,
                    int32_t* token_out, spp_gate_outcome* outcome, spp_summary* scan_out);

/* Sec. 3.6: clears the valid and decoded flags and bumps the epoch in the same call
 * as the mutation.  SPP_MUT_ROLLBACK sets n_s <- min(arg, n_s) (arg >= 0). */
spp_status spp_invalidate_on_mutation(spp_session_t session, spp_mutation kind, int32_t arg);

/* Sliding-window shift (Sec. 3.6, the mutation that relocates positions): drops the
 * oldest `delta` committed cells and moves the others down by delta positions in every
 * layer -- cell p goes to p - delta, its key turned back by delta positions (rotate-half
 * RoPE: the pair (k_i, k_{i+dh/2}) rotated by the angle -delta * rope_base^(-2i/dh)),
 * its value unchanged -- so n_s <- n_s - delta.  Invalidates the ready distribution and
 * drops the speculative entry in the same call.  Asynchronous on `stream`, ordered after
 * the session's earlier device work.  SPP_E_INVALID_ARG unless 1 <= delta <= n_s (then
 * nothing changes). */
spp_status spp_shift(spp_session_t session, int32_t delta, void* stream);

/* The fields of spp_session_info_t (Alg. 1's recorded position, decoded and valid
 * flags; the cell accounting; the epoch).  Reading `decoded` queries the device work's
 * completion, nothing else.  SPP_E_INVALID_ARG on a null pointer. */
spp_status spp_session_info(spp_session_t session, spp_session_info_t* out);
/* The same call under its earlier name. */
spp_status spp_session_info_get(spp_session_t session, spp_session_info_t* out);

/* ---- batched (many sessions of one model in one pass) ------------------------------ */

/* Alg. 1 for `n` sessions at once: the entries are packed into one pass so every
 * weight is read once for all of them.  Arrays of length n: sessions, entries (host
 * arrays), lengths, dists (device fp32[vocab] each).  Per-session results go to
 * out_status[i] (SPP_OK or SPP_SKIPPED_BUDGET) and out_ready[i].  A pass packs at most
 * the model's max_sessions entries (and max_tokens rows); more sessions take further
 * passes.  The return value is an error if any argument is invalid (then nothing ran):
 * a null pointer, a session of another model or listed twice, a length outside
 * [1, max_tokens], a token outside [0, vocab).  Asynchronous. */
spp_status spp_preposition_batch(int32_t n, const spp_session_t* sessions,
                                 const int32_t* const* entries, const int32_t* lengths,
                                 float* const* dists, void* stream, spp_ready_t* out_ready,
                                 spp_status* out_status);

/* Alg. 2 for n handles, as spp_gate in the relaxed mode (no realized entry): one scan
 * launch per 64 handles, one wait for all of them.  bitmaps (nullable) holds a device
 * bitmap or NULL per handle; taus[i] >= 0.  tokens_out[i] and outcomes[i] as in
 * spp_gate.  Handles of one call belong to one model.  Synchronous. */
spp_status spp_gate_batch(int32_t n, const spp_ready_t* ready, const float* taus,
                          const uint32_t* const* bitmaps, void* stream, int32_t* tokens_out,
                          spp_gate_outcome* outcomes);

/* For callers that cannot allocate memory -- code under HIP graph capture, tight serving
 * loops, harnesses that forbid allocation: spp_gate_batch with the scan's partials and
 * results in a static device array of the library (about 130 KB, one copy per device for
 * the life of the process) instead of the model's buffers.  Allocates nothing: no
 * hipMalloc, hipFree or allocating library call.  The results come back through one
 * device-to-host copy on `stream`, which is then synchronized.  At most 64 handles per
 * call (SPP_E_INVALID_ARG beyond, nothing run), all of models on the current device.
 * Outcomes and tokens as spp_gate_batch.  Every call on a device shares that device's
 * array: the library serializes such calls per device (a call waits for the previous
 * one's results), so overlapping calls do not race; every partial and result a call reads
 * is written by it, and the array's arrival counters are zero between calls (each call's
 * last workgroup clears them). */
spp_status spp_gate_batch_noalloc(int32_t n, const spp_ready_t* ready, const float* taus,
                                  const uint32_t* const* bitmaps, void* stream,
                                  int32_t* tokens_out, spp_gate_outcome* outcomes);

/* ---- paged caches ------------------------------------------------------------------ */

/* A pool of pages: the cells of many sequences in one caller-owned buffer, `page_cells`
 * cells of every layer to a page.  It serves a fall-through (Sec. 3.5) that decodes several
 * continuations of one state: a session's cells are imported once, forks share their pages,
 * and only the page a fork writes into becomes its own.  Sequences are numbered 0 ..
 * max_seqs - 1; a number is taken by spp_seq_create or spp_seq_fork and given back by
 * spp_seq_free.
 *
 * The bookkeeping (tables, references, free pages) is on the host and done when a call
 * returns.  The device work of a pool's calls -- copies and decode steps -- is enqueued on
 * the call's stream and ordered after that of the pool's earlier calls on whatever stream,
 * so a page freed and taken again is not written while earlier work reads it.  A pool's
 * calls may come from several threads: they are serialized.  Work that a caller enqueues on
 * the pages by itself (spp_paged_attention too) is the caller's to order: on the stream of a
 * spp_seq_reserve it follows the pool's earlier calls, and later calls have to be put behind
 * it (their stream, or an event).  A pool's calls are not for capture into a graph
 * (spp_paged_attention is). */
typedef struct spp_pool_s* spp_pool_t;

typedef struct {
  int32_t n_layers, n_kv_heads, head_dim;  /* of the models whose cells it holds; head_dim
                                              64 or 128                                  */
  int32_t dtype;            /* spp_dtype of the cells, or their spp_cell_codes            */
  int32_t page_cells;       /* cells per page: 16, 32, 64, 128 or 256                     */
  int32_t n_pages;          /* pages in the caller's buffer, >= 1                         */
  int32_t max_seqs;         /* most sequences alive at once, 1..65536                     */
} spp_pool_config;

/* Where cell (layer, head, cell, dim) of a page lives: byte offset from the buffer's start
 * of the K element = page*page_stride + layer*layer_stride + (head*k_stride[0] +
 * cell*k_stride[1] + dim*k_stride[2]) * elem_bytes; of the V element = page*page_stride +
 * layer*layer_stride + v_offset + (head*v_stride[0] + cell*v_stride[1] +
 * dim*v_stride[2]) * elem_bytes.  (K is [head][cell][dim], V [head][dim][cell].) */
typedef struct {
  int64_t page_stride, layer_stride, v_offset;  /* bytes    */
  int64_t k_stride[3], v_stride[3];             /* elements */
  int32_t elem_bytes;
} spp_page_layout;

typedef struct {
  int32_t n_pages, used_pages;   /* used: referred to by at least one sequence            */
  int32_t shared_pages;          /* referred to by more than one                          */
  int32_t n_seqs, max_seqs;
} spp_pool_info_t;

typedef struct {
  int32_t n_cells;               /* the sequence's length                                 */
  int32_t n_pages;               /* pages of its table (reserved ones among them)         */
  int32_t decoded;               /* 1 while spp_seq_summaries has a summary of it         */
} spp_seq_info_t;

/* Bytes of the buffer a pool needs (0 for a bad configuration), and its layout. */
size_t spp_pool_bytes(const spp_pool_config* cfg);
spp_status spp_pool_page_layout(const spp_pool_config* cfg, spp_page_layout* out);

/* A pool over a caller-owned device buffer of at least spp_pool_bytes() bytes, 16-byte
 * aligned, on the current device.  No page is touched.  SPP_E_INVALID_ARG on a null pointer,
 * a bad configuration, a short or misaligned buffer; SPP_E_NOMEM if the pool's device record
 * (32 bytes a sequence) cannot be allocated. */
spp_status spp_pool_create(const spp_pool_config* cfg, void* pages_dev, size_t bytes,
                           spp_pool_t* out);
/* Waits for the pool's device work, then releases it (no call may use it meanwhile). */
spp_status spp_pool_destroy(spp_pool_t pool);
spp_status spp_pool_info(spp_pool_t pool, spp_pool_info_t* out);

/* A sequence of n_cells cells with pages of its own, whose contents the caller has written
 * or will write (0: an empty one).  No stream waits here: earlier work of the pool may still
 * use these pages, and a caller that cannot rule it out starts with 0 cells, reserves and
 * commits.  Pages are taken lowest number first, here and below.
 * SPP_E_CAPACITY when the pages or the sequence numbers run out (then nothing changes, as
 * for every call below). */
spp_status spp_seq_create(spp_pool_t pool, int32_t n_cells, int32_t* seq_out);
/* Gives up a sequence: its pages lose a reference, those without any are free. */
spp_status spp_seq_free(spp_pool_t pool, int32_t seq);
spp_status spp_seq_info(spp_pool_t pool, int32_t seq, spp_seq_info_t* out);
/* The sequence's page numbers in order (host array of `cap` entries, at least its n_pages;
 * *n_out receives how many).  With table NULL only *n_out is written. */
spp_status spp_seq_table(spp_pool_t pool, int32_t seq, int32_t* table, int32_t cap,
                         int32_t* n_out);

/* `n` new sequences with the cells of `src`: they share its pages (those that hold cells),
 * nothing is copied yet.  seqs_out: host array of n.  SPP_E_CAPACITY when the sequence
 * numbers run out. */
spp_status spp_seq_fork(spp_pool_t pool, int32_t src, int32_t n, int32_t* seqs_out);

/* Makes the next `cells` cells of each of n distinct sequences writable: the page their
 * last cell shares with another sequence is copied to a page of their own (one launch for
 * all), and pages are added to their tables.  Lengths do not change.  spp_decode_batch does
 * this for its one cell; a caller that writes cells itself reserves, writes and then calls
 * spp_seq_commit.  Asynchronous on `stream`, on which what is enqueued next follows the
 * pool's earlier work, also where nothing is copied.  SPP_E_CAPACITY when the pages run out. */
spp_status spp_seq_reserve(spp_pool_t pool, int32_t n, const int32_t* seqs, int32_t cells,
                           void* stream);
/* Declares the next `cells` cells written: n_cells <- n_cells + cells.  SPP_E_STATE unless
 * pages of the sequence's own hold them, as after spp_seq_reserve. */
spp_status spp_seq_commit(spp_pool_t pool, int32_t seq, int32_t cells);
/* Discards cells: n_cells <- min(n_cells, n), and gives up the pages past them.  (What a discarded
 * cell made of its block's scale stays where the pool's cells are 8-bit codes.) */
spp_status spp_seq_truncate(spp_pool_t pool, int32_t seq, int32_t n);

/* The sequence becomes a copy of the session's committed cells (its former cells are given
 * up): every layer's cells [0, n_s) into pages of its own.  The session is only read.  Asynchronous
 * on `stream`, ordered after the device work of the session's model as well, and before its
 * next (as spp_seq_export); the session's buffer stays until the copy has run.
 * SPP_E_INVALID_ARG unless the session's model has the pool's layers, kv heads, head_dim and
 * dtype (any, where the pool's cells are 8-bit codes: they are quantised on the way in, and come
 * back as values of the session's dtype) and lives on its device; SPP_E_CAPACITY when the pages run
 * out. */
spp_status spp_seq_import(spp_pool_t pool, int32_t seq, spp_session_t session, void* stream);
/* The session's committed state becomes a copy of the sequence: its cells [0, n_cells) of
 * every layer are overwritten, n_s <- n_cells, its entry is dropped and its ready
 * distribution invalidated in the same call (Sec. 3.6).  Errors as for spp_seq_import;
 * SPP_E_CAPACITY when the cells exceed the session's capacity. */
spp_status spp_seq_export(spp_pool_t pool, int32_t seq, spp_session_t session, void* stream);

/* Moves the used pages together: with u pages in use, those numbered u and above move, in
 * ascending order, to the free ones below u, in ascending order, and the tables follow.
 * Afterwards pages [0, u) are in use and the buffer past them is free.  *n_moved (nullable):
 * the pages copied.  Asynchronous on `stream`. */
spp_status spp_pool_compact(spp_pool_t pool, void* stream, int32_t* n_moved);

/* One decode step of n distinct sequences at once (the decode of Eq. (fallthrough), batched):
 * tokens[i] (host array) is appended to seqs[i] -- its cells are written at n_cells of every
 * layer, into a page of the sequence's own (as spp_seq_reserve) -- and the fp32 logits after
 * it go to dists[i] (host array of device pointers, fp32[vocab] each); n_cells grows by one.
 * Every weight is read once for up to the model's max_sessions (and max_tokens) sequences;
 * more take further passes.  The model has the pool's layers, kv heads, head_dim and dtype (any,
 * where the pool's cells are 8-bit codes) and lives on its device.  Asynchronous on `stream`.
 * SPP_E_INVALID_ARG for a null pointer, n < 1, a sequence that does not exist or is listed
 * twice, a token outside [0, vocab);
 * SPP_E_CAPACITY when the pages run out or a sequence is SPP_MAX_CAPACITY cells long (then
 * nothing ran).  After SPP_E_HIP the sequences of finished passes have grown, the others not. */
spp_status spp_decode_batch(spp_pool_t pool, spp_model_t model, int32_t n, const int32_t* seqs,
                            const int32_t* tokens, float* const* dists, void* stream);
/* The reductions over the logits that the last spp_decode_batch of each sequence wrote (as
 * spp_ready_summary; position = n_cells after it).  Blocks until the pool's device work has
 * finished.  SPP_E_STATE for a sequence that has changed since, or was never decoded. */
spp_status spp_seq_summaries(spp_pool_t pool, int32_t n, const int32_t* seqs, spp_summary* out);

/* Attention of one new token per sequence over paged cells, the attention of
 * spp_decode_batch: for every sequence i and query head h (which reads kv head
 * h / (n_q_heads / n_kv_heads)),
 *   out = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale q.k_j),
 * over the cells j < lengths[i] of layer `layer` whose page is listed: cell j is in page
 * table[i][j / page_cells].  A table entry outside [0, n_pages) takes its cells out (a page
 * given up from the middle); lengths beyond max_pages*page_cells are cut to it, negative
 * ones are zero.  A sequence with no cell left gets zeros.  What lies in a page behind a sequence's
 * last cell, or in a page that is not listed, has no influence, NaN included.  Of a live cell, a
 * NaN of K makes the rows of the query heads that read it NaN, one of V its dimension of them; an
 * infinity of V makes its dimension infinite or NaN, and one of K makes infinite or NaN scores.  A
 * score of +inf or NaN makes its row NaN, one of -inf has no weight (a row of these alone gets zeros).
 * The products of bf16 cells run on bf16 matrix cores with q (unless it is bf16) and p in
 * two bf16 parts and fp32 sums: about 16 significant bits of both.  8-bit codes are taken as they
 * are, exactly, and likewise; their scales multiply scores and p_j in fp32.  A live cell whose scale
 * is NaN makes the rows that read it NaN. */
typedef struct {
  spp_pool_t pool;
  int32_t layer;
  int32_t n_seqs;            /* 0..65535 (0: nothing is done)                             */
  int32_t n_q_heads;         /* a multiple of the pool's n_kv_heads, at most 65535        */
  int32_t io_dtype;          /* spp_dtype of q and out                                    */
  const void* q;             /* device, [n_seqs] rows of [n_q_heads][head_dim]            */
  int64_t q_stride;          /* elements between rows, a multiple of 8; q 16-byte aligned */
  const int32_t* table;      /* device, [n_seqs] rows of max_pages page numbers           */
  int64_t table_stride;      /* entries between rows, >= max_pages                        */
  int32_t max_pages;         /* >= 1; max_pages*page_cells <= 2^30                        */
  const int32_t* lengths;    /* device, [n_seqs]                                          */
  float scale;               /* finite; 0 stands for 1 / sqrt(head_dim)                   */
  void* out;                 /* device, rows as q's                                       */
  int64_t out_stride;        /* as q_stride                                               */
} spp_paged_attn;
/* Bytes of workspace that suffice for the call, and for those with fewer sequences or a smaller
 * max_pages (0 for bad arguments, or none needed): a workspace made for the largest batch
 * serves it as sequences finish, which may need more than the largest itself.  The size depends on
 * n_seqs, n_q_heads, max_pages and the pool. */
size_t spp_paged_attention_work_bytes(const spp_paged_attn* a);
/* Only launches kernels (one or two) on `stream`: it may be captured into a graph, whose
 * replays read the table and the lengths as they are then.  The workspace (device, 16-byte
 * aligned) is written before it is read; two calls that may run at once need two.
 * SPP_E_INVALID_ARG for a null pointer or a value outside what the fields say. */
spp_status spp_paged_attention(const spp_paged_attn* a, void* work, size_t work_bytes,
                               void* stream);

/* ---- caches of 8-bit codes ----------------------------------------------------------- */

/* A pool whose dtype is an spp_cell_codes holds every element in 8 bits: half a bf16 cell, so that
 * attention reads half.  16 cells of one head (cells 16 b .. 16 b + 15 of a sequence) are a
 * block, keys and values apart, and share an fp32 scale, a power of two:
 *   s = the smallest with max |x| / s <= Q over the block's cells, at least 2^-100,
 *   code = x / s rounded to the nearest, ties to even,   Q = 127 (I8) or 448 (E4M3).
 * Cells appended to a block that holds cells already (a decode step, spp_paged_write) keep its s
 * at least what it was; where it grows, the codes there are rounded to the new one.  So what a
 * block holds depends on what was written and in which order.  The error of an element is at
 * most s / 2 (I8), or 2^-4 of it and 2^-10 s (E4M3), as it is written, and after any growth less
 * than s (I8), or 2^-4 of it and 2^-9 s (E4M3): I8 keeps 6 to 7 bits below the block's largest
 * element, E4M3 keeps 4 bits of each element down to 2^-13 of it.  A block that is given an
 * infinity or a NaN has the scale NaN and reads as NaN from then on, until it is written from its
 * first cell; magnitudes of 2^127 and more may come back infinite.  Cells of a block past the
 * last written one are undefined.  So, unlike in a pool of values, an append (a decode step,
 * spp_paged_write) writes the scale and the codes of up to 15 earlier cells of its sequence again: what
 * reads those is ordered against it.  And spp_seq_truncate takes cells away, not what they did to the
 * block that is cut: a scale that they made larger stays so, one that is NaN stays NaN.
 *
 * All calls of a pool serve such pools too: import and export convert, decode steps append,
 * forks, reserves and compaction copy pages with their scales. */

/* Where the scale of (layer, head, block of a page) lives: byte offset from the buffer's start
 * of K's = page*page_stride + layer*layer_stride + k_offset + (head*stride[0] + block*stride[1])
 * * 4, of V's likewise (the other strides in spp_page_layout). */
typedef struct {
  int64_t k_offset, v_offset;   /* bytes           */
  int64_t stride[2];            /* fp32 elements   */
  int32_t block_cells;          /* 16              */
} spp_scale_layout;
/* SPP_E_INVALID_ARG for a bad configuration, a null pointer, or cells that are no codes. */
spp_status spp_pool_scale_layout(const spp_pool_config* cfg, spp_scale_layout* out);

/* Cells of one layer of many sequences as rows of the caller's: row rows[i] + j of k and v is cell
 * first[i] + j of sequence i, for 0 <= j < rows[i + 1] - rows[i].  Tables as in
 * spp_paged_attention.  A sequence with first[i] < 0 or rows[i] < 0, rows from n_rows on, rows of a
 * sequence past max_cells and cells past its table are left out. */
typedef struct {
  spp_pool_t pool;           /* of 8-bit codes, at most 32767 kv heads                    */
  int32_t layer;
  int32_t n_seqs;            /* 0..65535 (0: nothing is done)                             */
  const int32_t* table;      /* device, [n_seqs] rows of max_pages page numbers           */
  int64_t table_stride;      /* entries between rows, max_pages..2^31 - 1                 */
  int32_t max_pages;         /* >= 1; max_pages*page_cells <= 2^30                        */
  const int32_t* first;      /* device, [n_seqs]                                          */
  const int32_t* rows;       /* device, [n_seqs + 1]                                      */
  int32_t n_rows;            /* rows of k and v, >= 0                                     */
  int32_t max_cells;         /* most cells of a sequence, 1..2^24; times n_kv_heads at most
                                63 * 2^23                                                 */
  int32_t io_dtype;          /* spp_dtype of k and v                                      */
  void* k;                   /* device, [n_rows] rows of [n_kv_heads][head_dim]           */
  int64_t k_stride;          /* elements between rows, a multiple of 8 below 2^35; k 16-byte
                                aligned                                                   */
  void* v;                   /* as k                                                      */
  int64_t v_stride;
} spp_paged_cells;

/* Quantises rows into cells (k and v are only read).  In the block of a sequence's first new cell,
 * the cells before that one, which have been written (their scale counts), keep their values as
 * described above; the cells past the last new one are undefined afterwards.  Cells whose page is
 * not listed are left out.  No block is written from two places of a call, in two sequences or
 * through a page that one lists twice (a spp_seq_reserve gives them pages of their own); what such
 * a block holds afterwards is undefined.  Only launches a kernel on `stream` and may be
 * captured into a graph, whose replays read tables, first, rows, k and v as they are then; it is
 * the caller's to order against the pool's other work, as spp_paged_attention.  SPP_E_INVALID_ARG
 * for a null pointer or a value outside what the fields say. */
spp_status spp_paged_write(const spp_paged_cells* a, void* stream);
/* The cells' values, code times scale, into the rows (exact in bf16, but for what lies beyond its
 * range).  Rows of cells whose page is not listed are zeros; rows that are no cell's stay as they
 * are.  Otherwise as spp_paged_write. */
spp_status spp_paged_read(const spp_paged_cells* a, void* stream);

/* ---- adjusted logits ---------------------------------------------------------------- */

/* One row of spp_adjust_logits.  For every token v:
 *   y = x                                          the logit src[v]
 *   y = y > 0 ? y / repetition : y * repetition    if v occurs in tokens
 *   y = y - frequency * c                          c: occurrences of v in tokens past the
 *   y = y - (c > 0 ? presence : 0)                    first n_prompt
 *   y = y + bias[i]                                if bias_tokens[i] = v (the last such i)
 *   y = fill                                       if the allowed set lacks v
 * every operation in fp32 with its own rounding.  Entries of tokens and bias_tokens
 * outside [0, vocab) are skipped: a row may keep one array of tokens, filled with -1 behind a
 * history that grows in place.  Every part of a row reads the whole list, so its length counts,
 * skipped entries too. */
typedef struct {
  const float* src;             /* device, [vocab]                                        */
  float* dst;                   /* device, [vocab]; may be src                            */
  const int32_t* tokens;        /* device, [n_tokens]: the prompt, then the answer so far */
  const int32_t* bias_tokens;   /* device, [n_bias]                                       */
  const float* bias;            /* device, [n_bias]                                       */
  const uint32_t* allowed;      /* device bitmap as the gate's fast-answer set; NULL: all */
  int32_t n_tokens, n_prompt;   /* 0 <= n_prompt <= n_tokens <= 2^30                      */
  int32_t n_bias;               /* 0..2^30                                                */
  float repetition;             /* finite, > 0; 1 changes nothing                         */
  float frequency, presence;    /* finite; 0 changes nothing                              */
  float fill;                   /* not NaN.  The gate never serves a distribution with an
                                   infinite value: fill with a finite one, such as
                                   -FLT_MAX, to gate the adjusted logits                  */
} spp_adjust;

/* Bytes of workspace that suffice for n rows with summaries, and for fewer (which may need more
 * than n rows themselves). */
size_t spp_adjust_logits_work_bytes(int32_t n, int32_t vocab);
/* Penalties for repeated tokens, biases and an allowed set (a grammar's next tokens) on n
 * rows of logits -- those of a resume or a decode step -- with the reductions a greedy step
 * reads.  rows: host array, read during the call.  No dst overlaps what another row reads or
 * writes, nor its own row's src unless it is the same; every pointer is 4-byte aligned and on
 * the current device.  summaries (nullable): device array of n
 * spp_summary: argmax (lowest index on ties), top1, top2, gap and lse over the adjusted
 * logits of the ALLOWED tokens, position 0, flags bit 0 if one of these is NaN or +-inf (lse
 * is then NaN; a NaN is never the argmax), bit 3 if no token is allowed (gap and lse are then
 * NaN).  Where no token qualifies argmax is -1 and top1 -inf; with one, top2 is -inf.  The
 * workspace (device, 16-byte aligned, needed only with summaries) is written before it is
 * read; two calls that may run at once need two.  Only launches kernels on `stream`: it may
 * be captured into a graph (the fields above are fixed then, what the pointers name is read
 * at each replay).  SPP_E_INVALID_ARG for n < 0, vocab outside [1, 2^24], a null pointer, or
 * a value outside what the fields say (then nothing ran). */
spp_status spp_adjust_logits(int32_t n, int32_t vocab, const spp_adjust* rows,
                             spp_summary* summaries, void* work, size_t work_bytes,
                             void* stream);

/* ---- log probabilities -------------------------------------------------------------- */

/* A row of logits and the tokens whose log probabilities are asked: logprobs[i] receives
 * log p(tokens[i]), p = softmax of the row; NaN for a token outside [0, vocab) (a list may be
 * filled with -1). */
typedef struct {
  const float* logits;       /* device, [vocab]                                           */
  const int32_t* tokens;     /* device, [n_tokens]                                        */
  float* logprobs;           /* device, [n_tokens]                                        */
  int32_t n_tokens;          /* 0..2^30                                                   */
} spp_logprob_row;

#define SPP_MAX_TOP 64

/* Bytes of workspace that suffice for n rows, and for fewer (0 for bad arguments). */
size_t spp_logprobs_work_bytes(int32_t n, int32_t vocab, int32_t n_top);
/* Log probabilities of given tokens over n rows of logits -- those of a resume, a decode step or
 * adjusted ones -- by which continuations of one state are compared, with what tells how sure the
 * model was: per row (each nullable) lse[i], the log of the sum of exp(x), and entropy[i] = -sum p
 * log p in nats; and the n_top (0..SPP_MAX_TOP) most probable tokens, top_tokens and top_logprobs
 * (device, [n][n_top]), in order, of equal logits the lower index first.
 * A logit of -inf has probability 0, log probability -inf, and is no alternative; where fewer
 * than n_top tokens are, the rest are -1 with -inf.  A NaN or +inf makes its row's log
 * probabilities, lse and entropy NaN (alternatives are still in the order of the logits, NaN left
 * out); a row without any logit above -inf has lse -inf, and NaN for its log probabilities and
 * entropy.  Sums are of fp32; the largest logit's own term is kept apart, so a log probability
 * near 0 keeps its relative precision, but for terms below 2^-126 of the largest (logits over 87 below
 * it), which may be lost.
 * rows: host array, read during the call.  No result overlaps another or a logit.  The workspace
 * (device, 16-byte aligned) is written before it is read; two calls that may run at once need
 * two.  Every pointer is 4-byte aligned and on the current device.  Only launches kernels on
 * `stream`: it may be captured into a graph, whose replays read logits and tokens as they are
 * then.  SPP_E_INVALID_ARG for n outside [0, 2^20], vocab outside [1, 2^24], a null pointer or a
 * value outside what the fields say (then nothing ran). */
spp_status spp_logprobs(int32_t n, int32_t vocab, const spp_logprob_row* rows, int32_t n_top,
                        int32_t* top_tokens, float* top_logprobs, float* lse, float* entropy,
                        void* work, size_t work_bytes, void* stream);

/* ---- gate calibration ------------------------------------------------------------- */

/* One threshold of the gate's risk-coverage curve (Sec. 2.4, Eqs. (coverage), (risk)):
 * `served` of the n decision points pass the gate (gap > tau and argmax in the set),
 * `wrong` of those disagree with the full-path output; coverage = served / n, risk =
 * wrong / served (NaN when nothing is served); Wilson score intervals for both. */
typedef struct {
  float tau;
  int32_t served, wrong;
  double coverage, coverage_lo, coverage_hi;
  double risk, risk_lo, risk_hi;
} spp_gate_point;

/* Host-side calibration of the gate threshold from n measured decision points (Sec. 2.4:
 * the smallest tau with r(tau) <= r_max, which maximizes coverage at bounded risk).
 * gaps[i]: the top-1 minus top-2 logit gap of decision point i's ready distribution;
 * in_set[i]: 1 if its argmax is in the fast-answer set; correct[i]: 1 if that argmax
 * equals the model's full-path output for the request.  Candidate thresholds are the
 * n_taus values in `taus` (each >= 0), or with n_taus = 0 every distinct gap >= 0 plus
 * 0 (coverage and risk change only where tau crosses a gap).  curve (nullable, curve_cap
 * points) receives the curve in ascending tau, *n_points its length; *tau_star the
 * smallest candidate with at least one point served and risk <= r_max, or +inf if none
 * qualifies (then the gate should not fire).  z: the normal quantile of the intervals
 * (1.959964 for 95%).  No device work.  SPP_E_INVALID_ARG on null pointers, n < 1, a
 * negative or NaN tau, r_max < 0, z <= 0, or a curve too short for the candidates. */
spp_status spp_gate_calibrate(int32_t n, const float* gaps, const uint8_t* in_set,
                              const uint8_t* correct, double r_max, double z, int32_t n_taus,
                              const float* taus, spp_gate_point* curve, int32_t curve_cap,
                              int32_t* n_points, float* tau_star);

/* ---- diagnostics ------------------------------------------------------------------- */

const char* spp_last_error(void);

/* Device time of the kernels of one pre-position step, measured with a start and a
 * stop HIP event carried by each kernel's own dispatch on `stream` (the kernel's
 * execution, without the launch gaps between kernels; a profiling run: it performs a
 * real pre-position with the same effects as spp_preposition, then waits).
 * times_us[k] receives the summed time of kernel class k over the step and counts[k]
 * its kernel launches, for k < n_classes (see spp_kernel_class_name).  Returns the
 * number of classes, or -1 on error (spp_last_error; an entry beyond the session's
 * headroom, which spp_preposition answers with SPP_SKIPPED_BUDGET, is an error here). */
int32_t spp_profile_preposition(spp_session_t session, const int32_t* entry, int32_t L_entry,
                                float* dist_dev, void* stream, int32_t n_classes,
                                float* times_us, int32_t* counts);
const char* spp_kernel_class_name(int32_t k);

/* spp_preposition_batch measured the same way: the same effects, then a wait; times_us[k]
 * and counts[k] summed over every pass of the batch.  Returns the number of classes, or
 * -1 on error (spp_last_error). */
int32_t spp_profile_preposition_batch(int32_t n, const spp_session_t* sessions,
                                      const int32_t* const* entries, const int32_t* lengths,
                                      float* const* dists, void* stream, spp_ready_t* out_ready,
                                      spp_status* out_status, int32_t n_classes, float* times_us,
                                      int32_t* counts);

/* Plain device copy of n bytes (both device pointers): the traffic reference the
 * HBM counters are calibrated against.  Asynchronous. */
spp_status spp_copy_reference(void* dst, const void* src, size_t n, void* stream);

#ifdef __cplusplus
}
#endif
#endif
