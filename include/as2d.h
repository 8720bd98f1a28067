/*
 * as2d.h -- C-ABI of the GB300 (sm_103a) target-side block verification
 * library, libas2d.so.
 *
 * The operation (paper: Section 3.2 "Target verification"; App. A.2
 * "Configuration and execution boundaries"; App. C.2 "Verification and state
 * repair"; App. C.4, Eq. 3 and Prop. 1):
 *   the target decoder holds a committed prefix in its KV cache (prefilled
 *   audio and instruction tokens plus every committed token except the last
 *   one) and a pending "known root" token -- the last committed token, not yet
 *   forwarded.  A verification call forwards the root followed by k drafter
 *   candidates c_1..c_k in one causal pass (physical width K = k + 1),
 *   takes the greedy token g_i after each row i, accepts the longest prefix
 *   c_1..c_n with c_{i+1} = g_i, and emits the correction g_n (the bonus
 *   token when n = k).  The cache keeps the root's and the accepted
 *   candidates' entries; the rejected rows' entries are dropped.  The
 *   correction is not forwarded: it becomes the next call's root, so full
 *   acceptance needs no extra single-token call (App. C.2, known-root
 *   carry).  With k = 0 the call is one plain greedy decode
 *   step of Eq. 3.
 *
 * Conventions shared by every entry point:
 *   - Pointers documented "device" are CUDA device pointers on the current
 *     device; "host" pointers are ordinary host memory, read before the call
 *     returns.  `stream` is a cudaStream_t (NULL = the legacy default stream).
 *   - Work is enqueued on `stream` and never synchronises with the host,
 *     except where an entry point says it does.  Device outputs are valid once
 *     the caller synchronises the stream.
 *   - Argument errors are found on the host before anything is enqueued and
 *     leave all state unchanged.  as2d_last_error() then describes the error
 *     (thread-local).
 *   - Every bf16 value is the upper 16 bits of an IEEE float (bfloat16).
 */
#ifndef AS2D_H
#define AS2D_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t as2d_status;
#define AS2D_OK 0
#define AS2D_ERR_INVALID_ARG (-1)   /* bad pointer, size or value            */
#define AS2D_ERR_CAPACITY (-2)      /* L + k + 1 would exceed the capacity   */
#define AS2D_ERR_CUDA (-3)          /* a CUDA runtime call failed            */
#define AS2D_ERR_UNSUPPORTED (-4)   /* shape outside what the kernels handle */
#define AS2D_ERR_DEVICE (-5)        /* a kernel reported an error or timeout */
#define AS2D_ERR_NO_MEMORY (-6)     /* a host allocation failed              */

/* Device-side error bits (as2d_kv_check's message names them; the static
   decode step returns them through its error_bits output). */
#define AS2D_DEVERR_BAD_TOKEN 1  /* a root or candidate id outside [0, vocab)  */
#define AS2D_DEVERR_ROLLBACK 2   /* a rollback beyond the committed length, or
                                    below what an eviction left               */
#define AS2D_DEVERR_TIMEOUT 4    /* a kernel's bounded wait gave up            */
#define AS2D_DEVERR_CAPACITY 8   /* a device-side length left no room for the
                                    call's rows (length < 0 or length + rows >
                                    capacity): that request was skipped       */
#define AS2D_DEVERR_BAD_TREE 16  /* a candidate's parent is no earlier row of
                                    its request                               */
#define AS2D_DEVERR_NO_TOKEN 32  /* a row's probabilities gave no token (NaN
                                    logits, or none above -inf)               */
#define AS2D_DEVERR_NOT_FINITE 64 /* NaN or an infinity was to be written into a
                                    cache of 4 bits                           */

/* Largest number of candidates per request in one call (the budget b of
   App. A.2; physical width K = k + 1 <= 17). */
#define AS2D_MAX_K 16
/* Largest number of requests verified together in one call. */
#define AS2D_MAX_BATCH 64

/* Decoder shape.  Requirements: hidden % 128 == 0, (n_q * head_dim) % 128
   == 0, ffn % 64 == 0, vocab % 8 == 0, head_dim in {64, 128},
   n_q % n_kv == 0, n_kv * head_dim % 128 == 0.  rope_theta is the rotary base (rotate-half
   pairing of dimensions i and i + head_dim/2, angle pos * theta^(-2i/d));
   rms_eps is added to the mean square before the root. */
typedef struct as2d_config {
  int32_t n_layers, hidden, n_q_heads, n_kv_heads, head_dim, ffn, vocab;
  float rope_theta, rms_eps;
} as2d_config;

/* Weights, as device pointers to bf16 in checkpoint (logical) layouts,
   row-major: embed, lm_head [vocab][hidden]; final_norm and the per-layer
   attn_norm, mlp_norm gains [hidden]; w_q [n_q*d][hidden], w_k, w_v
   [n_kv*d][hidden] (head j in rows [j*d, (j+1)*d)); w_o [hidden][n_q*d];
   w_gate, w_up [ffn][hidden]; w_down [hidden][ffn].  The per-layer members
   are HOST arrays of n_layers device pointers.  as2d_model_load copies every
   tensor into memory the model owns (re-laid out for the kernels); the caller
   may free its buffers once as2d_model_load has returned. */
typedef struct as2d_weights {
  const void* embed;
  const void* final_norm;
  const void* lm_head;
  const void* const* attn_norm;
  const void* const* w_q;
  const void* const* w_k;
  const void* const* w_v;
  const void* const* w_o;
  const void* const* mlp_norm;
  const void* const* w_gate;
  const void* const* w_up;
  const void* const* w_down;
} as2d_weights;

typedef struct as2d_model as2d_model;
typedef struct as2d_kv as2d_kv;

/* Outputs of one verification call.  rows = sum over requests of (k_b + 1),
   ordered request by request, each request's root row first.
   n_accepted, correction_token: device int32 [batch] (required).
   greedy: device int32 [rows], the greedy token after each row (nullable).
   logits: device float [rows][vocab], fp32 logits of every row (nullable;
   the paper's full-logits verification of App. B.2 stores [1, K, vocab]). */
typedef struct as2d_verify_out {
  int32_t* n_accepted;
  int32_t* correction_token;
  int32_t* greedy;
  float* logits;
} as2d_verify_out;

/* Load a model onto the current device.  Synchronises the device before it
   returns.  On success *out owns its device memory until as2d_model_free. */
as2d_status as2d_model_load(const as2d_config* cfg, const as2d_weights* w,
                            as2d_model** out);

/* Size this model's kernel grids for n_sms SMs (1 .. the device's count; the
   default is the device's count), so that the pass can share the GPU with
   other work confined to the remaining SMs -- for example a drafter on its
   own stream (as2d_session_run).  The projections' grids are of CTAs in
   groups of two, one CTA to an SM: an odd n_sms leaves one SM unused, 1 counts
   as 2, and the QKV projection, which has a CTA or more to each 128 of its
   rows, may start CTAs beyond n_sms that take the SMs in turn.  The other
   kernels are not sized.  The work split depends on (shape, n_sms)
   only: results stay batch invariant and bit-identical for a given budget;
   another budget adds partial sums in another order.  States created before
   a larger budget was set refuse to run (AS2D_ERR_INVALID_ARG): set the
   budget before as2d_kv_init_prefilled. */
as2d_status as2d_model_set_sm_budget(as2d_model* model, int32_t n_sms);

/* Bind a verification state of `batch` requests to a caller-allocated cache
   and its prefilled prefix (App. A.1: the retained audio KV plus the
   instruction, a valid prefix of the reference prompt).
   k_cache, v_cache: device bf16, layout [n_layers][batch][n_kv][capacity]
   [head_dim]; positions [0, kv_len[b]) of request b hold its prefilled keys
   (already rotated to their positions) and values.  The library writes the
   entries of forwarded rows; the caller keeps both buffers alive until
   as2d_kv_free.  kv_len, root_tokens: host int32 [batch]; root_tokens[b] is
   request b's pending known root (the first token chosen after prefill).
   capacity <= 65536 (AS2D_ERR_UNSUPPORTED above).  Allocates the state's
   device working memory.  Synchronises the device. */
as2d_status as2d_kv_init_prefilled(as2d_model* model, int32_t batch,
                                   const int32_t* kv_len, int32_t capacity,
                                   void* k_cache, void* v_cache,
                                   const int32_t* root_tokens, as2d_kv** out);

/* Verify one block per request (Section 3.2; App. C.2).
   candidates: device int32, packed: request b's k_b candidates start at
   index sum_{b' < b} k_{b'}.  k: host int32 [batch], 0 <= k_b <= AS2D_MAX_K.
   Request b forwards rows [root_b, c_1..c_{k_b}] at positions
   L_b .. L_b + k_b and afterwards holds L_b' = L_b + n_b + 1 and
   root_b' = correction_b, all on the device.  The host keeps only an upper
   bound of L_b (it grows by k_b + 1 per call); AS2D_ERR_CAPACITY is returned
   when that bound plus k_b + 1 would exceed the capacity (as2d_kv_read_state
   refreshes the bound).  Candidate ids outside [0, vocab) are a device-side
   error (as2d_kv_check).  Results are batch invariant: each row's logits are
   bitwise the same whatever the other rows of the call. */
as2d_status as2d_verify_block(as2d_kv* kv, const int32_t* candidates,
                              const int32_t* k, const as2d_verify_out* out,
                              void* stream);

/* Instruction-suffix prefill (App. A.1: processing the instruction with the
   retained, compatible audio KV gives the initial decoding state): forwards
   tokens[0..n) (device int32 [n], ids in [0, vocab)) at positions
   L .. L + n - 1 of a batch-1 state and keeps every entry, in passes of up
   to 256 rows through the verification pass (the first call allocates a
   working state for passes of 64, 128 or 256 rows, whichever holds its n, and
   a longer call a larger one, all kept until as2d_kv_free.  Under stream
   capture, or without the memory, a call uses the one there is, in more
   passes, or on first use makes one of 64 rows; that state is ready when the
   call returns, whether or not the captured graph ever runs.  Its attention
   buffers grow with the capacity, by about 3.7 MB per 1024 positions for the
   7B shape and 256 rows).  The LM head runs over the last row only.  The pending root
   before the call is discarded; afterwards L' = L + n and the root is the
   greedy token after tokens[n - 1] -- the first token of the response --
   also written to first_token (device int32 [1]) unless it is NULL.
   AS2D_ERR_UNSUPPORTED for batch > 1, AS2D_ERR_CAPACITY when the length
   bound plus n exceeds the capacity; bad token ids are device errors
   (as2d_kv_check): a pass that holds one keeps none of its rows, the other
   passes' rows are kept, the root is the greedy token after the last row kept
   (unchanged where there is none), and first_token is -1 if the last pass is
   the one.  Asynchronous on `stream`. */
as2d_status as2d_prefill(as2d_kv* kv, const int32_t* tokens, int32_t n,
                         int32_t* first_token, void* stream);

/* One greedy decode step for every request: as2d_verify_block with all
   k_b = 0 (App. C.2: with no ready candidate the target advances alone by one
   token). */
as2d_status as2d_decode_step(as2d_kv* kv, const as2d_verify_out* out,
                             void* stream);

/* Restore each request's state to an earlier committed prefix (App. C.4,
   requirement 2): length new_len[b] and pending root new_root[b] (host int32
   [batch]).  Entries [0, new_len[b]) must be ones this state holds; a
   new_len above the device-side length, or below the number of entries that the
   last as2d_kv_evict left, is a device error that leaves that request
   unchanged.  Asynchronous on `stream`. */
as2d_status as2d_kv_rollback(as2d_kv* kv, const int32_t* new_len,
                             const int32_t* new_root, void* stream);

/* Synchronise `stream`, copy the device-side lengths and roots into host
   int32 [batch] arrays (either may be NULL) and reset the host's length
   bounds to them. */
as2d_status as2d_kv_read_state(as2d_kv* kv, int32_t* len, int32_t* root,
                               void* stream);

/* Device pointers to the state's int32 [batch] lengths and roots, for
   consumers on the device (e.g. a drafter kernel that builds the next block
   without a host round trip).  Read-only for the caller. */
as2d_status as2d_kv_device_state(as2d_kv* kv, const int32_t** len,
                                 const int32_t** root);

/* Synchronise `stream` and return AS2D_ERR_DEVICE if any kernel of this
   state reported an error since the last check (then cleared), else
   AS2D_OK. */
as2d_status as2d_kv_check(as2d_kv* kv, void* stream);

/* Time limit, in nanoseconds, of the waits inside the kernels of this state's
   calls for a bulk copy, a tensor-core product or an accumulator (default
   2 s; this file's failure detection, not a paper mechanism).  A wait that
   runs out records AS2D_DEVERR_TIMEOUT, reported by as2d_kv_check, and its
   block of threads abandons that call's work: the call's outputs are then
   undefined, and the state should be restored with as2d_kv_rollback.  The
   waits by which a block drains its own outstanding copies and products
   before it ends keep the 2 s limit, so none is outstanding when it exits.
   A limit of 0 makes every wait that is not already satisfied give up at
   once, which exercises the failure path.  Takes effect for later calls. */
as2d_status as2d_kv_set_wait_limit(as2d_kv* kv, uint64_t ns);

/* One greedy decode step (k = 0) of a single request that allocates no
   memory.  The paper has no counterpart: this is for callers that must not
   allocate device memory when they decode -- for example a process whose
   device memory is handed out by another component under a fixed budget, or
   a real-time loop that cannot accept the latency or the possible failure of
   an allocation.  The model must have been loaded (as2d_model_load allocates,
   once, at set-up).  Every other byte a call needs lives in one array of
   9,735,424 bytes compiled into the library; each GPU that loads the library
   holds it until the process exits.
   k_cache, v_cache: device bf16 [n_layers][1][n_kv][capacity][head_dim] as
   for as2d_kv_init_prefilled.  len, root: device int32 [1], the request's
   state, updated in place (len += 1, root = correction) as by
   as2d_decode_step; *len must lie in [0, capacity - 1] when the step runs.
   correction_token: device int32 [1].  logits: device float [vocab] or NULL.
   error_bits: device int32 [1] or NULL; receives the step's AS2D_DEVERR_*
   bits (0 when it ran cleanly).
   Limits (AS2D_ERR_CAPACITY / AS2D_ERR_UNSUPPORTED on the host, before any
   work): capacity <= 4096, hidden <= 4096, ffn <= 20480, n_q * head_dim <=
   4096, n_kv <= 8, n_q / n_kv <= 16, vocab <= 262144, at most 192 SMs.
   The length lives on the device, so the host cannot check it: the kernels
   do.  A step whose *len is outside [0, capacity - 1], or whose root is
   outside [0, vocab), writes nothing to the cache, leaves len and root as
   they were, sets *correction_token to -1 and reports AS2D_DEVERR_CAPACITY
   (or AS2D_DEVERR_BAD_TOKEN) in error_bits.
   The first call on a device (and the first after a model of another shape)
   looks up the array's device address and builds descriptors of it; make
   that first call before any stream capture.  Calls from several host
   threads are enqueued one at a time, but all calls share the one array and
   each starts by clearing the parts that must start at zero, so calls that
   overlap on the GPU (other streams) race and give wrong results: issue
   them one after another on one stream, or synchronise between them.
   Device-side errors of this entry point are reported only through
   error_bits, not through as2d_kv_check. */
as2d_status as2d_decode_step_static(as2d_model* model, void* k_cache, void* v_cache,
                                    int32_t capacity, int32_t* len, int32_t* root,
                                    int32_t* correction_token, float* logits,
                                    int32_t* error_bits, void* stream);

/* Measurement support (not part of the verification step).  Kernel classes
   of one verification pass, in launch order per layer: */
#define AS2D_KERNEL_QKV 0        /* norm + QKV projection               */
#define AS2D_KERNEL_ATTENTION 1  /* RoPE + KV append + attention        */
#define AS2D_KERNEL_O 2          /* output projection + residual        */
#define AS2D_KERNEL_GATE_UP 3    /* norm + gate/up projection + SwiGLU   */
#define AS2D_KERNEL_DOWN 4       /* down projection + residual          */
#define AS2D_KERNEL_LM_HEAD 5    /* final norm + LM head + argmax       */
#define AS2D_KERNEL_OTHER 6      /* embedding gather, accept scan, ...  */
#define AS2D_KERNEL_CLASSES 7

/* Record a CUDA event pair on the call's stream around the launches of
   kernel class `kernel_class` (one pair per layer, or per call for the LM
   head) in later calls (-1 stops recording).  Also
   counts every kernel the library launches.  Events are created on demand. */
as2d_status as2d_kv_profile(as2d_kv* kv, int32_t kernel_class);

/* Synchronise the recorded events and return the number of recorded
   event pairs of the class, their summed device time in milliseconds, and the
   number of kernels the library launched since the last read; then reset. */
as2d_status as2d_kv_profile_read(as2d_kv* kv, int32_t* launches,
                                 double* total_ms, int64_t* all_launches);

void as2d_kv_free(as2d_kv* kv);
void as2d_model_free(as2d_model* model);

/* ---- Candidate buffer, read cursor and alignment -------------------------
   (Section 3.1 "Ordered publication and buffering"; Section 3.2 "Candidate
   alignment"; App. C.1 "Source records and incremental publication"; App. C.3
   "Candidate alignment"; Fig. 4.)  Host-side: one buffer per request and
   source.  The producer appends immutable batches of at most
   AS2D_CBUF_BATCH tokens; verification reads a snapshot of what is published
   from a read cursor that only alignment moves.  Alignment changes the
   cursor, never published tokens, committed tokens or the target's state, so
   the committed text is the target's greedy text whatever the buffer holds
   (Prop. 1).  Every entry point below is safe to call from several host
   threads at once (a producer thread publishing while the verifier reads):
   each one is atomic with respect to the others on the same buffer.

   Alignment, after a call that verified k candidates from cursor c,
   accepted n of them and ended with the target's token x (the correction,
   or the bonus token when n == k), with search bound W (the window):
     R1  x stands at buffer position m = c + n.  Once the buffer holds x at m
         (possible only after full acceptance; re-checked at each
         as2d_cbuf_candidates until m is published), the cursor steps over it
         to m + 1.
     R2  Otherwise m stays eligible: the next call verifies root x followed by
         the candidates from m (x may be a target insertion); if it accepts
         n >= 1, R1 applies to it.
     R3  If it accepts none, its token t is the first alignment anchor: the
         cursor moves to j + 1 for the first j in (m, m + W] holding t, else
         to j + 2 for the first j in [m, m + W] holding x, else the target
         decodes alone (k = 0).  While it does, its latest token is looked for
         before each call in the published positions [s, s + W) upwards, then
         [max(f, s - W), s) downwards, where f = m + 1 is where it began
         decoding alone and s starts at f and grows by one per token decoded
         alone; a match at j moves the cursor to j + 1. */
#define AS2D_CBUF_BATCH 8
#define AS2D_CBUF_NORMAL 0   /* candidates follow the cursor              */
#define AS2D_CBUF_REALIGN 1  /* R1/R2: waiting on the token at m          */
#define AS2D_CBUF_ALONE 2    /* R3: no usable candidates; k = 0           */

/* Source record of one published batch (App. C.1).  confidence is
   meaningful only when has_confidence != 0. */
typedef struct as2d_source_record {
  int32_t request, source, producer, offset;
  double time;
  float confidence;
  int32_t has_confidence;
} as2d_source_record;

typedef struct as2d_cbuf as2d_cbuf;

/* Create an empty buffer with search bound `window` in [1, 1024]. */
as2d_status as2d_cbuf_create(int32_t window, as2d_cbuf** out);

/* Append one batch: tokens host int32 [n], 1 <= n <= AS2D_CBUF_BATCH, every
   id >= 0; rec (host, required) is copied.  Published tokens never change. */
as2d_status as2d_cbuf_publish(as2d_cbuf* buf, const int32_t* tokens, int32_t n,
                              const as2d_source_record* rec);

/* The candidates for the next verification call: applies the checks that
   wait on publication (R1's step-over, R3's search while decoding alone),
   then copies up to b (0 <= b <= AS2D_MAX_K) published tokens from the cursor
   into host int32 tokens[b] and their number into *k (0 while the target
   decodes alone).  The next as2d_cbuf_after_call must report that k. */
as2d_status as2d_cbuf_candidates(as2d_cbuf* buf, int32_t b, int32_t* tokens,
                                 int32_t* k);

/* Report the call's outcome: the k of the last as2d_cbuf_candidates,
   n_accepted in [0, k] and the call's final token (correction or bonus,
   >= 0).  Moves the cursor by R1-R3. */
as2d_status as2d_cbuf_after_call(as2d_cbuf* buf, int32_t k, int32_t n_accepted,
                                 int32_t correction);

/* Published token count, cursor and mode (AS2D_CBUF_*); any may be NULL. */
as2d_status as2d_cbuf_state(as2d_cbuf* buf, int32_t* ready, int32_t* cursor,
                            int32_t* mode);

/* Tokens and batch records the buffer still holds (either may be NULL).
   Positions stay absolute, but tokens below both the cursor and the
   alignment position -- which no rule reads again -- are dropped once 4096
   of them have gathered, with the records of the batches wholly below them
   (App. C.1: exhausted records are discarded; the others keep their order
   and provenance), so a long session holds a bounded buffer. */
as2d_status as2d_cbuf_held(as2d_cbuf* buf, int32_t* tokens, int32_t* records);

/* Copy the source record of the batch that published `position`
   (AS2D_ERR_INVALID_ARG if the position is not published or was dropped). */
as2d_status as2d_cbuf_source_of(as2d_cbuf* buf, int32_t position,
                                as2d_source_record* out);

void as2d_cbuf_free(as2d_cbuf* buf);

/* One verification call driven by candidate buffers: bufs is a host array of
   kv's batch buffers (request r reads bufs[r]).  Takes up to b candidates
   from each buffer, copies them to the device, runs as2d_verify_block on
   `stream`, reads n_accepted and the correction back (this synchronises the
   stream) and reports them to each buffer.  Outputs (host, may be NULL):
   k_used int32 [batch]; committed int32 [batch][b + 1], row r holding the
   request's n_r + 1 committed tokens (accepted candidates, then the
   correction); n_committed int32 [batch] = n_r + 1.  The host's length
   bounds are tightened with the read-back n_r.  Device staging memory
   is allocated on the first call and kept until as2d_kv_free.  Errors of
   as2d_verify_block are returned as they are, before any buffer changes. */
as2d_status as2d_verify_from_buffers(as2d_kv* kv, as2d_cbuf* const* bufs, int32_t b,
                                     int32_t* k_used, int32_t* committed,
                                     int32_t* n_committed, void* stream);

/* ---- Producer / verifier sessions and their time accounting --------------
   (App. D.2 "Overlap, added work, and performance limits": the service
   intervals, D, V, O, H and the identity T = D + V - O + H;
   Section 3.1: the producer runs without target feedback and the target
   never waits for it.) */

/* A small decoder on the host cores: a producer placed on a different
   processor than the target, as the paper places drafter and target on
   different processors of one device.  fp32, one greedy decode step per
   call over its own cache (positions 0, 1, ...), matrix-vector products
   split over `threads` OpenMP threads.  w holds HOST float arrays in the
   layouts of as2d_weights (per-layer members: host arrays of host pointers);
   they are copied.  The shape rules of as2d_config do not apply (any
   positive sizes, n_q % n_kv == 0, even head_dim). */
typedef struct as2d_cpu_decoder as2d_cpu_decoder;
as2d_status as2d_cpu_decoder_create(const as2d_config* cfg, const as2d_weights* w,
                                    int32_t capacity, int32_t threads, int32_t root,
                                    as2d_cpu_decoder** out);
/* Forward the pending root at the next position, append its keys and values,
   make the greedy token the new root and return it in *token_out (may be
   NULL).  AS2D_ERR_CAPACITY when the cache is full. */
as2d_status as2d_cpu_decoder_step(as2d_cpu_decoder* d, int32_t* token_out);
/* The last step's logits: host float [vocab]. */
as2d_status as2d_cpu_decoder_logits(as2d_cpu_decoder* d, float* logits);
/* Back to an earlier length (<= the current one) with pending root `root`. */
as2d_status as2d_cpu_decoder_reset(as2d_cpu_decoder* d, int32_t len, int32_t root);
void as2d_cpu_decoder_free(as2d_cpu_decoder* d);

/* Service-interval accounting over [0, T].  p: host double [np][2] producer
   service intervals (start, end); v: host double [nv][2] verifier
   intervals; each is clipped to [0, T] and merged with the overlapping
   intervals of its own set.  out: host double [5] receives D = |P|, V = |V|,
   O = |P n V|, H = |[0, T] \ (P u V)| and T, so that T = D + V - O + H.
   AS2D_ERR_INVALID_ARG for an interval with end < start, T < 0 or counts
   < 0. */
as2d_status as2d_interval_accounting(const double* p, int32_t np, const double* v,
                                     int32_t nv, double T, double* out);

/* One request decoded to n_commit tokens by a producer publishing into a
   candidate buffer and a verifier drawing from it. */
typedef struct as2d_session_spec {
  as2d_kv* target;        /* batch-1 target state, advanced by the session          */
  as2d_kv* drafter;       /* batch-1 drafter state, one k = 0 decode step per
                             produced token on drafter_stream; NULL = no drafter
                             compute (tokens are published as fast as scripted)  */
  as2d_cbuf* buf;         /* the request's candidate buffer, written by the session */
  const int32_t* script;  /* host [n_script]: the token published by producer step i */
  int32_t n_script;
  int32_t b;              /* candidates per verification call, 0..AS2D_MAX_K       */
  int32_t publish_every;  /* producer steps per published batch, 1..AS2D_CBUF_BATCH */
  int32_t n_commit;       /* stop once at least this many tokens are committed     */
  int32_t overlapped;     /* 1: the producer runs on its own host thread and stream
                             alongside the verifier; 0: serial comparator -- the
                             producer runs (one batch) only while the verifier
                             waits, whenever fewer than b candidates are ready    */
  void* target_stream;
  void* drafter_stream;
  as2d_cpu_decoder* cpu_drafter;  /* when not NULL (and drafter is NULL): one
                                     host-core decode step per produced token */
} as2d_session_spec;

typedef struct as2d_session_stats {
  double T, D, V, O, H;   /* seconds: the accounting above over the session     */
  int32_t rounds;         /* verification calls (target-only rounds included)   */
  int32_t alone_rounds;   /* calls with k = 0                                    */
  int32_t committed;      /* tokens committed (accepted + one per call)          */
  int32_t accepted;       /* accepted candidates                                 */
  int32_t producer_steps; /* drafter steps run                                   */
  int32_t published;      /* tokens published                                    */
} as2d_session_stats;

/* Run a session.  Producer service intervals are the drafter steps with their
   publication; verifier intervals are the as2d_verify_from_buffers calls
   (verification, read-back, alignment).  Blocking; synchronises both
   streams, which should be distinct non-default streams for the two sides to
   overlap on the GPU.  The drafter's capacity must leave room for one
   position per scripted token.  committed: host int32 [n_commit + AS2D_MAX_K + 1] or NULL
   receives the committed tokens; stats (required) the accounting.  Errors of
   either side stop the session and are returned. */
as2d_status as2d_session_run(const as2d_session_spec* spec, int32_t* committed,
                             as2d_session_stats* stats);

/* ---- Offline budget selection -----------------------------------------------
   (Section 3.3 "Device-profiled configuration": device cost profiles and
   development traces choose one fixed proposal budget b; App. B, Eq. for
   R(K), the per-position cost reduction of width K; App. D.2 "Fixed
   configurations and development splits": budgets ranked by pooled
   throughput.) */

/* Estimate the pooled committed tokens per second of every budget b in
   0..b_max on development traces.  Each trace is replayed with the alignment
   rules above: the producer's whole text is published before the first call
   (in AS2D_CBUF_BATCH-token batches), each call takes up to b candidates,
   the target commits the trace's reference text (accepting the longest
   matching prefix, then one token) until n_commit tokens are committed, and
   each call of k candidates is charged cost_us[k].
   cost_us: host double [AS2D_MAX_K + 1], mean call time by k (> 0).
   refs, prods: host int32, the traces' reference and producer texts
   concatenated, with lengths ref_len, prod_len host int32 [n_traces];
   ref_len[t] >= n_commit + b_max + 1.  window: the alignment search bound.
   Outputs (host): tok_s double [b_max + 1]; calls int32 [b_max + 1] (may be
   NULL), the pooled call counts; *best_b, the budget with the highest
   estimate (the smallest such b on ties). */
as2d_status as2d_budget_select(const double* cost_us, const int32_t* refs,
                               const int32_t* ref_len, const int32_t* prods,
                               const int32_t* prod_len, int32_t n_traces,
                               int32_t n_commit, int32_t window, int32_t b_max,
                               double* tok_s, int32_t* calls, int32_t* best_b);

/* ---- Operators on caches and logits ------------------------------------------
   What a decoder around this library needs beside the chain of greedy
   candidates: attention of a tree of drafted tokens over a cache, the weight
   that attention gives each cache entry and eviction by it, probabilities at a
   temperature, and the acceptance of drafted tokens from given random numbers.
   They work on the caller's tensors; as2d_verify_tree, as2d_verify_sampled,
   as2d_kv_track_weights and as2d_kv_evict, further below, run them on a state.

   Each call is enqueued on `stream` without a host synchronisation and can be
   captured into a graph; nothing is kept from one call to the next.  Device
   addresses are multiples of their type's size, and of more where it is said;
   others are refused.  A
   workspace needs no initial contents, 256-byte alignment, and may serve any
   number of calls that run one after another: calls (or captured graphs) that
   may overlap on the GPU need one each. */

/* A caller's cache: device bf16 [n_layers][batch][n_kv][capacity][head_dim],
   16-byte aligned; head_dim 64 or 128, capacity <= 65536, batch <=
   AS2D_MAX_BATCH. */
typedef struct as2d_cache {
  void* k;
  void* v;
  int32_t n_layers, batch, n_kv, capacity, head_dim;
} as2d_cache;

#define AS2D_TYPE_BF16 0
#define AS2D_TYPE_F32 1
/* Most rows of one request in a call of as2d_tree_attention or
   as2d_attention_weights. */
#define AS2D_MAX_TREE 64

/* The query rows of a call.  Request b has rows[b] of them (0 .. AS2D_MAX_TREE),
   packed request by request; its cache holds kv_len[b] entries of the prefix
   and, right behind them, at [kv_len[b], kv_len[b] + rows[b]), the entries of
   these rows in row order.  Row i sees the whole prefix and those of its
   request's rows j whose bit j is set in visible[row] (itself only if bit i is;
   bits from rows[b] on are ignored): a tree of drafted tokens gives each row
   its ancestors and itself.  A row that sees nothing is allowed.
   q: device [sum rows][n_q][head_dim] of q_type, row r at element r q_stride
   (q_stride >= n_q head_dim); q and q_stride in bytes are multiples of 16.
   Query head h reads kv head h / (n_q / n_kv).  kv_len: device int32 [batch].
   max_len: host bound of the lengths, by which the launch is sized (0: the
   capacity); results do not depend on it beyond the order of sums.  rows: host
   int32 [batch].  visible: device uint64 [sum rows], or NULL for a chain (row i
   sees rows 0 .. i).  scale: the factor of q k (> 0, finite in 32 bits as a
   multiple of log2(e) too), usually 1 / sqrt(head_dim). */
typedef struct as2d_tree_rows {
  const void* q;
  int32_t q_type, n_q;
  int64_t q_stride;
  const int32_t* kv_len;
  int32_t max_len;
  const int32_t* rows;
  const uint64_t* visible;
  float scale;
} as2d_tree_rows;

/* Bytes of as2d_tree_attention's workspace on the current device, whatever the
   call. */
as2d_status as2d_tree_attention_workspace(const as2d_cache* cache, int64_t* bytes);

/* Softmax attention of the rows over one layer of a cache:
     out = sum_t p_t v_t,  p = softmax over the visible t of scale q k_t,
   and, unless lse is NULL, lse = ln sum_t e^(scale q k_t).  out: device [sum
   rows][n_q][head_dim] of q_type, 16-byte aligned; lse: device float [sum
   rows][n_q].  Scores, maxima and sums are held in 32 bits; 32-bit queries and the
   weights p enter the products as two bf16 parts, to 2^-17 of each (as the
   operands of this library's projections do).  A row that sees
   nothing gets out = 0 and lse = -inf.  What a row does not see does not reach
   its result, whatever it holds (NaN and infinities among it).  What it sees
   does as the formula has it: an infinite value makes its dim that infinity
   (values of both: NaN), a score of -inf is a weight of 0, and NaN or a score of +inf
   makes the row NaN in out and lse (scores are held as multiples of ln 2 too: beyond
   32 bits so, they are infinite).
   A request whose kv_len[b] is negative or leaves no room for its rows in the
   capacity is skipped: its rows of out and lse stay as they were and
   AS2D_DEVERR_CAPACITY is ORed into error_bits (device int32 [1], set to 0 by
   the caller beforehand, or NULL), as is AS2D_DEVERR_TIMEOUT where a bounded
   wait gave up (the outputs are then undefined).  out may not overlap q. */
as2d_status as2d_tree_attention(const as2d_cache* cache, int32_t layer,
                                const as2d_tree_rows* rows, void* out, float* lse,
                                void* workspace, int64_t workspace_bytes,
                                int32_t* error_bits, void* stream);

/* The weight that the rows' attention gives each entry of one layer's cache,
   added to what the entries have gathered: with lse as as2d_tree_attention
   leaves it, over the request's rows i and the query heads h of kv head g,
     weights[layer][b][g][t] += sum e^(scale q_ih k_t - lse_ih)   t < kv_len[b]
     weights[layer][b][g][t]  = the same sum       t in the rows' own entries
   (an entry starts with the weight its own call gives it).  What a row does
   not see adds 0.  weights: device float [n_layers][batch][n_kv][capacity];
   entries past the rows' own, and requests without rows, stay as they were.
   Requests are skipped and flagged as by as2d_tree_attention. */
as2d_status as2d_attention_weights(const as2d_cache* cache, int32_t layer,
                                   const as2d_tree_rows* rows, const float* lse,
                                   float* weights, int32_t* error_bits, void* stream);

/* Bytes of as2d_cache_evict's workspace. */
as2d_status as2d_cache_evict_workspace(const as2d_cache* cache, int64_t* bytes);

/* Evict entries by gathered weight, in place.  Of every (layer, request, kv
   head), each by itself, of a request with kv_len[b] > keep[b]: the latest
   min(recent, keep[b]) entries stay and, of the older ones, those of largest
   weight, keep[b] in all.  Equal weights: the lower position stays; -0 equals
   0, and NaN counts as less than every number.  The entries that stay keep
   their order and move, with their weights, to positions 0 .. keep[b] - 1;
   what lies behind stays as it was.  kv_len[b] becomes keep[b].  Other
   requests are left alone.  Keys keep the rotation of their old positions.
   weights: device float [n_layers][batch][n_kv][capacity]; kv_len: device int32
   [batch], in and out; keep: host int32 [batch], >= 0; recent >= 0.  A kv_len[b]
   outside [0, capacity] leaves that request alone. */
as2d_status as2d_cache_evict(const as2d_cache* cache, float* weights, int32_t* kv_len,
                             const int32_t* keep, int32_t recent, void* workspace,
                             int64_t workspace_bytes, void* stream);

/* Probabilities of rows of logits: probs = softmax(logits / temperature) over
   each row, sums in 32 bits or more.  logits, probs: device float [n_rows][vocab],
   4-byte aligned; probs may be logits.  temperature: finite, > 0.  Logits of -inf
   get 0; a row that holds nothing else gets all zeros; NaN or +inf in a row
   makes the row NaN.  vocab <= 2^24. */
as2d_status as2d_token_probs(const float* logits, int32_t n_rows, int32_t vocab,
                             float temperature, float* probs, void* stream);

/* Accept drafted tokens against the target's probabilities with given random
   numbers.  Request b drafted k[b] >= 0 candidates (packed in candidates, device
   int32 [sum k]) and owns k[b] + 1 rows of probs (device float [sum (k + 1)][vocab],
   row i the target's probabilities after the first i candidates) and of u
   (device float [sum (k + 1)], in [0, 1)).  draft_probs: device float [sum
   k][vocab], the drafter's probabilities that each candidate was drawn from, or
   NULL for candidates that the drafter gave with certainty.
     Candidate c at place i stands if u_i q_i(c) < p_i(c) (q_i(c) = 1 without
   draft_probs), exactly; n is the number of candidates before the first that
   does not.  The token after them is drawn, by u_k, from max(p_n - q_n, 0) if n <
   k (without draft_probs: p_n without candidate n) and from p_k otherwise: the
   lowest v at which the sum of the weights up to v exceeds u_k times their total
   (sums to some 48 bits where the total is 2^-100 or more; a total beyond 32-bit
   range gives token -1).  With u uniform the tokens follow the target's
   distribution.  Weights need not sum to 1; negative, infinite
   and NaN ones count as 0.  If max(p_n -
   q_n, 0) is 0 throughout the token is drawn from p_n; if that is too, token
   is -1.  A candidate outside [0, vocab) does not stand and takes nothing from
   p_n (with draft_probs its row is used as it is).
   k: host int32 [batch], 1 <= batch <= AS2D_MAX_BATCH, each <= AS2D_MAX_K;
   vocab <= 2^24; candidates may be NULL if all are 0.  n_accepted, token: device int32 [batch]. */
as2d_status as2d_accept_sampled(const float* probs, const float* draft_probs,
                                const int32_t* candidates, const int32_t* k, int32_t batch,
                                int32_t vocab, const float* u, int32_t* n_accepted,
                                int32_t* token, void* stream);

/* ---- Between a projection and its attention ------------------------------------
   The rows of a projection normed, rotated and appended to a cache; a cache held in
   4 bits, written as rows are appended or from a cache in bf16, read back, and
   attended to; attention of whole prompts.  As the operators above in all that
   concerns streams, captures, workspaces and addresses. */

/* A caller's cache in 4 bits, sizes as of as2d_cache.  k, v: device bytes
   [n_layers][batch][n_kv][capacity][head_dim / 2], 16-byte aligned; k_scale, v_scale:
   device bytes [n_layers][batch][n_kv][capacity][head_dim / 16], 8-byte aligned.
     Each 16 consecutive dims of an entry share a scale s and stand for s (c - 8),
   c their codes 0 .. 15.  A scale byte x has the 16-bit float x 2^7 as bits (five bits
   of exponent, three of fraction), at most 896: greater ones, whatever their bits,
   count as that.  Of 8 consecutive dims in a 32-bit little-endian word, dim 2e has
   bits 4e .. 4e + 3 and dim 2e + 1 bits 4e + 16 .. 4e + 19.  So every value that a
   cache can hold is finite and exact in bf16 and in 16-bit floats.
     What writes: s is the nearest scale to a seventh of the largest magnitude of
   the 16, ties to the even byte; c - 8 is the whole number nearest to x / s within
   -7 .. 7, ties to the even one, and 0 where s is 0; both as in exact arithmetic.  A
   value is off by at most s / 2, where s is neither capped nor below 2^-14.  NaN is written
   as 0 and an infinity as the largest magnitude of its sign that the 16 can have
   (s = 896; one that a norm or a rotation meets may count as NaN). */
typedef struct as2d_cache4 {
  uint8_t *k, *k_scale, *v, *v_scale;
  int32_t n_layers, batch, n_kv, capacity, head_dim;
} as2d_cache4;

/* Rows of a projection.  Request b has rows[b] >= 0 of them, packed request by
   request, which become the entries [kv_len[b], kv_len[b] + rows[b]) of its cache.
   q: device [sum rows][n_q][head_dim] of `type`, k and v: [sum rows][n_kv][head_dim];
   row r at element r q_stride (k_stride, v_stride), so that they may be parts of
   one tensor; addresses and strides in bytes are multiples of 16.
   q_norm, k_norm: device float [head_dim] or NULL: each head of a row is divided by
   its root mean square (mean of squares + eps; eps >= 0) and multiplied by these gains.
   rotary: dims 0 .. rotary - 1 of each head of q and k are rotated by position, dim j
   with dim j + rotary / 2 by the angle position theta^(-2j / rotary); a multiple of 32
   of at most head_dim, 0 for none.  theta > 0.  positions: device int32 [sum
   rows], or NULL: kv_len[b] + i for row i.  rows: host int32 [batch]; kv_len: device
   int32 [batch]. */
typedef struct as2d_new_rows {
  const void *q, *k, *v;
  int32_t type, n_q;
  int64_t q_stride, k_stride, v_stride;
  const int32_t* kv_len;
  const int32_t* rows;
  const int32_t* positions;
  const float *q_norm, *k_norm;
  float eps, theta;
  int32_t rotary;
} as2d_new_rows;

/* Finish rows and append them to one layer of a cache: q_out (device [sum
   rows][n_q][head_dim] of `type`, 16-byte aligned) gets the queries, normed and
   rotated, the cache the keys, normed and rotated, and the values as they are.
   Computed in 32 bits (of a head that is normed, the squares too: beyond their range it
   is not what the formula says), angles exactly reduced for every position, and rounded
   once.
   kv_len stays as it is.  A request whose kv_len[b] is negative or leaves no room
   for its rows in the capacity is skipped: its cache and its rows of q_out stay as they
   were and AS2D_DEVERR_CAPACITY is ORed into error_bits (device int32 [1] or
   NULL).  q_out may not overlap q, k or v.  At most 2^24 rows. */
as2d_status as2d_cache_append(const as2d_cache* cache, int32_t layer, const as2d_new_rows* rows,
                              void* q_out, int32_t* error_bits, void* stream);

/* The same into a cache in 4 bits: keys are rounded once, from their exact value.
   AS2D_DEVERR_NOT_FINITE is ORed into error_bits where a key or value is NaN or
   infinite. */
as2d_status as2d_cache4_append(const as2d_cache4* cache, int32_t layer, const as2d_new_rows* rows,
                               void* q_out, int32_t* error_bits, void* stream);

/* Write entries [start[b], end[b]) of each request of a cache in bf16 into the
   same places of one in 4 bits (as2d_cache4_write; flags AS2D_DEVERR_NOT_FINITE), or back
   (as2d_cache4_read, exactly).  The caches have the same sizes but for the
   capacities.  layer: one, or -1 for all.  start (NULL: 0), end: device int32
   [batch].  A request with start[b] >= end[b] has nothing to do; one with start[b] < 0 or
   end[b] past either capacity is skipped and flagged AS2D_DEVERR_CAPACITY.
   max_entries: host bound of end[b] - start[b], by which the launch is sized (0: the
   smaller capacity); results do not depend on it.  error_bits: device int32 [1] or
   NULL. */
as2d_status as2d_cache4_write(const as2d_cache4* to, const as2d_cache* from, int32_t layer,
                              const int32_t* start, const int32_t* end, int32_t max_entries,
                              int32_t* error_bits, void* stream);
as2d_status as2d_cache4_read(const as2d_cache4* from, const as2d_cache* to, int32_t layer,
                             const int32_t* start, const int32_t* end, int32_t max_entries,
                             int32_t* error_bits, void* stream);

/* Bytes of as2d_cache4_attention's workspace on the current device, whatever the
   call. */
as2d_status as2d_cache4_attention_workspace(const as2d_cache4* cache, int64_t* bytes);

/* as2d_tree_attention over a cache in 4 bits, which holds the entries of the rows
   too.  Queries enter the products in 16-bit floats with a power of two of their own,
   32-bit ones as two parts (to 2^-22 of a query's largest dim, or nearer), and so do the
   weights p (to 2^-11 for bf16 queries, 2^-22 for 32-bit ones).  What a row does not
   see does not reach its result.  A query that is not finite, or a score of +inf, makes its
   row NaN in out and lse.  What another max_len or other rows change is the order of sums
   and what the weights are relative to before they are rounded. */
as2d_status as2d_cache4_attention(const as2d_cache4* cache, int32_t layer,
                                  const as2d_tree_rows* rows, void* out, float* lse,
                                  void* workspace, int64_t workspace_bytes,
                                  int32_t* error_bits, void* stream);

/* Bytes of as2d_prompt_attention's workspace on the current device, whatever the
   call. */
as2d_status as2d_prompt_attention_workspace(const as2d_cache* cache, int64_t* bytes);

/* Causal attention of whole prompts over one layer of a cache: as as2d_tree_attention
   with rows[b] up to the capacity, row i of request b seeing the entries 0 ..
   kv_len[b] + i; visible is NULL, out 32-byte aligned.  bf16 queries (others: AS2D_ERR_UNSUPPORTED); the
   weights p enter the products in bf16 (relative to what max_len and the other rows of the
   call may change), their sum in 32 bits.  What a row does not see does
   not reach its result, whatever it holds; a value that it sees and that is not
   finite makes its dim not finite, and NaN or +inf among its scores the row NaN in out
   and lse.  At most 2^24 rows. */
as2d_status as2d_prompt_attention(const as2d_cache* cache, int32_t layer,
                                  const as2d_tree_rows* rows, void* out, float* lse,
                                  void* workspace, int64_t workspace_bytes,
                                  int32_t* error_bits, void* stream);

/* ---- The same on a verification state ------------------------------------------ */

/* Verify a tree of candidates per request in one pass: as as2d_verify_block, but
   parents (device int32, packed as candidates) gives each candidate the row it
   follows, 0 for the root and j for the request's candidate j (1 .. k_b), which
   must be an earlier one.  A candidate stands at position L_b + its depth and
   sees the prefix, its ancestors and itself.  From the root down, the candidate
   that follows the last one accepted and equals the greedy token there is
   accepted (the first, if several do); the greedy token after the last one
   is the correction.  Afterwards the cache holds the root's and the accepted
   candidates' entries at L_b .. L_b + n_b, as if they had been a chain.
   out: as for as2d_verify_block, n_accepted the accepted path's length, greedy
   and logits by row.  path: device int32 [batch][AS2D_MAX_K] or NULL: the
   accepted candidates' numbers in order, then -1.  A parent that is no earlier
   row is a device error (as2d_kv_check) that leaves that request unchanged with
   n_accepted = correction = -1, its path -1.  A row's logits depend on the other rows and
   requests of the call by the order of 32-bit sums only.  The first call
   allocates working memory, kept until as2d_kv_free. */
as2d_status as2d_verify_tree(as2d_kv* kv, const int32_t* candidates,
                             const int32_t* parents, const int32_t* k,
                             const as2d_verify_out* out, int32_t* path, void* stream);

/* as2d_verify_block with sampling in the place of the greedy rule: the rows'
   logits become probabilities at `temperature` (as2d_token_probs) and the
   candidates are accepted and the correction drawn by as2d_accept_sampled from
   them, draft_probs (device float [sum k][vocab] or NULL) and u (device float
   [sum (k + 1)] in [0, 1)).  probs: device float [rows][vocab], receives the
   probabilities.  out: as for as2d_verify_block, with logits NULL; greedy still
   holds each row's greedy token.  A row that gives no token is a device error
   that leaves that request unchanged with n_accepted = correction = -1. */
as2d_status as2d_verify_sampled(as2d_kv* kv, const int32_t* candidates, const int32_t* k,
                                const float* draft_probs, const float* u, float temperature,
                                const as2d_verify_out* out, float* probs, void* stream);

/* From now on every verification call of this state (as2d_verify_block,
   as2d_decode_step, as2d_verify_tree, as2d_verify_sampled and what calls them)
   adds the weight that its rows' attention gives each entry to `weights`
   (device float [n_layers][batch][n_kv][capacity], the caller's, who fills in
   what the entries of the prefix start with and keeps it alive), as
   as2d_attention_weights does, over all rows of the call whether accepted or
   not; NULL ends it.  A request that the call drops adds nothing, but for one
   whose rows give no token (AS2D_DEVERR_NO_TOKEN), which is known at the call's end
   only.  The weights of accepted entries move with them.  These calls take the
   attention of as2d_verify_tree, so that their logits differ from those of
   other calls by the order of 32-bit sums.  as2d_prefill is refused meanwhile
   (AS2D_ERR_UNSUPPORTED).  Allocates device memory on first use. */
as2d_status as2d_kv_track_weights(as2d_kv* kv, float* weights);

/* Cut every layer and kv head of each request b to the keep[b] entries
   (host int32 [batch], >= 0) that as2d_cache_evict chooses by the tracked weights,
   the latest `recent` among them; requests that hold no more are left alone.  The
   length becomes keep[b]; the pending root stays, and later rows take their
   positions as if nothing had been evicted.  Needs tracked weights
   (AS2D_ERR_INVALID_ARG).  Under stream capture the host's bound of the lengths
   stays as it was (as2d_kv_read_state reads them).  as2d_kv_rollback cannot go below keep[b] afterwards.
   Asynchronous on `stream`. */
as2d_status as2d_kv_evict(as2d_kv* kv, const int32_t* keep, int32_t recent, void* stream);

/* Thread-local description of the last error ("" if none). */
const char* as2d_last_error(void);

#ifdef __cplusplus
}
#endif
#endif
