/*
 * gs.h -- C ABI of libgs: greedy self-speculative draft/verify decoding with a
 * shared-parameter AR / block-diffusion decoder on one GB300 (sm_103a).
 *
 * The method (paper Sec. 4.3 "Self-Speculative Decoding", Fig. "Self-speculative
 * decoding", Appendix "Self-Speculative Decoding and KV-Cache Update"): every
 * round runs one DRAFT forward over [x0, [M] x K] with the hybrid mask (the
 * boundary row x0 causal to the cache, the K mask rows bidirectional inside
 * the window), then one VERIFY forward over [a0, d_1..d_K] with token-level
 * causal attention, accepts the longest prefix with d_j == a_j, commits
 * a0, d_1..d_A, a_{A+1} and rolls the KV cache back to the accepted prefix.
 * The first boundary x0 is the argmax at the prefill's last position.
 *
 * Conventions shared by every entry point
 *  - Device pointers are CUDA global-memory addresses on the current device;
 *    host pointers are ordinary process memory.  Each argument says which.
 *  - The caller owns every buffer it passes (weights, workspace, inputs,
 *    outputs) and the stream.  After gs_create the library allocates no
 *    device memory; it carves everything from the caller's workspace.
 *  - Work is enqueued asynchronously on the handle's stream unless stated.
 *  - bf16 tensors are bfloat16 bit patterns, fp16 tensors IEEE binary16
 *    bit patterns; all row-major.
 *  - Arithmetic: the model's weights arrive as bf16; gs_create re-encodes each
 *    matrix as an fp16 copy scaled by a power of two (exact for every weight
 *    whose magnitude is above 2^-31 of the tensor's largest).  Activations
 *    between kernels and the KV cache are fp16 (11 significant bits, against
 *    8 for bf16); every contraction accumulates in fp32; the residual stream
 *    and the softmax statistics are fp32.  A kernel that would store a value
 *    beyond the fp16 range raises the device error word (GS_ERR_DEVICE_CHECK).
 *  - Return value: GS_OK (0) or one of the GS_ERR_* codes below; the message
 *    of the last failure is available from gs_last_error().  Kernel-side
 *    checks (slot ids, token ids, bounded waits) raise a device error word
 *    that gs_sync_check() turns into GS_ERR_DEVICE_CHECK / GS_ERR_TIMEOUT.
 */
#ifndef GS_H_
#define GS_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  GS_OK = 0,
  GS_ERR_INVALID_ARG = 1,   /* bad pointer, size, slot or config value        */
  GS_ERR_OOM = 2,           /* workspace too small / KV page pool exhausted    */
  GS_ERR_UNSUPPORTED = 3,   /* valid request the library does not implement   */
  GS_ERR_CUDA = 4,          /* a CUDA runtime call failed                      */
  GS_ERR_DEVICE_CHECK = 5,  /* a kernel's bounds check fired                   */
  GS_ERR_TIMEOUT = 6        /* a kernel's bounded wait ran out                 */
};

/* Acceptance rule (paper Sec. 3 "Speculative Decoding"): greedy accepts drafts
 * while they equal the verifier's argmax; stochastic is the standard
 * acceptance-rejection rule of speculative sampling, which preserves the
 * target distribution (named by the paper, not used in its experiments):
 * a0 and the drafts are sampled at the handle's temperature (gs_set_sampling)
 * from the draft rows, d_j is accepted while r_j < P_j(d_j) / q_j(d_j), the
 * first rejected position takes a sample of max(0, P_j - q_j), a fully
 * accepted draft a bonus sample of P_{K+1}. */
typedef enum { GS_ACCEPT_GREEDY = 0, GS_ACCEPT_STOCHASTIC = 1 } gs_accept_rule;

/* Decoder shape and capacity.  The paper does not print the architecture; the
 * library implements a pre-norm decoder: RMSNorm (learned gain, eps) ->
 * grouped-query attention with rotate-half RoPE on all head dims at absolute
 * positions -> RMSNorm -> SwiGLU FFN; untied input/output embeddings, no
 * biases.  Requirements: head_dim 64, n_heads % n_kv_heads == 0, n_heads and
 * n_kv_heads even (a 128-row projection tile holds two whole heads),
 * d_model % 128 == 0, d_ffn % 64 == 0, vocab % 128 == 0. */
typedef struct {
  int n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ffn, vocab;
  float rope_theta, rms_eps;
  int mask_token_id;   /* the [M] embedding row (paper Sec. 4, "AR-to-Diffusion Conversion") */
  int eos_token_id;    /* stop token, -1 = none (Appendix step "Next round")              */
  int max_batch;       /* sequence slots                                                  */
  int max_ctx;         /* slots one sequence may reserve: prefix + max_new + max_K + 2   */
  int max_K;           /* largest block size a round may use                              */
  int max_prefill;     /* tokens per prefill chunk (longer prefixes run in chunks)        */
  int kv_pages;        /* 64-token pages in the KV pool; 0 = max_batch * ceil(max_ctx/64) */
  int split_pages;     /* attention pages per work item (decode); 0 = automatic           */
} gs_config;

/* Weights: device pointers to bf16 arrays owned by the caller, row-major
 * [out_features, in_features].  Per-layer fields are HOST arrays of n_layers
 * device pointers (copied by gs_create).
 *   embed [vocab, d]   lm_head [vocab, d]   final_norm [d]
 *   attn_norm [d]   w_qkv [(Hq + 2 Hkv) * 64, d]  (q heads, then k heads, then v heads)
 *   w_o [d, Hq * 64]   ffn_norm [d]   w_gate_up [2 d_ffn, d] (gate rows, then up rows)
 *   w_down [d, d_ffn]
 * Every pointer must be 16-byte aligned. */
typedef struct {
  const void *embed, *lm_head, *final_norm;
  const void *const *attn_norm, *const *w_qkv, *const *w_o,
             *const *ffn_norm, *const *w_gate_up, *const *w_down;
} gs_weights;

/* Forced acceptance (benchmark hook, not in the paper).  After the draft
 * argmax, for the sequence in slot s at round r with L = L_sched[row * L_stride + r]
 * (row = the sequence's index in this call's slot list, r = the number of
 * rounds the sequence has run since its prefill):
 *   d_j := teacher[row * teacher_stride + n + 1 + j]    for 1 <= j <= L
 *   d_{L+1} := (teacher[row * teacher_stride + n + 2 + L] + 1) mod vocab  if L < K
 * where n is the sequence's cached length at the round's start and teacher[p]
 * is the greedy token at absolute slot p.  All pointers are device int32. */
typedef struct {
  const int32_t *teacher;
  int64_t teacher_stride;
  const int32_t *L_sched;
  int64_t L_stride;
} gs_force;

/* Optional per-round diagnostics (device pointers, any may be NULL).  A round
 * given a non-NULL gs_debug runs outside the CUDA-graph cache.
 *   draft_tok  int32 [n_seq, K+1]   argmax of the draft rows (a0, d_1..d_K)
 *   verify_in  int32 [n_seq, K+1]   verify inputs after forcing (a0, d_1..d_K)
 *   verify_tok int32 [n_seq, K+1]   argmax of the verify rows (a_1..a_{K+1})
 *   draft_logits / verify_logits fp32 [n_seq, K+1, vocab] */
typedef struct {
  int32_t *draft_tok, *verify_in, *verify_tok;
  float *draft_logits, *verify_logits;
} gs_debug;

typedef struct gs_handle gs_handle;

/* Bytes of device workspace gs_create needs for this config (fp16 weight
 * copies, KV page pool, page table, per-sequence state, activations, split
 * scratch).  0 if the config is invalid. */
size_t gs_workspace_bytes(const gs_config *cfg);

/* Build a handle.  cfg, w: host structs (copied).  workspace: device memory of
 * at least gs_workspace_bytes(cfg) bytes, 256-byte aligned, owned by the
 * caller and not touched by anyone else until gs_destroy.  stream: a
 * cudaStream_t (NULL = legacy default stream).  Zeroes the workspace, writes
 * the scaled fp16 copies of the weight matrices into it (the caller's bf16
 * matrices are not read again; embed and the norm gains are read at every
 * forward) and builds the TMA descriptors; synchronises the stream before
 * returning.
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED (shape), GS_ERR_OOM
 * (workspace too small), GS_ERR_CUDA. */
int gs_create(const gs_config *cfg, const gs_weights *w, void *workspace, size_t ws_bytes,
              void *stream, gs_handle **out);

/* Release the handle (graphs, host tables).  Frees no caller memory. */
int gs_destroy(gs_handle *h);

/* Message of the last failure on this handle ("" if none).  NULL handle gives
 * the last failure of gs_create in this thread. */
const char *gs_last_error(gs_handle *h);

/* Prefill (paper Appendix step "State"; Sec. 3 task formulation: image I and
 * prompt c).  Reserves KV pages for n_vis + n_text + max_new + max_K + 2
 * slots in sequence slot `slot` (freeing whatever the slot held), runs a
 * causal forward over the visual rows then the text tokens, sets the cached
 * length to P = n_vis + n_text and the boundary x0 to the argmax at position
 * P-1, which is the first committed output token.
 *   vis_emb  device bf16 [n_vis, d_model] (may be NULL when n_vis == 0)
 *   text     device int32 [n_text], ids in [0, vocab)
 *   max_new  cap on committed output tokens, x0 included (>= 1)
 *   x0_out   device int32 [1] or NULL
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_OOM (pool exhausted or ctx too long). */
int gs_prefill(gs_handle *h, int slot, const void *vis_emb, int n_vis, const int32_t *text,
               int n_text, int max_new, int32_t *x0_out);

/* One self-speculative round for n_seq sequences (paper Appendix steps Draft
 * forward / Verify forward / Accept / Cache update / Next round).
 *   slots    device int32 [n_seq], distinct prefilled slots
 *   K        block size, 0 <= K <= max_K (K = 0 is two plain AR steps)
 *   rule     GS_ACCEPT_GREEDY, or GS_ACCEPT_STOCHASTIC (sampling at the
 *            handle's temperature and seed, see gs_set_sampling)
 *   force    NULL for natural drafting, else the forcing hook above (greedy only)
 *   out_tok  device int32 [n_seq, K+2]: committed tokens of this round
 *   out_cnt  device int32 [n_seq]: how many (0 for a sequence already done)
 *   out_done device int32 [n_seq]: 1 once the sequence hit EOS or max_new
 *   dbg      NULL, or diagnostics (see gs_debug)
 * Rounds with the same (n_seq, K, pointers) replay one cached CUDA graph; no
 * host synchronisation happens inside or between rounds. */
int gs_round(gs_handle *h, const int32_t *slots, int n_seq, int K, int rule, const gs_force *force,
             int32_t *out_tok, int32_t *out_cnt, int32_t *out_done, const gs_debug *dbg);

/* Sampling parameters of GS_ACCEPT_STOCHASTIC rounds (host values, kept by
 * the handle).  temperature > 0: tokens are sampled from softmax(logits / T).
 * seed: the 64-bit key of Philox4x32-10 (Salmon et al., SC 2011), whose
 * counter is (vocabulary entry / 4, window row, round of the sequence,
 * stream << 24 | slot); word (entry % 4) x gives the uniform
 * (2 * (x >> 9) + 1) * 2^-24 and token samples are Gumbel-max
 * (argmax of log-weight - log(-log u)).  Streams: 0 draft samples (a0, d_j),
 * 2 acceptance uniforms (row j, entry 0), 3 the replacement or bonus sample
 * (row j of the rejected position, K+1 for the bonus).  A round's draws thus
 * depend on the seed, the slot and the sequence's round count only.
 * Defaults: T = 1, seed = 0.  Errors: GS_ERR_INVALID_ARG. */
int gs_set_sampling(gs_handle *h, float temperature, uint64_t seed);

/* Direct block-diffusion decoding of one block per sequence (paper Appendix
 * "Direct Block-Diffusion Decoding"; Sec. 5 diffusion-vs-self-speculative
 * comparison).  From the same state as gs_round (the cache holds every
 * committed token but the boundary x0), a block of B [M] tokens at slots
 * n+1..n+B is denoised: each step is one forward over [x0, block] with the
 * draft's hybrid mask (x0 causal, block rows bidirectional in the window),
 * the prediction for position p read from the row at p-1; every still-masked
 * position whose argmax probability exceeds tau_c is revealed, or, if none
 * is, the single most confident one (ties to the lowest position); revealed
 * tokens stay fixed.  When every sequence's block is complete, one causal
 * forward over [x0, y_1..y_B] writes the cache (no LM head), and the block is
 * committed: y_1..y_B cut at the first EOS or at max_new, seq_len += B,
 * x0 = y_B.  All steps run inside one CUDA graph whose denoising loop is a
 * conditional (while) node: no host synchronisation; the loop is capped at B
 * steps (a sequence still open after B steps raises the device check).
 *   slots     device int32 [n_seq], distinct prefilled slots
 *   B         block size, 1 <= B <= max_K
 *   tau_c     confidence threshold (probabilities are in (0, 1]; tau_c >= 1
 *             reveals one position per step, tau_c < 0 the whole block at once)
 *   out_tok   device int32 [n_seq, B]: committed tokens of the block
 *   out_cnt   device int32 [n_seq]: how many (0 for a sequence already done)
 *   out_done  device int32 [n_seq]: 1 once the sequence hit EOS or max_new
 *   out_steps device int32 [n_seq] or NULL: denoising forwards of the block
 *             (the paper's TPF for this mode counts these, not the cache write)
 * Needs a handle created on a non-default stream.  Graphs are cached per
 * (n_seq, B, tau_c, pointers).  Errors: GS_ERR_INVALID_ARG, GS_ERR_CUDA. */
int gs_diffusion_block(gs_handle *h, const int32_t *slots, int n_seq, int B, float tau_c,
                       int32_t *out_tok, int32_t *out_cnt, int32_t *out_done, int32_t *out_steps);

/* A self-speculative round with multi-step drafting (paper Sec. 6 "Draft
 * Schedule", Fig. "Multi-step drafting versus one-shot drafting").  The draft
 * window [x0, [M] x K] is run repeatedly: prediction i (a0 for i = 0, d_i
 * otherwise, read from row i) is fixed once its argmax probability exceeds
 * tau_d, or, when no open prediction does, the single most confident one is;
 * a fixed prediction i < K is fed back at its own slot n+1+i in place of the
 * mask; after at most K+1 draft forwards the finished draft is verified,
 * accepted and committed exactly as by gs_round (GS_ACCEPT_GREEDY; the
 * forcing hook applies to the refined draft).  tau_d < 0 is the one-shot
 * round.  One graph launch with a conditional loop, no host synchronisation.
 *   out_tok [n_seq, K+2], out_cnt, out_done: as gs_round
 *   out_steps device int32 [n_seq] or NULL: draft forwards of the round
 * Needs a non-default stream.  Errors: GS_ERR_INVALID_ARG, GS_ERR_CUDA. */
int gs_round_refined(gs_handle *h, const int32_t *slots, int n_seq, int K, float tau_d,
                     const gs_force *force, int32_t *out_tok, int32_t *out_cnt, int32_t *out_done,
                     int32_t *out_steps);

/* Overwrite a sequence's per-slot state (resume/checkpoint: with the KV pages,
 * which keep their contents, the state is the cached length, the boundary
 * token, the output count and cap, the done flag and the round counter that
 * indexes a forcing schedule).  Rolling the cached length back to a value the
 * cache held before (e.g. the prefix length after a prefill) replays a decode.
 *   seq_len   1 <= seq_len and seq_len + max_K + 2 <= the slot's reservation
 *   x0        boundary token in [0, vocab); n_out >= 1 committed tokens (x0 included)
 *   max_new   output cap (>= n_out); done 0/1; rounds >= 0
 * Host values; enqueued on the stream.  Errors: GS_ERR_INVALID_ARG. */
int gs_seq_restore(gs_handle *h, int slot, int seq_len, int x0, int n_out, int max_new, int done,
                   int rounds);

/* Read one slot's state (synchronises the stream).  Any out pointer may be NULL. */
int gs_seq_state(gs_handle *h, int slot, int *seq_len, int *x0, int *n_out, int *done, int *rounds);

/* Number of kernel launches the most recent gs_round enqueued (or captured). */
int gs_round_launches(gs_handle *h);

/* Kinds of kernel reported by gs_round_profile (one per launch). */
enum {
  GS_KIND_WINDOW = 0,    /* draft window build or verify input build (Sec. 3.2) */
  GS_KIND_EMBED = 1,     /* token embedding + first RMSNorm input */
  GS_KIND_QKV = 2,       /* QKV projection + RoPE + KV-cache write */
  GS_KIND_ATTENTION = 3, /* hybrid-mask paged attention (Eq. 3 / Eq. 5 masks) */
  GS_KIND_O_PROJ = 4,    /* output projection + residual */
  GS_KIND_GATE_UP = 5,   /* gate/up projection + SwiGLU */
  GS_KIND_DOWN = 6,      /* down projection + residual */
  GS_KIND_LM_HEAD = 7,   /* LM head + greedy argmax */
  GS_KIND_ACCEPT = 8     /* longest-prefix acceptance and commit (Sec. 3.3) */
};

/* Measurement aid: one greedy round, with the same arguments and effects as
 * gs_round(h, slots, n_seq, K, GS_ACCEPT_GREEDY, force, out_tok, out_cnt,
 * out_done, NULL), captured (never from the graph cache) with a CUDA event
 * recorded after every kernel launch and replayed as one graph, so the host's
 * enqueue time never falls between two launches.  The paper has no
 * counterpart.
 *   ms[i]       device milliseconds between launch i-1's end event and launch
 *               i's end event (for i = 0, from an event recorded before the
 *               round).  An event between two kernels stops the second from
 *               starting early, so each figure is the kernel alone, from the
 *               front end starting it to its last CTA.
 *   kind[i]     GS_KIND_* of launch i.
 *   n_launches  number of launches written.
 * ms and kind are host arrays of max_launches entries.  Synchronises the
 * handle's stream (which must not be the default stream).
 * Errors: GS_ERR_INVALID_ARG (bad arguments, max_launches too small — the
 * round has then run), GS_ERR_CUDA. */
int gs_round_profile(gs_handle *h, const int32_t *slots, int n_seq, int K, const gs_force *force,
                     int32_t *out_tok, int32_t *out_cnt, int32_t *out_done, int max_launches,
                     float *ms, int *kind, int *n_launches);

/* Free the slot's KV pages (host bookkeeping only). */
int gs_release(gs_handle *h, int slot);

/* Synchronise the stream and report a kernel-side check or bounded-wait
 * failure raised since the last call (then clear it). */
int gs_sync_check(gs_handle *h);

/* Failure-detection self-test (the paper has no counterpart).  Enqueues on
 * the handle's stream one kernel that waits, through the same bounded
 * mbarrier wait every pipeline of the library uses, on a barrier nothing
 * arrives on; the wait gives up after limit_us microseconds of device time
 * (1 <= limit_us <= 2,000,000) and raises the timeout code in the handle's
 * error word, so the next gs_sync_check returns GS_ERR_TIMEOUT.  The context
 * stays usable: nothing else is in flight in the probe's CTA.
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_CUDA. */
int gs_wait_probe(gs_handle *h, int limit_us);

/* ---------------------------------------------------------------------------
 * Sub-steps exposed for the attention-only sweep and kernel parity tests.
 * ------------------------------------------------------------------------ */

/* Hybrid-mask attention over a paged fp16 KV cache (paper Appendix steps
 * Draft forward / Verify forward; mask semantics Sec. 4.2).  Standalone form
 * of the kernel the rounds use.
 *   mode 0 DRAFT:  query row i of sequence s sits at slot n_s + i;
 *                  row 0 sees keys 0..n_s, rows i >= 1 see keys 0..n_s + W - 1
 *   mode 1 VERIFY: query row i sits at slot n_s + 1 + i and sees keys 0..n_s + 1 + i
 *   q        device fp16 [n_seq, W, n_heads, 64] (RoPE already applied)
 *   kv       device fp16 page pool [n_pages][2][n_kv_heads][64][64]: per page and
 *            KV head, K as [64 tokens][64 dims] and V transposed, [64 dims][64 tokens]
 *   page_table device int32 [n_seq, pt_stride]: logical page -> physical page
 *   n        device int32 [n_seq]: n_s
 *   out      device fp16 [n_seq, W, n_heads, 64]
 *   scratch  device, >= gs_attention_scratch_bytes(...) bytes: the kernel's
 *            error word (first int32: 0 = no failure, 1 = bounds check,
 *            2 = bounded wait ran out, 3 = fp16 range; cleared by each call),
 *            key limits, the block -> page-table map, merge tickets and the
 *            fp32 partial rows (O, m, l) of every work item
 *   split_pages pages per work item (>= 1): item i of a sequence covers its
 *            logical pages [i * split_pages, (i + 1) * split_pages); items are
 *            reduced independently and merged in item order, so results depend
 *            on split_pages but not on n_seq, W or the other sequences.
 *            GS_ERR_UNSUPPORTED if ceil(pt_stride / split_pages) > 54 (the
 *            merge keeps each item's running max and sum of every row in the
 *            kernel's idle page ring, 54 KB).
 *   stream   cudaStream_t */
size_t gs_attention_scratch_bytes(int n_seq, int W, int n_heads, int n_kv_heads, int max_pages,
                                  int split_pages);
int gs_attention(int mode, const void *q, const void *kv, int n_pages, const int32_t *page_table,
                 int pt_stride, const int32_t *n, int n_seq, int W, int n_heads, int n_kv_heads,
                 void *out, void *scratch, size_t scratch_bytes, int split_pages, void *stream);

/* Y = X . W^T on the tcgen05 GEMM the decoder uses.
 *   x device fp16 [M, K] (row stride K), w device fp16 [N, K], y device [M, N]
 *   epilogue 0: y fp16 = acc;  1: y fp32 += acc (residual);  2: SwiGLU: w is
 *   [2N, K] (gate rows then up rows), y fp16 [M, N] = silu(gate) * up;
 *   3: argmax: y is uint64 [M] packed (ordered fp32 bits << 32 | ~index),
 *   combined with atomicMax (caller zeroes it first).
 *   split_k S: 1 or a divisor of K/64.  K is reduced as S consecutive chunks,
 *   each summed from zero in k order, then the chunks summed in order
 *   0..S-1.  Where the chunks are reduced (across a cluster of CTAs, inside
 *   one CTA, or through the scratch) depends on M; the sums do not, so a row's
 *   result is the same for any M.  scratch device >= gs_linear_scratch_bytes,
 *   any contents: the call clears the parts that must start at zero.  Its
 *   first int32 is the kernel's error word after the stream reaches the end
 *   of the call (0 = no failure, 1 = bounds check, 2 = bounded wait ran out,
 *   3 = a value beyond the fp16 range).
 *   Requirements: K % 64 == 0, N % 128 == 0 (N % 64 for epilogue 2), M >= 1;
 *   x, w and y 16-byte aligned. */
size_t gs_linear_scratch_bytes(int M, int N, int split_k);
int gs_linear(const void *x, const void *w, void *y, int M, int N, int K, int epilogue, int split_k,
              void *scratch, size_t scratch_bytes, void *stream);

/* ---------------------------------------------------------------------------
 * Allocation-free variant of gs_linear.  The paper has no counterpart: this
 * entry point exists for callers that cannot allocate device memory at the
 * call and have no workspace to pass (an operator inside another framework
 * with no workspace argument, a plugin host whose allocator owns all device
 * memory, a real-time path where cudaMalloc's implicit synchronisation is not
 * allowed).
 *
 * Same arguments and results as gs_linear minus the scratch pointer: the
 * split-K scratch (error word, per-tile counters, fp32 partials) lives in a
 * fixed device array of GS_NOALLOC_SCRATCH_BYTES inside the library, which
 * every GPU that loads the library keeps until the process exits.  The call
 * makes no cudaMalloc / cudaFree and calls no allocating library routine.
 *   - The first call on a device looks up that array's device address (with
 *     the device current); make that first call before any stream capture.
 *   - Every call clears the counters it uses and the error word before its
 *     kernel runs.  gs_linear_noalloc_status reports that call's kernel-side
 *     checks.
 *   - All calls share the one array: calls whose kernels overlap on the GPU
 *     (two streams, or two host threads on one device) race; serialise them.
 * Errors: as gs_linear; GS_ERR_OOM when split_k x tiles of partials for
 * (M, N) do not fit in GS_NOALLOC_SCRATCH_BYTES (e.g. M <= 32 rows, N = 2048,
 * split_k = 8 needs 2 MiB). */
#define GS_NOALLOC_SCRATCH_BYTES (8u << 20)
int gs_linear_noalloc(const void *x, const void *w, void *y, int M, int N, int K, int epilogue,
                      int split_k, void *stream);

/* Kernel-side status of the most recent gs_linear_noalloc on the current
 * device: synchronises `stream` (the one that call used), then returns GS_OK,
 * GS_ERR_DEVICE_CHECK (a bounds check fired or a value left the fp16 range)
 * or GS_ERR_TIMEOUT (a bounded wait ran out), and clears the word.  Call it
 * before the next gs_linear_noalloc, which clears the word again.  Allocates
 * nothing.  Errors: GS_ERR_CUDA. */
int gs_linear_noalloc_status(void *stream);

/* ---------------------------------------------------------------------------
 * One sampled decoding step over a paged cache, for decoders whose heads the
 * engine above does not cover and for sampling several continuations of one
 * prompt.  The paper has no counterpart: its rounds take the argmax or plain
 * temperature samples of one fixed decoder.  The four operators take a layer's
 * projected rows to the next token; the matrix products between them are
 * gs_linear's.  They need no handle: work is enqueued on the given stream, no
 * device memory is allocated, and every call may be captured in a CUDA graph.
 *
 * `err` (or the first int32 of the scratch) is a device error word: a kernel
 * that meets an index out of range stores 1 and goes on with the index clamped
 * or the write left out.  It is never cleared by a call: zero it once, read it
 * when convenient.
 * ------------------------------------------------------------------------ */

/* Element types. */
enum { GS_F16 = 0, GS_BF16 = 1, GS_F32 = 2 };

/* One layer of a paged cache.  A page holds 64 tokens, [2][n_kv_heads][64 *
 * head_dim] elements: keys as [64 tokens][head_dim], values transposed, as
 * [head_dim][64 tokens] (for head_dim 64 and fp16 the layout of the engine and
 * of gs_attention).  Token t of sequence s lies in page page_table[s][t / 64].
 *   kv          device, 16-byte aligned, n_pages pages
 *   head_dim    64 or 128; dtype GS_F16 or GS_BF16
 *   page_table  device int32 [n_seq, pt_stride]
 * Pages may be shared between sequences as long as no call writes them. */
typedef struct {
  void *kv;
  int n_pages, n_kv_heads, head_dim, dtype;
  const int32_t *page_table;
  int n_seq, pt_stride;
} gs_cache;

/* Rotary positions: the first rotary_dim dims of a head (a multiple of 16, at
 * most head_dim) are rotated in pairs, (i, i + rotary_dim / 2) in the half
 * layout or (2i, 2i + 1) in the interleaved one; the rest pass through.
 *   table   device fp32 [table_rows][rotary_dim / 2][2], 16-byte aligned: cos
 *           and sin of each position's angles (gs_rope_table) */
enum { GS_ROPE_HALF = 0, GS_ROPE_INTERLEAVED = 1 };
typedef struct {
  const void *table;
  int table_rows, rotary_dim, layout;
} gs_rope;

/* Frequencies theta^(-2i / rotary_dim) of pair i, stretched for contexts longer
 * than the trained one by `factor` (>= 1):
 *   GS_ROPE_LINEAR  every frequency divided by factor
 *   GS_ROPE_NTK     theta * factor^(R / (R - 2)) instead of theta
 *   GS_ROPE_YARN    pairs that turn more than beta_fast times in original_ctx
 *                   positions kept, those below beta_slow divided, a linear
 *                   ramp over the pairs between; cos and sin times magnitude
 *                   (0: 0.1 ln(factor) + 1)
 * Fields that a kind does not name are not read. */
enum { GS_ROPE_PLAIN = 0, GS_ROPE_LINEAR = 1, GS_ROPE_NTK = 2, GS_ROPE_YARN = 3 };
typedef struct {
  int kind;
  float theta, factor;
  int original_ctx;
  float beta_fast, beta_slow, magnitude;
} gs_rope_scaling;

/* Fill a rotary table: angles, cos and sin in 64 bits, rounded once to fp32.
 *   table  device fp32 [rows][rotary_dim / 2][2], 16-byte aligned
 * rotary_dim is a multiple of 16, at most 128.
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_CUDA. */
int gs_rope_table(const gs_rope_scaling *scaling, int rotary_dim, int rows, void *table,
                  void *stream);

/* Per-head RMS norm of queries and keys, their rotation, and the write of keys
 * and values into the cache, for T tokens of any sequences (a decode batch, a
 * prompt, or a mix).  Arithmetic in fp32, each output rounded once.
 *   qkv     device [T, (n_heads + 2 n_kv_heads) * head_dim] of the cache's
 *           type: query heads, key heads, value heads; row stride ld_qkv
 *           elements (a multiple of 8), 16-byte aligned
 *   q_gain, k_gain  device bf16 [head_dim], 16-byte aligned; both NULL: no norm
 *   seq     device int32 [T]: the token's row of the page table
 *   slot    device int32 [T]: its place in the sequence's cache; negative: the
 *           token's key and value are not written.  Two tokens of one call must
 *           not name the same place.
 *   pos     device int32 [T]: the position it is rotated to (row of the table)
 *   q_out   device [T, n_heads * head_dim], row stride ld_q (a multiple of 8);
 *           may be qkv itself with ld_q == ld_qkv
 *   err     device int32, see above (seq, slot, page or pos out of range: a
 *           write is left out, a position clamped)
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED (head_dim, too many rows),
 * GS_ERR_CUDA. */
int gs_rope_append(const gs_cache *cache, const gs_rope *rope, const void *qkv, int64_t ld_qkv,
                   int T, int n_heads, const void *q_gain, const void *k_gain, float eps,
                   const int32_t *seq, const int32_t *slot, const int32_t *pos, void *q_out,
                   int64_t ld_q, int32_t *err, void *stream);

/* Attention of one token per row over the paged cache:
 *   out = softmax(scale * q K^T) V over the keys max(0, n - window) .. n - 1
 * (all n keys if window is 0).  A row with n = 0 gives zeros and lse -inf.
 *   q       device [rows, n_heads * head_dim] of the cache's type, row stride
 *           ld_q (a multiple of 8), 16-byte aligned; out likewise with ld_out
 *   seq     device int32 [rows]: the row's sequence (page-table row), or NULL:
 *           row r is sequence r
 *   n       device int32 [rows]: cached keys, the new token's own included
 *   lse     device fp32 [rows, n_heads] or NULL: ln of the sum of exp of the
 *           scores (to join with attention over other keys)
 *   split_pages  pages per work item, 0 = chosen from rows, heads and pt_stride
 *           (or window).  Items are reduced independently and joined in a fixed
 *           order: a row's result depends on its own keys and the split only.
 *           The choice takes rows to be about as long as the table is wide: with
 *           much shorter ones, a split made for them is faster.
 *   scratch device, 256-byte aligned, at least
 *           gs_decode_attention_scratch_bytes(...) bytes (0 on a bad argument);
 *           its first int32 is the error word, the rest may hold anything.
 *           Calls that may run at the same time need scratch of their own.
 * What the cache holds at or beyond n, or before the window, has no influence.
 * Scores, maxima, sums and accumulators are fp32; the probabilities are rounded
 * to the cache's type for the product with V (relative error 2^-11 in fp16, down
 * to 2^-29 of the largest, 2^-8 in bf16), and the output to that type.
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED (head_dim, rows > 65535),
 * GS_ERR_OOM (scratch too small), GS_ERR_CUDA. */
size_t gs_decode_attention_scratch_bytes(const gs_cache *cache, int rows, int n_heads,
                                         int split_pages);
int gs_decode_attention(const gs_cache *cache, const void *q, int64_t ld_q, const int32_t *seq,
                        const int32_t *n, int rows, int n_heads, float scale, int window, void *out,
                        int64_t ld_out, float *lse, int split_pages, void *scratch,
                        size_t scratch_bytes, void *stream);

/* Per-row sampling settings: device arrays of `rows` entries, each may be NULL.
 *   temperature fp32, > 0 (NULL: 1).  0, negative or NaN: the row takes its
 *               largest logit, and u is not used
 *   top_p       fp32: below 1, the shortest prefix whose mass is at least top_p
 *   min_p       fp32: above 0, only tokens with at least min_p times the
 *               largest probability (at most 1 is used)
 *   top_k       int32: above 0, the k most likely tokens */
typedef struct {
  const float *temperature, *top_p, *min_p;
  const int32_t *top_k;
} gs_sample_params;

/* Draw one token per row.  With M the row's largest logit, token i has weight
 * w = exp((l_i - M) * (1 / T)), counted as the integer floor(w * 2^40): sums of
 * weights are exact, whatever their order, so a draw does not depend on how the
 * row was divided.  The tokens are ordered by falling logit, equal ones by
 * index; of that order min_p, then top_k, then top_p (a share of what is left)
 * keep a prefix of mass Z, and the draw is its first token whose cumulative
 * mass exceeds min(floor(u Z), Z - 1).  Tokens of weight 0 are neither drawn nor
 * counted.
 *   logits   device [rows, vocab] of dtype, row stride ld elements; NaN counts
 *            as -inf, logits of +inf have all the weight between them.  Rows
 *            need no alignment beyond the element's.
 *   u        device fp32 [rows], in [0, 1) (others are clamped, NaN is 0)
 *   token    device int32 [rows]; -1 where every logit is -inf
 *   logprob  device fp32 [rows] or NULL: ln of the token's share of Z
 *   kept     device int32 [rows] or NULL: tokens in the prefix
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED (vocab > 262,144, rows >
 * 2^24), GS_ERR_CUDA. */
int gs_sample(const void *logits, int64_t ld, int rows, int vocab, int dtype,
              const gs_sample_params *params, const float *u, int32_t *token, float *logprob,
              int32_t *kept, void *stream);

/* Copy n pages in every layer: page dst_ids[i] of dst becomes page src_ids[i]
 * of src, in one launch.  Both pools are [n_layers][pages][page_bytes] and may
 * be the same one; no page may be a destination twice, or a source and a
 * destination of one pool.
 *   page_bytes  a multiple of 16, at most 2^30; src, dst 16-byte aligned
 *   src_ids, dst_ids  device int32 [n] (an index out of range: nothing is
 *               copied for it and *err is raised)
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED (n_layers > 65535, page_bytes
 * > 2^30), GS_ERR_CUDA. */
int gs_pages_copy(const void *src, int src_pages, void *dst, int dst_pages, int n_layers,
                  int64_t page_bytes, const int32_t *src_ids, const int32_t *dst_ids, int n,
                  int32_t *err, void *stream);

/* ---------------------------------------------------------------------------
 * Verification of drafted trees over the paged cache, and products with 4-bit
 * weights.  The engine verifies one chain of its own drafts; these take a tree
 * of candidates from anywhere through one step of a decoder of the caller's:
 * its nodes are appended at slots n, n + 1, ... (gs_rope_append), attend to the
 * cache and their ancestors (gs_tree_attention), choose a token each (gs_sample,
 * or the largest logit), and the path of nodes that were chosen is kept
 * (gs_tree_accept, gs_tree_commit).  As each node's token is drawn from the
 * model's own distribution and a drafted one is only kept where it is that token,
 * the output is distributed as without drafts, whatever drafted them.
 *
 * Trees of one call have up to `nodes` <= 64 nodes each; arrays by node are
 * [trees, nodes].  Node 0 is the root: the last token chosen, not in the cache
 * yet.  A parent comes before its children.  Like the operators above these need
 * no handle, allocate nothing, may be captured, and raise an error word.
 * ------------------------------------------------------------------------ */

/* Attention of every node of each tree over the paged cache:
 *   out = softmax(scale * q K^T) V over the cached keys 0 .. n - 1 and, of the
 * nodes' own keys (at slots n .. n + count - 1), those in the node's mask.  A
 * node that sees nothing gives zeros and lse -inf.
 *   q       device [trees * nodes, n_heads * head_dim] of the cache's type, row
 *           stride ld_q (a multiple of 8), 16-byte aligned; out likewise
 *   seq     device int32 [trees]: the tree's row of the page table, or NULL: tree
 *           b is sequence b
 *   n       device int32 [trees]: cached keys before the tree
 *   count   device int32 [trees]: nodes in use, or NULL: all.  Rows of the others
 *           are left as they are, and their keys are not read.
 *   mask    device uint64 [trees, nodes]: bit j: the node sees node j (its own
 *           bit included, if it is to see itself).  Any pattern.
 *   pos     device int32 [trees, nodes]: positions (n + depth), read only with a
 *           window: cached keys at or below pos - window are not seen; a position
 *           below n counts as n.  The mask alone decides about nodes.  May be NULL
 *           without a window (0).
 *   lse     device fp32 [trees * nodes, n_heads] or NULL: ln of the sum of exp of
 *           the scores
 *   split_pages  pages per work item: items are reduced independently and joined in
 *           a fixed order, and a row's result depends on its own keys, the split and
 *           `nodes` only.  0: chosen; with more than 16 query rows of a KV head (nodes *
 *           n_heads / n_kv_heads) and at most 1024 trees the pages of all trees are
 *           then shared evenly, and how a row's sums are rounded depends on the other
 *           trees of the call (never on the order of execution: a repeated call
 *           gives the same bits).
 *   scratch device, 256-byte aligned, at least gs_tree_attention_scratch_bytes(...)
 *           bytes (0 on a bad argument); its first int32 is the error word: raised by
 *           a sequence, page, count or n out of range (n + count beyond the table, or
 *           a negative one), or 2 where a wait within the kernel ran out.  The rest
 *           may hold anything.  Calls that may run at the same time need scratch of
 *           their own; graphs that are replayed one after another may share it.
 * What the cache holds where a node does not see it has no influence on that node,
 * infinities and NaN included.  Scores, maxima, sums and accumulators are fp32;
 * the probabilities are rounded to the cache's type for the product with V (those
 * below 2^-29 of the largest lose bits in fp16, below 2^-21 with more than 16 rows).
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED (head_dim, nodes > 64, trees >
 * 65535, n_heads > 16383), GS_ERR_OOM (scratch too small), GS_ERR_CUDA. */
size_t gs_tree_attention_scratch_bytes(const gs_cache *cache, int trees, int nodes, int n_heads,
                                       int split_pages);
int gs_tree_attention(const gs_cache *cache, const void *q, int64_t ld_q, const int32_t *seq,
                      const int32_t *n, const int32_t *count, const uint64_t *mask,
                      const int32_t *pos, int trees, int nodes, int n_heads, float scale, int window,
                      void *out, int64_t ld_out, float *lse, int split_pages, void *scratch,
                      size_t scratch_bytes, void *stream);

/* The path of each tree that its model chose: from the root to the first child (by
 * number) whose token is its parent's choice, and so on.
 *   parent  device int32 [trees, nodes]: a lower number; node 0's is not read
 *   token   device int32 [trees, nodes]: drafted tokens; node 0's is not read
 *   choice  device int32 [trees, nodes]: the token that the model chose to follow
 *           each node; a negative one (gs_sample's -1) ends the path
 *   count   device int32 [trees]: nodes in use, or NULL: all
 *   most    device int32 [trees]: the longest path allowed, or NULL: any
 *   eos     a path ends at a node whose choice this is; -1: none
 *   path    device int32 [trees, nodes]: nodes on the path, then -1
 *   next    device int32 [trees, nodes]: their choices, the tokens that this step
 *           adds, then -1
 *   length  device int32 [trees]: how many; at least 1 (the root) unless count or
 *           most is 0
 *   err     device int32, raised by a parent that is not a lower number (the node
 *           is on no path) or a count out of range
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED (nodes > 64), GS_ERR_CUDA. */
int gs_tree_accept(const int32_t *parent, const int32_t *token, const int32_t *choice,
                   const int32_t *count, const int32_t *most, int eos, int trees, int nodes,
                   int32_t *path, int32_t *next, int32_t *length, int32_t *err, void *stream);

/* Keys and values of accepted paths moved together, in every layer by one launch:
 * slot n + path[i] goes to slot n + i for i < length.  Slots beyond are left as
 * they are, and so is what does not move.
 *   cache    layer 0; layer l lies l * n_pages pages behind it
 *   seq, n   as in gs_tree_attention
 *   path     device int32 [trees, nodes], rising, and length, device int32
 *            [trees], as gs_tree_accept gives them
 *   err      device int32, raised by a length, path, sequence, slot or page out of
 *            range; nothing of that tree is moved then
 * The slots' pages must not be shared with other sequences or trees.
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED (head_dim, nodes > 64, n_layers or
 * trees > 65535), GS_ERR_CUDA. */
int gs_tree_commit(const gs_cache *cache, int n_layers, const int32_t *seq, const int32_t *n,
                   const int32_t *path, const int32_t *length, int trees, int nodes, int32_t *err,
                   void *stream);

/* A matrix [N, K] of 4-bit weights (q - z) * s: whole numbers q in 0 .. 15, and for
 * each `group` of a row's neighbouring weights a scale s and a zero z in 0 .. 15.
 *   packed  device, 16-byte aligned, gs_qweight_bytes bytes, made by gs_qweight_pack
 *   group   32, 64 or 128; K is a multiple of it
 *   dtype   GS_F16 or GS_BF16: type of scales, inputs and outputs
 *   zeros   0: every z is 8
 *   gated   1: rows 0 .. N / 2 - 1 are a SwiGLU's gate and the others its up
 *           projection, laid out side by side for epilogue 2 */
typedef struct {
  void *packed;
  int N, K, group, dtype, zeros, gated;
} gs_qweight;

/* Bytes of the packed form (0 on a bad argument; `packed` is not read). */
size_t gs_qweight_bytes(const gs_qweight *w);

/* Lay weights out, once, in the order in which gs_qlinear reads them.
 *   q      device uint8 [N, K / 2]: two weights a byte, the first in the low bits
 *   scale  device [N, K / group] of dtype
 *   zero   device uint8 [N, K / group] (the low four bits count); NULL where zeros
 *          is 0
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED (another group, K > 2^20, N > 2^24),
 * GS_ERR_CUDA. */
int gs_qweight_pack(const gs_qweight *w, const void *q, const void *scale, const void *zero,
                    void *stream);

/* Y = X . W^T with 4-bit weights, made for the rows of a decoding step.
 *   x   device [M, K] of dtype, row stride ld_x (a multiple of 8), 16-byte aligned
 *   y   device [M, N], row stride ld_y.  epilogue 0: dtype, y = acc; 1: fp32, y +=
 *       acc; 2: dtype [M, N / 2], silu(gate) * up (gated weights, and only they)
 *   err device int32: 3 is stored where an fp16 output is beyond the type's range, 2
 *       where a wait within the kernel ran out (M > 32)
 * No weight is rounded: sums of q x and of x over each group are fp32, z times the
 * latter is taken off, and s multiplies in fp32; the error before the output's
 * rounding is that of fp32 sums of terms up to 15 s |x| (31 s |x| in bf16).  A row's
 * result is the same for any M up to 32, and for any M beyond.  A row of x that holds an
 * infinity or a NaN, or (bf16) values beyond 2^110, may give NaN where the sum would be
 * infinite or finite; other rows are not touched by it.
 * Errors: GS_ERR_INVALID_ARG, GS_ERR_UNSUPPORTED (as above, M > 2^21), GS_ERR_CUDA. */
int gs_qlinear(const gs_qweight *w, const void *x, int64_t ld_x, void *y, int64_t ld_y, int M,
               int epilogue, int32_t *err, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* GS_H_ */
