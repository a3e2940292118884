/*
 * spec.h -- C ABI of the MI355X speculative verify-and-commit library
 * (libspecdec.so, gfx950).
 *
 * The library runs the propose / verify / commit loop of two-reasoner
 * speculative decoding (Sec. 3.2 and Sec. 4.1 of "Reasoning-aware Speculative
 * Decoding for Efficient Vision-Language-Action Models in Autonomous
 * Driving"):
 *   draft_step   one step of the routine reasoner, which proposes the next token
 *                with FlatRoPE (Eq. propose, Eq. flatrope-proj); K calls give d_1..d_K.
 *   spec_verify  the deliberative reasoner (target, 3D M-RoPE, Eq. rope-3d)
 *                evaluates [pending, d_1..d_K] in one forward pass, takes the
 *                greedy token of every row (Eq. verify) and the longest matching
 *                prefix l (Eq. accept).
 *   spec_commit  commits (d_1..d_l, r*_{l+1}), advances the lengths by l+1 and
 *                rolls back both KV caches (Eq. commit).
 *
 * Conventions
 *   - Every entry point returns a spec_status; nothing throws or exits.
 *   - "device" pointers are HIP device memory on the device that is current at
 *     spec_init; "host" pointers are ordinary memory.
 *   - bf16 means IEEE bfloat16 stored as 16-bit words; matrices are row-major
 *     [out_features][in_features].  All row lengths must be multiples of 8
 *     elements and all device pointers 16-byte aligned.
 *   - All work is enqueued on the stream given to spec_init and returns
 *     without waiting, except the calls documented as synchronising.
 *   - Arguments are validated on the host before anything is enqueued; on an
 *     error the context is left unchanged.  A HIP runtime error poisons the
 *     context: afterwards only spec_last_error and spec_destroy are valid.
 *   - One context is not safe to use from two threads at once.
 */
#ifndef SPECDEC_SPEC_H
#define SPECDEC_SPEC_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPEC_MAX_K      16   /* draft block size limit (the paper verifies blocks of 16) */
#define SPEC_MAX_BATCH  16   /* sequences per context */
#define SPEC_MAX_LAYERS 256
#define SPEC_MAX_ROWS   160  /* batch*(K+1): rows of one verify pass */
#define SPEC_KV_PAGE    64   /* KV slots per cache page */

typedef struct spec_ctx spec_ctx;   /* opaque; owned by the library */

typedef enum spec_status {
  SPEC_OK = 0,
  SPEC_E_INVAL = 1,     /* bad argument, or a token id out of range was seen on the device */
  SPEC_E_STATE = 2,     /* call out of order (see the state machine below) */
  SPEC_E_CAPACITY = 3,  /* workspace too small or sequence capacity exceeded */
  SPEC_E_HIP = 5,       /* HIP runtime error; the context is poisoned */
  SPEC_E_NUMERIC = 6    /* NaN logits were seen on the device */
} spec_status;

/* Shape of one decoder stack.  The block is pre-norm: RMSNorm -> q,k,v (no
 * bias) -> rotary -> causal grouped-query attention -> o projection + residual
 * -> RMSNorm -> SwiGLU (silu(gate) * up) -> down projection + residual. */
typedef struct spec_dims {
  int32_t layers;            /* 1..SPEC_MAX_LAYERS */
  int32_t hidden;            /* model width; multiple of 16 */
  int32_t q_heads;           /* query heads; multiple of kv_heads */
  int32_t kv_heads;          /* key/value heads */
  int32_t head_dim;          /* 64 or 128 */
  int32_t ffn;               /* SwiGLU inner width; multiple of 16 */
  int32_t mrope_section[3];  /* (s_T, s_H, s_W) rotary pairs per axis, summing to
                                head_dim/2 (Eq. rope-3d); ignored by the draft unless
                                SPEC_FLAG_DRAFT_MROPE */
  int32_t interleaved;       /* 0: blocked axis assignment, 1: d mod 3 (Eq. axis-assign) */
  float rope_base;           /* theta_d = rope_base^(-2d/head_dim) (Eq. mrope-phase) */
  float rms_eps;             /* RMSNorm epsilon */
} spec_dims;

#define SPEC_FLAG_NO_GRAPHS 1      /* launch kernels one by one instead of replaying HIP graphs */
/* (values 2 and 4 are not used; unknown flag bits are rejected with SPEC_E_INVAL) */
#define SPEC_FLAG_ROWMAJOR 8       /* stream the caller's row-major weights directly.  Without it, passes
                                      of at most 32 rows (batch*(K+1) <= 32), or of
                                      rows the batched-row GEMM takes, stream a tile-packed copy of every
                                      weight matrix that spec_init writes into the workspace (its size is
                                      part of spec_workspace_bytes) */
#define SPEC_FLAG_BLOCK_DRAFT 32   /* draft_step proposes all K tokens in one forward of the draft (the
                                      block-diffusion draft family, Sec. 4.1): rows [pending, MASK x K],
                                      the pending row attending causally and every MASK row attending to
                                      the prefix and the whole block; MASK row i proposes d_i.  Accepted
                                      proposals of the previous round are first re-encoded causally.
                                      Needs a draft. */
#define SPEC_FLAG_COND 64          /* the draft is conditioned on target hidden states (Sec. 4.1; fused
                                      EAGLE-3 style, Sec. 5): every verify keeps the target's residual
                                      stream after layers cond_layers[0..2]; for the rows whose inputs get
                                      committed, f = w_fuse [h0; h1; h2] (3*hidden -> hidden) becomes the
                                      slot's feature, and a draft row at slot t takes the layer-0 input
                                      e + w_in [e; f(t-1)] (2*hidden -> hidden; f = 0 where no verified
                                      feature exists: prompt slots and the draft's proposal rows).
                                      Needs a draft with w_fuse and w_in. */
#define SPEC_FLAG_COND_CROSS 256   /* with SPEC_FLAG_COND: the fused features f are the draft's layer-0
                                      cross-attention context (Sec. 4.1: target hidden states fed to the
                                      draft as cross-attention K/V) instead of the input term.  After each
                                      commit, every committed slot s gets k = rot_s(W_k RMSNorm(f_s)) and
                                      v = W_v RMSNorm(f_s) (the draft's layer-0 norm and projections) in
                                      the draft's layer-0 cache; the prompt slots keep the given draft
                                      prompt K/V.  A draft row at slot t attends in layer 0 to the context
                                      slots s < min(t, seq_len) only, and takes the plain embedding as
                                      input (w_in may be null).  Not with SPEC_FLAG_BLOCK_DRAFT. */
#define SPEC_FLAG_FULL_DRAFT_ROWS 128  /* every draft step runs the pass of batch*(K+1) rows.  Without it,
                                      a chained draft step after the first of a round (each live sequence
                                      then consumes exactly one token, its previous proposal) runs as a
                                      pass of one row per sequence on the tile-packed GEMV, when the
                                      batch is at most 32, a packed weight copy exists and neither
                                      SPEC_FLAG_BLOCK_DRAFT nor SPEC_FLAG_COND is set */
#define SPEC_FLAG_KV8 512          /* the target's prompt cache in 8 bits: every whole page of a prompt is held
                                      as spec_kv8_pack packs it (after rotation), the prompt's last slots and
                                      all later ones in bf16, as spec_kv8_attn reads them.  What a round rolls
                                      back never enters an 8-bit page, so greedy output stays the same for
                                      every K.  The prompts' whole pages take half the bytes.  Each kind's
                                      pages lie in a pool of their own, in the order of their page_table
                                      numbers.
                                      The attention-budget readout of the target is not available. */
#define SPEC_FLAG_DRAFT_MROPE 16   /* the draft rotates with 3D M-RoPE (its own mrope_section and
                                      interleaved, validated as the target's) instead of FlatRoPE: the
                                      comparison arm of the attention-budget readout (Sec. 4.2) */

typedef struct spec_config {
  spec_dims target;          /* deliberative reasoner (3D M-RoPE) */
  spec_dims draft;           /* routine reasoner (FlatRoPE); draft.layers = 0 means no draft.
                                hidden, head_dim and rope_base must equal the target's: the draft
                                shares the embedding and the theta table (Sec. 4.2). */
  int32_t vocab;             /* tied embedding / LM head rows; multiple of 16 */
  int32_t K;                 /* draft block size, 0..SPEC_MAX_K (0: plain greedy decoding) */
  int32_t batch;             /* independent sequences, 1..SPEC_MAX_BATCH; batch*(K+1) <= SPEC_MAX_ROWS */
  int32_t max_new_tokens;    /* committed-token budget per sequence, >= 1 */
  int32_t stop_token;        /* committing this token ends a sequence; -1: none */
  int32_t flags;             /* SPEC_FLAG_* */
  int32_t mask_token;        /* SPEC_FLAG_BLOCK_DRAFT: input token of the MASK rows, in [0, vocab) */
  int32_t cond_layers[3];    /* SPEC_FLAG_COND: target layers (0-based) whose output is fused */
} spec_config;

/* Borrowed device pointers (bf16).  They must stay valid until spec_destroy. */
typedef struct spec_layer_weights {
  const void* attn_norm;     /* [hidden]                        */
  const void* wq;            /* [q_heads*head_dim][hidden]      */
  const void* wk;            /* [kv_heads*head_dim][hidden]     */
  const void* wv;            /* [kv_heads*head_dim][hidden]     */
  const void* wo;            /* [hidden][q_heads*head_dim]      */
  const void* ffn_norm;      /* [hidden]                        */
  const void* w_gate;        /* [ffn][hidden]                   */
  const void* w_up;          /* [ffn][hidden]                   */
  const void* w_down;        /* [hidden][ffn]                   */
} spec_layer_weights;

typedef struct spec_model_weights {
  const spec_layer_weights* layers;  /* host array of dims.layers entries */
  const void* final_norm;            /* [hidden] bf16, device */
  const void* w_fuse;                /* draft, SPEC_FLAG_COND: [hidden][3*hidden] bf16; else ignored */
  const void* w_in;                  /* draft, SPEC_FLAG_COND: [hidden][2*hidden] bf16; else ignored */
} spec_model_weights;

/* A (t, h, w) grid of vision patches occupying sequence indices
 * [start, start + t*h*w), stored t-major, then h, then w.  Its patch (t, h, w)
 * gets the 3D position (start+t, start+h, start+w); every index outside the
 * blocks is text and gets (i, i, i) (Sec. 3.3, Sec. 4.2). */
typedef struct spec_vision_block {
  int32_t start, t, h, w;
} spec_vision_block;

/* One sequence's prompt.  Its first prefix_len KV slots are filled from the
 * given pre-rotation keys and values; index prefix_len holds pending_token,
 * the first row of the first verify. */
typedef struct spec_seq_init {
  int32_t prefix_len;                 /* >= 1 */
  int32_t n_blocks;
  const spec_vision_block* blocks;    /* host; inside [0, prefix_len), non-overlapping */
  int32_t pending_token;              /* in [0, vocab) */
  const void* const* tgt_k;           /* host array [target.layers] of device pointers to
                                         [prefix_len][kv_heads][head_dim] bf16 keys before rotation */
  const void* const* tgt_v;           /* same shape, values */
  const void* const* drf_k;           /* host array [draft.layers]; NULL without a draft */
  const void* const* drf_v;
  const int32_t* page_table;          /* host; NULL, or the physical cache page of each of this
                                         sequence's spec_seq_pages() pages of SPEC_KV_PAGE slots
                                         (slot s lives in page page_table[s / SPEC_KV_PAGE]) */
} spec_seq_init;

/* KV pages one sequence owns: ceil((prefix_len + max_new_tokens + K + 2) /
 * SPEC_KV_PAGE).  Each model's caches are one pool of the sum of these over
 * the batch; a page holds SPEC_KV_PAGE slots of every kv head of one layer.
 * Either every sequence gives a page_table or none does.  Given tables must
 * together name every pool page exactly once (a permutation of
 * [0, pool pages)); without them sequence b owns the pages after those of
 * sequences 0..b-1, in order.  Both models use the same table. */
int32_t spec_seq_pages(const spec_config* cfg, const spec_seq_init* seq);

/* Bytes of device workspace spec_init needs (KV caches, positions, rotary
 * table, activations, partial sums, per-sequence state). */
spec_status spec_workspace_bytes(const spec_config* cfg, const spec_seq_init* seqs /* [batch] */,
                                 size_t* bytes);

/* Creates a context.  embed: [vocab][hidden] bf16 device, the tied token
 * embedding and LM head shared by target and draft.  draft must be NULL
 * exactly when cfg->draft.layers == 0 (then draft_step is unavailable and
 * spec_verify needs explicit draft tokens).
 * The workspace (device, 256-byte aligned, at least spec_workspace_bytes) is
 * owned by the caller and must outlive the context; the library allocates no
 * device memory of its own.  Prefix K/V may be freed once the stream has
 * passed this call.  Builds the 3D position table and the cos/sin table,
 * rotates the prefix keys of every layer into the caches, and leaves the
 * context READY. */
spec_status spec_init(const spec_config* cfg, const void* embed,
                      const spec_model_weights* target, const spec_model_weights* draft,
                      const spec_seq_init* seqs, void* workspace, size_t workspace_bytes,
                      hipStream_t stream, spec_ctx** out);

/* One draft step (Eq. propose as a chain of single-token steps; with
 * SPEC_FLAG_BLOCK_DRAFT the single-forward block proposal, which writes all K
 * columns of d_draft_tokens and counts as the round's K steps).  The draft
 * first consumes the committed tokens it has not yet seen (one row normally,
 * up to K+1 after the verifier overrode its proposals), then proposes a token
 * from its last row with a greedy argmax.  Call j (0-based) of a round writes
 * column j of d_draft_tokens [batch][K] (device int32; may be NULL).
 * State: READY or DRAFTING with fewer than K steps taken -> DRAFTING. */
spec_status draft_step(spec_ctx* ctx, int32_t* d_draft_tokens);

/* n draft steps in one call: the same as n calls of draft_step (columns j..j+n-1
 * of d_draft_tokens), issued as one launch sequence so that the steps follow
 * each other on the device without a gap between them.  1 <= n <= K minus the
 * steps already taken this round; the state rules are those of draft_step. */
spec_status draft_steps(spec_ctx* ctx, int32_t n, int32_t* d_draft_tokens);
/* (With SPEC_FLAG_BLOCK_DRAFT, draft_steps(ctx, K, out) is the block proposal
 * and n must be K.) */

/* One verify pass (Eq. verify, Eq. accept).  Rows [pending, d_1..d_K] of every
 * sequence go through the target in one forward pass; row j's greedy token is
 * r*_{j+1} (argmax over fp32 logits, lowest index on ties, NaN as -inf).
 * d_draft_tokens: [batch][K] device int32 proposals, or NULL to use the
 * draft's own K proposals of this round.  d_logits: [batch][K+1][vocab] bf16
 * device output, or NULL.  Finished sequences are skipped.
 * State: READY (with d_draft_tokens, or K == 0) or DRAFTING after K steps -> VERIFIED. */
spec_status spec_verify(spec_ctx* ctx, const int32_t* d_draft_tokens, void* d_logits);

/* ---- verify without allocation ------------------------------------------- */

#define SPEC_SCRATCH_BYTES (32u << 20)   /* size of the library's static scratch array per GPU */

/* For callers that cannot allocate or instantiate anything while they run:
 * code under HIP stream capture (this call can be captured into the caller's
 * own graph), tight serving loops, harnesses that forbid allocation.
 * Same arguments, state rules, device outputs and results as spec_verify, with
 * two differences:
 *   - the pass's scratch (split-KV attention partials, partial tiles and
 *     k-split sums of the projections, the per-workgroup argmax pairs of the LM
 *     head, their arrival counters and the bf16 logits staging) lives in one
 *     static device array of SPEC_SCRATCH_BYTES bytes that the library holds
 *     on each GPU it runs on until the process ends (its address is looked up
 *     in spec_init), not in the context's workspace;
 *   - every kernel is launched directly on the context's stream: no HIP graph
 *     is captured, instantiated or launched.
 * It calls no hipMalloc, hipFree or other allocating routine.  The counters
 * that must start at zero are cleared by a fill kernel at the start of the
 * call.  Every call on one GPU, from any context, shares that GPU's array,
 * which keeps the last call's contents: calls on one GPU that overlap in time
 * (other streams or threads) race and give wrong results, so serialise them.
 * Returns SPEC_E_CAPACITY, with nothing enqueued and the context unchanged,
 * when the context's verify needs more than SPEC_SCRATCH_BYTES of scratch (the
 * error text gives the need; it grows with batch*(K+1) rows, query heads,
 * sequence capacity and vocabulary).  Any other error is spec_verify's. */
spec_status spec_verify_scratch(spec_ctx* ctx, const int32_t* d_draft_tokens, void* d_logits);

/* Commit (Eq. commit): appends (d_1..d_l, r*_{l+1}), cut after a stop token
 * or at the token budget, to each unfinished sequence; the target keeps KV
 * slots up to the new length and the draft keeps the slots whose inputs still
 * match the committed tokens (the rest are rolled back and later
 * overwritten).  Optional device outputs (int32): d_accept_len [batch] = l,
 * d_committed [batch][K+1] (first d_n_committed[b] entries valid),
 * d_n_committed [batch], d_finished [batch].
 * State: VERIFIED -> READY. */
spec_status spec_commit(spec_ctx* ctx, int32_t* d_accept_len, int32_t* d_committed,
                        int32_t* d_n_committed, int32_t* d_finished);

/* Attention-budget readout (Sec. 4.2, Table attn-budget): arms the next pass
 * of `model` (0: the target, i.e. the next spec_verify; 1: the draft, i.e. the
 * next draft step) to also report where attention layer `layer` (0-based) puts
 * its softmax mass.  Cache slots are classed as visual (inside a vision
 * block), trajectory/text (any other prompt slot) or generated (index >=
 * prefix_len).  For every row j < the pass's row count of sequence b and
 * every query head h of that model, the pass writes d_out[((b*(K+1) + j) *
 * q_heads + h)*4 + c] (device float32, 16-byte aligned):
 *   c = 0, 1, 2  attention mass on visual / trajectory-text / generated slots
 *                (the three sum to 1 up to rounding);
 *   c = 3        entropy of the attention restricted to trajectory/text slots
 *                and renormalised, divided by ln(number of those slots)
 *                (0 when the prompt has at most one such slot).
 * Rows a pass does not run (finished sequences, rows past a draft pass's
 * count) are left unchanged.  The armed pass is launched kernel by kernel
 * (no graph replay); the readout then disarms.  d_out = NULL disarms.
 * Any state; the target of a SPEC_FLAG_KV8 context has no readout
 * (SPEC_E_STATE). */
spec_status spec_attn_readout(spec_ctx* ctx, int32_t model, int32_t layer, float* d_out);

/* Synchronising: waits for the stream, then reports how many sequences have
 * finished (*n_finished, may be NULL) and returns SPEC_E_INVAL / SPEC_E_NUMERIC
 * if a device-side check failed since spec_init (an out-of-range draft token,
 * which was replaced by token 0, or NaN logits). */
spec_status spec_sync(spec_ctx* ctx, int32_t* n_finished);

void spec_destroy(spec_ctx* ctx);

/* Text of the last error of this context (or of the last failed spec_init if
 * ctx is NULL).  Valid until the next call on the context. */
const char* spec_last_error(const spec_ctx* ctx);

/* ---- inspection (synchronising; for tests and tools) --------------------- */

/* 3D positions (p_T, p_H, p_W) of sequence b's slots 0..len-1 into
 * host_out [3][len] int32.  len <= capacity. */
spec_status spec_debug_positions(spec_ctx* ctx, int32_t b, int32_t* host_out, int32_t len);

/* Sequence b's state into host_out [8] int32: seq_len (slots with target KV =
 * index of the pending token), draft_len, pending token, committed-token
 * count, finished, accept length of the last verify, tokens committed by the
 * last commit, device error bits. */
spec_status spec_debug_state(spec_ctx* ctx, int32_t b, int32_t* host_out);

/* Cached keys (which = 0, after rotation) or values (which = 1) of sequence
 * b, model 0 = target / 1 = draft, layer, slots [pos0, pos0+npos) into
 * host_out [npos][kv_heads][head_dim] bf16 (of 8-bit pages the values they
 * stand for). */
spec_status spec_debug_kv(spec_ctx* ctx, int32_t b, int32_t model, int32_t layer, int32_t which,
                          int32_t pos0, int32_t npos, void* host_out);

/* SPEC_FLAG_COND: the fused target features of sequence b's slots [slot0,
 * slot0+n) into host_out [n][hidden] bf16 (zero for slots never verified). */
spec_status spec_debug_feature(spec_ctx* ctx, int32_t b, int32_t slot0, int32_t n, void* host_out);

/* Execution path of the context's passes into *path:
 * SPEC_PATH_ROWMAJOR (one kernel per layer step over the caller's row-major weights),
 * SPEC_PATH_PACKED (one kernel per layer step over the tile-packed weight copy). */
#define SPEC_PATH_ROWMAJOR 0
#define SPEC_PATH_PACKED 1
spec_status spec_debug_path(const spec_ctx* ctx, int32_t* path);

/* Cache pages one attention workgroup takes in every pass (with SPEC_FLAG_KV8,
 * every target pass) of a context opened with these arguments, into *pages (a pass with an armed readout takes one).
 * Does not synchronise; needs no context. */
spec_status spec_debug_attn_pages(const spec_config* cfg, const spec_seq_init* seqs /* [batch] */, int32_t* pages);

/* Per-kernel timing with HIP events on the context's stream.  While enabled,
 * calls launch kernels one by one (no graph replay), each through
 * hipExtLaunchKernelGGL with a start/stop event pair, and every pass begins
 * with a bounded device-side wait (a few ms) so that the host has enqueued the
 * whole pass before its first kernel runs.  spec_timing_read (synchronising) returns, for kernel class
 * `kind`, the number of launches, their summed duration in milliseconds and
 * the summed algorithmic bytes (weights and activations each launch must
 * move, cached keys and values excluded; 0 for kinds without a byte model)
 * since timing was last enabled. */
enum spec_kernel_kind {
  SPEC_KERNEL_QKV = 0,       /* fused Q/K/V projection with rotary and KV append */
  SPEC_KERNEL_O = 1,         /* attention output projection with the residual add */
  SPEC_KERNEL_GATEUP = 2,    /* fused gate/up projection with SwiGLU */
  SPEC_KERNEL_DOWN = 3,      /* down projection partial sums (split over the FFN width) */
  SPEC_KERNEL_LMHEAD = 4,    /* tied LM head with the fused per-tile argmax */
  SPEC_KERNEL_ATTN = 5,      /* split-KV attention */
  SPEC_KERNEL_OTHER = 6,     /* embed, attention combine, down reduction, accept, commit */
  SPEC_KERNEL_KINDS = 7
};
spec_status spec_timing(spec_ctx* ctx, int32_t enable);

/* Read-only streaming reference (no context): reads `bytes` (a multiple of
 * 16) of device memory at d_buf (16-byte aligned) once with non-temporal
 * 16-byte loads, each wave taking 8 KB chunks (eight 1 KB loads in flight),
 * in sink_words / 4 workgroups of 256 threads, and writes one checksum word
 * per wave to d_sink [sink_words]
 * (device; sink_words a positive multiple of 4).  Enqueued on `stream`.  Used
 * to measure the HBM read rate a kernel reaches on this device and to
 * calibrate byte counters against a known read volume. */
spec_status spec_stream_read(const void* d_buf, size_t bytes, uint32_t* d_sink, int32_t sink_words,
                             hipStream_t stream);
spec_status spec_timing_read(spec_ctx* ctx, int32_t kind, int64_t* launches, double* ms, double* bytes);

/* ---- operators without a context ------------------------------------------ */

/* They take device memory of the current device and enqueue on `stream` of that
 * device without waiting; nothing is allocated, and every call can be captured
 * into a graph.  A failed call enqueues nothing, and spec_last_error(NULL) gives
 * its text.  Workspaces are the caller's: 256-byte aligned, of at least the bytes
 * that the matching _workspace_bytes names, their contents of no matter before a
 * call and after it.  Calls that may overlap in time (other streams, graphs that
 * replay together) need workspaces of their own. */

/* A KV cache of one layer whose leading pages are held in 8 bits.  Sequence b's
 * page i (slots [64 i, 64 i + 64)) is page table[b][i] of the 8-bit pool for i <
 * packed[b], else of the bf16 pool, which is laid out as a context's own pages.
 * 8-bit pages hold e4m3 codes (sign, 4 exponent, 3 mantissa bits; no infinity) and
 * one scale for each page and kv head: the value is scale * code. */
typedef struct spec_kv8 {
  int32_t kv_heads;
  int32_t head_dim;          /* 64 or 128 */
  int32_t pages8, pages16;   /* pages of the two pools (either may be 0, its pointers then NULL) */
  void* k8;                  /* [pages8][kv_heads][SPEC_KV_PAGE][head_dim], 16-byte aligned */
  void* v8;                  /* [pages8][kv_heads][head_dim][SPEC_KV_PAGE] (transposed), 16-byte aligned */
  float* k_scale;            /* [pages8][kv_heads], positive and finite */
  float* v_scale;
  const void* k16;           /* bf16 [pages16][kv_heads][SPEC_KV_PAGE][head_dim], 16-byte aligned */
  const void* v16;           /* bf16 [pages16][kv_heads][head_dim][SPEC_KV_PAGE] */
} spec_kv8;

/* Packs the keys (as the cache holds them, after rotation) and values of `rows`
 * (1..2^28) tokens of at most 65535 kv heads into 8-bit pages: rows [64 i, 64 i + 64)
 * into pool page d_pages[i] (device int32, ceil(rows / 64) entries, no page twice).
 * k, v: bf16 rows of [kv_heads][head_dim], 16-byte aligned, row_stride elements apart
 * (a multiple of 8; the rows may lie in a fused projection).  A page and head's scale
 * is the smallest power of two s, at least 2^-126, with max |x| <= 448 s over its finite
 * values (1 if all are zero); codes are x / s to nearest even.  NaN and infinities
 * become NaN.  Slots past the rows are set to zero.  What a page stands for is
 * exact in bf16 (but for magnitudes from 248 * 2^120, which round to 2^128).  An
 * entry of d_pages outside the pool is skipped and sets *d_err (device int32, may be
 * NULL; otherwise left alone) to SPEC_E_INVAL. */
spec_status spec_kv8_pack(const spec_kv8* cache, const void* k, const void* v, int64_t row_stride, int32_t rows,
                          const int32_t* d_pages, int32_t* d_err, hipStream_t stream);

/* Grouped-query attention of a pass's rows over such a cache: row j of sequence b
 * sees slots [0, n) with n = d_visible[b*rows + j], and for query head h of kv head
 * h / (q_heads / kv_heads)
 *   out = sum_s p_s v_s,  p = softmax(scale * q . k_s),  lse = ln sum_s e^(scale * q . k_s).
 * n = 0: out = 0 and lse = -infinity.  n < 0: no such row; its out and lse are left
 * as they were.  Slots that a row does not see have no influence on it, whatever
 * they hold.  An infinite value that a row sees makes its result infinite however
 * small its p (NaN against the other infinity).  1 <= batch*rows <= SPEC_MAX_ROWS;
 * rows*q_heads/kv_heads <= 1048560; q_heads*head_dim <= 2^20; table_stride < 2^25;
 * batch*kv_heads*table_stride <= 2^27.
 *   scale        positive, at most 2^127
 *   d_table      [batch][table_stride] device int32; entries past a sequence's
 *                visible pages are not read
 *   d_packed     [batch] device int32
 *   d_visible    [batch][rows] device int32, at most table_stride * 64
 *   q, out       bf16, row b*rows + j at (b*rows + j) * stride, [q_heads][head_dim];
 *                strides are multiples of 8, pointers 16-byte aligned
 *   d_lse        [batch*rows][q_heads] device float, or NULL
 *   d_err        device int32 or NULL: set to SPEC_E_INVAL, else left alone, if a
 *                table entry lay outside its pool or a scale was not positive and
 *                finite (the page is then taken as not visible; a row that sees no
 *                other has NaN in out and -infinity in lse), or a row wanted more
 *                slots than the table has (it sees those there are)
 * Scores, softmax and sums are formed in 32 bits, in an order fixed by the arguments
 * and lengths; p meets the values as the sum of two bf16 numbers, within 2^-16 of
 * itself. */
spec_status spec_kv8_attn(const spec_kv8* cache, int32_t batch, int32_t rows, int32_t q_heads, const int32_t* d_table,
                          int32_t table_stride, const int32_t* d_packed, const int32_t* d_visible, const void* q,
                          int64_t q_stride, float scale, void* out, int64_t out_stride, float* d_lse, int32_t* d_err,
                          void* workspace, size_t workspace_bytes, hipStream_t stream);
spec_status spec_kv8_attn_workspace_bytes(const spec_kv8* cache, int32_t batch, int32_t rows, int32_t q_heads,
                                          int32_t table_stride, size_t* bytes);

#define SPEC_MAX_TOP 32      /* alternatives of a row */
#define SPEC_BF16 0          /* element types of logits */
#define SPEC_F16 1
#define SPEC_F32 2

/* Scores of rows of logits, such as those a spec_verify hands out, under p =
 * softmax(row).  logits: `dtype` (SPEC_BF16 / F16 / F32), row r at r * row_stride
 * elements (>= vocab; any), 1 <= vocab <= 2^20, 1 <= rows <= 65535.
 *   d_logprob      [rows][n_tokens] float: ln p of the tokens d_tokens
 *                  [rows][n_tokens] (int32); NaN for an id outside [0, vocab)
 *   d_entropy      [rows] float: -sum p ln p, or NULL
 *   d_top_token    [rows][top] int32: the `top` (0..SPEC_MAX_TOP, at most vocab) most
 *                  probable tokens, most probable first, the lowest index on ties, NaN as
 *                  -infinity (spec_verify's rule); d_top_logprob [rows][top]: their ln p
 * Logits of -infinity have p = 0 and ln p = -infinity.  A row with a NaN or
 * +infinity, or with nothing above -infinity, has no distribution: its log
 * probabilities and entropy are NaN.  Arrays of no elements may be NULL. */
spec_status spec_logprobs(const void* logits, int32_t dtype, int32_t rows, int32_t vocab, int64_t row_stride,
                          const int32_t* d_tokens, int32_t n_tokens, int32_t top, float* d_logprob, float* d_entropy,
                          int32_t* d_top_token, float* d_top_logprob, void* workspace, size_t workspace_bytes,
                          hipStream_t stream);
spec_status spec_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t top, size_t* bytes);

/* A pass over trees of drafted tokens.  Where spec_verify checks one chain of
 * proposals, a tree holds several alternatives for a position: each row continues
 * its parent, a row sees its ancestors and no sibling, and the longest path that
 * greedy decoding confirms is committed.  Three operators, over pages laid out as a
 * context's own: spec_kv_append writes the rows' keys and values to the cache,
 * spec_tree_attn is the attention of each layer, and spec_tree_commit, after the
 * target's greedy tokens are known, takes the path and moves its keys and values to
 * consecutive slots in every layer. */

/* A model's KV cache in bf16 pages. */
typedef struct spec_kv {
  int32_t kv_heads;          /* 1..65535 */
  int32_t head_dim;          /* 64 or 128 */
  int32_t pages;             /* pages of a layer's pool, >= 1 */
  int32_t layers;            /* 1..SPEC_MAX_LAYERS */
  int64_t layer_stride;      /* elements from a layer's pool to the next one's, the same for keys and
                                values: a multiple of 8, at least a pool (any value for one layer) */
  void* k;                   /* bf16 [layers][pages][kv_heads][SPEC_KV_PAGE][head_dim], 16-byte aligned */
  void* v;                   /* bf16 [layers][pages][kv_heads][head_dim][SPEC_KV_PAGE] (transposed), 16-byte aligned */
} spec_kv;

/* The rows of a pass.  Sequence b has rows d_first[b] .. d_first[b + 1] - 1 (none is
 * allowed), row d_first[b] + j standing for slot d_len[b] + j: page d_table[b][slot / 64]
 * of the pool, offset slot % 64.  Rows outside every sequence are left as they were in
 * every output.
 * What the host cannot see is checked on the device, which sets *d_err to SPEC_E_INVAL
 * (else leaves it alone) and goes on in bounds: if d_first decreases or leaves [0, rows], no
 * sequence has rows; one whose d_len is negative or more than its table's slots has none (one
 * without rows anyway may have any d_len and is not reported); a parent that is not an earlier
 * row of the sequence counts as -1; slots past the table, and pages outside the pool, are not
 * written, not moved and not visible.
 * No page may belong to two sequences where one of them writes it. */
typedef struct spec_rows {
  int32_t batch;             /* 1..SPEC_MAX_ROWS */
  int32_t rows;              /* rows of the buffers: 1..SPEC_MAX_ROWS (spec_kv_append without trees: to 2^28) */
  const int32_t* d_first;    /* [batch + 1] device int32 */
  const int32_t* d_len;      /* [batch] slots in use before the pass */
  const int32_t* d_table;    /* [batch][table_stride]; entries of pages that a call does not touch are not read */
  int32_t table_stride;      /* 1..2^25 - 16 */
  const int32_t* d_parent;   /* [rows] row of the same sequence (counted from its first) that the row continues, an
                                earlier one, or -1; NULL: chains, each row continues the one before it */
  int32_t* d_err;            /* device int32 or NULL */
} spec_rows;

/* Rotary positions: pair d of a head (dimensions 2d, 2d + 1) turns by
 * base^(-2d/head_dim) times the position on its axis, T, H or W, assigned as
 * spec_dims does (FlatRoPE: section {head_dim/2, 0, 0}). */
typedef struct spec_rope {
  float base;                /* > 1 */
  int32_t section[3];        /* pairs per axis, summing to head_dim/2 */
  int32_t interleaved;       /* 1: pair d takes axis d mod 3, whatever the sections */
} spec_rope;

/* Writes a pass's rows to their slots of layer `layer`: keys rotated, values
 * transposed; queries are rotated into q_out (q may be NULL with q_heads = 0; q_out may be
 * q itself with the same stride; otherwise outputs overlap no input).
 *   d_pos   [3][rows] device int32: positions on T, H and W (axes without pairs are not
 *           read), or NULL: on every axis d_len[b] + the number of the row's
 *           ancestors (then rows <= SPEC_MAX_ROWS if d_parent is given)
 *   q, k, v bf16 rows of [q_heads] and [kv_heads] x head_dim, 16-byte aligned, q_stride and
 *           kv_stride elements apart (multiples of 8; they may lie in a fused projection)
 * q_heads need not be a multiple of kv_heads; q_heads*head_dim <= 2^20, q_heads +
 * 2 kv_heads <= 65535.  Angles are
 * formed in 64 bits, a result is rounded to bf16 once, values are copied as they are. */
spec_status spec_kv_append(const spec_kv* cache, int32_t layer, const spec_rows* rows, const spec_rope* rope,
                           const int32_t* d_pos, int32_t q_heads, const void* q, int64_t q_stride, const void* k,
                           const void* v, int64_t kv_stride, void* q_out, int64_t q_out_stride, hipStream_t stream);

/* Grouped-query attention of a pass's rows over layer `layer`, whose slots hold the
 * rows' own keys and values already.  A row of sequence b sees slots [0, d_len[b]),
 * its ancestors' slots and its own; for query head h of kv head h / (q_heads / kv_heads)
 *   out = sum_s p_s v_s,  p = softmax(scale * q . k_s),  lse = ln sum_s e^(scale * q . k_s).
 * Slots that a row does not see have no influence on it, whatever they hold.  An
 * infinite value that a row sees makes its result infinite however small its p
 * (NaN against the other infinity).  A row that sees no slot (its page lies outside the pool) has
 * NaN in out and -infinity in lse.
 *   scale   positive, at most 2^127
 *   q, out  bf16, row r at r * stride, [q_heads][head_dim]; strides are multiples of 8,
 *           pointers 16-byte aligned; they do not overlap
 *   d_lse   [rows][q_heads] device float, or NULL
 * q_heads is a multiple of kv_heads; q_heads*head_dim <= 2^20; batch*kv_heads*table_stride <= 2^27.
 * Scores, softmax and sums are formed in 32 bits, in an order fixed by the arguments and
 * lengths; p meets the values as the sum of two bf16 numbers, within 2^-16 of itself.  A row
 * with a score beyond 2^30, or one that is not a number, may be NaN. */
spec_status spec_tree_attn(const spec_kv* cache, int32_t layer, const spec_rows* rows, int32_t q_heads, const void* q,
                           int64_t q_stride, float scale, void* out, int64_t out_stride, float* d_lse, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);
spec_status spec_tree_attn_workspace_bytes(const spec_kv* cache, const spec_rows* rows, int32_t q_heads, size_t* bytes);

/* Accept and commit of a tree (Eq. accept, Eq. commit on the tree's paths).  Row 0 of a
 * sequence is its pending token.  The path begins there and goes from row j on to the
 * lowest row whose parent is j and whose token is j's greedy token, as long as there is one;
 * the greedy tokens along the path, l + 1 of them, are committed, cut after a stop token or
 * at the budget.  Of n committed tokens, the first n rows of the path move to slots
 * d_len[b] .. d_len[b] + n - 1, in every layer, and the sequence goes on with n more
 * slots and the last committed token pending.  Other slots are left as they were.
 *   d_tokens     [rows] device int32: token of each row
 *   d_greedy     [rows]: the target's greedy token after each row
 *   stop_token   -1: none
 *   d_budget     [batch]: tokens that may yet be committed (a sequence with none left commits none), or NULL
 *   d_path       [rows]: entry d_first[b] + i is the i-th committed step's row of the sequence
 *   d_committed  [rows]: ... its greedy token (entries past n are left as they were in both)
 *   d_n          [batch]: n;  d_new_len [batch]: d_len + n
 * Any of d_path, d_committed, d_n and d_new_len may be NULL; none may overlap an input or another. */
spec_status spec_tree_commit(const spec_kv* cache, const spec_rows* rows, const int32_t* d_tokens, const int32_t* d_greedy,
                             int32_t stop_token, const int32_t* d_budget, int32_t* d_path, int32_t* d_committed,
                             int32_t* d_n, int32_t* d_new_len, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* SPECDEC_SPEC_H */
