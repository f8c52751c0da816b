/*
 * mcd.h -- C ABI of libmcd, the MI355X (gfx950) multi-codebook audio decode head.
 *
 * One decode step of the output stage of a delay-pattern speech LM served with
 * paired classifier-free guidance (arXiv 2607.02119):
 *   - K codebook head projections of every row's hidden state (Sec. 2.1: each
 *     of the S parallel heads maps h_t to its logits; head k is the k-th audio
 *     slice of the shared head, its stream-embedding term folds into a bias);
 *   - the in-batch CFG merge of each conditional (Main) row with its
 *     unconditional (Companion) partner, w * l_cond + (1 - w) * l_uncond, per
 *     codebook (Eq. 1), only for audio rows (Sec. 2.4);
 *   - temperature, top-k and top-p selection and a Gumbel-max draw from a
 *     counter-based generator in two levels (Philox, Salmon et al., SC'11):
 *     once per (row, codebook, step) vector, Philox4x64-10 with key (seed, 0)
 *     and counter (0, k, t, rng_key) gives the key material D; id v then takes
 *     word v mod 4 of Philox4x32-10 with key (lo D0, hi D0) and counter
 *     (v / 4, lo D1, hi D1, lo D2).  All K streams of a row are drawn in the
 *     same step (synchronous multi-stream sampling, Sec. 2.3);
 *   - the delay pattern: codebook k at step t carries frame t - d_k (Sec. 2.1);
 *     positions with no frame (before the stream starts, or in the drain that
 *     flushes the last S-1 steps, Sec. 2.3) carry the pad id;
 *   - the sampled Main token copied to the Companion row, whose own outputs
 *     stay hidden (Sec. 2.4), and each frame scattered into a per-request
 *     frame grid (the de-interleaved S x T codebook matrix, Sec. 2.1 / 2.3).
 *
 * Conventions
 *   - Pointers are DEVICE pointers unless marked [host].  Every buffer is owned
 *     by the caller; the library never allocates device memory, never
 *     synchronises (except mcd_read_device_status) and launches only on the
 *     stream it is given.
 *   - Row-major layouts; sizes in elements unless named *_bytes.
 *   - Errors: argument and shape errors return MCD_E_INVALID or
 *     MCD_E_UNSUPPORTED before anything is launched; a failed launch returns
 *     MCD_E_HIP.  mcd_last_error() gives a thread-local description of the last
 *     non-OK return.  No call aborts or throws.  Conditions only the device can
 *     see (a parameter value out of range, a grid cell outside the grid, a
 *     corrupt plan) set bits of a sticky status word in the workspace and make
 *     the affected tokens the pad id (the grid cell is then not written); read
 *     it with mcd_read_device_status.
 *   - Calls that share a workspace must not overlap in time.
 */
#ifndef MCD_H
#define MCD_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MCD_OK = 0,
  MCD_E_INVALID = 1,      /* bad argument, shape or batch structure */
  MCD_E_UNSUPPORTED = 2,  /* valid but outside what the kernels implement */
  MCD_E_WORKSPACE = 3,    /* workspace missing or too small */
  MCD_E_HIP = 4           /* the HIP runtime reported an error */
} mcd_status;

typedef enum { MCD_F32 = 0, MCD_BF16 = 1 } mcd_dtype;

/* Row kinds of a continuous batch (Sec. 2.4: a Main request with CFG scale
 * w > 1 gets a Companion; both are scheduled together). */
enum { MCD_ROW_COND = 0, MCD_ROW_UNCOND = 1, MCD_ROW_SOLO = 2, MCD_ROW_TEXT = 3 };

/* Bits of the device status word. */
enum {
  MCD_DEV_BAD_PARAM = 1u,   /* temperature < 0 or NaN, top_p <= 0 or NaN, non-finite w */
  MCD_DEV_GRID_RANGE = 2u,  /* grid_slot >= n_slots or frame >= F_max: cell not written */
  MCD_DEV_BAD_PLAN = 4u,    /* device plan does not match the counts of the call */
  MCD_DEV_BAD_TOKEN = 8u,   /* mcd_next_input: a token outside its table */
  MCD_DEV_BAD_PAGE = 16u,   /* mcd_cache_*: a slot, length or page id out of range */
  MCD_DEV_NO_PAGE = 32u     /* mcd_cache_reserve: no free page left for a token */
};

#define MCD_MAX_K 32         /* codebooks per head */
#define MCD_MAX_V 4096       /* audio sub-vocabulary size per codebook */

typedef struct mcd_head mcd_head;   /* opaque, immutable after creation, thread-safe */

/* Head description.  The weights are borrowed: they must stay valid and
 * unchanged while the handle is used.
 *
 * Streams of unequal size (heterogeneous codebooks, e.g. one SSL stream and
 * eight codec streams): V_stream[k] ids for stream k, V the largest of them.
 * Stream k's block of the N = sum_k V_stream[k] columns starts at
 * off_k = sum_{j<k} V_stream[j]: rows off_k + v of W and entries of bias, and
 * the same columns of every scores row.  With V_stream NULL every stream has
 * V ids, off_k = k*V and N = K*V. */
typedef struct {
  int32_t H;                 /* hidden size; multiple of 64 for MCD_BF16, of 4 for MCD_F32 */
  int32_t K;                 /* codebooks (streams), 1..MCD_MAX_K */
  int32_t V;                 /* audio sub-vocabulary per codebook (the largest), 1..MCD_MAX_V */
  int32_t pad_id;            /* token emitted where the delay pattern has no frame */
  const int32_t *delays;     /* [host][K] d_k >= 0; copied at creation */
  mcd_dtype dtype;           /* element type of hidden, W and W_text */
  const void *W;             /* [N][H]: row off_k + v is head k's weight for id v */
  const float *bias;         /* [N] or NULL: stream-embedding term W_k e_k */
  int32_t V_text;            /* text vocabulary of the text head, 0 if none */
  const void *W_text;        /* [V_text][H] or NULL */
  const int32_t *V_stream;   /* [host][K] ids of each stream (1..MCD_MAX_V), or NULL;
                                copied at creation */
  int32_t T_text;            /* text-phase vocabulary mask (Sec. 2.3): ids [0, T_text) of the
                                text head are text tokens, the rest mark other modalities.
                                0 or V_text: no mask; else a multiple of 32 below V_text */
} mcd_head_desc;

/* Creates the handle.  A bf16 head with a text head also creates, on the
 * current device, the second stream and the two events its mixed batches use
 * (MCD_E_HIP if that fails); nothing is created later, in a step. */
mcd_status mcd_head_create(const mcd_head_desc *desc, mcd_head **out);
void mcd_head_destroy(mcd_head *head);

/* ---- batch plan -----------------------------------------------------------
 * Built on the host once per batch composition (not per step) from the pair
 * map and row kinds, then copied to device memory by the caller.
 *   pair_map[r]: partner row of a COND or UNCOND row, -1 for SOLO and TEXT rows;
 *   partners must point at each other and be one COND and one UNCOND row.
 * The plan fixes the "sampled order" of audio rows: the Main rows of the pairs
 * in ascending row order, then the SOLO rows in ascending row order.  Scores
 * are laid out in that order (see mcd_step_args.scores). */
typedef struct {
  int32_t n_pairs, n_solo, n_text;
} mcd_batch_counts;

size_t mcd_plan_words(int32_t R);   /* int32 words of a plan for R rows */

/* [host] Validate the batch and write the plan.  No HIP call.  Fails with
 * MCD_E_INVALID (and writes nothing) for an inconsistent pair map, an unknown
 * row kind, or TEXT rows on a head without a text head. */
mcd_status mcd_batch_plan(const mcd_head *head, int32_t R, const int32_t *pair_map,
                          const uint8_t *row_kind, int32_t *plan, size_t plan_words,
                          mcd_batch_counts *counts);

/* [host] Physical row of sampled index s (0 <= s < n_pairs + n_solo) and its
 * companion row (-1 for a SOLO row), read from a host copy of the plan. */
mcd_status mcd_plan_sampled_row(const int32_t *plan, int32_t s, int32_t *row, int32_t *companion);

/* Workspace bytes for a batch of up to R rows; the workspace must be 256-byte
 * aligned and zero-filled once before first use (the status word lives in it). */
size_t mcd_workspace_bytes(const mcd_head *head, int32_t R);

/* ---- one decode step -----------------------------------------------------*/
typedef struct {
  int32_t R;                 /* rows in the batch */
  mcd_batch_counts counts;   /* as returned by mcd_batch_plan */
  const int32_t *plan;       /* device copy of the plan words */
  const void *hidden;        /* [R][H] of the head's dtype, 16-byte aligned */
  /* Per-row arrays, [R] each: every one is required when R > 0 (MCD_E_INVALID
     otherwise), whatever the row kinds, since the kernels read them at every
     row; only rng_key may be NULL. */
  const float *cfg_w;        /* [R] CFG scale, used on COND rows (any finite w) */
  const float *temperature;  /* [R] >= 0; 0 selects greedy decoding */
  const int32_t *top_k;      /* [R] <= 0 or >= V: no top-k */
  const float *top_p;        /* [R] in (0, 1); >= 1: no top-p */
  const uint64_t *rng_key;   /* [R] stable request id (Main row's for a pair), or NULL: row index */
  const int32_t *step;       /* [R] decode step t of the row */
  const int32_t *n_frames;   /* [R] frames of the request, -1 if open-ended */
  const int32_t *grid_slot;  /* [R] frame-grid slot of a Main or SOLO row, -1 for none */
  uint64_t seed;             /* Philox key word 0 */
  int32_t *tokens_out;       /* [R][K]: COND/SOLO sampled, UNCOND = its Main row's,
                                TEXT: [r][0] greedy text id, the rest pad_id */
  int32_t *frame_grid;       /* [n_slots][K][F_max] or NULL; cell [slot][k][t - d_k] written */
  uint8_t *modality_out;     /* [R] or NULL: for TEXT rows, 1 when the argmax over all text-head
                                ids lies outside [0, T_text) (the model asks to leave the
                                text phase), else 0; other rows untouched */
  int32_t n_slots, F_max;
  float *scores;             /* [n_pairs + n_solo][N] fp32 in sampled order: the merged,
                                temperature-divided logits (greedy rows: merged only).
                                Output of mcd_head_step, input of mcd_sample_step. */
  void *workspace;
  size_t workspace_bytes;
} mcd_step_args;

/* The whole hot path of one step: projection + merge + temperature (scores),
 * text-head greedy argmax, selection, draw, pads, companion copy, grid scatter.
 * Equal to mcd_head_logits followed by mcd_sample_step: kernel launches on
 * `stream` (for some batches with both audio and text rows the text
 * projection runs on a second stream of the head, forked from and joined back
 * to `stream`); no device allocation, no synchronisation. */
mcd_status mcd_head_step(const mcd_head *head, const mcd_step_args *args, hipStream_t stream);

/* ---- allocation-free step ---------------------------------------------------
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc) and so
 * cannot size mcd_head_step's workspace, whose text-head partials grow with
 * the batch: the same step through the same kernels, with those partials in a
 * device array the library holds per GPU (MCD_NOALLOC_SCRATCH_BYTES, from the
 * first call on a device until the process ends).  Arguments as for
 * mcd_head_step, except args->workspace: the status word region only
 * (workspace_bytes >= 256, 256-byte aligned, zero-filled once; read it with
 * mcd_read_device_status).  MCD_E_UNSUPPORTED, before anything is launched,
 * when the text partials of the batch (n_text x ceil(V_text / 32) fp32 values
 * and int32 ids, each block rounded up to 256 bytes) exceed the array: 220
 * text rows at V_text = 151936.  No allocation, no synchronisation.  Every
 * call on one GPU shares that GPU's array: calls that overlap in time on one
 * GPU race.  A step's partials are written by its projection before its
 * sampler reads them, so nothing carries over between calls. */
#define MCD_NOALLOC_SCRATCH_BYTES (8u << 20)
mcd_status mcd_head_step_noalloc(const mcd_head *head, const mcd_step_args *args,
                                 hipStream_t stream);

/* First half of a step: the K head projections of every audio row with the
 * CFG merge (Eq. 1) and temperature applied in the GEMM epilogue, written to
 * args->scores, and the text-head projection of the TEXT rows reduced to
 * per-32-column (max, lowest argmax) partials kept in the workspace.  Tokens
 * and the grid are not touched. */
mcd_status mcd_head_logits(const mcd_head *head, const mcd_step_args *args, hipStream_t stream);

/* Second half of a step, from the scores in args->scores (same layout as
 * above; they may come from mcd_head_logits or from the caller): selection,
 * draw, pads, companion copy and grid scatter for the audio rows.  TEXT rows
 * take their greedy token from the partials the last mcd_head_logits call left
 * in the same workspace; a batch with TEXT rows must therefore follow such a
 * call (args->hidden is not read). */
mcd_status mcd_sample_step(const mcd_head *head, const mcd_step_args *args, hipStream_t stream);

/* ---- delay pattern (Sec. 2.1) --------------------------------------------
 * De-interleave at request completion: grid[r][k][f] = streams[r][f + d_k][k]
 * for f < T - max_k d_k.  streams: [n_req][T][K], grid: [n_req][K][T - max d]. */
mcd_status mcd_deinterleave(const int32_t *streams, int32_t n_req, int32_t T, int32_t K,
                            const int32_t *delays /*[host][K]*/, int32_t *grid,
                            hipStream_t stream);
/* Inverse: streams[r][t][k] = grid[r][k][t - d_k] where 0 <= t - d_k < F, else
 * pad_id.  grid: [n_req][K][F], streams: [n_req][F + max d][K]. */
mcd_status mcd_interleave(const int32_t *grid, int32_t n_req, int32_t F, int32_t K,
                          const int32_t *delays /*[host][K]*/, int32_t pad_id,
                          int32_t *streams, hipStream_t stream);

/* ---- mixed-modality phases (Sec. 2.3) -------------------------------------
 * Each request moves through a text phase (TEXT rows: greedy over the text
 * ids, the mask of mcd_head_desc.T_text), a transition that injects
 * deterministic bridging tokens, an audio phase (audio rows: all K streams),
 * and a drain of S - 1 steps that flushes the delayed streams, then back to
 * text.  The switch out of text is read from the unmasked distribution
 * (mcd_step_args.modality_out).  The caller re-plans its batch when a
 * request's row kind changes (TEXT rows in the text phase, audio rows in the
 * audio and drain phases; the drain ends the request's frames through
 * n_frames). */
enum { MCD_PHASE_TEXT = 0, MCD_PHASE_BRIDGE = 1, MCD_PHASE_AUDIO = 2, MCD_PHASE_DRAIN = 3 };

typedef struct {
  int32_t n_bridge;          /* bridging tokens between text and audio, >= 0 */
  const int32_t *bridge;     /* [host][n_bridge] their ids */
  int32_t audio_end;         /* stream-0 token that ends the audio phase */
  int32_t drain_steps;       /* steps of the drain: the largest delay (S - 1), >= 0 */
} mcd_phase_desc;

/* [host] One decode step of n requests' phases, in place.  For request i:
 * phase[i], count[i] (bridging tokens emitted / audio steps / drain steps);
 * token0[i]: its stream-0 token of this step (the masked text token of a
 * text-phase row); modality[i]: its modality flag (text phase only).  emit[i]
 * receives the token the request emits this step outside the head's audio
 * output (text token or bridging token), or -1.
 *   TEXT:   modality 0 -> stay, emit token0; modality 1 -> emit bridge[0] and
 *           go to BRIDGE (AUDIO if that was the only one; with none, emit
 *           token0 and go to AUDIO).
 *   BRIDGE: emit bridge[count]; after the last, AUDIO.
 *   AUDIO:  token0 == audio_end -> DRAIN (TEXT if drain_steps is 0).
 *   DRAIN:  after drain_steps steps, TEXT.
 * MCD_E_INVALID for bad sizes, an unknown phase or a count out of range (the
 * arrays are then unchanged from that request on). */
mcd_status mcd_phase_advance(const mcd_phase_desc *desc, int32_t n, uint8_t *phase,
                             int32_t *count, const int32_t *token0, const uint8_t *modality,
                             int32_t *emit);

/* ---- next-step input (Sec. 2.1, delay pattern) ----------------------------
 * The backbone's input for the next step aggregates the embeddings of the K
 * tokens each row emitted at this step, one per stream (each for its own
 * delayed frame).  Read as their sum:
 *   out[r][h] = sum_k E[k][row_k][h],   row_k = tokens[r][k], or V for pad_id;
 * TEXT rows (row_kind MCD_ROW_TEXT) take E_text[tokens[r][0]][h].  The sum is
 * formed in fp64 and rounded once, to nearest even, to the table type: the
 * exact sum rounded once whenever the values' exponents span at most 40 bits
 * (bf16) or 24 bits (fp32).  After mcd_head_step a Companion row holds its
 * Main row's tokens, so both get the same input. */
typedef struct {
  int32_t R;                 /* rows, >= 0 */
  int32_t H;                 /* embedding width, >= 1 */
  int32_t K;                 /* streams, 1..MCD_MAX_K */
  int32_t V;                 /* audio sub-vocabulary per stream, >= 1 */
  int32_t pad_id;            /* outside [0, V): selects row V of every stream's table */
  mcd_dtype dtype;           /* element type of E, E_text and out */
  const void *E;             /* [K][V + 1][H]; row V of stream k is its pad embedding */
  int32_t V_text;            /* rows of E_text, 0 if none */
  const void *E_text;        /* [V_text][H] or NULL */
  const uint8_t *row_kind;   /* [R] MCD_ROW_* of every row */
  const int32_t *tokens;     /* [R][K], e.g. the tokens_out of a step */
  void *out;                 /* [R][H] of dtype; must not overlap the inputs */
  void *workspace;           /* a step workspace (its status word), or NULL */
} mcd_next_input_args;

/* Launches on `stream`; no allocation, no synchronisation.  MCD_E_INVALID for
 * bad sizes, a pad_id inside [0, V), or E, E_text or out not 16-byte aligned.
 * A token outside [0, V) other than pad_id, a text id outside [0, V_text), or
 * a TEXT row without a text table makes that row's output zero and sets
 * MCD_DEV_BAD_TOKEN in the workspace status word (when a workspace is given). */
mcd_status mcd_next_input(const mcd_next_input_args *args, hipStream_t stream);

/* ---- log probabilities ------------------------------------------------------
 * How likely the given tokens were, under the softmax of each of K vectors of
 * logits of n rows: the head's scores (mcd_step_args.scores after a step: fp32,
 * its sampled rows in plan order, so token_row holds each one's batch row), or any
 * other logits (K = 1: a text head's).  For vector x of a row and stream, with
 * p = softmax(x):
 *   logprob:      log p of its token; 0 for pad_id (no choice)
 *   entropy:      - sum p log p, natural
 *   top_ids, top_logprobs: the T largest logits, ties to the lower id, and their
 *                 log p; -1 and -infinity past the ids that are not -infinity
 * A logit of -infinity has p = 0.  A vector with a NaN, with +infinity or with
 * nothing but -infinity has no distribution: NaN for all of it, ids -1 (0 for
 * pad_id all the same).  A token outside its stream other than pad_id, or a row of
 * tokens that is not there, gives NaN and sets MCD_DEV_BAD_TOKEN.  Sums and log
 * probabilities are in fp32; log p near 0 keeps its leading digits (terms of the sum
 * below 2^-126 are 0). */
#define MCD_MAX_TOP 32

typedef struct {
  int32_t n;                 /* rows, >= 0 */
  int32_t K;                 /* vectors of a row (streams), 1..MCD_MAX_K */
  int32_t V;                 /* logits of a vector (the largest), 1..2^19 */
  int32_t T;                 /* alternatives, 0..MCD_MAX_TOP */
  int32_t pad_id;            /* outside [0, V) */
  mcd_dtype dtype;           /* of logits */
  const void *logits;        /* [n][N]: vector k at column off_k, N = K V, or with V_stream
                                off_k and N its sums (as in mcd_head_desc) */
  int64_t logits_stride;     /* elements between rows, >= N */
  const int32_t *V_stream;   /* [host][K] logits of each vector (1..V), or NULL: V */
  int32_t token_rows;        /* rows of tokens */
  const int32_t *tokens;     /* [token_rows][K] */
  const int32_t *token_row;  /* [n] row of tokens of every row, or NULL: its index */
  float *logprob;            /* [n][K] */
  float *entropy;            /* [n][K] or NULL */
  int32_t *top_ids;          /* [n][K][T]; this or top_logprobs may be NULL */
  float *top_logprobs;       /* [n][K][T] */
  void *workspace;
  size_t workspace_bytes;    /* mcd_logprobs_workspace_bytes() */
} mcd_logprobs_args;

/* Workspace bytes for these sizes and smaller ones, 0 for invalid sizes; 256-byte
 * aligned, its first 256 bytes (the status word) zeroed once before first use.  A call
 * takes fewer than 2^26 - 3 vectors (n K) for V <= 1024, and fewer than 2^24 pieces
 * of 8192 logits otherwise (MCD_E_UNSUPPORTED). */
size_t mcd_logprobs_workspace_bytes(int32_t n, int32_t K, int32_t V, int32_t T);

/* Launches on `stream`; no allocation, no synchronisation.  The arrays written
 * overlap no other of the call.  The same inputs give the same bits. */
mcd_status mcd_logprobs(const mcd_logprobs_args *args, hipStream_t stream);

/* ---- paired co-scheduling (Sec. 2.4 input allocation and co-scheduling) ---
 * [host] A continuous-batching scheduler for CFG requests; no HIP calls.
 *   - Auto-allocation: a request with cfg_w > 1 becomes a unit of two rows, its
 *     Main row and a Companion row with a null prompt; other requests are
 *     one-row units.
 *   - Atomic unit: a unit is admitted with all its rows or not at all, holds
 *     them until it finishes, and its rows finish together.
 *   - Equal budget: in a step, each member of a pair is granted the same
 *     number of prompt tokens, c = min(floor(left / 2), the larger remaining
 *     prompt), and the pair is charged 2c whether or not the shorter prompt
 *     uses its share.
 *   - CFG only in the audio phase (Sec. 3.4): a decoding request first emits text_len
 *     text tokens (its Main row is a TEXT row of the head; the Companion is
 *     not run), then n_frames + drain_steps audio steps (Main COND and
 *     Companion UNCOND rows, or one SOLO row).  The Companion joins the audio
 *     phase with a copy of the Main sequence (a prefix-cache hit: no prompt
 *     tokens).
 * One step: mcd_sched_plan builds the batch (decode rows of running units
 * first, one token each; then prompt chunks of prefilling units in admission
 * order; then strict first-come admission while rows and budget remain), and
 * mcd_sched_commit applies it.  A unit whose prompts complete in a step
 * decodes from the next step on.  A scheduler is not thread-safe: one caller
 * at a time. */
typedef struct mcd_sched mcd_sched;

typedef struct {
  int32_t max_rows;          /* rows of the batch (Main and Companion rows), >= 1 */
  int32_t token_budget;      /* backbone tokens per step, >= max_rows */
  int32_t null_prompt_len;   /* prompt tokens of a Companion, >= 1 */
  int32_t drain_steps;       /* audio steps after the last frame (largest delay), >= 0 */
  int32_t max_requests;      /* requests held at once (waiting and running), >= 1 */
} mcd_sched_desc;

typedef struct {
  float cfg_w;               /* > 1: a pair with a Companion */
  int32_t prompt_len;        /* >= 1 */
  int32_t text_len;          /* text tokens before the audio, >= 0 */
  int32_t n_frames;          /* audio frames, >= 1 */
} mcd_sched_request;

/* The planned step; the arrays belong to the scheduler and stay valid until
 * the next mcd_sched_plan or mcd_sched_destroy. */
typedef struct {
  int32_t n_rows;            /* backbone rows of the step (rows with tokens) */
  const int32_t *row_req;    /* [n_rows] request id */
  const uint8_t *row_member; /* [n_rows] 0 Main, 1 Companion */
  const int32_t *row_slot;   /* [n_rows] the row's slot in [0, max_rows) */
  const int32_t *row_tokens; /* [n_rows] tokens this step (prompt chunk, or 1) */
  const int32_t *row_context;/* [n_rows] tokens already in the row's context */
  int32_t R;                 /* head rows: the decoding rows, in backbone order */
  const int32_t *head_row;   /* [R] backbone row of each head row */
  const int32_t *pair_map;   /* [R] head index of the partner, -1 */
  const uint8_t *row_kind;   /* [R] MCD_ROW_* */
  const float *cfg_w;        /* [R] */
  const int32_t *step;       /* [R] audio step (text rows: text step) */
  const int32_t *n_frames;   /* [R] */
  const int32_t *grid_slot;  /* [R] Main's slot for audio Main/SOLO rows, else -1 */
} mcd_sched_batch;

mcd_status mcd_sched_create(const mcd_sched_desc *desc, mcd_sched **out);
void mcd_sched_destroy(mcd_sched *s);
/* Queue a request; *id receives its id (0, 1, ... in submission order).
 * MCD_E_INVALID for bad fields, a pair on a one-row batch, or a full table. */
mcd_status mcd_sched_submit(mcd_sched *s, const mcd_sched_request *req, int32_t *id);
/* Plan the next step.  MCD_E_INVALID if the last planned step is not yet
 * committed. */
mcd_status mcd_sched_plan(mcd_sched *s, mcd_sched_batch *out);
/* Apply the planned step.  The ids of the requests that finished with it go
 * to finished[0 .. *n_finished) (at most cap; MCD_E_INVALID and nothing
 * applied if more would finish). */
mcd_status mcd_sched_commit(mcd_sched *s, int32_t *finished, int32_t cap, int32_t *n_finished);
/* Requests waiting and running. */
mcd_status mcd_sched_counts(const mcd_sched *s, int32_t *waiting, int32_t *running);

/* ---- 4-bit key/value cache ----------------------------------------------------
 * The cache between mcd_next_input and the head: what the backbone's attention
 * layers read for every row the scheduler plans (mcd_sched_batch: row_slot,
 * row_context, row_tokens).  One mcd_cache is one layer's.
 *
 * A slot is a sequence of positions 0, 1, ... in pages of MCD_CACHE_PAGE tokens:
 * position t lies in page table[slot][t / 64] at token t % 64.  Slots may share
 * pages (a Companion that joins with a copy of its Main row's prefix) as long as
 * no call writes to a shared page: with refs, such pages are left alone and
 * MCD_DEV_BAD_PAGE is set.  Keys are cached as attention multiplies
 * them (after any rotary embedding), so positions may later be dropped.
 *
 * A page holds, for each K/V head, mcd_cache_page_bytes(D) bytes (66 D + 128):
 * e2m1 codes of the keys and values (a sign and 0, 1/2, 1, 3/2, 2, 3, 4, 6) and
 * their scales.
 *   Keys: one power of two 2^(b - 127) for every token and 32 channels, the
 *   smallest with max|k| <= 7 * 2^(b - 127), b in 1..254; b = 255 where a key of
 *   the 32 is not finite: they read as NaN.
 *   Values: one bfloat16 for every token, max|v| * (1/6) in fp32 rounded to
 *   nearest even; NaN where a value of the token is not finite.
 *   Codes: the nearest multiple of the scale, ties to the even code, at most 6.
 * In bytes, with nb = D / 32:
 *   [0, 32 D)        key codes [token][channel], the lower channel in the low bits
 *   [32 D, 64 D)     value codes, 8 tokens of one channel to a 32-bit word: token
 *                    32 h + 16 j + 4 g + i in bits 4 (4 j + i) of word
 *                    [h][c / 4][16 g + m][c % 4], whose channel is
 *                    (m / 4) (D / 4) + 4 c + m % 4
 *   [64 D, 66 D)     key scales: token 16 t + m, block b at byte (m nb + b) 4 + t
 *   [66 D, + 128)    value scales: token 16 t + 4 g + i at bfloat16 16 g + 4 t + i
 *
 * The device arrays (table, slot, context, start, length) are read when the
 * kernels run, so a captured graph may be replayed with new contents.  A slot
 * outside [0, n_slots), a page id outside [0, n_pages), a length beyond the
 * table or beyond the call's max_* bounds sets MCD_DEV_BAD_PAGE in the workspace
 * status word; the positions concerned are skipped (not written, not seen). */
#define MCD_CACHE_PAGE 64

typedef struct {
  int32_t Hkv;               /* K/V heads, >= 1 */
  int32_t D;                 /* channels of a head: 64, 128 or 256 */
  int32_t n_slots, max_pages;/* rows and columns of table, >= 1 */
  int32_t n_pages;           /* pages, >= 1 */
  void *pages;               /* [n_pages][Hkv][mcd_cache_page_bytes(D)], 16-byte aligned */
  const int32_t *table;      /* [n_slots][max_pages] page ids; read up to a slot's length only */
  float *weight;             /* [n_slots][Hkv][max_pages * 64] attention weight every position
                                has received, or NULL */
  const int32_t *refs;       /* [n_pages] how many table entries hold each page
                                (mcd_cache_pages.refs): append, and evict into this cache,
                                write to no page that more than one holds; or NULL */
} mcd_cache;

/* The rows of a step and their new tokens; tokens of row r are start[r] ..
 * start[r + 1] - 1 of the packed token arrays, at positions context[r],
 * context[r] + 1, ... of its slot.  n_tokens, max_tokens and max_context are
 * bounds: the device arrays may hold fewer (a replayed step in which some rows
 * are idle, start[r] == start[r + 1]). */
typedef struct {
  int32_t R;                 /* rows, >= 0 */
  int32_t n_tokens;          /* tokens of all rows at most (start[R] <= n_tokens), >= 0 */
  int32_t max_tokens;        /* no row has more tokens, >= 0 */
  int32_t max_context;       /* no row has more positions (context + tokens), >= 0 */
  const int32_t *slot;       /* [R] slot of each row (no two alike), or NULL: its index */
  const int32_t *context;    /* [R] positions before the row's first token */
  const int32_t *start;      /* [R + 1], ascending from 0; NULL: one token in every row
                                (n_tokens == R, max_tokens == 1) */
} mcd_cache_rows;

size_t mcd_cache_page_bytes(int32_t D);   /* bytes of one page and head; 0 for another D */

/* Workspace bytes of mcd_cache_attend for rows of these bounds (0 for invalid
 * sizes); with a cache that has weights that is also room for the scores of
 * rows of few query heads, from which their received weight is added up (1 GiB
 * at most).  Enough for every step of no more rows, tokens, tokens of a row and
 * positions as well, with weight_out or without.  Attention that adds up no
 * weight may be given the cache with weight NULL, and needs no such room.  The
 * other calls need the 256-byte status word only.  The
 * workspace must be 256-byte aligned and zero-filled once before first use. */
size_t mcd_cache_workspace_bytes(const mcd_cache *cache, const mcd_cache_rows *rows, int32_t Hq);

/* Quantises the tokens' keys and values (k, v: [n_tokens][Hkv][D] of dtype, rows
 * k_stride and v_stride elements apart) into their pages and, when the cache has
 * weights, sets the new positions' weight to 0.  k, v and the strides in bytes
 * must be multiples of 16.  The pages must be in the table already. */
mcd_status mcd_cache_append(const mcd_cache *cache, const mcd_cache_rows *rows, mcd_dtype dtype,
                            const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                            void *workspace, size_t workspace_bytes, hipStream_t stream);

/* What the rows' positions stand for, rounded once to dtype: positions
 * context[r] + i into token start[r] + i of k and v (layout and alignment as in
 * mcd_cache_append).  Skipped positions are left as they are. */
mcd_status mcd_cache_read(const mcd_cache *cache, const mcd_cache_rows *rows, mcd_dtype dtype,
                          void *k, int64_t k_stride, void *v, int64_t v_stride,
                          void *workspace, size_t workspace_bytes, hipStream_t stream);

typedef struct {
  int32_t Hq;                /* query heads, a multiple of Hkv; head n reads K/V head n / (Hq / Hkv) */
  mcd_dtype dtype;           /* of q and out */
  float scale;               /* > 0, finite: logits are scale * q . k */
  const void *q;             /* [n_tokens][Hq][D], rows q_stride elements apart */
  int64_t q_stride;
  void *out;                 /* [n_tokens][Hq][D], rows out_stride elements apart; q itself, or
                                apart from it, and apart where there is weight_out */
  int64_t out_stride;
  float *lse;                /* [n_tokens][Hq] or NULL: log of the sum of exp(logits), natural;
                                -infinity for a token that sees nothing */
  float *weight_out;         /* NULL, or laid out as cache->weight (it, or apart from it): receives
                                cache->weight (0 where that is NULL) plus, at every position of
                                the rows' slots (of rows without a token too), the softmax weight
                                summed over the row's tokens and the query heads of the K/V head */
  void *workspace;
  size_t workspace_bytes;    /* mcd_cache_workspace_bytes() */
} mcd_cache_attend_args;

/* Attention of every new token over its row's cache, causal within the row:
 * token i of row r sees positions 0 .. context[r] + i (append first; context[r]
 * = length - 1 with one token attends over a cache that nothing was appended
 * to).  A token that sees no position (context[r] + i < 0) gets zeros, one that
 * sees a key or value that is not finite gets NaN.  Values may be as large as
 * fp32 holds (with logits below 2^29).  Logits,
 * softmax and sums are in fp32; softmax weights enter the product with the
 * values to 16 bits when dtype is MCD_BF16 and to 24 when it is MCD_F32.  The
 * same inputs give the same bits.  q, out and the strides in bytes
 * must be multiples of 16. */
mcd_status mcd_cache_attend(const mcd_cache *cache, const mcd_cache_rows *rows,
                            const mcd_cache_attend_args *args, hipStream_t stream);

/* Rows that begin with the same pages (several continuations of one prompt, several
 * questions about one document): groups of consecutive rows of a step.  Rows
 * start[g] .. start[g + 1] - 1 are group g's, and the table entries of the whole
 * pages of their first prefix[g] positions (prefix[g] / 64 of them) are the same for
 * all of them, rows without a token too: they are read from the group's first row.
 * Every row of a group that has tokens continues past those pages (context >=
 * prefix[g] / 64 * 64).  The groups hold all rows (start[0] = 0, start[n] = R); a
 * row that shares nothing is a group of its own.  The arrays are read when the kernels run, the max_* are bounds as in
 * mcd_cache_rows (n groups of max_rows rows of max_tokens hold n_tokens).  Where the
 * rows are few or the prefixes short, every row is read by itself, from its own
 * table entries, and the groups are not looked at.  Otherwise MCD_DEV_BAD_PAGE is
 * set past a bound, and for a row that breaks the above: positions past a bound are
 * not seen, a row outside the groups, short of its prefix or past max_rows sees
 * nothing. */
typedef struct {
  int32_t n;                 /* groups, 0..65535 */
  int32_t max_rows;          /* no group has more rows */
  int32_t max_prefix;        /* no prefix is longer */
  int32_t max_own;           /* no row has more positions past its group's shared pages */
  const int32_t *start;      /* [n + 1], ascending */
  const int32_t *prefix;     /* [n] */
} mcd_cache_groups;

/* Workspace bytes of mcd_cache_attend_shared for these bounds (0 for invalid sizes),
 * enough for every step of no more rows, tokens, groups and positions too; as
 * mcd_cache_attend's otherwise, which it also serves for a cache with weight NULL
 * (with weights that call asks for more, whether any are added up or not). */
size_t mcd_cache_shared_workspace_bytes(const mcd_cache *cache, const mcd_cache_rows *rows,
                                        const mcd_cache_groups *groups, int32_t Hq);

/* mcd_cache_attend of rows in groups, to the same accuracy and with the same refusals,
 * where a group's shared pages are read once for all of its rows.  weight_out is not
 * supported (MCD_E_UNSUPPORTED). */
mcd_status mcd_cache_attend_shared(const mcd_cache *cache, const mcd_cache_rows *rows,
                                   const mcd_cache_groups *groups,
                                   const mcd_cache_attend_args *args, hipStream_t stream);

/* Eviction by received weight.  Row r's source slot holds length[r] positions.
 * In every K/V head the `recent` newest stay and, of the others, the keep -
 * recent that received the most weight (from->weight; equal weights: the lower
 * position first; NaN below every number), in their order.  Their codes, scales
 * and weights become positions 0, 1, ... of slot r of `to`, whose pages must be
 * in its table and must not be pages of a source slot of the call (from and to
 * may share the page array).  A row of at most keep positions is copied whole,
 * so this also gives a Companion a copy of its own.
 *   kept: [R][Hkv][keep] the positions kept, -1 past the row's new length
 *   length_out: [R] min(length[r], keep)
 * The arrays written must overlap none that the call reads (length_out is not
 * length; where from and to share weights, no source slot is below R).
 * to->weight may be NULL; from->weight may be NULL when keep >= max_length. */
typedef struct {
  int32_t R;
  int32_t max_length;        /* no row is longer, >= 0 */
  int32_t keep, recent;      /* 0 <= recent <= keep, keep >= 1 */
  const int32_t *slot;       /* [R] source slots, or NULL: the row's index */
  const int32_t *length;     /* [R] */
  int32_t *kept;
  int32_t *length_out;
  void *workspace;
  size_t workspace_bytes;    /* the status word */
} mcd_cache_evict_args;

mcd_status mcd_cache_evict(const mcd_cache *from, const mcd_cache *to,
                           const mcd_cache_evict_args *args, hipStream_t stream);

/* ---- page tables on the GPU ---------------------------------------------------
 * A cache's table (mcd_cache.table), and how many of its entries hold each page.
 * The table may be one for several layers' caches.  A page that no entry holds is
 * free.  The calls below keep both, without the host: a captured step can take
 * pages, give them back, and let rows begin on the pages of another slot's prefix.
 *   entry:  a page id, or below 0: no page
 *   refs:   entries that hold the page
 * Calls on one table must not overlap in time.  Which pages a call hands out
 * depends on the table alone.  Conditions that only the device sees set bits of
 * the workspace's status word: a slot or page id out of range, a length below 0
 * or beyond the table, a page given back more often than counted
 * (MCD_DEV_BAD_PAGE, what it concerns is skipped); no free page left
 * (MCD_DEV_NO_PAGE). */
typedef struct {
  int32_t n_slots, max_pages;/* rows and columns of table, >= 1 */
  int32_t n_pages;           /* pages, >= 1 */
  int32_t *table;            /* [n_slots][max_pages] */
  int32_t *refs;             /* [n_pages] */
} mcd_cache_pages;

/* Workspace bytes of mcd_cache_reserve for R rows and fewer (0 for invalid sizes);
 * the other calls need the 256-byte status word only.  256-byte aligned, the
 * status word zeroed once before first use. */
size_t mcd_cache_pages_workspace_bytes(const mcd_cache_pages *pages, int32_t R);

/* refs from the table's entries, for a table that the host has written. */
mcd_status mcd_cache_count(const mcd_cache_pages *pages, void *workspace, size_t workspace_bytes,
                           hipStream_t stream);

/* Slot slot[r] (slot NULL: r) keeps the pages of its first length[r] positions
 * (length NULL: none) and gives back those of the columns past them.  A slot may
 * be named more than once (the shortest length holds).  A length below 0 or beyond
 * the table gives nothing back (MCD_DEV_BAD_PAGE). */
mcd_status mcd_cache_release(const mcd_cache_pages *pages, int32_t R, const int32_t *slot,
                             const int32_t *length, void *workspace, size_t workspace_bytes,
                             hipStream_t stream);

/* The whole pages of source[r]'s first length[r] positions (length[r] / 64 of them)
 * become slot[r]'s too (slot NULL: r).  Positions past the whole pages are the
 * caller's to append again, to a page of the slot's own.  An entry of slot[r] that
 * holds a page already keeps it, and a source without a page gives none
 * (MCD_DEV_BAD_PAGE): release first.  No source of a call is among its slots, and
 * no slot is named twice. */
mcd_status mcd_cache_share(const mcd_cache_pages *pages, int32_t R, const int32_t *slot,
                           const int32_t *source, const int32_t *length, void *workspace,
                           size_t workspace_bytes, hipStream_t stream);

/* Pages for the next step's tokens, and the step's rows.  Row r of slot[r] has
 * tokens[r] new tokens at positions context[r], context[r] + 1, ...: every column
 * of theirs without a page takes a free one, in the order of the rows and of their
 * positions the free pages in the order of their ids.  (A page that other entries
 * hold too is no place for a new token, as after a release to a length within it:
 * MCD_DEV_BAD_PAGE, and where is -1.  mcd_cache_append goes by the table, not by where:
 * give its cache the refs, or it writes there all the same.)
 *   start:    [R + 1] sums of tokens before each row, for mcd_cache_rows
 *   where:    [n_tokens] page * 64 + position % 64 of each packed token, -1: no page
 *   row, position: [n_tokens] of each packed token
 * Entries of where, row and position past start[R] are left as they were, and each
 * of the three may be NULL.  tokens[r] is taken within 0 .. max_tokens, and tokens past
 * n_tokens or positions from max_context on get no place (MCD_DEV_BAD_PAGE).  The
 * arrays written overlap no other of the call. */
typedef struct {
  int32_t R;                 /* rows, 0..65535 */
  int32_t n_tokens;          /* tokens of all rows at most, >= 0 */
  int32_t max_tokens;        /* of a row at most, 0..n_tokens */
  int32_t max_context;       /* positions of a row (context + tokens) at most */
  const int32_t *slot;       /* [R] slot of each row (no two alike), or NULL: its index */
  const int32_t *context;    /* [R] */
  const int32_t *tokens;     /* [R] */
  int32_t *start;
  int64_t *where;
  int32_t *row, *position;
  void *workspace;
  size_t workspace_bytes;    /* mcd_cache_pages_workspace_bytes() */
} mcd_cache_reserve_args;

mcd_status mcd_cache_reserve(const mcd_cache_pages *pages, const mcd_cache_reserve_args *args,
                             hipStream_t stream);

/* ---- device status ----------------------------------------------------------
 * Synchronises `stream`, returns the status word of the workspace in *code
 * (MCD_DEV_* bits) and clears it. */
mcd_status mcd_read_device_status(void *workspace, uint32_t *code, hipStream_t stream);

const char *mcd_status_string(mcd_status s);
const char *mcd_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* MCD_H */
