/*
 * dvi.h -- C-ABI of the GB300 (sm_103a) DVI library.
 *
 * DVI (Draft, Verify & Improve, arxiv 2510.05421) splits one decoder at layer
 * k (Sec. 3.1): layers 1..k plus a LoRA drafter head greedily propose k_spec
 * tokens; the frozen layers k+1..L plus the LM head verify the whole block in
 * one multi-query pass; the longest agreeing prefix is committed and the KV
 * cache rolled back past it (Sec. 3.3); the logged accept/reject tuples drive
 * an online KL->RL update of the drafter head (Sec. 3.4).
 *
 * Conventions shared by every call
 *  - Memory.  The caller owns all device memory: weights, the workspace and
 *    every input/output buffer.  The library never allocates or frees device
 *    memory.  A context keeps raw pointers to the weights and the workspace;
 *    both must outlive it.
 *  - Asynchrony.  Every call only enqueues work on the context's stream and
 *    returns.  Argument errors are reported synchronously through the return
 *    value.  Errors found on the device (non-finite logits or loss, KV or
 *    buffer capacity, a bounded wait that ran out) set bits of a device
 *    status word that dvi_get_stats() reads.
 *  - Threads.  A context is used by one host thread at a time.  No C++
 *    exception crosses this interface.
 *  - Layout.  Matrices are row-major with the output feature as the row
 *    (torch nn.Linear layout): W[out][in].  Token ids are int32.
 */
#ifndef DVI_H_
#define DVI_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct dvi_ctx dvi_ctx;           /* opaque, host-side */
typedef struct CUstream_st* dvi_stream;   /* a cudaStream_t */

typedef enum {
  DVI_OK = 0,
  DVI_ERR_INVALID_ARG = -1,
  DVI_ERR_CAPACITY = -2,
  DVI_ERR_NONFINITE = -3,
  DVI_ERR_CUDA = -4,
  DVI_ERR_UNIMPLEMENTED = -5,
  DVI_ERR_TIMEOUT = -6
} dvi_status;

/* bits of dvi_stats.device_status */
enum {
  DVI_DEV_NONFINITE = 1,   /* a NaN/Inf logit, or a non-finite update loss (update skipped) */
  DVI_DEV_TIMEOUT = 2,     /* a bounded device wait gave up */
  DVI_DEV_KV_FULL = 4,     /* a KV row fell past max_seq_len (row not written) */
  DVI_DEV_BAD_TOKEN = 8,   /* a token id outside [0, vocab) */
  DVI_DEV_LOG_FULL = 16    /* the replay buffer was full; tuples of a step were dropped */
};

typedef enum { DVI_F32 = 0, DVI_BF16 = 1 } dvi_dtype;

/* The decoder (Sec. 3.1; the backbone is Llama-style: pre-norm RMSNorm,
 * RoPE rotate-half, SwiGLU, GQA).  dtype is the storage type of the weight
 * matrices and the KV cache.  The residual stream, norm gains, LoRA factors
 * and logits are float32; with bf16, the activations that meet a weight
 * matrix in a tensor-core product (and the queries and probabilities of the
 * attention) enter it as a bf16 pair hi + lo, so the products carry the
 * rounding of the stored weights and cache only. */
typedef struct {
  int n_layers;       /* L */
  int d_model;        /* d, a multiple of 128 */
  int n_heads;        /* H_q */
  int n_kv_heads;     /* H_kv, divides H_q */
  int head_dim;       /* 64 or 128 */
  int d_ffn;          /* F */
  int vocab;          /* V */
  int split_k;        /* k: draft path = layers 1..k, verify path = k+1..L; 1 <= k <= L */
  int lora_rank;      /* r of A_s [V][r], B_s [r][d]; 0 = no LoRA */
  float lora_gamma;   /* gamma_s */
  float rms_eps;      /* 1e-5 */
  float rope_theta;   /* 10000 */
  int dtype;          /* dvi_dtype */
} dvi_model_config;

typedef struct {
  int batch;            /* B sequences decoded together */
  int k_spec;           /* K: drafted tokens per step, 1 <= K <= 16 (K + bonus <= 16) */
  int max_seq_len;      /* KV rows per sequence: prompt + generated + K */
  int log_steps;        /* decode steps the replay buffer holds between updates (U) */
  int head_mode;        /* 0: train LoRA A_s, B_s on the frozen W^(S); 1: train W^(S) itself
                           (the LoRA factors, if any, stay frozen; the workspace then holds
                           the Adam moments of W^(S), an f32 master copy of it when dtype is
                           bf16, and the gradient buffer: 12 (f32) or 16 (bf16) B per entry) */
  int max_prefill_chunk;/* rows per prefill pass, a multiple of 16: bf16 16..4096 (0 = 1024),
                           f32 16..128 (0 = 128).  A bf16 pass runs its projections on the
                           prefill kernel (128 token rows x 256 features per tile), so the
                           weights stream from HBM about once per pass. */
  int use_graphs;       /* capture the decode step in a CUDA graph on first use */
  int bonus;            /* 0: verify the K drafted rows and commit min(m+1, K) tokens (Sec. 3.3
                           emits y*_{n+m+1}, which the K verify rows hold only for m < K);
                           1: one more shallow pass on t~_K and a (K+1)-th verify row, so the
                           correction y*_{n+K+1} exists at m = K and every step commits m+1
                           tokens.  K + bonus <= 16. */
  int persistent;       /* 0: one kernel per projection.  1: bf16 decode passes of up to 64
                           rows run each layer's O, gate/up and down projections and the next
                           layer's QKV as one persistent launch (attention stays a launch of
                           its own); the context then needs every CTA of that launch resident
                           at once (two per SM) and ignores the flag when they do not fit.
                           Results differ from mode 0 in summation order only. */
  int chain_counters;   /* 0: each launch of a decode pass waits for its predecessor's whole
                           grid (programmatic dependent launch).  1: bf16 decode passes
                           (draft, verify, AR step; not with persistent = 1) chain their
                           projection, attention and head launches through per-launch
                           completion counters: each CTA adds 1 with release semantics
                           after its last write and the next launch polls the count with
                           acquire semantics (bounded: DVI_DEV_TIMEOUT).  Same arithmetic,
                           bit-identical results. */
  int megakernel;       /* 0: the draft passes run one kernel per projection, attention and
                           head.  1: bf16 contexts of at most 2 sequences with k <= 16 draft
                           layers (GQA groups of 1, 2, 4 or 8 -- 8 at head_dim 64 only --,
                           head_dim 64 or 128, d a multiple of 128)
                           run the whole draft phase -- every draft pass's k layers, the
                           drafter head with its argmax, the hand-off of h_k to the verify
                           rows -- as one persistent launch of one CTA per SM (Sec. 3.3
                           draft rollout), and the greedy AR step runs its first k layers
                           the same way, so the DVI stream stays bit-identical to AR.  Its
                           projections are row-split GEMVs on f32 activations and its
                           attention runs on warp MMAs (online softmax per warp); its phases
                           meet at tagged words and completion counters, all waits bounded.
                           Ignored when the
                           shape or the device does not allow it (stats: megakernel_ctas). */
} dvi_runtime_config;

typedef struct {
  const void* attn_norm;   /* [d] f32 */
  const void* wq;          /* [H_q*hd][d] */
  const void* wk;          /* [H_kv*hd][d] */
  const void* wv;          /* [H_kv*hd][d] */
  const void* wo;          /* [d][H_q*hd] */
  const void* ffn_norm;    /* [d] f32 */
  const void* w_gate;      /* [F][d] */
  const void* w_up;        /* [F][d] */
  const void* w_down;      /* [d][F] */
} dvi_layer_weights;

/* Device pointers, caller-owned, read for the whole life of the context.
 * final_norm and lora_b must be 16-byte aligned (dvi_create returns
 * DVI_ERR_INVALID_ARG otherwise), and so must every bf16 weight matrix.
 * draft_head (W^(S)) may alias lm_head (W^(V)) only when head_mode == 0.
 * lora_a / lora_b are updated in place by dvi_update_drafter (head_mode 0);
 * draft_head is updated in place in head_mode 1: with dtype bf16 the
 * optimizer steps an f32 master copy (taken from draft_head by dvi_create)
 * and writes its bf16 rounding back to draft_head after every update.
 * Everything else is frozen, and its first tiles may be read ahead of the
 * kernels that precede a call on the stream: what writes it must be complete
 * before dvi_create. */
typedef struct {
  const void* embed;              /* [V][d] */
  const dvi_layer_weights* layers;/* host array of L entries */
  const void* final_norm;         /* [d] f32 */
  const void* lm_head;            /* W^(V) [V][d], frozen */
  void* draft_head;               /* W^(S) [V][d] */
  float* lora_a;                  /* A_s [V][r] f32 */
  float* lora_b;                  /* B_s [r][d] f32 */
} dvi_weights;

/* Drafter-update hyper-parameters (Sec. 3.4).  objective: 0 = the KL->RL
 * schedule (L_fast, plus L_policy once t >= t_warmup), 1 = KL only, 2 = PG
 * only (REINFORCE), 3 = reward-masked CE only (the ablations of Sec. 4.3).
 * optimizer: 0 = bias-corrected Adam, 1 = SGD. */
typedef struct {
  int objective;
  int optimizer;
  float lr, beta1, beta2, adam_eps;
  float tau;                                  /* KD temperature */
  float lambda0, lambda_kl_min, lambda_pg_max;
  int t_warmup, t_ramp;
  float w_ce, w_ent, w_rl_max;
  float beta0, beta_min, t_beta;              /* beta(t) of L_policy */
  float baseline_rho;                         /* EMA constant of the reward baseline b */
  int keep_grad_w;                            /* head_mode 1: also store dL/dW^(S) in DVI_BUF_GRAD_W
                                                 (4 more bytes of traffic per W^(S) entry) */
} dvi_update_config;

typedef struct {
  int64_t steps;          /* draft_verify_commit calls */
  int64_t drafted;        /* sum over sequences of K per step */
  int64_t accepted;       /* sum of m (mean accepted length = accepted / (steps * B)) */
  int64_t committed;      /* tokens committed by decode steps */
  int64_t updates;        /* drafter updates applied */
  int64_t kernel_launches;/* kernels this context enqueued (graph replays count their nodes) */
  float last_loss;        /* objective of the last update */
  float last_kl, last_pg, last_ce, last_ent, last_rl, last_kl1;
  float last_accept_rate; /* accepted / logged rows of the last update's buffer */
  float baseline_b;       /* EMA reward baseline after the last update */
  int update_t;           /* completed updates t (the schedule's clock) */
  int device_status;      /* DVI_DEV_* bits */
  int persistent_ctas;    /* grid of the persistent projection launch (runtime option
                             persistent = 1 in effect), else 0 */
  int megakernel_ctas;    /* grid of the draft-phase megakernel (runtime option megakernel = 1
                             in effect), else 0 */
} dvi_stats;

/* Bytes of device workspace a context needs (KV caches, residual streams,
 * replay buffer, optimizer state, scratch).  0 for an invalid config. */
size_t dvi_workspace_bytes(const dvi_model_config* cfg, const dvi_runtime_config* rt);

/* "Load split model" (Sec. 3.1): validate the config, keep the weight
 * pointers, carve `workspace` (>= dvi_workspace_bytes, 256-byte aligned,
 * contents arbitrary) and enqueue its initialisation on `stream`.  Builds
 * the TMA descriptors of every weight matrix. */
dvi_status dvi_create(const dvi_model_config* cfg, const dvi_runtime_config* rt,
                      const dvi_weights* weights, void* workspace,
                      size_t workspace_bytes, dvi_stream stream, dvi_ctx** out);

/* Reset sequence `seq` and run its prompt (device int32 [n_tokens]) through
 * all L layers, filling the KV cache; the greedy next token (the first
 * generated token, committed) becomes the pending token of the sequence and
 * is written to d_first_token (device int32 [1]) when non-null. */
dvi_status dvi_prefill(dvi_ctx* ctx, int seq, const int32_t* d_tokens, int n_tokens,
                       int32_t* d_first_token);

/* One DVI step for all B sequences (Sec. 3.3): K greedy draft passes through
 * layers 1..k and the drafter head, one verify pass of the K (K+1 with the
 * bonus row) rows through layers k+1..L and the LM head, accept length m,
 * commit and rollback, and (when logging is on) the replay-buffer tuples of
 * positions 1..min(m+1, K).  Outputs (device, may be null): d_out_ids
 * [B][K + bonus] committed ids (the first d_n_committed[b] entries of row b
 * are valid: min(m+1, K), or m+1 with the bonus row), d_n_accepted [B] = m. */
dvi_status dvi_draft_verify_commit(dvi_ctx* ctx, int32_t* d_out_ids,
                                   int32_t* d_n_committed, int32_t* d_n_accepted);

/* Replay-buffer logging on (1, the default) or off (0) for later steps. */
dvi_status dvi_log(dvi_ctx* ctx, int enable);

/* One drafter-head update on every tuple logged since the last update
 * (Sec. 3.4), then clear the buffer and advance t.  With the per-row logit
 * gradients G [N][V] of the loss, head_mode 0 steps A_s and B_s with
 * dA = gamma G^T (U B^T) and dB = gamma (G A)^T U; head_mode 1 steps W^(S)
 * with dW = G^T U.  A non-finite loss skips the parameter step and sets
 * DVI_DEV_NONFINITE.  DVI_ERR_UNIMPLEMENTED in head_mode 0 without LoRA
 * factors (nothing to train). */
dvi_status dvi_update_drafter(dvi_ctx* ctx, const dvi_update_config* ucfg);

/* Baseline: one greedy autoregressive step of the full model for every
 * sequence (the speedup denominator of Sec. 4.1); commits one token each.
 * d_out_ids: device int32 [B] or null. */
dvi_status dvi_ar_step(dvi_ctx* ctx, int32_t* d_out_ids);

/* Synchronise the context's stream and copy the counters to *out. */
dvi_status dvi_get_stats(dvi_ctx* ctx, dvi_stats* out);

/* Message of the last synchronous error on this context ("" if none). */
const char* dvi_last_error(const dvi_ctx* ctx);

/* Free the host-side context (never the caller's device memory). */
dvi_status dvi_destroy(dvi_ctx* ctx);

/* Inspection of internal device buffers for tests and tools: sets *dptr and
 * *bytes for buffer `which` (DVI_BUF_*).  The memory stays owned by the
 * workspace. */
enum {
  DVI_BUF_LENS = 0,        /* int32 [B] committed KV length n per sequence */
  DVI_BUF_PENDING = 1,     /* int32 [B] pending (last committed) token */
  DVI_BUF_DRAFT_IDS = 2,   /* int32 [B][K+1]: pending, t~_1..t~_K of the last step */
  DVI_BUF_LOG_U = 3,       /* logged head inputs u = RMSNorm_final(h_k): f32 [cap][d]; bf16
                              [2][cap][d], a hi plane then a lo plane, u = hi + lo */
  DVI_BUF_LOG_LOGITS = 4,  /* f32 [cap][V] logged verifier logits */
  DVI_BUF_LOG_META = 5,    /* int32 [cap][6]: valid, a, r, i, prev_id, y* */
  DVI_BUF_GRAD_A = 6,      /* f32 [V][r] last dL/dA */
  DVI_BUF_GRAD_B = 7,      /* f32 [r][d] last dL/dB */
  DVI_BUF_X_DRAFT = 8,     /* f32 [B][d] residual stream of the draft pass */
  DVI_BUF_X_VERIFY = 9,    /* f32 [B*K][d] h_k rows, then h_L after verify */
  DVI_BUF_K_CACHE = 10,    /* dtype [L][B][H_kv][max_seq_len][hd] */
  DVI_BUF_V_CACHE = 11,
  DVI_BUF_STATUS = 12,     /* int32 device status word */
  DVI_BUF_GRAD_W = 13,     /* f32 [V][d] last dL/dW^(S) (head_mode 1, written when keep_grad_w) */
  DVI_BUF_Z = 14,          /* f32 [cap][V] drafter logits z of the buffer rows: logged by the drafter
                              head while drafting (head_mode 0; A, B and W^(S) change only at an
                              update, which empties the buffer), else recomputed by the update */
  DVI_BUF_COUNT
};
dvi_status dvi_debug_buffer(dvi_ctx* ctx, int which, void** dptr, size_t* bytes);

/* Device timing of the phases for measurement: while enabled, CUDA events
 * are recorded on the context's stream around the draft phase (0), the
 * verify phase (1) and the drafter update (2) of every call. */
dvi_status dvi_timing(dvi_ctx* ctx, int enable);

/* Synchronise the stream, then return per phase the summed milliseconds
 * ms[3] and the number of timed calls counts[3] since the last read. */
dvi_status dvi_get_timing(dvi_ctx* ctx, double* ms, int* counts);

/* Y[M][n_out] = X[M][K] . W[n_out][K]^T through the library's projection
 * kernel (tcgen05 for bf16, FP32 FMA for f32), with X float32 (for bf16
 * weights carried as a bf16 pair hi + lo, about 16 significant bits) and Y
 * float32, on the context's stream.  M <= 256.  d_w and d_x may come from the
 * work enqueued just before the call (another call's d_y, a trained W^(S)):
 * neither is read before that is done.
 * A building block exposed for tests of the projection kernel itself. */
dvi_status dvi_linear(dvi_ctx* ctx, const void* d_w, int n_out, int k_in,
                      const float* d_x, int m_rows, float* d_y);

/* Y[M][n_out] = X[M][K] . W[n_out][K]^T like dvi_linear, for callers that
 * cannot allocate device memory (code inside another framework's memory
 * pool or a fixed device-memory budget, plug-ins that are handed only their
 * input and output buffers).  It needs no context and allocates nothing:
 * the split-K scratch is a fixed array inside the library, 8 MiB of partial
 * sums plus 4096 tile counters, which every GPU that loads the library
 * holds until the process exits.  The paper has no counterpart to this
 * call; it is a deployment convenience.
 *  - dtype: DVI_BF16 (tcgen05 path; k_in % 8 == 0, 16-byte aligned d_w and
 *    d_x) or DVI_F32 (FP32 FMA path).  d_w [n_out][k_in] in that dtype,
 *    d_x [m_rows][k_in] f32, d_y [m_rows][n_out] f32, all device pointers
 *    owned by the caller, on the current device; 1 <= m_rows <= 256.  With
 *    bf16 weights the kernel carries each f32 input as a bf16 pair hi + lo
 *    (about 16 significant bits), so only the weights are rounded.
 *  - Every device of the process has its own scratch and its own kernel
 *    attributes, each set up on the first call with that device current.
 *  - Shapes whose split plan needs more scratch than the fixed array holds
 *    return DVI_ERR_CAPACITY (with a message on stderr); for example a
 *    4096 x 4096 weight fits for up to 32 rows.
 *  - The first call on a device looks up the scratch address for that
 *    device; make that first call before any stream capture.
 *  - d_w and d_x may come from the work enqueued on `stream` just before the
 *    call (another call's d_y, a W^(S) that an update steps): neither is read
 *    before that is done.
 *  - All calls on a device share the one scratch array, and it keeps the
 *    last call's contents (f32 calls whose splits meet there clear its
 *    counters at their start, bf16 calls use none): calls that overlap on
 *    the GPU, e.g. on two streams, race. */
dvi_status dvi_linear_noalloc(int dtype, const void* d_w, int n_out, int k_in, const float* d_x,
                              int m_rows, float* d_y, dvi_stream stream);

/* ---------------------------------------------------------------- paged 8-bit KV cache
 * Keys and values in pages of 8-bit codes with an f32 scale for each page
 * and KV head (value = code * scale), for programs that serve many sequences
 * of changing length.  The calls need no context: the caller owns the page
 * pool, the page tables and the lengths, all on the device, and every call
 * only enqueues work on `stream` (a graph may capture them).  A call's rows
 * of sequence b take the positions lens[b], lens[b] + 1, ..., so one pass is
 * dvi_paged_append, then dvi_paged_attend with the same batch; the caller
 * then advances lens by the rows it keeps.  Lowering a length rolls rows back.
 *
 * Pointers and row strides (in bytes) are multiples of 16.  Errors found on
 * the device set DVI_DEV_* bits of `status` (a device int32 the caller zeroes
 * and reads, or null). */
typedef enum { DVI_KV_INT8 = 0, DVI_KV_E4M3 = 1 } dvi_kv_format;

typedef struct {
  int n_pages;
  int n_kv_heads;       /* H_kv */
  int page_tokens;      /* P: 16, 32, 64 or 128 */
  int head_dim;         /* 64 or 128 */
  int format;           /* dvi_kv_format */
  void* k;              /* codes [n_pages][H_kv][P][head_dim]: int8, or e4m3 bytes */
  void* v;
  float* k_scale;       /* [n_pages][H_kv], positive where the page is in use */
  float* v_scale;
} dvi_paged_cache;

typedef struct {
  int n_seqs;                 /* 1..1024 */
  int max_pages;              /* columns of the page table */
  int n_rows;                 /* rows of the call, all sequences together */
  int max_rows;               /* no sequence has more (more are dropped: DVI_DEV_KV_FULL); the kernels are chosen by
                                 it where row_start is given: a close bound is a faster one */
  const int32_t* table;       /* [n_seqs][max_pages] pages of each sequence, in order; a negative entry is a
                                 page that is not held: its positions are not attended to (an entry past
                                 n_pages counts as one, DVI_DEV_KV_FULL) */
  const int32_t* lens;        /* [n_seqs] positions before the call's rows */
  const int32_t* row_start;   /* [n_seqs + 1] first row of each sequence, or null: n_rows / n_seqs each */
  int32_t* status;
} dvi_paged_batch;

/* Append n_rows rows of keys and values: k, v [n_rows][H_kv][head_dim] with
 * ld_k, ld_v elements from row to row (a slice of a projection's output).
 * rotary: [n_pos][rot_dim / 2] pairs (cos, sin) by which dims d and
 * d + rot_dim / 2 of the keys (d < rot_dim / 2; rot_dim a multiple of 16) are
 * rotated at their position, or null.  q (or null): the call's queries
 * [n_rows][n_heads][head_dim], rotated alike into q_out (which may be q;
 * rows of no sequence stay as they are).  dtype (dvi_dtype) is that of k, v, q
 * and q_out; the arithmetic is f32.
 *
 * A page's scale is the largest magnitude it has held since its first row was
 * written, over 127 (int8) or 448 (e4m3), at least 2^-80; when it grows, the
 * page's earlier codes are rounded again to the new scale.  NaN is stored as
 * 0 and an infinity as the largest code (DVI_DEV_NONFINITE), rows whose page
 * is not held are dropped (DVI_DEV_KV_FULL), positions past the rotary table
 * are not rotated (DVI_DEV_KV_FULL).  No two sequences of a call may append
 * to the same page. */
dvi_status dvi_paged_append(const dvi_paged_cache* cache, const dvi_paged_batch* batch, int dtype, const void* d_k,
                            int64_t ld_k, const void* d_v, int64_t ld_v, const float* d_rotary, int rot_dim,
                            int n_pos, const void* d_q, int64_t ld_q, void* d_q_out, int64_t ld_q_out, int n_heads,
                            dvi_stream stream);

/* Options of dvi_paged_attend: score = scale (q . k), then softcap * tanh(score
 * / softcap) where softcap > 0 (more than 1e-30 of scale), then + slopes[head]
 * (p_key - p_row) where slopes (device f32 [n_heads]) is given.  A row at
 * position p sees the held positions up to p, and with window > 0 only those
 * past p - window. */
typedef struct {
  int n_heads;          /* a multiple of H_kv: heads h G .. h G + G - 1 read KV head h */
  float scale;
  float softcap;
  int window;
  const float* slopes;
} dvi_paged_options;

/* Attention of the call's rows, already appended: q, o [n_rows][n_heads]
 * [head_dim] with ld_q, ld_o elements from row to row, in dtype.  Scores, their
 * maxima and all sums are f32; a softmax weight, its page's value scale in it,
 * enters the product with the codes rounded to f16 (by 2^-11 of it; f32 rows: as
 * two f16 numbers, 2^-21), one below 2^-19 of the row's largest by up to 2^-30 of
 * that.  A row
 * that sees nothing gets zeros, a row of no sequence (before the first row start,
 * from the last on, or dropped past max_rows) stays as it is.  workspace:
 * dvi_paged_workspace_bytes, 256-byte aligned, its first
 * dvi_paged_counter_bytes zeroed once before its first use (a call leaves them
 * zeroed; the rest may hold anything).  Calls that may overlap need one each,
 * the replays of a graph among them; those of one stream follow each other, also
 * from several host threads, and share one. */
dvi_status dvi_paged_attend(const dvi_paged_cache* cache, const dvi_paged_batch* batch,
                            const dvi_paged_options* options, int dtype, const void* d_q, int64_t ld_q, void* d_o,
                            int64_t ld_o, void* workspace, size_t workspace_bytes, dvi_stream stream);

/* Bytes of workspace that dvi_paged_attend needs on the current device for
 * any batch of this head_dim; 0 for one that it does not take. */
size_t dvi_paged_workspace_bytes(int head_dim);
size_t dvi_paged_counter_bytes(void);

/* An id of the capture that `stream` is in, 0 if it is in none: the calls of one
 * capture on one stream follow each other and may share a workspace, which is then
 * the graph's own. */
uint64_t dvi_paged_capture(dvi_stream stream);

/* Cached rows as values, in dtype: positions lens[b] .. of each sequence (the
 * batch's rows) to k_out, v_out [n_rows][H_kv][head_dim].  Rows of a page that
 * is not held are zeros, those of no sequence stay as they are. */
dvi_status dvi_paged_read(const dvi_paged_cache* cache, const dvi_paged_batch* batch, int dtype, void* d_k_out,
                          void* d_v_out, dvi_stream stream);

/* ---------------------------------------------------------------- page plans
 * The pages of a paged cache handed out on the device, from the lengths alone:
 * no copy to the host between the passes of a decoder, and a graph may capture
 * the call.  The pool is the caller's: a stack of the pages that nobody holds,
 * and for each of n_seqs slots its page table and how many pages it holds. */
typedef struct {
  int n_pages;          /* of the cache */
  int page_tokens;      /* P: 16, 32, 64 or 128 */
  int n_seqs;           /* 1..1024 */
  int max_pages;        /* columns of the page table */
  int32_t* stack;       /* [n_pages]: its first *n_free entries are the free pages, the last of them is taken first */
  int32_t* n_free;      /* [1] */
  int32_t* table;       /* [n_seqs][max_pages]: a slot's pages in order, -1 behind them */
  int32_t* held;        /* [n_seqs] pages of each slot */
  int32_t* status;      /* DVI_DEV_* bits, or null */
} dvi_page_pool;

/* Bring every slot b to the ceil((lens[b] + rows[b]) / P) pages that rows[b]
 * (d_rows, or rows_each of every slot where it is null) more positions behind
 * lens[b] need.  First the pages past that go back: slot after slot, in order of
 * the table, onto the stack; their table entries become -1.  Then pages that are
 * missing come off the stack's top, in the same order.  A slot whose missing
 * pages are not all there, or not all in its table, gets none of them
 * (DVI_DEV_KV_FULL) and the slots after it are served still.  With rows of 0 the
 * call gives back what a rejected block or (lens[b] = 0) a sequence that ended
 * held.  Negative lens and rows count as 0.
 *
 * d_row_start [n_seqs + 1] (or null): the first row of each slot when their rows
 * lie one after another, as dvi_paged_append and dvi_paged_attend take it.
 * d_slots, d_positions [n_rows] (or null): for each of those rows the place of
 * its position in the cache, page * P + position % P (-1 where its page is not
 * held), and the position; both -1 behind the last row.  Rows past n_rows have no
 * entry (DVI_DEV_KV_FULL).
 *
 * A pool out of order (a count or page out of its range) is not written past its
 * arrays; pages out of range are not handed out (DVI_DEV_KV_FULL). */
dvi_status dvi_paged_plan(const dvi_page_pool* pool, const int32_t* d_lens, const int32_t* d_rows, int rows_each,
                          int n_rows, int32_t* d_row_start, int64_t* d_slots, int32_t* d_positions,
                          dvi_stream stream);

/* ---------------------------------------------------------------- sampling
 * Speculative decoding with sampled tokens (the greedy step's counterpart for
 * programs that sample): probabilities of logits, and the verification of
 * drafted tokens against them.  No context; every call only enqueues work on
 * `stream`, allocates nothing and takes its random numbers as inputs.  Rows may
 * lie apart (ld elements from row to row) and need only their elements'
 * alignment.  vocab is at most 262144 (2^18).  d_status: as above, or null. */
typedef struct {
  const float* temperature;   /* device [n_rows], or null: temperature_all of every row */
  const int32_t* top_k;       /* device [n_rows], or null: top_k_all */
  const float* top_p;         /* device [n_rows], or null: top_p_all */
  float temperature_all;      /* >= 0 */
  int top_k_all;              /* >= 0 */
  float top_p_all;            /* >= 0 */
} dvi_sampling;

/* Probabilities of n_rows rows of logits x (in dtype, dvi_dtype): with tokens
 * ordered by logit, equal ones by index, and w_i = exp((x_i - max x) / T), the
 * first top_k tokens stay (0: all), of those the fewest first ones whose w sum to
 * top_p of theirs (at least one; 1 or more: all), and their w over the sum of what
 * stays are the probabilities; 0 elsewhere.  T = 0: 1 at the first of the largest
 * logits.  T counts as 2^-100 below that and as 2^100 above.  A row of -inf alone
 * gets zeros.
 *
 * Which tokens stay is decided on w as whole multiples of 2^-44 of the row's largest
 * (off by less than one of them, and by less than 2^-31 of themselves), so it does not depend on the
 * order of any sum.  NaN logits count as -inf and +inf as the largest finite number
 * (DVI_DEV_NONFINITE).  Of settings in device arrays, T that is negative or NaN counts
 * as 0, top_k below 0 as 0, top_p NaN as 1 (NaN: DVI_DEV_NONFINITE).  d_probs may be
 * d_logits itself (f32, the same ld); rows that overlap in another way are refused.
 *
 * Long rows with cuts are shared by CTAs that wait for each other's sums.  Where such a wait runs out (a second)
 * the whole row gets zeros (DVI_DEV_TIMEOUT). */
dvi_status dvi_token_probs(int dtype, const void* d_logits, int64_t ld_logits, int n_rows, int vocab,
                           const dvi_sampling* sampling, float* d_probs, int64_t ld_probs, int32_t* d_status,
                           dvi_stream stream);

typedef struct {
  int n_seqs;                 /* at most 65536 */
  int vocab;
  int n_drafts;               /* drafted tokens of all sequences together */
  int max_drafts;             /* no sequence has more (more are not looked at) */
  int bonus;                  /* 1: every sequence has a target row behind those of its drafts */
  const int32_t* draft_start; /* device [n_seqs + 1] first draft of each sequence, or null: n_drafts / n_seqs each */
  const int32_t* draft_ids;   /* device [n_drafts] */
  const float* u_accept;      /* device [n_drafts], uniform in [0, 1) */
  const float* u_token;       /* device [n_seqs], uniform in [0, 1) */
  int32_t* status;
} dvi_draft_batch;

/* Verify drafted tokens x_1 .. x_K of each sequence (Sec. 3.3 with sampling in
 * the argmax's place): with the target's probabilities p_j and the drafter's q_j
 * of the place of x_j, x_j is accepted while u_accept_j q_j(x_j) < p_j(x_j); m is
 * how many are before the first that is not.  Then one token more comes from
 * max(p_{m+1} - q_{m+1}, 0) (from p_{m+1} where that is zero everywhere), or at m =
 * K from the bonus row: the first token up to which the numbers sum to more than
 * u_token of their total.  Committed tokens are so distributed as the target's own.
 *
 * d_target: f32 rows, sequence b's first is row draft_start[b] + b * bonus, its
 * drafts' in order and then its bonus row.  d_draft: f32 rows, one a draft, or null
 * for tokens that were drafted greedily (q_j is 1 at x_j).  Numbers need not sum to
 * 1; a negative one counts as 0, NaN and infinities too (DVI_DEV_NONFINITE).  Without
 * drafts and with bonus = 1 the call samples a token of each row.
 *
 * d_out_ids [n_seqs][max_drafts + bonus]: x_1 .. x_m and the token, -1 behind them;
 * d_n_committed [n_seqs]: m + 1, or K at m = K without a bonus row; d_n_accepted
 * [n_seqs]: m.  A drafted id outside [0, vocab) is rejected (DVI_DEV_BAD_TOKEN) and
 * its row's q taken as it is (greedy: as 0).  Of draft_start, an entry outside [0,
 * n_drafts] counts as the nearest in it, one below its sequence's first as that
 * (DVI_DEV_BAD_TOKEN).  A row that is zero everywhere gives no token
 * (DVI_DEV_NONFINITE): n_committed is m. */
dvi_status dvi_verify_drafts(const dvi_draft_batch* batch, const float* d_target, int64_t ld_target,
                             const float* d_draft, int64_t ld_draft, int32_t* d_out_ids, int32_t* d_n_committed,
                             int32_t* d_n_accepted, dvi_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* DVI_H_ */
