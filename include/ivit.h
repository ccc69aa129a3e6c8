/*
 * ivit -- incremental ViT encoding of streaming camera frames on one GB300 (sm_103a).
 *
 * The library implements temporal token reuse (Sec. III-B of "Reducing Temporal
 * Redundancy for Efficient Vision-Language-Action Inference"): a frame is encoded
 * in full once (the paper's "odd chunk"); every later frame re-encodes only the
 * tokens whose patch embedding changed (Eq. 3 score, threshold or top-k selection),
 * with their queries attending over all tokens and the other tokens' per-layer K/V
 * read from a resident cache (Eq. 4-5); reused tokens keep their cached outputs.
 *
 * Conventions for every entry point:
 *  - Return value: IVIT_OK (0) or a negative IVIT_ERR_* code.  Nothing throws or
 *    aborts across the ABI; ivit_last_error() describes the last failure.
 *  - Device pointers ("_dev") are caller-owned CUDA global memory on the device the
 *    handle was created on; host pointers ("_host") are caller-owned host memory.
 *    The library never frees caller memory.  All work is enqueued on the caller's
 *    cudaStream_t (passed as void*, NULL = legacy default stream) and is
 *    asynchronous: outputs are valid once that stream has reached the call.
 *  - A handle owns the weights (copied at create), every per-view cache and all
 *    workspaces.  One handle may be used from one host thread at a time; calls on
 *    one handle must be ordered on one stream (or explicitly synchronised).
 *  - Shapes: S = n_streams camera streams, V = n_views views each, SV = S*V
 *    independent views (each with its own caches), N = (img_h/patch)*(img_w/patch)
 *    tokens per view, D = dim, L = depth, F = mlp_dim.
 */
#ifndef IVIT_H
#define IVIT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define IVIT_OK 0
#define IVIT_ERR_ARG (-1)      /* null handle/pointer, bad enum, out-of-range index */
#define IVIT_ERR_SHAPE (-2)    /* configuration the kernels do not support */
#define IVIT_ERR_OOM (-3)      /* device allocation failed */
#define IVIT_ERR_CUDA (-4)     /* a CUDA runtime/driver call failed */
#define IVIT_ERR_DEVICE (-5)   /* a kernel reported an error (bounded wait expired) */

#define IVIT_GELU_TANH 0       /* 0.5x(1+tanh(sqrt(2/pi)(x+0.044715x^3))) (SigLIP) */
#define IVIT_GELU_ERF 1        /* 0.5x(1+erf(x/sqrt 2)) (ViT) */
#define IVIT_SEL_THRESHOLD 0   /* update token i iff sim(i) < threshold (strict) */
#define IVIT_SEL_TOPK 1        /* update the topk lowest sims, ties by lower index */
#define IVIT_REF_PREV_FRAME 0  /* reference = previous frame's embeddings (all tokens) */
#define IVIT_REF_LAST_REFRESH 1 /* reference of token i updated only when i is updated */
#define IVIT_SCORE_EMBED 0     /* Eq. 3 on patch embeddings (before position embedding) */
#define IVIT_SCORE_KEY0 1      /* Eq. 3 as printed: first-layer keys W_K LN1(e+pos) + b_K */
#define IVIT_SCHED_INCREMENTAL 0 /* every ivit_encode_incremental call is incremental */
#define IVIT_SCHED_ODD_EVEN 1  /* odd calls encode in full, even calls incrementally */
#define IVIT_MLP_UPDATED 0     /* every block runs on the updated tokens only */
#define IVIT_MLP_ALL 1         /* attention on the updated tokens, residual + MLP on all */

/* Encoder + selection configuration.
 * Supported by the kernels: patch >= 1 dividing img_h and img_w; N <= 1024;
 * dim % 64 == 0, dim <= 2048, heads dividing dim with head_dim = dim/heads a multiple of 8,
 * at most 128; mlp_dim % 8 == 0; SV <= 4096. */
typedef struct ivit_config {
  int32_t img_h, img_w;  /* frame size in pixels */
  int32_t patch;         /* patch edge P; patch k-vector is P*P*3 (HWC order) */
  int32_t dim;           /* D */
  int32_t depth;         /* L transformer blocks (pre-LN) */
  int32_t heads;         /* H */
  int32_t mlp_dim;       /* F */
  int32_t n_streams;     /* S */
  int32_t n_views;       /* V */
  float ln_eps;          /* layer-norm epsilon (1e-6) */
  int32_t gelu;          /* IVIT_GELU_* */
  int32_t select_mode;   /* IVIT_SEL_* */
  float threshold;       /* IVIT_SEL_THRESHOLD: refresh where sim < threshold */
  int32_t topk;          /* IVIT_SEL_TOPK: tokens refreshed per view, clamped to [0, N] */
  int32_t ref_mode;      /* IVIT_REF_* */
  int32_t score_source;  /* IVIT_SCORE_*: what Eq. 3's cosine compares (Sec. III-B) */
  int32_t schedule;      /* IVIT_SCHED_*: odd/even chunking of Sec. III-B, or none */
  int32_t mlp_tokens;    /* IVIT_MLP_*: which tokens go through the residual addition and
                            the MLP after attention (Sec. III-B, the passage after Eq. 5).
                            IVIT_MLP_ALL keeps every token's attention-block output
                            W_o O + b_o per layer (fp32 [L][SV][N][D]); reused tokens take
                            theirs from that cache, every token runs LN2 + MLP and the
                            final LN, and every output token is recomputed. */
} ivit_config;

typedef struct ivit_handle ivit_handle;

/* Number of bf16 elements of the weight buffer for `cfg`, 0 if cfg is invalid.
 * Layout (row-major tensors, back to back):
 *   W_pe[D][P*P*3] (column k = (ky*P+kx)*3+c, applied to pixel-128), b_pe[D], pos[N][D],
 *   per layer: ln1_g[D] ln1_b[D] W_qkv[3D][D] b_qkv[3D] W_o[D][D] b_o[D]
 *              ln2_g[D] ln2_b[D] W_1[F][D] b_1[F] W_2[D][F] b_2[D],
 *   lnf_g[D] lnf_b[D].
 * W_qkv rows: query block, key block, value block; head h owns rows h*dh..h*dh+dh-1
 * of each block (Eq. 4: Q = W_Q T, K = W_K T, V = W_V T). */
size_t ivit_weights_size(const ivit_config* cfg);

/* Creates a handle on the current CUDA device: validates cfg, copies the weights
 * (bf16 bit patterns, host memory, ivit_weights_size(cfg) elements) to the device,
 * allocates every cache and workspace, and marks every view cold.
 * On failure *out is NULL and the code says why. */
int ivit_create(const ivit_config* cfg, const uint16_t* weights_bf16_host,
                ivit_handle** out);

/* Full encode of one frame per view (the paper's full forward that seeds the
 * reference, Sec. III-B).  frames_dev: uint8 [SV][img_h][img_w][3], any byte address.
 * The kernels read frames and write tokens and counts at the caller's addresses; frames
 * at an odd address, a misaligned output (tokens 16 bytes, counts 4) and memory that is
 * not the handle's GPU's go through one more copy on `stream`.
 * tokens_out_dev: bf16 [SV][N][D] final tokens (after the final LN), or NULL.
 * Re-seeds every cache and reference and marks every view warm. */
int ivit_encode_full(ivit_handle* h, const uint8_t* frames_dev, uint16_t* tokens_out_dev,
                     void* stream);

/* Incremental encode (Sec. III-B, Eq. 3-5): scores every token's patch embedding, or
 * its first-layer key (score_source), against its reference (cosine, fp32), selects
 * the tokens to update per view, runs
 * every block on those tokens only (their queries attend over all N tokens of the
 * view, the others' K/V come from the cache), and returns all tokens: updated ones
 * recomputed, the rest from the final-token cache.  A cold view updates every token.
 * tokens_out_dev: bf16 [SV][N][D] or NULL.  changed_count_dev: int32 [SV] number of
 * updated tokens per view, or NULL.  No host synchronisation happens inside.  With
 * schedule = IVIT_SCHED_ODD_EVEN the 1st, 3rd, ... call encodes in full (count N).
 * With mlp_tokens = IVIT_MLP_ALL the blocks after attention run on every token (see
 * ivit_config). */
int ivit_encode_incremental(ivit_handle* h, const uint8_t* frames_dev,
                            uint16_t* tokens_out_dev, int32_t* changed_count_dev,
                            void* stream);

/* Copies the ascending updated-token list of view `sv` from the last encode call:
 * idx_dev int32 [N] (first *count entries valid), count_dev int32 [1] (either may be
 * NULL).  Enqueued on `stream`.  IVIT_ERR_ARG if sv is outside [0, SV). */
int ivit_get_changed(ivit_handle* h, int sv, int32_t* idx_dev, int32_t* count_dev,
                     void* stream);

/* Copies per-view state for inspection: which = 0 key cache of `layer`, 1 value cache
 * of `layer`, 2 final-token cache (all bf16 [SV][N][D]), 3 reference score vectors
 * (patch embeddings or first-layer keys, fp32 [SV][N][D]), 4 attention-block outputs of
 * `layer` (fp32 [SV][N][D], mlp_tokens = IVIT_MLP_ALL only).  dst_dev must hold that
 * many bytes.  IVIT_ERR_ARG for a NULL destination, an unknown `which` (4 without that
 * reading) or, for 0, 1 and 4, a layer outside [0, L). */
int ivit_get_cache(ivit_handle* h, int which, int layer, void* dst_dev, void* stream);

/* Marks the views of camera stream `stream_index` (all streams if -1) cold: the next
 * incremental call recomputes every token of those views.  Host-side only.
 * IVIT_ERR_ARG if stream_index is outside [-1, n_streams). */
int ivit_reset(ivit_handle* h, int stream_index);

/* Kernel timeline.  With enable != 0 every later call records, for each of its kernel
 * launches, the global time at which each CTA started its work (after the wait on the
 * previous kernel) and finished; the captured CUDA graphs are rebuilt with the
 * recording in them, so the calls still run as replayed graphs (enable = 0 rebuilds
 * them without it).  Allocates 16 KB of device memory per launch of a call on first use.
 * ivit_timeline_read synchronises `stream` and reads the last call: per kernel family
 * (index 0 tensor-core GEMMs, 1 attention, 2 layer norms, 3 patchify / score /
 * selection / gather / output copy) the sum over its launches of (last CTA end - first CTA start)
 * in ms and the number of launches (arrays of 4, either may be NULL), the algorithmic
 * bytes of the GEMM launches (weights + input rows + outputs + bias, with this call's
 * updated-row count), and the span from the first start to the last end in ms.  Only
 * the first 1024 CTAs of a launch record.  IVIT_ERR_ARG when timeline mode is off. */
int ivit_timeline(ivit_handle* h, int enable);
int ivit_timeline_read(ivit_handle* h, void* stream, double* family_ms, int64_t* family_launches,
                       double* gemm_bytes_total, double* span_ms);

/* Reads and clears the device error word (0 = none; nonzero = a kernel's bounded
 * wait expired, the kernel skipped its work and returned).  Synchronises `stream`. */
int ivit_device_status(ivit_handle* h, void* stream);

/* Execution paths: one kernel per operation, chained with programmatic dependent launch
 * and replayed as a CUDA graph, is what every call runs.  On request (environment
 * variable IVIT_PATH read at create): IVIT_PATH=persistent, every transformer block of a
 * call in one persistent cooperative kernel with grid barriers (at most 256 tokens per
 * view); IVIT_PATH=stream, the incremental calls without cold views in one cooperative
 * weight-streaming kernel that keeps each SM's share of the next weights in flight
 * through a shared-memory ring.  All give the same result within the bf16 rounding. */

/* Number of the library's kernel launches made by the last encode call. */
int64_t ivit_last_launch_count(const ivit_handle* h);

/* Releases the handle and every device buffer, CUDA graph and stream it owns (weights,
 * caches, workspaces).  The device memory is freed with cudaFree, which waits for work
 * in flight on the device; the caller must not use `h` from another thread meanwhile or
 * afterwards.  NULL does nothing. */
void ivit_destroy(ivit_handle* h);

/* Token selection that allocates nothing.  The paper has no counterpart: this entry
 * point exists for callers that cannot call cudaMalloc when they need the lists --
 * code enqueuing work while a stream is captured into a CUDA graph (allocation is not
 * permitted there), plugins whose host framework forbids allocation inside its enqueue
 * callback, and real-time loops that allocate only at start-up.
 *
 * It computes what the selection step of ivit_encode_incremental computes (cosine of
 * each token against its reference in fp32, then threshold or top-k), from embeddings
 * the caller holds: e_cur_dev and e_ref_dev fp32 [n_views][n_tok][dim], 16-byte
 * aligned (they are read with 128-bit loads).  Outputs, all caller-owned device memory,
 * 4-byte aligned: idx_out_dev int32 [n_views][n_tok] (ascending updated indices, then
 * -1), counts_out_dev int32 [n_views].  A NULL or misaligned pointer returns
 * IVIT_ERR_ARG before any device work.  Enqueued on `stream`; no handle.
 *
 * Its scratch (one fp32 score per token) is a file-scope device array of
 * IVIT_NOALLOC_MAX_TOKENS floats (256 KiB) that every GPU loading the library holds
 * until the process exits.  n_views * n_tok above that maximum returns IVIT_ERR_SHAPE
 * (message via ivit_last_error(NULL)); no cudaMalloc, cudaFree or allocating library
 * routine is ever called.  The first call on a device, with that device current, looks
 * up the array's device address (cudaGetSymbolAddress) and caches it: make that first
 * call before any stream capture.  cudaDeviceReset invalidates the cached address:
 * do not call this entry point on a device after resetting it in the same process.
 * All calls share the array; each call writes every
 * score it reads, so nothing carries over, but calls that overlap on the GPU (two
 * streams, or two threads) race on it and must be serialised by the caller. */
#define IVIT_NOALLOC_MAX_TOKENS 65536
int ivit_select_noalloc(const float* e_cur_dev, const float* e_ref_dev, int32_t n_views,
                        int32_t n_tok, int32_t dim, int32_t select_mode, float threshold,
                        int32_t topk, int32_t* idx_out_dev, int32_t* counts_out_dev,
                        void* stream);

/* The 2-step action combine of the flow-matching head (Sec. III-C, Eq. 9):
 *   xT[s][i] = x0[s][i] + alpha[s] v0[s][i] + beta[s] v7[s][i] + b[s][i]
 * for `batch` samples of `dim` action values (row-major [batch][dim], fp32, device
 * memory; alpha, beta fp32 [batch]; b may be NULL, read as zero).  v0 and v7 are the
 * solver's anchor velocities (first and eighth step) and (alpha, beta, b) the adaptor's
 * prediction, all computed by the caller: this library holds neither network.  Needs no
 * handle; enqueued on `stream`, no allocation.  IVIT_ERR_ARG for negative sizes, a
 * NULL required pointer or a pointer that is not 4-byte aligned (checked before any
 * device work); batch * dim == 0 does nothing.  128-bit accesses are used when the arrays
 * are 16-byte aligned, scalar ones otherwise. */
int ivit_action_combine(const float* x0_dev, const float* v0_dev, const float* v7_dev,
                        const float* alpha_dev, const float* beta_dev, const float* b_dev,
                        int32_t batch, int32_t dim, float* xT_dev, void* stream);

/* ------------------------------------------------------- language backbone
 * The operators that a policy's language backbone needs around the encoder's tokens: its
 * keys and values live in a cache of pages, its queries and keys are normalised per head
 * and rotated by positions of one or several axes, and a step answers with one token or a
 * tree of drafted tokens that is verified in one pass.  None needs a handle, allocates or
 * synchronises; all work is enqueued on `stream`; arrays named *_dev are device memory of
 * the current device.  Failures are described by ivit_last_error(NULL).
 *
 * A request's step: ivit_step_plan reserves pages for its new rows and gives their slots,
 * positions and tree masks; per layer ivit_qk_norm_rope turns the projections into queries
 * and keys (prompt rows go straight into the cache) and ivit_tree_attention lets the new
 * rows attend over the cached tokens and over each other; after the verification
 * ivit_kv_write puts the accepted rows of every layer into their slots.
 *
 * Slot s of a cache is token s % page_size of page s / page_size.  Rows of a call are the
 * new tokens of all requests back to back (cu_rows[i] .. cu_rows[i + 1] are request i's). */
#define IVIT_BF16 0
#define IVIT_FP16 1

/* Keys (and, in an array of its own with the same layout, values) of one layer: element d of
 * head h of token t of page p is at p * page_stride + t * token_stride + h * head_stride + d.
 * Supported: page_size a power of two up to 1024, n_pages * page_size < 2^31, head_dim a
 * multiple of 8 up to 256, kv_heads up to 256, strides multiples of 8 elements, arrays
 * 16-byte aligned. */
typedef struct ivit_cache_layout {
  int32_t n_pages, page_size, kv_heads, head_dim;
  int32_t dtype;         /* IVIT_BF16 or IVIT_FP16: the cache's type and that of the rows */
  int32_t reserved;      /* 0 */
  int64_t page_stride, token_stride, head_stride;  /* in elements */
} ivit_cache_layout;

/* Limits: n_req up to 4096, max_rows and max_pages up to 262144, page_size as above,
 * n_pages * page_size < 2^31, mask_words up to 32768. */
typedef struct ivit_plan_config {
  int32_t n_req;         /* requests of the step */
  int32_t max_rows;      /* rows that the row arrays have room for */
  int32_t max_pages;     /* columns of the block table */
  int32_t page_size;
  int32_t n_pages;       /* pages of the cache = places of the ring of free pages */
  int32_t mask_words;    /* 32-bit words of a row's tree mask, 0: no mask */
} ivit_plan_config;

/* Pages, slots, positions and tree masks of a step, from the requests' lengths.
 * In (int32): held_dev [n_req] tokens for which request i holds pages, base_dev [n_req]
 * tokens that it has in the cache, new_dev [n_req] rows that it adds; parent_dev [max_rows]
 * the row that a drafted row hangs on, counted from the request's first (-1, or anything
 * that is not an earlier row of the request: a root), or NULL: the rows are a run;
 * ring_dev [n_pages] the ids of the free pages, as a ring of which ring_in_dev[1] places
 * from ring_in_dev[0] on are filled; table_dev [n_req][max_pages] the block table.
 * A request needs pages for base + new tokens: what it lacks is taken from the ring's front
 * and entered in the table, what it holds beyond is put behind the ring's end (a finished
 * request has base = new = 0).  Pages that are returned are free from the next call on.
 * Out: table_dev and ring_dev in place (so a repeated call with the same inputs gives the
 * same result), ring_out_dev [2] (may not be ring_in_dev), cu_rows_dev [n_req + 1], and per
 * row: req_dev the request, slot_dev the slot of token base + j for the request's row j,
 * pos_dev base + depth in the tree (base + j without one), mask_dev [max_rows][mask_words]
 * with bit k set for the row itself and its ancestors (rows past 32 * mask_words have no
 * bit).  req_dev, pos_dev and mask_dev may be NULL.  Rows past the step's get -1, -1, 0, 0.
 * The new held lengths are base + new.
 * status_dev [1]: 0, or why the step was refused -- 1 too few free pages, 2 a request has
 * more pages than the table, 4 more rows than max_rows, 8 a negative length or an invalid
 * ring (one whose free pages and those that are returned are more than n_pages, too).  A refused step takes and returns no page, ring_out = ring_in, and every row is
 * marked as past the step's (cu_rows 0). */
int ivit_step_plan(const ivit_plan_config* cfg, const int32_t* held_dev, const int32_t* base_dev,
                   const int32_t* new_dev, const int32_t* parent_dev, int32_t* ring_dev,
                   const int32_t* ring_in_dev, int32_t* table_dev, int32_t* cu_rows_dev, int32_t* req_dev,
                   int32_t* slot_dev, int32_t* pos_dev, uint32_t* mask_dev, int32_t* ring_out_dev,
                   int32_t* status_dev, void* stream);

/* Norm and rotation of heads of head_dim values (a multiple of 8, up to 256), the first
 * rot_dim (a multiple of 8) of which are rotated; heads and kv_heads up to 256, up to 2^30 rows. */
typedef struct ivit_rope_config {
  int32_t heads, kv_heads, head_dim, rot_dim;
  int32_t n_axes;        /* axes of a position (1: text; 3: time, height, width), up to 4 */
  int32_t interleaved;   /* pairs (2f, 2f + 1) if 1, (f, f + rot_dim / 2) if 0 */
  int32_t dtype;         /* IVIT_BF16 or IVIT_FP16 */
  float eps;             /* of the norm, >= 0 */
} ivit_rope_config;

/* For every row and every head of q [n_rows][heads][head_dim] and k [n_rows][kv_heads][..]:
 *   y = x / sqrt(mean(x^2) + eps) * weight       (weight [head_dim]; NULL: y = x)
 *   (u, w) -> (u cos a - w sin a, w cos a + u sin a), a = pos[axis[f]][row] * freq[f]
 * for the pairs f = 0 .. rot_dim / 2 - 1; values past rot_dim are not rotated.  freq fp32 and
 * axis int32 (0 .. n_axes - 1; others count as 0) [rot_dim / 2]; pos int32, axis a of row r at
 * a * pos_stride + r (pos_stride 0: all axes share one position), exact up to 2^24 either way.
 * All arithmetic is fp32, rounded once.  The *_stride of a row array is the number of elements
 * from one row to the next (a multiple of 8; heads are contiguous in a row), so that q, k and v
 * can be parts of one projection's output.
 * q_out; k_out (or NULL); and with `cache` also k and v into the slots slot_dev [n_rows] of
 * k_cache_dev and v_cache_dev (slots outside the cache, as -1, are skipped; slots of a call
 * are distinct).  Without `cache`, v and the cache arguments are NULL.  q_out may be q and
 * k_out may be k.  Arrays 16-byte aligned (freq, axis, pos, slot 4). */
int ivit_qk_norm_rope(const ivit_rope_config* cfg, int32_t n_rows, const void* q_dev, int64_t q_stride,
                      const void* k_dev, int64_t k_stride, const void* v_dev, int64_t v_stride,
                      const void* q_weight_dev, const void* k_weight_dev, const int32_t* pos_dev,
                      int64_t pos_stride, const float* freq_dev, const int32_t* axis_dev, void* q_out_dev,
                      int64_t q_out_stride, void* k_out_dev, int64_t k_out_stride,
                      const ivit_cache_layout* cache, void* k_cache_dev, void* v_cache_dev,
                      const int32_t* slot_dev, void* stream);

/* Gradients of the above: from grad_q, grad_k (of q_out, k_out) and the inputs q, k to dq, dk
 * (which may be grad_q, grad_k, or q, k, with the same strides) and, where
 * there is a weight, dq_weight_dev, dk_weight_dev fp32 [head_dim] (or NULL), summed over rows
 * and heads in an order that depends on the sizes alone.  workspace_dev (needed for weight
 * gradients alone): 16-byte aligned, workspace_bytes at least
 * ivit_qk_norm_rope_backward_workspace(cfg) (which gives 0 for an invalid cfg), of no meaning
 * between calls; calls that overlap on the GPU need one each. */
size_t ivit_qk_norm_rope_backward_workspace(const ivit_rope_config* cfg);
int ivit_qk_norm_rope_backward(const ivit_rope_config* cfg, int32_t n_rows, const void* grad_q_dev,
                               int64_t grad_q_stride, const void* grad_k_dev, int64_t grad_k_stride,
                               const void* q_dev, int64_t q_stride, const void* k_dev, int64_t k_stride,
                               const void* q_weight_dev, const void* k_weight_dev, const int32_t* pos_dev,
                               int64_t pos_stride, const float* freq_dev, const int32_t* axis_dev,
                               void* dq_dev, int64_t dq_stride, void* dk_dev, int64_t dk_stride,
                               float* dq_weight_dev, float* dk_weight_dev, void* workspace_dev,
                               size_t workspace_bytes, void* stream);

#define IVIT_MASK_CAUSAL 0     /* a row sees itself and the request's rows before it */
#define IVIT_MASK_ALL 1        /* a row sees all of the request's rows */
#define IVIT_MASK_TREE 2       /* a row sees the rows whose bits are set in its mask */

/* Limits: n_req up to 4096, heads up to 256 and a multiple of the cache's kv_heads, max_new up
 * to 65536, max_pages * page_size < 2^31 - 2^20, mask_words up to 32768. */
typedef struct ivit_attention_config {
  int32_t n_req;
  int32_t heads;         /* query heads; head h reads key / value head h * kv_heads / heads */
  int32_t max_pages;     /* columns of the block table */
  int32_t max_new;       /* most new rows of a request (further ones are not computed) */
  int32_t mask_mode;     /* IVIT_MASK_* */
  int32_t mask_words;    /* IVIT_MASK_TREE: words of a mask row; rows past 32 * mask_words are unseen */
  float scale;           /* of the scores, > 0 (usually 1 / sqrt(head_dim)) */
} ivit_attention_config;

/* New rows over the cached tokens and over each other.  For row r of request i and head h:
 *   o = sum_j exp(scale q.k_j) v_j / sum_j exp(scale q.k_j),  lse = log sum_j exp(scale q.k_j)
 * over the request's len_dev[i] cached tokens (all of which a row sees) and the new rows that
 * the mask lets it see, whose keys and values are k_new, v_new [n_rows][kv_heads][head_dim]
 * (not read from the cache, so that drafts need no slots before they are accepted).  A row that
 * sees nothing gets o = 0, lse = -inf; keys whose scores are -inf take no part; what a row does
 * not see does not reach it, NaN and infinities included.  Sums and the softmax are fp32;
 * probabilities enter the product with V as sums of two 16-bit values up to 16 rows (new rows x heads of the
 * group) per key head, 32 on pages of fewer than 8 tokens, and as one 16-bit value above.
 * table_dev int32 [n_req][max_pages]; len_dev int32 [n_req] (more than the table holds counts as
 * that much, pages outside the cache read as zeros); cu_rows_dev int32 [n_req + 1];
 * mask_dev uint32 [n_rows][mask_words] for IVIT_MASK_TREE, else NULL; out [n_rows][heads]
 * [head_dim], lse_dev fp32 [n_rows][heads] or NULL.  Row strides as in ivit_qk_norm_rope, but
 * positive; rows that belong to no request are left as they are.  max_new is a bound that the
 * caller vouches for; it chooses the kernel (tcgen05 for more than 16 rows per key head, where
 * pages have at least 8 tokens and key heads at most 128 query heads).  workspace_dev: 16-byte aligned,
 * workspace_bytes at least ivit_tree_attention_workspace(cfg, cache) (0: invalid arguments), needs
 * no initialisation; calls that overlap on the GPU need one each.  Its first int32 is 0 after a
 * call, or not if one of the kernel's bounded waits expired (then outputs are not valid). */
size_t ivit_tree_attention_workspace(const ivit_attention_config* cfg, const ivit_cache_layout* cache);
int ivit_tree_attention(const ivit_attention_config* cfg, const ivit_cache_layout* cache, int32_t n_rows,
                        const void* q_dev, int64_t q_stride, const void* k_new_dev, int64_t k_new_stride,
                        const void* v_new_dev, int64_t v_new_stride, const void* k_cache_dev,
                        const void* v_cache_dev, const int32_t* table_dev, const int32_t* len_dev,
                        const int32_t* cu_rows_dev, const uint32_t* mask_dev, void* out_dev,
                        int64_t out_stride, float* lse_dev, void* workspace_dev, size_t workspace_bytes,
                        void* stream);

/* Row src_row_dev[i] of k and v ([n_layers][n_src][kv_heads][head_dim], row and layer strides in
 * elements, multiples of 8) into slot slot_dev[i] of every layer's cache (k_cache_dev,
 * v_cache_dev: layer l begins cache_layer_stride * l elements in), for i < n.  Entries whose row
 * is outside [0, n_src) or whose slot is outside the cache are skipped; slots of a call are
 * distinct. */
int ivit_kv_write(const ivit_cache_layout* cache, int32_t n_layers, int32_t n, int32_t n_src, const void* k_dev,
                  const void* v_dev, int64_t row_stride, int64_t layer_stride, const int32_t* src_row_dev,
                  const int32_t* slot_dev, void* k_cache_dev, void* v_cache_dev, int64_t cache_layer_stride,
                  void* stream);

/* ---- a cache of 8 bits
 * Half the bytes of a decoding step: keys and values as e4m3 codes, with one fp32 scale for each block
 * of `block` consecutive tokens of a page (tokens 0 .. block - 1, block .. 2 block - 1, ...) and head.  Code c of a
 * block with scale s stands for c * s.  Element d of head h of token t of page p is at p * page_stride +
 * t * token_stride + h * head_stride + d of an array of codes, the scale of that token's block at
 * ((p * (page_size / block) + t / block) * kv_heads + h) of an array of scales; keys and values have
 * arrays of their own of the same layout.  Supported: as for ivit_cache_layout, and block a power of two up to
 * page_size; codes' arrays 8-byte aligned, scales' 4-byte.  16-byte aligned arrays with strides and a head_dim that
 * are multiples of 16 take wider copies. */
typedef struct ivit_quantised_layout {
  int32_t n_pages, page_size, kv_heads, head_dim;
  int32_t dtype;         /* IVIT_BF16 or IVIT_FP16: the type of rows (not of the cache) */
  int32_t block;         /* tokens that share a scale */
  int64_t page_stride, token_stride, head_stride;  /* in bytes (= elements), multiples of 8 */
} ivit_quantised_layout;

/* ivit_kv_write for a cache of 8 bits: row src_row_dev[i] of k and v ([n_layers][n_src][kv_heads][head_dim], row and
 * layer strides in elements, multiples of 8) into slot slot_dev[i] of every layer's cache, for i < n; entries whose row is outside
 * [0, n_src) or whose slot is outside the cache are skipped; slots of the others are distinct, and those of one block lie
 * next to each other in the list, as those of ivit_step_plan do (skipped ones may be between, whatever slots they have).
 * At most 2^20 entries and 4096 layers.
 * Of a block that is written, tokens before the last written one stay, if they are not written themselves, and what lies
 * behind it is of no meaning from then on (a block whose first token is written with the rest behind it starts afresh, so
 * that a page's next owner finds no old scale).  The new scale is the smallest power of two from 2^-60 to 2^60 by which
 * the finite new values are at most 448, and not below the old scale where tokens stay; those are rounded again
 * if the scale grew (a power of two: exact but for codes that leave the normal range).  Codes are rounded to nearest even;
 * values that are not finite become NaN, finite ones beyond 448 * 2^60 the largest code.  A repeated call changes nothing.
 * Layer l's codes begin cache_layer_stride * l bytes in (a multiple of 8), its scales scale_layer_stride * l elements in. */
int ivit_kv_quantise(const ivit_quantised_layout* cache, int32_t n_layers, int32_t n, int32_t n_src, const void* k_dev,
                     const void* v_dev, int64_t row_stride, int64_t layer_stride, const int32_t* src_row_dev,
                     const int32_t* slot_dev, void* k_cache_dev, void* v_cache_dev, int64_t cache_layer_stride,
                     float* k_scale_dev, float* v_scale_dev, int64_t scale_layer_stride, void* stream);

/* Cached tokens back as rows: slot slot_dev[i] of every layer into row i of k and v ([n_layers][n][kv_heads][head_dim],
 * strides as above), code * scale rounded once to the rows' type, for i < n.  Rows whose slot is outside the cache
 * are left as they are. */
int ivit_kv_dequantise(const ivit_quantised_layout* cache, int32_t n_layers, int32_t n, const int32_t* slot_dev,
                       const void* k_cache_dev, const void* v_cache_dev, int64_t cache_layer_stride,
                       const float* k_scale_dev, const float* v_scale_dev, int64_t scale_layer_stride, void* k_dev,
                       void* v_dev, int64_t row_stride, int64_t layer_stride, void* stream);

/* ivit_tree_attention over a cache of 8 bits: the operation, arguments, limits and workspace rules are those given
 * there, with cached keys code * k_scale and values code * v_scale; new rows (q, k_new, v_new, out) are of the layout's
 * 16-bit type.  Scales other than ivit_kv_quantise's have to be within 2^-60 .. 2^60 (one that is not positive and
 * finite counts as 0 for keys and 2^-80 for values).  Of products of a key's probability and its block's scale of values,
 * those of 2^-126 of a row's largest and less may be left out of the sums, of 2^-34 and less of the product with V.  Codes enter the products as they are, as 16-bit values that hold them exactly; a
 * block's scale of keys multiplies their scores and one of values their probabilities, in fp32.  Up to 40 rows (new rows x heads of
 * the group) per key head, 24 for heads above 128, probabilities of cached keys enter the product with V as one fp16 value for bf16
 * rows and two for fp16 ones, above as one of the rows' type; those of new rows as two of that type or, above, one.
 * bf16 queries are scaled by powers of two to fp16 up to there (exact but for values 2^-28 of a row's largest and less).
 * Above 40 rows per key head (24 for heads above 128) it saves the cache's room, not time: ivit_tree_attention is faster there. */
size_t ivit_tree_attention_quantised_workspace(const ivit_attention_config* cfg, const ivit_quantised_layout* cache);
int ivit_tree_attention_quantised(const ivit_attention_config* cfg, const ivit_quantised_layout* cache, int32_t n_rows,
                                  const void* q_dev, int64_t q_stride, const void* k_new_dev, int64_t k_new_stride,
                                  const void* v_new_dev, int64_t v_new_stride, const void* k_cache_dev,
                                  const void* v_cache_dev, const float* k_scale_dev, const float* v_scale_dev,
                                  const int32_t* table_dev, const int32_t* len_dev, const int32_t* cu_rows_dev,
                                  const uint32_t* mask_dev, void* out_dev, int64_t out_stride, float* lse_dev,
                                  void* workspace_dev, size_t workspace_bytes, void* stream);

/* Limits: n_req up to 65536, vocab up to 2^24, max_new up to 1024. */
#define IVIT_FP32 2
typedef struct ivit_verify_config {
  int32_t n_req;
  int32_t vocab;
  int32_t max_new;       /* most rows of a request (further ones are not looked at: never accepted) */
  int32_t dtype;         /* of the logits: IVIT_BF16, IVIT_FP16 or IVIT_FP32 */
} ivit_verify_config;

/* Verification of drafted tokens against the target's probabilities, from given random numbers: tokens that are accepted
 * and the one that follows them are distributed as if the target had been sampled token by token.
 * Row r of a step is a token, token_dev[r], and the target's logits after it, logits_dev [n_rows][vocab]; rows of a
 * request lie back to back (cu_rows_dev [n_req + 1]), its first is the known token and is always accepted, the others
 * are drafts.  parent_dev [n_rows] says which row a draft hangs on, as in ivit_step_plan (NULL: a run); a draft that hangs on none is
 * never accepted.  draft_prob_dev fp32 [n_rows][vocab]: row r has the probabilities q from which the drafts that hang on row
 * r were drawn, independently of each other; NULL: drafts were not drawn (q is 1 at the draft's token).
 * temperature_dev fp32 [n_req]: the target is p = softmax(logits / temperature); 0 or less (or NaN), or NULL for
 * all requests: the first of the likeliest tokens has probability 1.
 * From the first row on, with w = p and W = 1: of the drafts that hang on the last accepted row, in their order, draft x in
 * row r is accepted if uniform_dev[r] * W * q(x) < w(x), and its row is the last accepted one then (w = p, W = 1);
 * else w loses what was tried, w = max(w - W q, 0) (without q: w(x) = 0), and W = sum(w).  When no draft is left, next_dev[i] is the
 * token with the largest w / noise among positive ones, the first of equals, where noise_dev fp32 [n_req][vocab] has exponential random numbers
 * (those that are not positive take no part).  If no w is left then w = p; if no token has a probability (no logit above
 * -inf; NaN counts as -inf) the next token is -1.  A token outside [0, vocab) is never accepted and changes nothing.
 * uniform_dev fp32 [n_rows], of [0, 1); it and noise_dev may be NULL if temperature_dev is.
 * Out: accepted_dev [n_req] the number of accepted rows (0 for a request without rows, whose next token is -1), next_dev [n_req],
 * and path_dev [n_rows]: at cu_rows[i] + j the j-th accepted row of request i, -1 past them, so that path_dev and
 * ivit_step_plan's slots are what ivit_kv_write and ivit_kv_quantise take; entries of no request are left as they are.
 * Row strides in elements, at least vocab (16-byte aligned rows take wider loads).  All arithmetic is fp32 (W without q: what is left
 * of the last sum over all tokens, made again when half of it or 32 drafts are gone); sums are made in an order that depends on the
 * sizes, on whether all rows are 16-byte aligned, and on the device's number of SMs, so that equal calls give equal results, and the
 * same values at another alignment may decide otherwise where a draft is within the sums' rounding of its border. */
int ivit_tree_verify(const ivit_verify_config* cfg, int32_t n_rows, const void* logits_dev, int64_t logits_stride,
                     const float* draft_prob_dev, int64_t draft_prob_stride, const int32_t* token_dev,
                     const int32_t* parent_dev, const int32_t* cu_rows_dev, const float* temperature_dev,
                     const float* uniform_dev, const float* noise_dev, int64_t noise_stride, int32_t* path_dev,
                     int32_t* accepted_dev, int32_t* next_dev, void* stream);

/* Message of the last failure on `h` (or of the last failed create if h is NULL). */
const char* ivit_last_error(const ivit_handle* h);

#ifdef __cplusplus
}
#endif
#endif /* IVIT_H */
