/*
 * libcas: multi-cartridge prefix attention for AMD Instinct MI355X (gfx950).
 *
 * One attention layer of a frozen LLM in which each query token attends over
 * a concatenation of trainable KV prefixes ("cartridges") followed by the
 * row's own tokens under causal masking, with the backward pass that returns
 * dQ and the dK/dV of every cartridge and of the self tokens.
 *
 * The operation (paper: Section "Cartridges at Scale (CAS) Training",
 * Background paragraph, for the cartridge as a trainable KV prefix whose keys
 * and values alone receive gradients; Section "Inference" for the
 * concatenation of several cartridges in order ahead of the prompt; the
 * Limitations paragraph "Cartridge KV position" for ordinary causal masking of
 * the tokens that follow; the Budget Manager and Pool rotation paragraphs for
 * cartridges that move between host memory and the GPU):
 *
 *   For batch row b, query head h, query position t and kv = h / group_size,
 *   the visible keys are, in order, every token of every segment of row b,
 *   then self tokens 0..t. With s_j = softmax_scale * q . k_j:
 *     LSE = ln sum_j exp(s_j),  P_j = exp(s_j - LSE),  O = sum_j P_j v_j.
 *   Backward, given dO:  D = dO . O,  dS_j = P_j (dO . v_j - D),
 *     dQ = scale * sum_j dS_j k_j,  dK_j += scale * dS_j q,  dV_j += P_j dO,
 *   summed over every query (all heads of the group) that sees key j.
 *
 * The attention takes keys and queries as given (post-RoPE): cas_rope and
 * cas_paged_append apply the positions before it. All calls are asynchronous on the caller's HIP stream; results are
 * valid once the stream reaches them.
 *
 * Thread safety: calls may be made from several host threads; the error
 * message is thread-local.
 */
#ifndef CAS_H_
#define CAS_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define CAS_ABI_VERSION 4

/* Bytes of the device scratch each GPU holds for cas_prefix_attn_fwd_noalloc. */
#define CAS_NOALLOC_SCRATCH_BYTES ((size_t)16 << 20)

typedef enum {
  CAS_OK = 0,
  CAS_ERR_INVALID_ARGUMENT = 1, /* bad pointer, size, shape, segment table or aliasing */
  CAS_ERR_UNSUPPORTED = 2,      /* valid but not implemented (head_dim, dtype, table size) */
  CAS_ERR_ALIGNMENT = 3,        /* pointer or stride not a multiple of 16 bytes */
  CAS_ERR_NOT_PINNED = 4,       /* staging source is pageable host memory */
  CAS_ERR_WORKSPACE = 5,        /* workspace NULL or smaller than the size query returned */
  CAS_ERR_HIP = 6,              /* a HIP runtime call failed; see cas_last_error_message */
  CAS_ERR_IO = 7,               /* a file operation of the pool's moment tier failed */
  CAS_ERR_PAGES = 8             /* a page table has fewer free pages than the call needs */
} cas_status_t;

typedef enum {
  CAS_DTYPE_BF16 = 0, /* bfloat16 tensors; MFMA in bf16 with fp32 accumulation */
  CAS_DTYPE_FP32 = 1  /* float32 tensors; MFMA in fp32 (no down-conversion anywhere) */
} cas_dtype_t;

/*
 * One cartridge block as seen by one batch row (one entry of the segment table).
 *
 * k, v:   device pointers. Element (token j, kv head h, channel c) lives at
 *         base + j*stride_tok + h*stride_head + c (in elements of the dtype).
 *         The channel stride is 1. Token-major [len, Hkv, d] and head-major
 *         [Hkv, len, d] storage, and padded token strides, are all expressible.
 * dk, dv: device pointers with the same strides, receiving the gradient
 *         (backward only; ignored by the forward). NULL means "do not return
 *         this gradient".
 * len:    tokens, >= 0. A zero-length entry is skipped and its pointers are
 *         not read.
 *
 * Entries with equal (k, v, len, stride_tok, stride_head) are the same
 * cartridge, referenced several times (by several rows, or twice in one row);
 * they must carry equal dk and dv, which then receive the SUM over all
 * references. Any other overlap between a gradient buffer and any tensor the
 * call reads or writes is rejected with CAS_ERR_INVALID_ARGUMENT.
 */
typedef struct {
  const void *k;
  const void *v;
  void *dk;
  void *dv;
  int64_t len;
  int64_t stride_tok;
  int64_t stride_head;
} cas_segment_t;

/*
 * Problem description, read only during the call (the host arrays may be
 * reused as soon as the call returns).
 *
 * Two query layouts. With q_offsets == NULL every batch row has q_len >= 1
 * query tokens (fixed-length batch). Otherwise the batch rows are packed
 * samples of different lengths (the training layout in which several
 * conversations, each with its own cartridges, share one token axis;
 * paper: Section "Training with Multiple Cartridges" and Eq. mixing):
 * q_offsets is a host array of batch+1 non-decreasing int32 with
 * q_offsets[0] == 0, row b owns tokens q_offsets[b] .. q_offsets[b+1]-1 of a
 * token axis of T = q_offsets[batch] >= 1 tokens, q_len must be 0, and each
 * row's self keys are its own tokens only (block-diagonal causal masking).
 * Rows may be empty. In both layouts let T be the token count (batch*q_len
 * when fixed) and Hq = num_kv_heads*group_size.
 *
 * Shapes (contiguous, in elements of dtype):
 *   q, o, d_o, dq:                    [T, Hq, head_dim]
 *   k_self, v_self, dk_self, dv_self: [T, num_kv_heads, head_dim]
 *   lse (always float32, natural log): [batch, Hq, q_len] (fixed) or [Hq, T] (packed)
 * (a fixed-length batch is [batch, q_len, ...] in these terms).
 * Query head h reads kv head h / group_size (contiguous GQA groups).
 * head_dim is 64 or 128. softmax_scale must be finite and > 0. T * Hq must
 * stay below 2^31.
 * seg_offsets is a host array of batch+1 non-decreasing int32 with
 * seg_offsets[0] == 0; row b uses segments[seg_offsets[b] .. seg_offsets[b+1]).
 * segments may be NULL when seg_offsets[batch] == 0.
 */
typedef struct {
  cas_dtype_t dtype;
  int32_t batch;
  int32_t q_len;
  int32_t num_kv_heads;
  int32_t group_size;
  int32_t head_dim;
  float softmax_scale;
  const cas_segment_t *segments;
  const int32_t *seg_offsets;
  const int32_t *q_offsets; /* NULL (fixed q_len per row) or batch+1 token offsets (packed) */
} cas_problem_t;

/*
 * Bytes of device workspace a forward (backward == 0) or backward
 * (backward != 0) call on this problem needs, written to *bytes. The size
 * depends on the problem, the current tuning (cas_set_tuning) and, through
 * the automatic key-axis splits, the compute-unit count of the current
 * device (the same on every whole MI355X): query it with the device current
 * that will run the call. Workspace is caller-owned, 256-byte aligned, and
 * may be reused by the next call once the stream has passed the previous
 * one. Besides the
 * segment tables and per-row statistics, a bf16 backward keeps a transposed
 * copy of q and d_o in it (about twice the bytes of q).
 */
cas_status_t cas_prefix_attn_workspace_size(const cas_problem_t *p, int backward, size_t *bytes);

/*
 * Forward (paper: Section "Inference", several cartridges concatenated in
 * order ahead of the prompt; Limitations, "Cartridge KV position", ordinary
 * causal masking of the tokens that follow): softmax attention of every
 * query over its row's segments in table order, then its own tokens 0..t.
 * Writes o (dtype) and, when lse != NULL, the row log-sum-exp lse
 * (float32, natural log). All tensors are device memory, 16-byte aligned
 * (lse 4-byte aligned). hip_stream is a hipStream_t (NULL = default stream).
 * Validation happens before anything is enqueued; on error nothing is
 * launched and the outputs are untouched.
 */
cas_status_t cas_prefix_attn_fwd(const cas_problem_t *p, const void *q, const void *k_self,
                                 const void *v_self, void *o, float *lse, void *workspace,
                                 size_t ws_bytes, void *hip_stream);

/*
 * Backward (paper: Section "Cartridges at Scale (CAS) Training", Background
 * paragraph: the model is frozen and only the cartridges' keys and values
 * are trained, so the gradient flows through the attention into every
 * referenced cartridge; a cartridge used several times gets the sum).
 * Backward of sum(d_o * o): consumes q, the self and segment K/V, and the o
 * and lse written by cas_prefix_attn_fwd on the same inputs, and OVERWRITES
 * dq, dk_self, dv_self and every non-NULL segments[i].dk / .dv (NULL outputs
 * are skipped). Gradients are returned in the input dtype; accumulation is in
 * fp32. Same pointer, alignment, stream and error rules as the forward.
 */
cas_status_t cas_prefix_attn_bwd(const cas_problem_t *p, const void *q, const void *k_self,
                                 const void *v_self, const void *o, const float *lse,
                                 const void *d_o, void *dq, void *dk_self, void *dv_self,
                                 void *workspace, size_t ws_bytes, void *hip_stream);

/*
 * The forward without any allocation, for callers that cannot allocate
 * (code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc). Same problem, tensors, results and error rules as
 * cas_prefix_attn_fwd, without the workspace arguments: the workspace is a
 * static device array of CAS_NOALLOC_SCRATCH_BYTES that the library holds on
 * every GPU it runs on until the process ends, and the launch tables reach it
 * as kernel arguments (no pinned staging buffer). The call allocates nothing:
 * no hipMalloc, hipHostMalloc, hipFree or event creation (the first call on a
 * device only looks up that device's scratch address).
 *
 * When the forward would split the key axis into more partials than the
 * scratch holds, fewer splits are used (the result changes only in rounding
 * order). A problem whose launch tables alone exceed the scratch returns
 * CAS_ERR_UNSUPPORTED before anything is enqueued.
 *
 * All calls on one GPU share its scratch: calls that may overlap on that GPU
 * (different streams without ordering, or several host threads) race and
 * give wrong results; calls ordered on one stream are safe. Nothing in the
 * scratch needs clearing between calls.
 */
cas_status_t cas_prefix_attn_fwd_noalloc(const cas_problem_t *p, const void *q, const void *k_self,
                                         const void *v_self, void *o, float *lse, void *hip_stream);

/*
 * Cartridge staging (paper: Budget Manager and Pool rotation paragraphs,
 * cartridges offloaded to host memory and moved back onto the GPU).
 * Enqueues n host->device copies on side_stream (a hipStream_t) and, when
 * done_event (a hipEvent_t) is non-NULL, records it after the last copy so a
 * compute stream can hipStreamWaitEvent on it. Every host_src must lie in
 * pinned (page-locked) host memory, else CAS_ERR_NOT_PINNED and nothing is
 * enqueued: a pageable copy would silently serialise with the host. The
 * caller keeps host_src alive and unmodified until the event completes.
 * Consecutive entries whose source and destination both continue the
 * previous entry's are moved as one transfer (list a pool's cartridges in
 * address order to get large transfers); copies run in the given order.
 */
typedef struct {
  const void *host_src;
  void *dev_dst;
  size_t bytes;
} cas_stage_copy_t;

cas_status_t cas_cartridge_stage(const cas_stage_copy_t *copies, int32_t n, void *side_stream,
                                 void *done_event);

/*
 * Optimizer step of the trainable cartridges (paper: Section "Optimization
 * Dynamics", paragraphs "Optimizer" and "Per-cartridge LR warmup"; the
 * hyperparameter table's Adam (FP32), per-cartridge warmup W_c = 20 and one
 * frozen token). Adam (Kingma and Ba, Algorithm 1) with fp32 moments on bf16
 * parameters, one fused launch over every listed cartridge's K and V.
 *
 * For each element x of k and v (and its gradient g from dk / dv), with
 * t = step + 1 and lr_c = lr * cas_adam_lr_scale(step, warmup_steps,
 * warmup_buckets):
 *   m1 = beta1 m1 + (1 - beta1) g;   m2 = beta2 m2 + (1 - beta2) g g
 *   x  = bf16_rne(x - lr_c (m1 / (1 - beta1^t)) / (sqrt(m2 / (1 - beta2^t)) + eps))
 * all in fp32 with one rounding per operation, in this order (1 - beta^t is
 * evaluated in double and rounded to fp32). The first frozen_tokens tokens
 * of each cartridge (the BOS token) are neither read nor written.
 *
 * k, v, dk, dv: bf16 device tensors with the strides of cas_segment_t
 *   (element (j, h, c) at base + j*stride_tok + h*stride_head + c).
 * m1_k, m2_k, m1_v, m2_v: fp32 device moments, contiguous
 *   [len, num_kv_heads, head_dim], zero before a cartridge's first step.
 * step: optimizer steps the cartridge has already received (the caller
 *   increments it after the call; moving a cartridge out of the GPU pool and
 *   back keeps its step count and moments).
 * Every pointer 16-byte aligned, strides multiples of 8 elements; parameters
 * may not overlap their gradients or moments, or another cartridge's
 * tensors. Validation happens before anything is enqueued; on error nothing
 * runs. The workspace holds the launch tables (size from
 * cas_cartridge_adam_workspace_size; reusable once the stream has passed).
 */
typedef struct {
  void *k;
  void *v;
  const void *dk;
  const void *dv;
  float *m1_k;
  float *m2_k;
  float *m1_v;
  float *m2_v;
  int64_t len;
  int64_t stride_tok;
  int64_t stride_head;
  int32_t step;
  int32_t frozen_tokens;
} cas_adam_cartridge_t;

typedef struct {
  float lr;               /* eta_t of the global schedule at this step, >= 0 */
  float beta1, beta2;     /* in [0, 1) */
  float eps;              /* > 0 */
  int32_t warmup_steps;   /* W_c; 0 disables the per-cartridge warmup */
  int32_t warmup_buckets; /* N_b >= 1 */
} cas_adam_config_t;

/*
 * Per-cartridge warmup factor (host only): min(1, step / warmup_steps)
 * rounded up to one of warmup_buckets levels 1/N_b, 2/N_b, ..., 1 (the first
 * level also for step 0), so at most N_b distinct learning rates occur in a
 * step. 1 when warmup_steps <= 0; NaN for warmup_buckets < 1 or step < 0.
 */
float cas_adam_lr_scale(int32_t step, int32_t warmup_steps, int32_t warmup_buckets);

cas_status_t cas_cartridge_adam_workspace_size(const cas_adam_cartridge_t *carts, int32_t n,
                                               int32_t num_kv_heads, int32_t head_dim,
                                               size_t *bytes);

cas_status_t cas_cartridge_adam(const cas_adam_cartridge_t *carts, int32_t n, int32_t num_kv_heads,
                                int32_t head_dim, const cas_adam_config_t *cfg, void *workspace,
                                size_t ws_bytes, void *hip_stream);

/*
 * Short-query / decode attention over paged cartridges (paper: Section
 * "Inference" and paragraph "Cartridge RAG": the top-k retrieved cartridges'
 * KV caches are concatenated ahead of the prompt; appendix on cartridge
 * sizes: cartridges are whole 16-token pages of the serving engine's paged
 * KV cache). Forward only.
 *
 * K and V live in a page pool: k_pages, v_pages are bf16 device tensors
 * [num_pages, page_size, num_kv_heads, head_dim], contiguous. Request b owns
 * kv_lens[b] keys, stored in the pages page_ids[page_offsets[b] ..
 * page_offsets[b+1]) in key order (ceil(kv_lens[b] / page_size) pages; the
 * last may be partly filled): typically the pages of its selected cartridges
 * (shared with other requests, never copied) followed by the pages of its
 * own prompt and generated tokens. Its n_b = q_offsets[b+1] - q_offsets[b]
 * queries (1 <= n_b <= kv_lens[b]; n_b = 1 for a decode step) are the last
 * n_b positions of that key sequence: query i sees keys 0 .. kv_lens[b] -
 * n_b + i (causal among the new tokens). q and o are [Tq, Hq, head_dim]
 * (Tq = q_offsets[batch]), lse is [Hq, Tq] fp32 (may be NULL); query head h
 * reads kv head h / group_size. page_size is 16, 32, 64 or 128; head_dim 64
 * or 128; page ids lie in [0, num_pages). The key axis of each request is
 * split over several workgroups when the requests alone would not fill the
 * GPU (partials merged by their LSE). Validation before anything is
 * enqueued; on error nothing runs and the outputs are untouched.
 */
typedef struct {
  int32_t batch;
  int32_t num_kv_heads;
  int32_t group_size;
  int32_t head_dim;
  float softmax_scale;
  int32_t page_size;
  int64_t num_pages;
  const int32_t *q_offsets;    /* host, batch+1 */
  const int32_t *kv_lens;      /* host, batch */
  const int32_t *page_offsets; /* host, batch+1 */
  const int32_t *page_ids;     /* host, page_offsets[batch] entries */
} cas_decode_problem_t;

/* Workspace bytes of a cas_paged_decode_fwd call (launch tables and the
 * partials), written to *bytes; like the prefix-attention query it depends on
 * the compute-unit count of the current device. Page runs that requests share
 * are streamed once, which takes a partial per request and run: with them the
 * size is larger. A workspace of that size also serves any other page ids with
 * the same counts and lengths: where it is too small for what they share, the
 * call streams every request's keys by themselves. */
cas_status_t cas_paged_decode_workspace_size(const cas_decode_problem_t *p, size_t *bytes);

/*
 * Launch plan of a paged decode call (host-side; no device access). For tests
 * and profiling tools. rows and work may be NULL; otherwise they receive the
 * plan's tables, 3 * info->num_rows and 9 * info->workgroups values (ask for
 * the counts first):
 *   rows: per query row of a segment of keys its row of q at KV head 0, the
 *         last key of the segment it sees, its first partial (-1: none, the
 *         result goes straight to o);
 *   work: per workgroup the segment's first entry of page_ids and key count,
 *         the last key every row sees, KV head, first and one past the last
 *         32-key tile, first row, row count, and which piece of its segment.
 */
typedef struct {
  int64_t key_tiles;        /* 32-key tiles streamed by all workgroups */
  int32_t workgroups;
  int32_t num_rows;
  int32_t row_blocks;       /* 16-row blocks of one workgroup (1 or 2) */
  int32_t max_partials;     /* most partials of one request (1: no merge) */
  int32_t shared_runs;      /* page runs streamed once for several readers */
  int32_t reserved;
  size_t ws_bytes;
} cas_decode_plan_info_t;

cas_status_t cas_paged_decode_plan_info(const cas_decode_problem_t *p, cas_decode_plan_info_t *info, int32_t *rows,
                                        int32_t *work);

cas_status_t cas_paged_decode_fwd(const cas_decode_problem_t *p, const void *q, const void *k_pages,
                                  const void *v_pages, void *o, float *lse, void *workspace,
                                  size_t ws_bytes, void *hip_stream);

/*
 * The same in two steps, so that a step's planning is done once for its size
 * and all its calls (the attention layers of a model share one set of tables):
 * create validates and plans for the current device and writes the workspace
 * bytes to *ws_bytes; run is cas_paged_decode_fwd of the planned problem, from
 * any thread and on any stream. The plan has copies of the problem's tables; runs
 * already enqueued do not need it.
 */
typedef struct cas_decode_plan cas_decode_plan_t;

cas_status_t cas_paged_decode_plan_create(const cas_decode_problem_t *p, cas_decode_plan_t **plan, size_t *ws_bytes);
cas_status_t cas_paged_decode_run(const cas_decode_plan_t *plan, const void *q, const void *k_pages,
                                  const void *v_pages, void *o, float *lse, void *workspace,
                                  size_t ws_bytes, void *hip_stream);
cas_status_t cas_paged_decode_plan_destroy(cas_decode_plan_t *plan);
/* Whether plan is one of problem p as its values and tables are now (1) or not (0). */
int32_t cas_paged_decode_plan_matches(const cas_decode_plan_t *plan, const cas_decode_problem_t *p);

/*
 * Rotary positions (paper: paragraph "Pool rotation", the queries' positions
 * are offset by the tokens of the active cartridges ahead of them; Su et al.
 * 2021 for the rotation). Of every head's first rotary_dim channels, pair i <
 * rotary_dim / 2 at position t is turned by the angle a = 2 pi t turns[i]:
 *   (x, y) -> scale (x cos a - y sin a, x sin a + y cos a).
 * The pair is channels (i, rotary_dim/2 + i) in the HALF layout and (2i, 2i+1)
 * in the INTERLEAVED one; the channels from rotary_dim on are copied. The
 * angle is taken modulo a turn in double precision with the exact product, so at any
 * int32 position it is that of the given turns (whose own rounding to doubles is up
 * to 2^-53 of the whole angle, 2.4e-7 at 2^31 radians); cos, sin and the products
 * are fp32, rounded once to the dtype.
 *
 * turns: device array of rotary_dim / 2 doubles, 8-byte aligned, which
 *   cas_rope_frequencies fills in host memory, or any others.
 */
typedef enum { CAS_ROPE_HALF = 0, CAS_ROPE_INTERLEAVED = 1 } cas_rope_layout_t;

typedef struct {
  int32_t layout;       /* cas_rope_layout_t */
  int32_t rotary_dim;   /* a multiple of 16, 16 .. head_dim */
  const double *turns;
  float scale;          /* finite and > 0: 1, or a long-context scaling's factor */
} cas_rope_t;

/*
 * Frequencies for long contexts, with f_i = base^(-2i / rotary_dim) radians
 * per position:
 *   NONE      f_i
 *   LINEAR    f_i / factor (Chen et al. 2023, position interpolation)
 *   NTK       f_i with base * factor^(rotary_dim / (rotary_dim - 2))
 *   BY_PARTS  (1 - w) f_i / factor + w f_i, where a pair that turns r times
 *             within original_len tokens has w = (r - low) / (high - low),
 *             clamped to [0, 1] (Peng et al. 2023, "NTK-by-parts")
 * Host only: writes f_i / (2 pi) to turns[0 .. rotary_dim / 2).
 */
typedef enum { CAS_ROPE_NONE = 0, CAS_ROPE_LINEAR = 1, CAS_ROPE_NTK = 2, CAS_ROPE_BY_PARTS = 3 } cas_rope_scaling_t;

cas_status_t cas_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double original_len,
                                  double low, double high, double *turns);

/*
 * One rotated tensor: x is read, y written, [tokens, heads, head_dim] with unit
 * channel stride (element (t, h, c) at base + t*stride_tok + h*stride_head +
 * c). y == x with equal strides rotates in place. Tokens and heads of x may
 * have stride 0 (one that several share); those of y are distinct.
 */
typedef struct {
  const void *x;
  void *y;
  int64_t x_stride_tok, x_stride_head;
  int64_t y_stride_tok, y_stride_head;
  int32_t heads;
} cas_rope_tensor_t;

/*
 * Rotates n (1 .. 4) tensors of the same tokens (a layer's queries and keys)
 * in one launch. dtype: a cas_dtype_t. positions: device array of `tokens` (at
 * most 2^24) int32 (any sign). inverse != 0 gives the gradient: the same with
 * -a, so that for y = R x and a gradient dy the call returns dx = R^T dy.
 * head_dim is 64 or 128; x and y are 16-byte aligned with strides of multiples of
 * 16 bytes. An output may overlap no other tensor of the call; rows or heads that
 * interleave (slices of one projection's output, [tokens, Hq + 2 Hkv, d] or
 * [tokens, heads, 3, d]) do not. Nothing is allocated and no workspace is used, so
 * the call can be captured into a HIP graph.
 */
cas_status_t cas_rope(const cas_rope_t *rope, int32_t dtype, int32_t head_dim, int64_t tokens, const int32_t *positions,
                      const cas_rope_tensor_t *tensors, int32_t n, int32_t inverse, void *hip_stream);

/*
 * Appending to the paged cache. The requests, pages and counts are those of
 * the paged attention (cas_decode_problem_t) with the new tokens counted in:
 * request b's n_b = q_offsets[b+1] - q_offsets[b] new tokens (0 allowed here)
 * are the last n_b of its kv_lens[b] keys, and the call writes them to those
 * places of its pages: token t of k and v, rows of [Tq, num_kv_heads, head_dim],
 * t counted over the requests. With a rope the keys are rotated on the way, by
 * the position that their request's first new token has in `starts` (host,
 * batch entries; NULL: its place among the keys) and the ones that follow;
 * with q and q_out the queries are too ([Tq, Hq, head_dim], q_out contiguous).
 * Every other row of the pools stays as it is. The values equal those that
 * cas_rope gives.
 *
 * A row that the call writes may not be a key of another request, or a key
 * twice in its own (pages of cartridges are shared by reference; a request
 * whose last page is shared needs a copy of it first): such tables are refused.
 * Strides as for cas_rope (16 bytes aligned). q may be NULL (no query is
 * rotated); rope may be NULL if q is. q_out == q is allowed where q is
 * contiguous. No workspace; nothing is allocated on the device, and the call
 * can be captured (a replay writes the same places).
 */
typedef struct {
  const void *k, *v;
  int64_t k_stride_tok, k_stride_head, v_stride_tok, v_stride_head;
  const void *q;
  int64_t q_stride_tok, q_stride_head;
  void *q_out;
  const int32_t *starts;
} cas_append_t;

/* In two steps, as with cas_paged_decode_plan_create: the plan (with copies of the tables) is checked once for all the
 * layers of a step. */
typedef struct cas_append_plan cas_append_plan_t;

cas_status_t cas_paged_append(const cas_decode_problem_t *p, const cas_rope_t *rope, const cas_append_t *t, void *k_pages,
                              void *v_pages, void *hip_stream);
cas_status_t cas_paged_append_plan_create(const cas_decode_problem_t *p, cas_append_plan_t **plan);
cas_status_t cas_paged_append_run(const cas_append_plan_t *plan, const cas_rope_t *rope, const cas_append_t *t, void *k_pages,
                                  void *v_pages, void *hip_stream);
int32_t cas_paged_append_plan_matches(const cas_append_plan_t *plan, const cas_decode_problem_t *p);
cas_status_t cas_paged_append_plan_destroy(cas_append_plan_t *plan);

/*
 * Attention of a chunk of new tokens over the paged cache: prompts that are
 * prefilled piece by piece behind their cartridges, and single decode tokens
 * mixed with them in one step (paper: Section "Inference", several cartridges
 * concatenated in order ahead of the prompt; ordinary causal masking of the
 * tokens that follow). The problem, tensors and results are those of
 * cas_paged_decode_fwd (the new tokens' K/V already in their pages:
 * cas_paged_append); requests without new tokens are allowed. That call streams
 * the keys once for every 32 rows (tokens x heads of a group) and is for steps
 * of a few tokens per request; this one takes up to 256 rows at a time on the
 * matrix cores. Requests of one new token next to each other whose pages are
 * shared go through that call's kernels. Rows of q and o behind the last
 * request's are neither read nor written; lse is [Hq, Tq]. Keys past a query's
 * own position do not reach it, whatever they and their values hold (NaN and
 * infinities included).
 *
 * A short problem needs no workspace: its size is 0 then, and NULL will do. Calls
 * that run at the same time need a workspace each. A call made while the launch
 * tables of sixteen before it have not reached the device yet may wait for one of
 * them, for 10 ms at most. Under stream capture the launch tables travel as kernel
 * arguments; a captured call uses its workspace at every replay, so graphs that may
 * run at the same time need one each, too.
 */
cas_status_t cas_paged_chunk_workspace_size(const cas_decode_problem_t *p, size_t *bytes);
cas_status_t cas_paged_chunk_fwd(const cas_decode_problem_t *p, const void *q, const void *k_pages, const void *v_pages,
                                 void *o, float *lse, void *workspace, size_t ws_bytes, void *hip_stream);

/* In two steps, as with cas_paged_decode_plan_create: planned once for a step's size and its layers. */
typedef struct cas_chunk_plan cas_chunk_plan_t;

cas_status_t cas_paged_chunk_plan_create(const cas_decode_problem_t *p, cas_chunk_plan_t **plan, size_t *ws_bytes);
cas_status_t cas_paged_chunk_run(const cas_chunk_plan_t *plan, const void *q, const void *k_pages, const void *v_pages,
                                 void *o, float *lse, void *workspace, size_t ws_bytes, void *hip_stream);
int32_t cas_paged_chunk_plan_matches(const cas_chunk_plan_t *plan, const cas_decode_problem_t *p);
cas_status_t cas_paged_chunk_plan_destroy(cas_chunk_plan_t *plan);

/*
 * A plan's launch table (host only; for tests and profiling tools). items may be
 * NULL; otherwise it receives 11 values per item: first token and token count of
 * the request, its key count, its first granule (16 key rows; counted over the
 * requests of the table, whole tiles of four each), the block's first row
 * (tokens x group heads), KV head, first and one past the last 64-key tile, the
 * partial that it writes (-1: the result), its workgroup's next item (-1: none),
 * and one past the block's last row. Workgroup i, in dispatch order, begins with item i.
 */
typedef struct {
  int32_t workgroups;
  int32_t items;
  int32_t partials;
  int32_t max_partials;   /* most of one block of rows (1: no merge) */
  int64_t key_tiles;      /* 64-key tiles walked by all workgroups */
  int32_t decode_parts;   /* runs of requests that the decode kernels take, and their new tokens */
  int32_t decode_tokens;
  size_t ws_bytes;
} cas_chunk_plan_info_t;

cas_status_t cas_paged_chunk_plan_info(const cas_chunk_plan_t *plan, cas_chunk_plan_info_t *info, int32_t *items);

/*
 * Pages of the cache. A page table says which pages of the paged cache (page_ids
 * of cas_decode_problem_t) hold whose keys: sequences are lists of pages with a
 * length, which share pages by reference (paper: Section "Inference" and
 * paragraph "Cartridge RAG", requests over the same retrieved cartridges; the
 * beams of a request over its prompt), and a page is free when no sequence has
 * it. Host only: what has to move on the GPU comes back as a list for
 * cas_pages_copy, which the caller enqueues before whatever writes or reads the
 * pages next, in the order of the calls.
 *
 * Sequences are named by ids that are not given out again. New pages are the
 * free ones with the lowest ids. Calls on one table must not overlap. On an error
 * the table stays as it was; CAS_ERR_PAGES: too few pages are free.
 */
typedef struct cas_page_table cas_page_table_t;

/* The first `rows` rows (tokens) of page src go to those of page dst. */
typedef struct {
  int32_t src, dst, rows;
} cas_page_copy_t;

typedef struct {
  int64_t sequences;
  int64_t pages_used;   /* by one sequence or more */
  int64_t pages_free;
  int64_t pages_end;    /* one past the highest page in use: a pool of that many pages holds everything */
} cas_page_table_info_t;

/* page_size is 16, 32, 64 or 128, num_pages in [1, 2^31). */
cas_status_t cas_page_table_create(int64_t num_pages, int32_t page_size, cas_page_table_t **table);
cas_status_t cas_page_table_destroy(cas_page_table_t *table);
cas_status_t cas_page_table_info(const cas_page_table_t *table, cas_page_table_info_t *info);

/* A new sequence of the keys of n others, one behind the other, by reference: none (an empty sequence), one (a fork of it,
 * whatever its length), or several (cartridges ahead of a prompt), each of which but the last fills whole pages. */
cas_status_t cas_page_table_add(cas_page_table_t *table, const int64_t *parts, int32_t n, int64_t *seq);
/* Room for counts[i] >= 0 more keys at the end of each of n different sequences. Where they begin in a page that another
 * sequence has, too, the sequence gets a page of its own for it and copies[] an entry (room for n of them). */
cas_status_t cas_page_table_extend(cas_page_table_t *table, const int64_t *seqs, int32_t n, const int32_t *counts,
                                   cas_page_copy_t *copies, int32_t *n_copies);
/* Each of n different sequences gets the keys that seqs[parents[i]] has before the call, by reference (beams that go on
 * from others). */
cas_status_t cas_page_table_reorder(cas_page_table_t *table, const int64_t *seqs, int32_t n, const int32_t *parents);
/* Leaves a sequence its first len keys. */
cas_status_t cas_page_table_truncate(cas_page_table_t *table, int64_t seq, int64_t len);
/* Removes n different sequences. */
cas_status_t cas_page_table_free(cas_page_table_t *table, const int64_t *seqs, int32_t n);
/* Moves at most `most` pages, highest first, to free ones below them, until the pages in use are the lowest ones. copies
 * (room for `most` entries) are the moves, of the rows that hold keys. Page lists from before the call are void. */
cas_status_t cas_page_table_compact(cas_page_table_t *table, int32_t most, cas_page_copy_t *copies, int32_t *n_copies);
/* The tables of cas_decode_problem_t for n sequences (one may come several times): kv_lens [n], page_offsets [n + 1], and
 * page_ids, unless NULL, of room for cap ids (ask for page_offsets first). */
cas_status_t cas_page_table_lists(const cas_page_table_t *table, const int64_t *seqs, int32_t n, int32_t *kv_lens,
                                  int32_t *page_offsets, int32_t *page_ids, int64_t cap);

/*
 * Copies rows of pages within each of n_pools pools (K and V of every layer): pools
 * are device pointers to [num_pages, page_size, row_bytes] bytes, contiguous,
 * 16-byte aligned, row_bytes a multiple of 16 (num_kv_heads * head_dim elements
 * of any type). All copies are made as if at once: a page that is written is named
 * once, and read by no copy of the call. Pages and rows that the list does not
 * name stay as they are; rows behind a copy's `rows` too.
 *
 * The copies are host memory, read during the call. Up to 240 travel as kernel
 * arguments. The list of more goes through a workspace of the size that
 * cas_pages_copy_workspace_size gives for n copies (0 up to 240, where NULL will
 * do; no larger from 65,536 on); calls that run at the same time need a workspace
 * each, as do captured graphs that may.
 */
cas_status_t cas_pages_copy_workspace_size(int32_t n, size_t *bytes);
cas_status_t cas_pages_copy(void *const *pools, int32_t n_pools, int64_t num_pages, int32_t page_size, int64_t row_bytes,
                            const cas_page_copy_t *copies, int32_t n, void *workspace, size_t ws_bytes, void *hip_stream);

/*
 * A step of beam search: of the candidates of a batch entry, every token after
 * every one of its beams, the k with the best scores. For beam i with the logits x,
 *   score(i, v) = scores[i] + (x_v - max x) - ln sum_w exp(x_w - max x).
 * A beam with finished[i] != 0 has one candidate, pad_token at the score that it
 * has, and its logits are not read. Every other candidate's score is -inf: those
 * of a finished beam, of tokens whose logit is -inf (that the caller rules out),
 * and of a beam without anything to choose from: one whose own score is not
 * finite, whose logits are all -inf, or among whose logits is a NaN or +inf (such a
 * beam leaves the search; the others of the batch entry go on).
 *
 * Candidates are ordered by their exact scores, equal ones by beam and then token,
 * lowest first. Those of one beam are ordered by its logits. Two beams' that sums in
 * 32 bits do not tell apart are compared with sums in 64, which do if their scores
 * differ by more than 2^-52 (vocab / 512 + 140) (1e-13 for 131,072 tokens) and a few
 * units of 64 bits of the scores; rows that are equal, or so but for a constant, have
 * equal sums.
 * out_scores are within 6e-6 of the exact ones, and rounded once. Should there be
 * fewer than k above -inf, the others follow in that order with the score -inf:
 * parents and tokens are always in range.
 *
 * logits: [batch, beams, vocab] bf16 or fp32, device memory, aligned to its type,
 *   rows row_stride >= vocab elements apart (any number: columns behind vocab are not read).
 * scores: [batch, beams] fp32: sums of the tokens' log-probabilities so far (a
 *   request's first step: 0 for one beam and -inf for the others).
 * finished: [batch, beams] bytes, or NULL: none is.
 * out_scores (fp32), out_parents (the beam, 0 .. beams - 1) and out_tokens
 *   (int32): [batch, k].
 * beams and k are at most 64, k at most beams * vocab, vocab at most 2^30, batch * beams
 * at most 2^20. Outputs may not overlap the inputs or each other. The workspace is
 * 16-byte aligned; calls that run at the same time need one each.
 */
typedef struct {
  int32_t dtype;        /* of the logits: a cas_dtype_t */
  int32_t batch;        /* >= 0 */
  int32_t beams;
  int32_t k;
  int64_t vocab;
  int64_t row_stride;
  int32_t pad_token;    /* in [0, vocab) */
} cas_beam_problem_t;

cas_status_t cas_beam_select_workspace_size(const cas_beam_problem_t *p, size_t *bytes);
cas_status_t cas_beam_select(const cas_beam_problem_t *p, const void *logits, const float *scores, const uint8_t *finished,
                             float *out_scores, int32_t *out_parents, int32_t *out_tokens, void *workspace, size_t ws_bytes,
                             void *hip_stream);

/*
 * States that are kept per beam (token histories, dense caches) follow the
 * surviving beams: for every batch entry b and j < beams_out,
 *   y[b, j] = x[b, parents[b, j]],
 * for 1 to 8 tensors in one launch. parents: device array [batch, beams_out] of
 * beams of the same batch entry, 0 .. beams_in - 1; a row with any other parent is
 * left as it was. A row is row_bytes bytes (0 allowed) in a row; strides are
 * bytes, of any alignment (16 is the fastest: a tensor whose addresses and strides
 * are multiples of 4 only takes twice as long, any other five times; the bytes of a
 * row behind its last 16 or 4 go one by one). beams_in and beams_out are at most
 * 64. y == x with equal strides and beams_in == beams_out reorders in place; any
 * other overlap is refused.
 */
typedef struct {
  const void *x;
  void *y;
  int64_t row_bytes;
  int64_t x_stride_batch, x_stride_beam, y_stride_batch, y_stride_beam;
} cas_beam_state_t;

cas_status_t cas_beam_reorder(const int32_t *parents, int32_t batch, int32_t beams_in, int32_t beams_out,
                              const cas_beam_state_t *states, int32_t n, void *hip_stream);

/*
 * Budget manager (paper: paragraphs "Budget Manager" and "Pool rotation";
 * hyperparameter table: budget B = 20, rotation interval R = 10, swap
 * fraction phi = 0.5, least-trained cartridges first, Adam moments of
 * CPU-resident cartridges offloaded to NVMe). The pool owns a pinned host
 * copy of every cartridge's bf16 K/V and step count, and B active device
 * slots, plus floor(phi * B) staging slots into which the next rotation's
 * cartridges are copied ahead of time on the pool's own stream while the
 * current ones train.
 *
 * The fp32 Adam moments of the cartridges that are not on the GPU live in
 * one of two tiers: pinned host memory next to their K/V (moment_dir NULL),
 * or a file on a local (NVMe) file system (moment_dir names its directory:
 * the pool creates an unnamed file there, removed when the pool is
 * destroyed or the process ends, and keeps in pinned memory only two sets
 * of floor(phi * B) (at least one) moment buffers for the cartridges in
 * transit). The file tier's reads and writes run on a pool thread: an
 * eviction's moments are written after their copy back has landed, and the
 * next admissions' moments are read and copied to the GPU ahead of the
 * rotation that admits them, overlapped with the training steps between
 * rotations.
 *
 * Rotation, after every R-th cas_pool_end_step: the n = min(floor(phi * B),
 * N - B) active cartridges with the most optimizer steps (ties: lower id)
 * are copied back to host (parameters and moments, after the compute
 * stream's work so far) and leave the active set; the prefetched cartridges,
 * the n offloaded ones with the fewest steps (ties: lower id), take their
 * place; then the next admissions are prefetched into the freed slots.
 * Offloaded cartridges receive no gradient. cas_pool_plan_rotation is that
 * policy on its own (host only).
 *
 * Use: create; fill the host copies (cas_pool_host_cartridge: pinned views,
 * moments zero, step 0); cas_pool_load; then per training step read the
 * active set (cas_pool_active: device views of K/V, their gradient buffers
 * dk/dv, moments and step counts, ready for cas_cartridge_adam) and call
 * cas_pool_end_step after the optimizer step. cas_pool_flush copies every
 * active cartridge back and waits, after which all host copies (and the
 * moment file) are current. Calls on one pool must not overlap; streams are
 * the caller's except the pool's own copy stream (default priority). A
 * failed file read or write of the moment tier is reported as CAS_ERR_IO by
 * the next call on the pool; the pool is then unusable except for destroy.
 */
typedef struct cas_pool cas_pool_t;

typedef struct {
  int32_t num_cartridges;   /* N >= 1 */
  const int64_t *lens;      /* host, N token counts (>= 1) */
  int32_t num_kv_heads;
  int32_t head_dim;         /* 64 or 128 */
  int32_t budget;           /* B, 1 <= B <= N */
  int32_t rotate_every;     /* R >= 1 */
  float swap_fraction;      /* phi in [0, 1] */
  int32_t frozen_tokens;    /* reported in the views (BOS: 1) */
  const char *moment_dir;   /* NULL: moments in pinned host memory; else the file tier's directory */
} cas_pool_config_t;

cas_status_t cas_pool_plan_rotation(const int32_t *steps, const uint8_t *active, int32_t n, int32_t budget,
                                    float swap_fraction, int32_t *evict, int32_t *admit, int32_t *n_swap);
cas_status_t cas_pool_create(const cas_pool_config_t *cfg, cas_pool_t **pool);
cas_status_t cas_pool_destroy(cas_pool_t *pool);
/* Pinned host views of cartridge cart: k, v, step and frozen tokens, and
 * with the host moment tier its moments (NULL with the file tier: use
 * cas_pool_read_moments). */
cas_status_t cas_pool_host_cartridge(cas_pool_t *pool, int32_t cart, cas_adam_cartridge_t *host_view);
cas_status_t cas_pool_load(cas_pool_t *pool, void *compute_stream);
cas_status_t cas_pool_active(cas_pool_t *pool, int32_t *cart_ids, cas_adam_cartridge_t *views, int32_t cap,
                             int32_t *n);
cas_status_t cas_pool_end_step(cas_pool_t *pool, void *compute_stream);
cas_status_t cas_pool_flush(cas_pool_t *pool, void *compute_stream);
/*
 * Copies cartridge cart's fp32 moments, m1_k, m2_k, m1_v, m2_v (each
 * [len, num_kv_heads, head_dim], contiguous), into the host buffer dst
 * (4 * len * num_kv_heads * head_dim floats), from whichever tier holds
 * them. Current for every cartridge before cas_pool_load and after
 * cas_pool_flush; during training an active cartridge's copy is the one of
 * its last admission. Waits for the pool's pending file I/O.
 */
cas_status_t cas_pool_read_moments(cas_pool_t *pool, int32_t cart, float *dst);

/* Static description of a status code. */
const char *cas_status_string(cas_status_t s);
/* Message of the last failed call on this thread ("" if none). */
const char *cas_last_error_message(void);
/* Workspace bytes that the last call on this thread which returned
 * CAS_ERR_WORKSPACE needs (0 before any): what the size query for that call
 * would return. */
size_t cas_last_workspace_needed(void);
/* CAS_ABI_VERSION of the built library. */
int32_t cas_abi_version(void);

/*
 * Tuning knobs (process-wide; 0 = automatic). They change the launch plan,
 * never the result beyond rounding order.
 *   fwd_splits:  key-axis splits of the forward (partial O/LSE merged after)
 *   dq_splits:   key-axis splits of the dQ pass (fp32 partials summed after)
 */
typedef struct {
  int32_t fwd_splits;
  int32_t dq_splits;
} cas_tuning_t;

cas_status_t cas_set_tuning(const cas_tuning_t *t);
cas_status_t cas_get_tuning(cas_tuning_t *t);

/*
 * Launch plan of a problem (host-side; no device access). For tests and
 * profiling tools.
 */
typedef struct {
  int32_t fwd_splits;       /* key-axis splits used by the forward */
  int32_t dq_splits;        /* key-axis splits used by the dQ pass */
  int32_t fwd_workgroups;   /* forward grid size */
  int32_t dkdv_workgroups;  /* dK/dV work: 128-key tiles x KV heads */
  int32_t unique_segments;  /* distinct cartridges after alias folding */
  int32_t total_key_tiles;  /* dK/dV key tiles over unique cartridges and self */
  int64_t max_prefix_len;   /* longest row prefix, tokens */
  size_t ws_fwd_bytes;
  size_t ws_bwd_bytes;
} cas_plan_info_t;

cas_status_t cas_plan_info(const cas_problem_t *p, cas_plan_info_t *out);

/*
 * Per-kernel timing with HIP events, recorded on the stream each kernel is
 * launched on (a profiling aid; off by default). While enabled, every kernel
 * a call launches is bracketed by two events. cas_timing_read waits for the
 * recorded events and returns, per kernel name, the number of launches and
 * their summed duration since the last reset.
 */
typedef struct {
  char name[48];
  int32_t launches;
  double total_ms;
} cas_kernel_time_t;

cas_status_t cas_timing_enable(int enable);
cas_status_t cas_timing_reset(void);
cas_status_t cas_timing_read(cas_kernel_time_t *out, int32_t cap, int32_t *n_out);

#ifdef __cplusplus
}
#endif

#endif /* CAS_H_ */
