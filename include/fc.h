/*
 * fc.h — C ABI of the FlowCache hot path for NVIDIA B200 (sm_100a).
 *
 * FlowCache (arXiv 2602.10825) is a chunkwise caching scheme for autoregressive
 * video diffusion transformers.  This library implements the per-denoising-step
 * chunk pipeline as four calls, all enqueued on a caller-supplied CUDA stream:
 *
 *   fc_chunk_decide       which chunks are recomputed at this step   (Eqs. 5, 8)
 *   fc_chunk_attention    attention of the recomputed chunks' queries over the
 *                         fixed-budget KV cache plus the denoising window (Sec. 3.3)
 *   fc_kv_score           importance / redundancy score of cached tokens (Eqs. 9-12)
 *   fc_kv_select_compact  per-head top-B and retention of the chosen K/V rows
 *
 * and a fifth for the step around the forward pass:
 *
 *   fc_chunk_cache_apply  chunks that were not recomputed are served from the
 *                         activation cache (Sec. 3.2)
 *
 * Four more calls, not in the paper, make the queries and keys that the store holds
 * and keep its clean region in 4 bits:
 *
 *   fc_qk_norm_rope         norms of queries and keys per head and the rotation over
 *                           (time, height, width), in one pass
 *   fc_kv4_pack             rows into a 4-bit store, gathered through a kept list
 *   fc_kv4_unpack           rows of a 4-bit store as plain rows (what fc_kv_score reads)
 *   fc_chunk_attention_kv4  fc_chunk_attention over [4-bit clean region | window]
 *
 * And, for generations that roll on and branch, a clean region in pages of 8-bit rows:
 *
 *   fc_kv8_append           rows of several sequences into their pages
 *   fc_kv8_unpack           tokens of the pages as plain rows
 *   fc_pages_take, _drop    pages for sequences that grow; pages that sequences let go of
 *   fc_pages_fork           a sequence that begins as another one did, sharing its pages
 *   fc_pages_compact        the used pages moved to the front of their pool
 *   fc_chunk_attention_kv8  fc_chunk_attention over [tokens in pages | window], with a sliding window and first tokens
 *                           that stay visible
 *   fc_chunk_attention_span the same over plain rows alone
 *
 * Conventions
 *   - Plain C types only.  Every pointer argument says whether it is a HOST or a
 *     DEVICE pointer.  The caller owns every buffer, including the workspace,
 *     whose size the matching fc_*_workspace_bytes() returns.  No call allocates
 *     or frees device memory, synchronises the host with the device, or uses a
 *     stream other than `stream` (a cudaStream_t passed as void*; NULL is the
 *     default stream).
 *   - Tensors are [heads, tokens, d] with d contiguous and explicit head / token
 *     strides counted in elements.  Device base pointers must be 16-byte aligned
 *     and every stride a multiple of 16 bytes.
 *   - dtype is the storage type of the tensors (FC_BF16 or FC_F32); sums and
 *     softmax statistics are always kept in fp32 or wider.
 *   - Return value: FC_OK (0) or a negative fc_status.  On an error nothing has
 *     been launched.  Data-dependent conditions that can only be seen on the
 *     device (a NaN score, a bounded wait that expired) set bits in the optional
 *     DEVICE word `status` (OR-ed in, never cleared by the library); the caller
 *     reads it after its own synchronisation.
 *   - The library keeps no state between calls except immutable per-device
 *     attributes inside fc_ctx.  Calls on different streams may overlap as long
 *     as their buffers and workspaces do not.
 *   - One exception to the two points above: fc_chunk_decide_static takes no
 *     workspace; its scratch is an array inside the library that all its calls
 *     on a device share (see its comment for what that implies).
 */
#ifndef FC_H_
#define FC_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  FC_OK = 0,
  FC_ERR_INVALID_ARG = -1, /* NULL where a pointer is required, negative size, even pool_k ... */
  FC_ERR_UNSUPPORTED = -2, /* d not in {64,128}, unknown dtype, too many chunks / segments */
  FC_ERR_MISALIGNED = -3,  /* a base pointer or stride is not a multiple of 16 bytes */
  FC_ERR_WORKSPACE = -4,   /* ws is NULL or ws_bytes is below fc_*_workspace_bytes() */
  FC_ERR_DEVICE = -5,      /* the device is not compute capability 10.x */
  FC_ERR_CUDA = -6,        /* a CUDA runtime / driver call failed (see fc_last_cuda_error) */
  FC_ERR_UNIMPLEMENTED = -7,
  FC_ERR_TOO_LARGE = -8    /* the problem needs more scratch than a no-allocation entry point holds */
} fc_status;

typedef enum { FC_BF16 = 0, FC_F32 = 1 } fc_dtype;

/* Reuse policy of fc_chunk_decide: the paper's chunkwise rule, or the uniform policy it compares with. */
typedef enum { FC_POLICY_CHUNKWISE = 0, FC_POLICY_UNIFORM = 1 } fc_policy;

/* Bits of the device status word. */
enum {
  FC_DEV_TIMEOUT = 1u,   /* a bounded in-kernel wait expired; the affected outputs are invalid */
  FC_DEV_NAN_SCORE = 2u, /* a NaN score was ranked as -inf by the selection */
  FC_DEV_BAD_INDEX = 4u, /* an index read from device memory was out of range and was skipped */
  FC_DEV_NONFINITE = 8u, /* an infinity or a NaN was packed: a 4-bit store's group of elements reads as NaN, an 8-bit store's element */
  FC_DEV_NO_PAGES = 16u  /* fewer pages were free than a call asked for; the entries left over hold -1 */
};

enum { FC_MAX_CHUNKS = 64, FC_MAX_SEGMENTS = 64 };

typedef struct fc_ctx fc_ctx;

/* Create / destroy a context for CUDA device `device` (made current by the call).  Reads the
 * device attributes (SM count, shared-memory limit) and resolves the driver entry point used to
 * encode TMA tensor maps.  Fails with FC_ERR_DEVICE unless the device is compute capability 10.x. */
int fc_create(fc_ctx** out, int device);
int fc_destroy(fc_ctx* ctx);
const char* fc_status_string(int status);
/* Text of the last CUDA error a call on this thread ran into ("" if none). */
const char* fc_last_cuda_error(void);
/* Number of SMs the context's persistent kernels size their grids by. */
int fc_sm_count(const fc_ctx* ctx);

/* Self-test of the bounded waits (no counterpart in the paper).  Every wait on a barrier inside the tensor-core
 * kernels gives up after a wall-time limit instead of spinning forever; the kernel then runs to its normal end
 * and sets FC_DEV_TIMEOUT.  This call launches one warp that waits, with the same routine and a limit of
 * `limit_ns` (clamped to 1 us .. 1 s), on a barrier nobody signals.  After the caller's synchronisation `status`
 * (DEVICE, required) has FC_DEV_TIMEOUT set and `waited_ns` (DEVICE [1] or NULL) holds how long the warp waited.
 * Nothing faults or hangs; the context stays usable. */
int fc_selftest_bounded_wait(fc_ctx* ctx, void* stream, uint64_t limit_ns, uint32_t* status, uint32_t* waited_ns);

/* ------------------------------------------------------------------------------------------
 * fc_chunk_decide — per-chunk reuse decision.
 *
 * Paper: the relative L1 distance of chunk i between consecutive denoising steps (Eq. 5, the
 * per-chunk form of Eq. 4) is accumulated per chunk and compared with a threshold (Eq. 8):
 *     r_i = sum|cur_i - prev_i| / sum|prev_i|           (the denominator is the earlier state)
 *     s_i = acc_i + r_i                                 (fp32)
 *     recompute_i = chunk_step[i] < warmup_m  ||  force[i]  ||  s_i > eps      (strict)
 *     acc_i <- 0 if recompute_i else s_i
 * A zero denominator yields r = +inf if the numerator is positive, else 0.
 *
 * policy = FC_POLICY_UNIFORM is the "traditional reuse" the paper compares with (caption of Fig. 3): all chunks of
 * a step share one compute / reuse status, except chunks that must be computed anyway (chunk_step[i] < warmup_m
 * or force[i]: a newly initialised chunk).  Over the sharing chunks S taken as one tensor (Eq. 4):
 *     r = sum_S |cur - prev| / sum_S |prev|,   s = acc[first chunk of S] + r   (fp32)
 *     recompute_i = (i not in S) || s > eps;   every acc[i] <- 0 if s > eps (or S is empty) else s
 * and l1rel[i] = r for i in S, the chunk's own indicator otherwise.
 *
 *   cur, prev        DEVICE, `dtype` elements; chunk i occupies elements
 *                    [chunk_elem_off[i], chunk_elem_off[i+1]) of both.  The vectorised path
 *                    is taken when every offset is a multiple of 16 bytes.
 *   chunk_elem_off   HOST [n_chunks+1], non-decreasing; n_chunks <= FC_MAX_CHUNKS.
 *   chunk_step       DEVICE [n_chunks]: number of steps chunk i has already taken.
 *   force            DEVICE [n_chunks] or NULL: non-zero forces a recompute (a newly
 *                    initialised chunk must be computed).
 *   acc              DEVICE [n_chunks], in/out: the accumulator f of Eq. 8.
 *   l1rel            DEVICE [n_chunks] out or NULL: r_i.
 *   recompute        DEVICE [n_chunks] out: 1 = recompute, 0 = serve from cache.
 *   active_ids       DEVICE [n_chunks] out: ids of recomputed chunks, ascending; entries at
 *                    and after n_active are set to -1.
 *   n_active         DEVICE [1] out.
 * Sums are fixed-order (run-to-run bit-reproducible): fp32 inside a thread's 32-element run,
 * fp64 above that.  Workspace: fc_chunk_decide_workspace_bytes(total elements, n_chunks). */
size_t fc_chunk_decide_workspace_bytes(int64_t total_elems, int n_chunks);
int fc_chunk_decide(fc_ctx* ctx, void* stream, const void* cur, const void* prev, int dtype,
                    const int64_t* chunk_elem_off, int n_chunks, const int32_t* chunk_step,
                    int warmup_m, float eps, const uint8_t* force, int policy, float* acc, float* l1rel,
                    uint8_t* recompute, int32_t* active_ids, int32_t* n_active,
                    uint32_t* status, void* ws, size_t ws_bytes);

/* fc_chunk_decide_static — fc_chunk_decide without a workspace argument.
 *
 * The paper has no counterpart: this entry point exists for callers that may not allocate device
 * memory at the point of the call — code running inside a memory-pool or allocator callback, a
 * real-time loop that must not touch the allocator, a host that was handed fixed buffers by
 * another runtime — and therefore have no workspace to pass.  The (num, den) slab pairs go to an
 * array of fc_chunk_decide_static_max_bytes() = 1 MiB that is part of the library image: every
 * GPU that loads the library holds it until the process exits.  Inputs, outputs and semantics are
 * exactly those of fc_chunk_decide.
 *
 *   - Limit: fc_chunk_decide_workspace_bytes(total elements, n_chunks) must not exceed the
 *     array, which holds 65,536 slab pairs: about 268 million elements over all chunks together,
 *     whatever the dtype.  Beyond it the call returns FC_ERR_TOO_LARGE and launches nothing.
 *   - The call never allocates or frees device memory.  The array's device address is looked up
 *     once per device (a driver query, made with that device current) by fc_create; should that
 *     have failed, the first call on the device repeats it, so create the context, or make that
 *     first call, before starting any stream capture.
 *   - All calls on a device share the one array, and it keeps the previous call's contents.
 *     Nothing in it has to start at zero (each slab pair is written before it is read), but two
 *     calls that overlap on the GPU (different streams, no dependency) race on it: serialise
 *     them, or use fc_chunk_decide with separate workspaces. */
size_t fc_chunk_decide_static_max_bytes(void);
int fc_chunk_decide_static(fc_ctx* ctx, void* stream, const void* cur, const void* prev, int dtype,
                           const int64_t* chunk_elem_off, int n_chunks, const int32_t* chunk_step,
                           int warmup_m, float eps, const uint8_t* force, int policy, float* acc, float* l1rel,
                           uint8_t* recompute, int32_t* active_ids, int32_t* n_active,
                           uint32_t* status);

/* ------------------------------------------------------------------------------------------
 * fc_chunk_cache_apply — serving the chunks that were not recomputed from the activation cache.
 *
 * Paper (Sec. 3.2, text after Eq. 8): when the rule says reuse, the chunk's cached activations are
 * reused instead of a forward pass; the cache is one tensor the size of the model input (efficiency
 * appendix).  The cache holds, per chunk, the residual output - input of the chunk's last computed
 * forward; a reused chunk's output is its current input plus that residual.  For every element e of
 * chunk i (flat layout as in fc_chunk_decide):
 *     recompute[i] != 0:  cache[e] <- y[e] - x[e]       (y holds the fresh output of the forward)
 *     recompute[i] == 0:  y[e]     <- x[e] + cache[e]   (the cache is left as it is)
 * in fp32, rounded once to `dtype` (round to nearest even for bf16).  Call it after the forward of
 * the active chunks, with the recompute flags fc_chunk_decide left on the device.
 *
 *   x_in             DEVICE, `dtype`: the chunks' inputs at this step.
 *   y_io             DEVICE, `dtype`, in/out: outputs; only skipped chunks are written.
 *   cache            DEVICE, `dtype`, in/out: only computed chunks are written.
 *   chunk_elem_off   HOST [n_chunks+1]; recompute DEVICE [n_chunks].
 * The three tensors must not overlap.  Needs no workspace.  Moves 3 x (elements x element size)
 * bytes with 16-byte accesses when every offset is a multiple of 16 bytes. */
int fc_chunk_cache_apply(fc_ctx* ctx, void* stream, const void* x_in, void* y_io, void* cache, int dtype,
                         const int64_t* chunk_elem_off, int n_chunks, const uint8_t* recompute,
                         uint32_t* status);

/* ------------------------------------------------------------------------------------------
 * fc_chunk_attention — chunk-causal attention of the active chunks.
 *
 * Paper (Sec. 3.3): the chunks being denoised attend to the compressed clean-chunk region of
 * the KV buffer followed by the current denoising region; generation is causal over chunks.
 * For every active chunk c, head h and query row r of c:
 *     O[h, r, :] = softmax_j( Q[h, r, :] . K[g(h), p(j), :] * scale ) V[g(h), p(j), :],
 *     j over the first kv_visible_len[c] LOGICAL tokens, g(h) = h / (H_q / H_kv),
 * where p maps a logical token to a physical row of the K/V store: through the segment table
 * (logical range [seg_logical_off[s], seg_logical_off[s+1]) starts at physical row
 * seg_phys_off[s]) or, if given, through the per-head token map kv_token_index[g][j] (this is
 * how a cache is read through the kept-index list of fc_kv_select_compact without moving it).
 * All tokens of a chunk's own range are visible to all its rows (no mask inside a chunk).
 * Rows of chunks that are not in active_ids are never written: their cached outputs stay.
 */
typedef struct {
  int32_t H_q, H_kv, d, W;                   /* query heads, kv heads, head dim (64|128), chunks */
  int64_t q_hs, q_rs, k_hs, k_rs, v_hs, v_rs; /* element strides: head, row */
  int64_t o_hs, o_rs;
  int64_t kv_rows;                           /* physical rows per head in the K/V store */
  float scale;                               /* 0 => 1/sqrt(d) */
  int32_t impl;                              /* 0 auto; 1 force the CUDA-core kernel; 2 force the tcgen05
                                                kernel (FC_ERR_UNSUPPORTED where it does not apply) */
} fc_attn_desc;

/*   Q, O             DEVICE [H_q, rows, d]; K, V DEVICE [H_kv, kv_rows, d]; `dtype` elements.
 *   q_chunk_row_off  HOST [W+1]: chunk c owns query rows [off[c], off[c+1]).  W <= FC_MAX_CHUNKS.
 *   kv_visible_len   HOST [W].
 *   seg_logical_off  HOST [n_seg+1], seg_phys_off HOST [n_seg]; n_seg <= FC_MAX_SEGMENTS.
 *                    Ignored (may be NULL, n_seg 0) when kv_token_index is given.
 *   kv_token_index   DEVICE [H_kv, kv_index_hs] int32 or NULL.
 *   active_ids       DEVICE [<= W], n_active DEVICE [1] (as written by fc_chunk_decide): the
 *                    work list is read on the device, so no host synchronisation is needed
 *                    between the decision and the attention.
 *   lse              DEVICE [H_q, lse_hs] fp32 or NULL: natural-log sum-exp of each computed row.
 * bf16 runs on tcgen05 tensor cores (fp32 accumulation in tensor memory, TMA-fed); fp32 runs
 * on CUDA cores with fp32 accumulation.  With a token map the tensor-core kernel fetches K / V rows
 * by index (four rows per copy instruction), at roughly three quarters of the segment-table rate;
 * it needs K's and V's head strides to be whole numbers of rows, otherwise the CUDA-core kernel
 * takes the call.  An index outside [0, kv_rows) sets FC_DEV_BAD_INDEX and is not followed.
 * Physical rows that no visible logical token maps to (rows behind a segment's end, slots of
 * the store that were never written) are never used, whatever they hold.
 * Workspace: fc_chunk_attention_workspace_bytes(). */
size_t fc_chunk_attention_workspace_bytes(const fc_attn_desc* desc);
int fc_chunk_attention(fc_ctx* ctx, void* stream, const fc_attn_desc* desc, const void* Q,
                       const void* K, const void* V, int dtype, const int32_t* q_chunk_row_off,
                       const int32_t* kv_visible_len, const int32_t* seg_logical_off,
                       const int32_t* seg_phys_off, int n_seg, const int32_t* kv_token_index,
                       int64_t kv_index_hs, const int32_t* active_ids, const int32_t* n_active,
                       void* O, float* lse, int64_t lse_hs, uint32_t* status, void* ws,
                       size_t ws_bytes);

/* ------------------------------------------------------------------------------------------
 * fc_kv_score — joint importance / redundancy score of the candidate tokens.
 *
 * Paper: Imp_j = mean over the observation queries (and the query heads of a kv head's group)
 * of softmax_j(q K_cand^T * scale) (Eq. 9); Imp~ = stride-1 max-pool of width pool_k with
 * -inf padding (Eq. 10); Red_j = softmax_j of the column means of the cosine-similarity matrix
 * of the l2-normalised keys with a zeroed diagonal (Eq. 11), evaluated through the mean-key
 * identity of the paper's efficiency appendix, column mean_j = (mean_i khat_i).khat_j -
 * |khat_j|^2 / L_k, with khat = k / max(|k|, 1e-12); Score = lambda*Imp~ - (1-lambda)*Red (Eq. 12).
 *
 * Query granularity (the paper's ablation of token / frame / chunk observation queries): up to
 * 128 query rows per kv head take the streaming pipelines (the paper's setting, the last 50
 * tokens); more than that - a latent frame or a whole chunk of queries, bf16, H_q == H_kv, up
 * to 8192 - take the frame-level pipeline, in which both passes over the logits run on the
 * tensor cores.
 */
/* How the softmax argument of the redundancy (Eq. 11) is evaluated.
 *   FC_RED_MEANKEY    the mean-key identity of the efficiency appendix (default; O(L_k d) per head)
 *   FC_RED_TILED      Eq. 11 as written: 128 x 128 tiles of the cosine matrix on the tensor cores, diagonal
 *                     zeroed, column sums in the epilogue, the matrix never stored (O(L_k^2 d) per head: the
 *                     dense work the identity avoids; for checking it and as the base of the next mode)
 *   FC_RED_TILED_MAX  not in the paper: the column MAXIMUM over the other tokens instead of the column mean,
 *                     a statistic no mean key can express (same tiles, another epilogue)
 * The tiled modes need bf16 keys. */
typedef enum { FC_RED_MEANKEY = 0, FC_RED_TILED = 1, FC_RED_TILED_MAX = 2 } fc_red_mode;

typedef struct {
  int32_t H_q, H_kv, d, L_q, L_k;  /* n = L_q * (H_q/H_kv) queries per kv head: n <= 128, or bf16 with n <= 8192 and
                                      either H_q == H_kv or the query heads stored one after the other (q_hs = L_q q_rs) */
  int64_t q_hs, q_rs, k_hs, k_rs;  /* element strides */
  float scale;                     /* 0 => 1/sqrt(d) */
  float lambda;                    /* mixing coefficient (paper: 0.07) */
  int32_t pool_k;                  /* odd, >= 1 */
  int32_t impl;                    /* 0 auto; 1 force the CUDA-core kernels; 2 force tcgen05 */
  int32_t red_mode;                /* fc_red_mode */
} fc_score_desc;

/*   Q_obs            DEVICE [H_q, L_q, d]; K_cand DEVICE [H_kv, L_k, d]; `dtype` elements.
 *   imp_accum        DEVICE [H_kv, L_k] fp32 or NULL; accum_phase: 0 single shot (imp_accum
 *                    unused); 1 imp_accum += Imp of this call, nothing else is written; 2
 *                    imp_accum += Imp, then Imp := imp_accum / n_steps and the scores are
 *                    finalised (mean importance over the steps of a chunk).
 *   imp, red         DEVICE [H_kv, L_k] fp32 out, either may be NULL.
 *   score            DEVICE [H_kv, L_k] fp32 out (required unless accum_phase == 1).
 * Deterministic: no floating-point atomics.  Workspace: fc_kv_score_workspace_bytes(). */
size_t fc_kv_score_workspace_bytes(const fc_score_desc* desc);
int fc_kv_score(fc_ctx* ctx, void* stream, const fc_score_desc* desc, const void* Q_obs,
                const void* K_cand, int dtype, float* imp_accum, int accum_phase, int n_steps,
                float* imp, float* red, float* score, uint32_t* status, void* ws,
                size_t ws_bytes);

/* ------------------------------------------------------------------------------------------
 * fc_kv_select_compact — per-head top-B and retention of the selected rows.
 *
 * Paper: for each head keep the B tokens with the highest Score (text after Eq. 12); the kept
 * K/V form the compressed clean region (Sec. 3.3).  Total order: score descending, index
 * ascending (so ties keep the lowest indices); NaN ranks as -inf and sets FC_DEV_NAN_SCORE;
 * -0 equals +0.  B >= L_k keeps everything (identity).
 *
 *   score            DEVICE [n_heads, L_k] fp32.
 *   K_src, V_src     DEVICE [n_heads, L_k, d] with strides src_hs / src_rs (elements);
 *   K_dst, V_dst     DEVICE [n_heads, >= min(B,L_k), d] with strides dst_hs / dst_rs; must not
 *                    overlap the sources.  All four NULL => selection only.
 *   kept_idx         DEVICE [n_heads, min(B, L_k)] int32 out, ascending per head.
 *   n_kept           DEVICE [1] out or NULL: min(B, L_k).
 * Row r of head h of the destination is source row kept_idx[h][r], copied byte for byte with
 * 16-byte accesses; bytes outside the kept rows are not touched; dropped rows are not read. */
typedef struct {
  int64_t src_hs, src_rs, dst_hs, dst_rs;
} fc_compact_strides;

size_t fc_kv_select_compact_workspace_bytes(int n_heads, int L_k);
int fc_kv_select_compact(fc_ctx* ctx, void* stream, const float* score, int n_heads, int L_k,
                         int B, const void* K_src, const void* V_src, void* K_dst, void* V_dst,
                         int dtype, int d, const fc_compact_strides* strides, int32_t* kept_idx,
                         int32_t* n_kept, uint32_t* status, void* ws, size_t ws_bytes);

/* fc_kv_select_compact_ex — the same selection at a coarser key granularity and / or with a protected tail.
 *
 * Paper: the key-granularity ablation (Table 4) compresses with frame- or chunk-level keys instead of tokens (and
 * finds token-level keys best, which is why fc_kv_select_compact is the default).  Here a unit is `unit`
 * consecutive tokens (a latent frame, a chunk), kept or dropped as a whole; a unit's score is the mean of its
 * tokens' scores (fp64 sum, rounded to fp32); L_k and B must be whole numbers of units.  n_protect (not in the
 * paper) keeps the units of the last n_protect tokens - the newest ones - whatever their score; the others rank
 * by (score descending, index ascending), NaN as -inf.  unit = 1, n_protect = 0 is fc_kv_select_compact.
 * Workspace (only for unit > 1): fc_kv_select_compact_ex_workspace_bytes().  All other arguments as above;
 * kept_idx lists the kept tokens ascending, n_kept = min(B, L_k). */
typedef struct {
  int32_t unit;      /* tokens per selection unit, >= 1 */
  int32_t n_protect; /* newest tokens always kept, >= 0 */
} fc_select_opts;

size_t fc_kv_select_compact_ex_workspace_bytes(int n_heads, int L_k, int unit);
int fc_kv_select_compact_ex(fc_ctx* ctx, void* stream, const float* score, int n_heads, int L_k, int B,
                            const fc_select_opts* opts, const void* K_src, const void* V_src, void* K_dst,
                            void* V_dst, int dtype, int d, const fc_compact_strides* strides, int32_t* kept_idx,
                            int32_t* n_kept, uint32_t* status, void* ws, size_t ws_bytes);

/* ------------------------------------------------------------------------------------------
 * fc_qk_norm_rope — RMS norms of queries and keys for each head and the position rotation over
 * several axes, in one pass.
 *
 * Not in the paper, whose method starts from given Q and K.  The norm is of each head's row; a model that norms a projection's whole row
 * does that before the call and takes FC_NORM_NONE.
 * For every token n and head, with x the head's d elements (fp32 throughout, one rounding to `dtype`; a row whose sum of squares
 * leaves the range of fp32 has no meaningful norm):
 *     y = x * w / sqrt(mean(x^2) + eps)                      norm = FC_NORM_RMS; w = 1 where the weight is NULL
 *     y = x                                                  norm = FC_NORM_NONE
 * The first axis_dim[0] elements turn with the token's position on axis 0 (time), the next axis_dim[1]
 * with axis 1 (height), the next axis_dim[2] with axis 2 (width); elements behind them pass through: y as it is, infinities and
 * signs of zero too.
 * Pair i of a section of n elements is (2i, 2i+1) (FC_ROPE_PAIRS) or (i, i + n/2) (FC_ROPE_HALVES):
 *     (y0, y1) <- (y0 cos a - y1 sin a, y0 sin a + y1 cos a),   a = position * theta^(-2i/n)
 * The angle is reduced in 64-bit fixed point, so that it is as exact at position 2^31 as at 1, and rounded to fp32 after that (off by
 * 2^-24 of itself, which is at most half a turn).  Negative positions turn back: the rotation by -p undoes the rotation by p, and the rotation of an already
 * rotated key by (new - old) position moves it there.
 *
 *   Q, Q_out         DEVICE [H_q, T, d], K, K_out DEVICE [H_kv, T, d]; `dtype` elements with the strides of the
 *                    descriptor (any order of heads and tokens, e.g. slices of a fused projection).  H_q or
 *                    H_kv may be 0 (its pointers are then ignored), T too.  An output may be its own input (same pointer
 *                    and strides); other overlap is not allowed, nor rows of an output that overlap one another.
 *   q_weight, k_weight  DEVICE [d] fp32 or NULL; ignored for FC_NORM_NONE.
 *   pos              DEVICE [T, 3] int32, contiguous, or NULL: token n then stands at
 *                    (grid_t0 + n / (grid_h grid_w), n / grid_w % grid_h, n % grid_w).
 *   inv_freq         HOST [sum of axis_dim / 2] double or NULL: the pairs' radians per position in place of theta^(-2i/n),
 *                    section by section.
 * Needs no workspace. */
typedef enum { FC_NORM_NONE = 0, FC_NORM_RMS = 1 } fc_norm;
typedef enum { FC_ROPE_PAIRS = 0, FC_ROPE_HALVES = 1 } fc_rope_pairing;

typedef struct {
  int32_t H_q, H_kv, d, T;                       /* d in {64, 128} */
  int64_t q_hs, q_rs, k_hs, k_rs;                /* element strides of the inputs: head, token */
  int64_t qo_hs, qo_rs, ko_hs, ko_rs;            /* and of the outputs */
  int32_t axis_dim[3];                           /* even, >= 0, sum <= d */
  int32_t pairing;                               /* fc_rope_pairing */
  int32_t norm;                                  /* fc_norm */
  float eps;                                     /* >= 0 */
  double theta;                                  /* > 0; ignored where inv_freq is given */
  int32_t grid_t0, grid_h, grid_w;               /* ignored where pos is given, or nothing turns */
} fc_rope_desc;

int fc_qk_norm_rope(fc_ctx* ctx, void* stream, const fc_rope_desc* desc, const void* Q, const void* K, int dtype,
                    const float* q_weight, const float* k_weight, const int32_t* pos, const double* inv_freq,
                    void* Q_out, void* K_out);

/* ------------------------------------------------------------------------------------------
 * The 4-bit store.
 *
 * A row of d elements is d/2 bytes of codes and d/32 bf16 scales: 4.5 bits an element, so that a budget
 * of B tokens takes 0.28 of its bf16 bytes.  Each group of 32 consecutive elements shares a scale s:
 *     s = the least number with five significant bits that is >= max|x| / 7 (divided in fp32), clamped to
 *         [2^-126, 2^122]; 0 if all are 0; NaN if one is not finite (FC_DEV_NONFINITE)
 *     code = 8 + min(max(round_half_even(x / s), -7), 7),   value = (code - 8) * s
 * A value has at most eight significant bits: it is exactly a bf16 number, so attention over the store is
 * attention over these values without another rounding.  In each little-endian 32-bit word of eight
 * elements, element 2i is at bits 4i of the low half and element 2i+1 at bits 4i of the high half (i = 0..3).
 * Rows that the calls below write may not overlap one another, nor what the same call reads.
 * The pointers are DEVICE pointers inside a HOST struct; K and V share strides.  Code bases and strides are
 * multiples of 16 bytes, scale bases and strides of a row's scales (d/32 elements). */
typedef struct {
  void *k_codes, *k_scales, *v_codes, *v_scales;
  int64_t code_hs, code_rs;   /* bytes: head, row (row >= d/2) */
  int64_t scale_hs, scale_rs; /* bf16 elements: head, row (row >= d/32) */
  int64_t rows;               /* rows per head that the buffers hold */
} fc_kv4_cache;

/* fc_kv4_pack — writes rows dst_row .. dst_row + n_out - 1 of the store `dst` (all heads, K and V).
 *
 * Output row r of head h is logical row i = kept_idx[h * kept_hs + r], or i = r without a kept list:
 *     i <  n_old   row i of the store `old`, codes and scales byte for byte (no second rounding)
 *     i >= n_old   row i - n_old of K_src / V_src, quantised
 * With the kept list of fc_kv_select_compact over [clean region | finished chunk] this is the compaction of a
 * 4-bit clean region; with n_old = 0 and no list it appends n_out rows.
 *
 *   K_src, V_src     DEVICE [H, n_new, d], `dtype` (may be NULL if n_new is 0).
 *   old              HOST struct or NULL (n_old 0); its rows >= n_old.  Its first n_old rows must not overlap the rows that are
 *                    written: refused, by their addresses and strides (`dst` itself with dst_row < n_old; slices of one store that
 *                    share rows; stores of different strides whose heads lie between one another's).
 *   kept_idx         DEVICE [H, >= n_out] int32 or NULL (n_out <= n_old + n_new then).  An index outside
 *                    [0, n_old + n_new) sets FC_DEV_BAD_INDEX; its output row is left as it was.
 * Rows outside the written range are not touched.  Needs no workspace. */
typedef struct {
  int32_t H, d;                    /* d in {64, 128} */
  int32_t n_old, n_new, n_out;     /* rows per head; n_out may be 0 */
  int64_t dst_row;
  int64_t k_hs, k_rs, v_hs, v_rs;  /* element strides of K_src, V_src */
} fc_kv4_pack_desc;

int fc_kv4_pack(fc_ctx* ctx, void* stream, const fc_kv4_pack_desc* desc, const void* K_src, const void* V_src, int dtype,
                const fc_kv4_cache* old, const int32_t* kept_idx, int64_t kept_hs, const fc_kv4_cache* dst,
                uint32_t* status);

/* fc_kv4_unpack — the values of rows src_row .. src_row + n - 1 of every head as plain rows.
 *   K_dst, V_dst     DEVICE [H, n, d], `dtype` (exact in both types); either may be NULL (the score needs the keys
 *                    only).  Needs no workspace. */
typedef struct {
  int32_t H, d;
  int32_t n;                       /* may be 0 */
  int64_t src_row;
  int64_t k_hs, k_rs, v_hs, v_rs;  /* element strides of K_dst, V_dst */
} fc_kv4_unpack_desc;

int fc_kv4_unpack(fc_ctx* ctx, void* stream, const fc_kv4_unpack_desc* desc, const fc_kv4_cache* src, void* K_dst,
                  void* V_dst, int dtype);

/* fc_chunk_attention_kv4 — fc_chunk_attention over a 4-bit clean region and a plain window.
 *
 * Logical token j < n_cache is row j of the 4-bit store; j >= n_cache is token j - n_cache of the window, found in
 * K / V through the segment table, whose logical offsets count from the window's start.  kv_visible_len counts both.
 * Everything else is as in fc_chunk_attention: chunks, active list, grouped heads, rows of inactive chunks left as they are; rows that see no
 * token get zeros (lse -inf).  There is no token map: a 4-bit store is compacted by fc_kv4_pack.
 *
 *   desc             as above; k_* and v_* strides and kv_rows describe the window.  impl: 0 auto; 1 force the
 *                    CUDA-core kernel; 2 (bf16 only) unpack into the workspace and run the tcgen05 kernel of
 *                    fc_chunk_attention over [workspace | window]; 3 force the kernel for few rows, which reads the packed keys
 *                    in one pass and is also the path of fp32.
 *   active_ids       as above; an id outside [0, W) sets FC_DEV_BAD_INDEX and is ignored.  A chunk named again is one chunk.
 *   cache            HOST struct, rows >= n_cache; may be NULL if n_cache is 0.
 *   K, V             DEVICE [H_kv, kv_rows, d], the window; may be NULL if n_seg is 0 (no window).
 *   kv_visible_len   as above, at most 2^31 - 4097.
 *   n_seg            <= FC_MAX_SEGMENTS - 1.  n_cache and the window's tokens together are at most 2^31 - 4097.
 * Logits, maxima, sums and outputs are kept in fp32.  Softmax weights too for fp32 tensors and with impl 1; otherwise they are rounded to bf16
 * on their way to V, as in fc_chunk_attention (each by 2^-8 at most, which adds about as much to the output's error as its
 * own rounding).  The kernel for few rows (impl 3, or chosen by 0) takes along what the rounding leaves (2^-17 then) where no chunk has more
 * than eight rows times heads of a group.
 * An infinity in a row of V that is seen makes what it reaches infinite or NaN; in fp32 one in q, K or V makes it NaN, and a
 * magnitude that rounds to a bf16 infinity (2^128 - 2^119 and above) counts as one.
 * Deterministic.  Workspace: fc_chunk_attention_kv4_workspace_bytes() of the same arguments (0 for arguments
 * that the call refuses). */
size_t fc_chunk_attention_kv4_workspace_bytes(const fc_ctx* ctx, const fc_attn_desc* desc, int dtype,
                                              const int32_t* q_chunk_row_off, const int32_t* kv_visible_len, int n_cache);
int fc_chunk_attention_kv4(fc_ctx* ctx, void* stream, const fc_attn_desc* desc, const void* Q, const fc_kv4_cache* cache,
                           int n_cache, const void* K, const void* V, int dtype, const int32_t* q_chunk_row_off,
                           const int32_t* kv_visible_len, const int32_t* seg_logical_off, const int32_t* seg_phys_off,
                           int n_seg, const int32_t* active_ids, const int32_t* n_active, void* O, float* lse,
                           int64_t lse_hs, uint32_t* status, void* ws, size_t ws_bytes);

/* ------------------------------------------------------------------------------------------
 * The paged 8-bit store.
 *
 * A pool of n_pages pages holds K and V of any number of sequences.  A page is `page` tokens (16, 32, 64 or 128) of all heads;
 * token j of a sequence is row j % page of page table[j / page], where `table` is the sequence's row of a DEVICE
 * int32 array [sequences, entries] (row stride table_cs elements).  An entry of -1 is no page (never given, or dropped).
 * A block, one page of one head, is `page` rows of d E4M3 codes (a sign, four bits of exponent with bias 7, three of mantissa; no
 * infinities; +-448 the largest), one row behind the other, with a scale s for K and one for V:
 *     s = the least number with four significant bits whose 448-fold is not below max|x|, clamped to [2^-117, 2^119]; 0 if all
 *         are 0 (elements that are not finite are left out)
 *     code = x / s rounded to the nearest code, ties to even, +-448 at most; NaN if x is not finite (FC_DEV_NONFINITE)
 *     value = code * s
 * A value has at most eight significant bits: it is exactly a bf16 number.
 * The pointers are DEVICE pointers inside a HOST struct; K and V share strides.  Blocks must not overlap. */
typedef struct {
  void *k_codes, *v_codes;        /* bytes, 16-byte aligned */
  float *k_scales, *v_scales;
  int64_t code_ps, code_hs;       /* bytes, multiples of 16 below 2^36: page, head */
  int64_t scale_ps, scale_hs;     /* elements, below 2^31 */
  int32_t n_pages, page;
} fc_kv8_pool;

/* fc_kv8_append — rows row_off[c] .. row_off[c+1] - 1 of K_src / V_src become tokens pos[c], pos[c] + 1, ... of sequence c.
 *
 * Where pos[c] falls inside a page, the block's scale becomes the larger of its own and the new rows', and where it grows the rows before
 * pos[c] are rounded again: code' = code * s / s' rounded as above.  Rows of that block from pos[c] on are what a rewound
 * sequence leaves behind: they are written over, or left as they are, and count for nothing but the scale.  A page
 * whose first row is written starts with a scale of its own.
 *
 *   K_src, V_src     DEVICE [H, rows, d], `dtype`.
 *   row_off          HOST [W+1], non-decreasing; pos HOST [W]; W <= FC_MAX_CHUNKS.  pos[c] + rows <= 2^31 - 4097.
 *   table            DEVICE [W, table_cs] (table_cs covers every entry that is used where W > 1: rows of the table do not overlap).
 *   ref              DEVICE [n_pages] int32 or NULL: how many entries name each page (see below).  With it, only pages with a
 *                    count of 1 are written to.  One that more entries name, or that is free, is left as it is
 *                    (FC_DEV_BAD_INDEX): fork a sequence, or take its pages, before it is written to.
 * An entry outside [0, n_pages) sets FC_DEV_BAD_INDEX and its rows are dropped.  Two sequences of a call may not name the same
 * page where they write.  Needs no workspace. */
typedef struct {
  int32_t H, d, W;                /* d in {64, 128} */
  int64_t k_hs, k_rs, v_hs, v_rs; /* element strides of K_src, V_src (fc_kv8_unpack: of K_dst, V_dst) */
} fc_kv8_rows;

int fc_kv8_append(fc_ctx* ctx, void* stream, const fc_kv8_rows* desc, const void* K_src, const void* V_src, int dtype,
                  const int32_t* row_off, const int32_t* pos, const fc_kv8_pool* pool, const int32_t* table,
                  int64_t table_cs, const int32_t* ref, uint32_t* status);

/* fc_kv8_unpack — tokens first[c], first[c] + 1, ... of sequence c as rows row_off[c] .. row_off[c+1] - 1 of K_dst / V_dst.
 *   K_dst, V_dst     DEVICE [H, rows, d], `dtype` (exact in both); either may be NULL (the score needs the keys only).
 *   table            as above; table_cs may be 0 (several ranges of one sequence).
 * Rows of an entry outside [0, n_pages) are zeros, and FC_DEV_BAD_INDEX is set.  Needs no workspace. */
int fc_kv8_unpack(fc_ctx* ctx, void* stream, const fc_kv8_rows* desc, const fc_kv8_pool* pool, const int32_t* table,
                  int64_t table_cs, const int32_t* first, const int32_t* row_off, void* K_dst, void* V_dst, int dtype,
                  uint32_t* status);

/* ------------------------------------------------------------------------------------------
 * The pages of a pool.
 *
 *   ref              DEVICE [n_pages] int32, 16-byte aligned: how many table entries name each page; 0: the page is free.
 *   table            DEVICE [sequences, table_cs] int32, as above.
 * The caller sets `ref` to 0 and `table` to -1 once; the calls keep the two in step.  All of them are deterministic, and none asks the
 * host: pages are found on the device.  Calls that work on the same counts belong on one stream.
 *
 * fc_pages_take — entries first[c] .. last[c] - 1 of sequence c get pages of their own.  Sequence by sequence and entry by
 * entry, each takes the free page of the lowest number.  Where none is left, entries get -1 and FC_DEV_NO_PAGES is set.
 * What the entries held before is forgotten, not dropped.
 *
 * fc_pages_drop — entries first[c] .. last[c] - 1 of sequence c let go of their pages and become -1.  A page that nobody
 * names any more is free; its content stays until somebody takes it.  An entry of -1 is passed over; one that names no
 * page of the pool, or a free one, sets FC_DEV_BAD_INDEX.
 *
 *   first, last      HOST [W], 0 <= first <= last; W <= FC_MAX_CHUNKS.  Rows of the table may not overlap (W > 1: table_cs >= every last). */
int fc_pages_take(fc_ctx* ctx, void* stream, int32_t* ref, int n_pages, int32_t* table, int64_t table_cs, int W,
                  const int32_t* first, const int32_t* last, uint32_t* status);
int fc_pages_drop(fc_ctx* ctx, void* stream, int32_t* ref, int n_pages, int32_t* table, int64_t table_cs, int W,
                  const int32_t* first, const int32_t* last, uint32_t* status);

/* fc_pages_fork — sequence dst[i] begins as the first tokens[i] tokens of sequence src[i].  Pages that these fill are shared; the
 * last one, if they fill it in part, is copied into a page of its own (taken as above, fork by fork), so that both
 * sequences may go on.  Entries that are -1 (dropped) stay -1.  dst's entries behind these are left as they are, and what it named before is
 * forgotten: drop it first.
 *   src, dst         HOST [n], rows of the table: 0 <= . < n_seq; no dst twice, and none among the src.
 *   tokens           HOST [n], >= 0; ceil(tokens / page) <= table_cs.  n <= FC_MAX_CHUNKS.
 * Where no page is left for a copy, the entry gets -1 and FC_DEV_NO_PAGES is set.  An entry of src that names no page of the pool
 * sets FC_DEV_BAD_INDEX and becomes -1.  So does one that names a free page; filled in part it becomes a page of dst's own into which
 * nothing is copied.  H, d as for fc_kv8_append.  Workspace: fc_pages_workspace_bytes(n_pages).
 *
 * fc_pages_compact — the n used pages of the pool become pages 0 .. n - 1: those with numbers from n on, in ascending order, move into
 * the free ones below n, in ascending order; counts go with them, and entries 0 .. entries - 1 of all n_seq rows
 * of the table are rewritten.  What the pages hold that are free afterwards is left as it is.
 *   n_used           DEVICE [1] int32 out or NULL: n.
 * Tables that are not among those rows would point at the wrong pages.  An entry that names no page, or a free one from n on, sets
 * FC_DEV_BAD_INDEX and is left.  Workspace: fc_pages_workspace_bytes(n_pages). */
size_t fc_pages_workspace_bytes(int n_pages);
int fc_pages_fork(fc_ctx* ctx, void* stream, const fc_kv8_pool* pool, int H, int d, int32_t* ref, int32_t* table,
                  int64_t table_cs, int n_seq, int n, const int32_t* src, const int32_t* dst, const int32_t* tokens,
                  uint32_t* status, void* ws, size_t ws_bytes);
int fc_pages_compact(fc_ctx* ctx, void* stream, const fc_kv8_pool* pool, int H, int d, int32_t* ref, int32_t* table,
                     int64_t table_cs, int n_seq, int entries, int32_t* n_used, uint32_t* status, void* ws,
                     size_t ws_bytes);

/* ------------------------------------------------------------------------------------------
 * fc_chunk_attention_kv8 — fc_chunk_attention over a paged 8-bit clean region and a plain window, each chunk with a sliding window
 * and first tokens that stay visible.
 *
 * The logical tokens of chunk c are the first cache_len[c] tokens of its sequence, in pages, followed by the plain tokens
 * window_first[c], window_first[c] + 1, ... of K / V (in the order of the segment table).  Its rows see
 *     j < kv_visible_len[c]   and   (j < n_sink   or   j >= kv_begin[c])
 * and O and lse are the softmax over those tokens, as in fc_chunk_attention; rows that see none get zeros (lse -inf).  The chunks of a
 * generation share a row of the table (table_cs 0) and see one another's plain tokens; sequences of a batch have rows of their own,
 * and window_first points each at its own plain tokens.
 *
 *   desc             as for fc_chunk_attention; k_*, v_* and kv_rows describe the plain tokens.  impl: 0 auto; 2 (bf16
 *                    only) unpack what is seen into the workspace and run the tcgen05 kernel; 3 the kernel for few rows, which
 *                    reads the pages in place and is also the path of fp32.
 *   pool, table      as above; both may be NULL if every cache_len is 0.
 *   cache_len        HOST [W] or NULL (all 0).  kv_visible_len HOST [W]; kv_begin HOST [W] or NULL (all 0: no sliding window); window_first
 *                    HOST [W] or NULL (all 0).  Tokens that no active chunk sees need no page.
 *   K, V, seg_*      as in fc_chunk_attention_kv4: the plain tokens; n_seg 0 if there are none.
 * Everything else is as in fc_chunk_attention_kv4: the active list, grouped heads, rows of inactive chunks.  Logits, maxima, sums and outputs are kept
 * in fp32.  Softmax weights are rounded on their way to V: for fp32 tensors by 2^-22 at most (over pages by 2^-43 of the row's largest so far
 * where that is more); by the tcgen05 kernel to bf16; by the
 * kernel for few rows to fp16 over pages (2^-11 of a weight, or 2^-32 of the row's largest so far where that is more) and to bf16 over
 * plain rows, where what that leaves is taken along if no tile has more than eight rows times heads of a group.
 * Before they are divided by their sum, weights are at most 1 in the kernel for few rows and at most 2^8 in the tcgen05 kernel; the sum of
 * weights times values has to stay below 2^128, which it does where the tokens that are seen, times the largest |value|, times that bound do.
 * What lies in tokens that a chunk does not see never reaches its rows, whatever it is.  A NaN in a token that is seen makes what it reaches NaN, and so
 * does an infinity in Q.  One in a plain token's K or V that is seen makes what it reaches infinite or NaN, or leaves the token out where its logit is -inf;
 * in fp32 it makes it NaN, and a magnitude in Q, K or V over plain tokens that rounds to a bf16 infinity (2^128 - 2^119 and above) counts as one.  A row
 * all of whose logits are -inf is NaN.  Head strides of K and V are not 0 where there are several heads.
 * An entry outside [0, n_pages) of whose tokens an active chunk sees one sets FC_DEV_BAD_INDEX; K and V of its tokens count as zeros.
 * Deterministic.  Workspace: fc_chunk_attention_kv8_workspace_bytes() of the same arguments (0 for arguments that the call
 * refuses). */
size_t fc_chunk_attention_kv8_workspace_bytes(const fc_ctx* ctx, const fc_attn_desc* desc, int dtype, int page, int64_t table_cs,
                                              const int32_t* cache_len, const int32_t* q_chunk_row_off,
                                              const int32_t* kv_visible_len, int n_sink, const int32_t* kv_begin,
                                              const int32_t* window_first, const int32_t* seg_logical_off, int n_seg);
int fc_chunk_attention_kv8(fc_ctx* ctx, void* stream, const fc_attn_desc* desc, const void* Q, const fc_kv8_pool* pool,
                           const int32_t* table, int64_t table_cs, const int32_t* cache_len, const void* K, const void* V,
                           int dtype, const int32_t* q_chunk_row_off, const int32_t* kv_visible_len, int n_sink,
                           const int32_t* kv_begin, const int32_t* window_first, const int32_t* seg_logical_off,
                           const int32_t* seg_phys_off, int n_seg, const int32_t* active_ids, const int32_t* n_active,
                           void* O, float* lse, int64_t lse_hs, uint32_t* status, void* ws, size_t ws_bytes);

/* fc_chunk_attention_span — the same over plain rows alone: fc_chunk_attention in which chunk c sees tokens
 *     j < kv_visible_len[c]   and   (j < n_sink   or   j >= kv_begin[c])
 * of the segment table, from single tokens, whose keys are shared out among all SMs, to whole chunks.  Arguments, types and impl as above.
 * Workspace: fc_chunk_attention_span_workspace_bytes() of the same arguments. */
size_t fc_chunk_attention_span_workspace_bytes(const fc_ctx* ctx, const fc_attn_desc* desc, int dtype,
                                               const int32_t* q_chunk_row_off, const int32_t* kv_visible_len, int n_sink,
                                               const int32_t* kv_begin, const int32_t* seg_logical_off, int n_seg);
int fc_chunk_attention_span(fc_ctx* ctx, void* stream, const fc_attn_desc* desc, const void* Q, const void* K, const void* V,
                            int dtype, const int32_t* q_chunk_row_off, const int32_t* kv_visible_len, int n_sink,
                            const int32_t* kv_begin, const int32_t* seg_logical_off, const int32_t* seg_phys_off, int n_seg,
                            const int32_t* active_ids, const int32_t* n_active, void* O, float* lse, int64_t lse_hs,
                            uint32_t* status, void* ws, size_t ws_bytes);

#ifdef __cplusplus
}
#endif
#endif /* FC_H_ */
