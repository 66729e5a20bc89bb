/*
 * xattn.h -- C ABI of the MI355X (gfx950) XAttention prefill library.
 *
 * XAttention (arXiv 2503.16428) replaces dense prefill attention by three
 * steps (Fig. 1): (1) strided antidiagonal block scoring, (2) threshold block
 * selection, (3) attention on the selected blocks only. Each step is one call
 * here, plus a dense reference mode and a chained forward.
 *
 * Conventions shared by every call
 *   - Plain C; no HIP or torch types. `stream` is a hipStream_t passed as
 *     void* (NULL = the default stream). Every call only validates its
 *     arguments on the host and enqueues kernels on `stream`: it never
 *     allocates, never synchronises and never throws. Results are ready when
 *     the caller synchronises the stream.
 *   - All array pointers are DEVICE pointers owned by the caller; the library
 *     keeps none of them after the call returns. Arrays are dense and
 *     row-major in the shapes stated below; tensors of bfloat16 values are
 *     passed as `const void*`.
 *   - Heads: query head h (0 <= h < batch*hq) reads key/value head
 *     (h / hq) * hkv + (h % hq) / (hq / hkv)  (contiguous GQA grouping).
 *   - Shapes use L = dims->seq, D = dims->head_dim, NB = L / block,
 *     HQ = batch * hq, HKV = batch * hkv.
 *   - Return value: XATTN_OK or an error code; on error nothing has been
 *     enqueued (argument errors) or the HIP launch failed (XATTN_ERR_HIP).
 *     xattn_last_error() gives a message for the calling thread.
 *   - Results are deterministic: the same inputs give bitwise equal outputs.
 *   - The calls for serving after the prefill (rotary positions, paged cache, one
 *     new token's attention, eviction) keep these conventions; their shapes
 *     stand with them.
 *
 * Supported today: head_dim 128, block 128, stride S in {1,2,4,8,16,32,64},
 * seq a multiple of 128 and at most 262144 (NB <= 2048).
 */
#ifndef XATTN_H
#define XATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum xattn_status {
    XATTN_OK = 0,
    XATTN_ERR_ARG = 1,          /* invalid argument (null pointer, bad shape, tau <= 0 or NaN) */
    XATTN_ERR_UNSUPPORTED = 2,  /* valid but not implemented (e.g. head_dim != 128) */
    XATTN_ERR_WORKSPACE = 3,    /* workspace pointer null or smaller than required */
    XATTN_ERR_HIP = 4           /* a HIP runtime call or kernel launch failed */
};

/* Problem shape. Layouts: Q [batch][hq][seq][head_dim], K and V
 * [batch][hkv][seq][head_dim], all bfloat16. causal: 1 = query i attends to
 * keys k <= i (decoder prefill), 0 = bidirectional (e.g. video DiT). */
typedef struct xattn_dims {
    int32_t batch;
    int32_t hq;
    int32_t hkv;
    int32_t seq;
    int32_t head_dim;
    int32_t causal;
} xattn_dims;

/*
 * Step 1 -- strided antidiagonal block scoring (Sec. 3.1-3.2, Algorithm 1).
 *
 * For query head h, query block b and key block j, with nr = block / stride
 * reduced rows per block and reduced row R = b*nr + r:
 *   x[R][c]  = (1 / (sqrt(D) * S)) * sum_{t<S} q[R*S + S-1-t] . k[c*S + t]
 *              (the product of Algorithm 1's strided reshapes: the sum over
 *              the antidiagonal of every S x S sub-block of Q K^T),
 *   A[R][c]  = softmax over the valid reduced columns c (c <= R when causal),
 *   scores[h][b][j] = (1/nr) * sum_{r<nr} sum_{c in block j} A[R][c],
 * so every row sums to 1. Entries with j > b (causal) are written as 0.
 *   q        bf16 [HQ][L][D]          k  bf16 [HKV][L][D]
 *   scores   fp32 [HQ][NB][NB]        (output, fully written)
 *   workspace  device scratch of at least xattn_score_workspace_size() bytes;
 *              its contents on entry are ignored, on exit unspecified.
 * Products are bf16 x bf16 on the matrix cores with fp32 accumulation; the
 * softmax and block sums are fp32.
 */
int xattn_score_workspace_size(const xattn_dims *dims, int block, int stride,
                               size_t *bytes);
int xattn_score(const void *q, const void *k, const xattn_dims *dims, int block,
                int stride, float *scores, void *workspace, size_t workspace_bytes,
                void *stream);

/*
 * Step 1 with another sampling pattern inside each S x S sub-block (the
 * pattern ablation, Sec. 4.5, Table 4): the S summed positions are
 * (query sub-row qsub[t], key sub-row t), t < S, so
 *   X[R][c] = (1 / (S sqrt(D))) sum_{t<S} q[R*S + qsub[t]] . k[c*S + t].
 * qsub[t] = S-1-t is xattn_score (the antidiagonal); qsub[t] = t the main
 * diagonal; any other permutation (e.g. a seeded random one) the random
 * pattern, which keeps one position per sub-block row and column.
 *   qsub  host array of `stride` int32, a permutation of 0 .. stride-1; read
 *         during the call only (copied into the launch)
 * Everything else as xattn_score. XATTN_ERR_ARG if qsub is NULL or not a
 * permutation.
 */
int xattn_score_pattern(const void *q, const void *k, const xattn_dims *dims, int block,
                        int stride, const int32_t *qsub, float *scores, void *workspace,
                        size_t workspace_bytes, void *stream);

/*
 * Step 2 -- threshold block selection, find_blocks (Sec. 3.2, equation of
 * find_blocks; Algorithm 1). Per row (h, b) the candidates are j <= b
 * (causal) or all j. Each candidate's mass is taken as the integer
 * u_j = floor(clamp(scores[h][b][j], 0, 1) * 2^32); T = sum of u_j over the
 * candidates. The selected set is the shortest prefix (length >= 1) of the
 * candidates ordered by (u_j descending, j ascending) whose integer sum
 * reaches ceil(tau * T) (tau * T as one fp64 product). tau >= 1 selects every
 * candidate. Integer masses make the result independent of summation order.
 *   scores  fp32 [HQ][NB][NB]   (input; only candidate entries are read)
 *   tau     threshold, 0 < tau; values >= 1 mean "all candidates"
 *   idx     int32 [HQ][NB][NB]  (output) row (h, b): idx[h][b][0 .. cnt) are
 *           the selected key blocks in ascending order; later entries are
 *           left unchanged
 *   cnt     int32 [HQ][NB]      (output) number selected, >= 1
 */
int xattn_select(const float *scores, const xattn_dims *dims, int block, float tau,
                 int32_t *idx, int32_t *cnt, void *stream);

/*
 * Step 2 with one threshold per query head (the per-head thresholds that the
 * minimum-threshold prediction of Sec. 3.3 produces). Row (h, b) of batch
 * element n uses tau_h[h] (rows are indexed n * hq + h); otherwise exactly
 * xattn_select.
 *   tau_h  host array of dims->hq floats, each > 0 (values >= 1: all
 *          candidates); read during the call only (copied into the launch)
 * Errors: XATTN_ERR_ARG for a NULL array or a tau <= 0 / NaN,
 * XATTN_ERR_UNSUPPORTED for hq > 256.
 */
int xattn_select_heads(const float *scores, const xattn_dims *dims, int block,
                       const float *tau_h, int32_t *idx, int32_t *cnt, void *stream);

/*
 * Fixed-size block selection of the selection-strategy ablation (Sec. 4.5,
 * Table 6: Top-K and Top-Ratio against threshold selection). Per row the
 * candidates are ordered as in xattn_select, by (u_j descending, j
 * ascending) with u_j = floor(clamp(score, 0, 1) * 2^32), and the first k are
 * selected, k clamped to [1, m] for m candidates; output as xattn_select.
 *   Top-K:     k = k_h[h] key blocks (the paper quotes K in tokens: K tokens
 *              correspond to K / block blocks); host array of dims->hq
 *              int32, each >= 1
 *   Top-Ratio: k = floor(ratio_h[h] * m + 0.5) (fp32 ratio, product in
 *              fp64), at least 1; host array of dims->hq floats, each finite
 *              and > 0 (>= 1 keeps every candidate)
 * The arrays are read during the call only. Errors as xattn_select_heads.
 */
int xattn_select_topk(const float *scores, const xattn_dims *dims, int block,
                      const int32_t *k_h, int32_t *idx, int32_t *cnt, void *stream);
int xattn_select_ratio(const float *scores, const xattn_dims *dims, int block,
                       const float *ratio_h, int32_t *idx, int32_t *cnt, void *stream);

/*
 * Step 3 -- block-sparse attention (Fig. 1, right): for query i in block b of
 * head h, with K_i the keys of the listed key blocks idx[h][b][0 .. cnt)
 * (intersected with k <= i when causal):
 *   o[h][i]   = sum_{k in K_i} softmax_k(q_i . k_k / sqrt(D)) v_k
 *   lse[h][i] = log sum_{k in K_i} exp(q_i . k_k / sqrt(D))   (natural log)
 * A query with no visible key gets o = 0 and lse = -inf. Lists must hold
 * distinct ascending block indices in [0, NB); cnt in [0, NB].
 *   q  bf16 [HQ][L][D]; k, v bf16 [HKV][L][D]
 *   idx int32 [HQ][NB][NB], cnt int32 [HQ][NB]  (e.g. from xattn_select)
 *   o   bf16 [HQ][L][D] (output)
 *   lse fp32 [HQ][L] (output) or NULL
 * QK^T and PV run on the bf16 matrix cores with fp32 accumulation; the
 * online softmax is fp32 and P is rounded to bf16 for the PV product. The
 * normaliser sums the same rounded P (so o is a weighted mean of the values
 * with consistent weights); lse carries that rounding, at most 2^-8 relative
 * in the sum, i.e. below 0.004 in lse.
 */
int xattn_block_sparse_attn(const void *q, const void *k, const void *v,
                            const xattn_dims *dims, int block, const int32_t *idx,
                            const int32_t *cnt, void *o, float *lse, void *stream);

/*
 * Dense reference mode (the paper's speedup denominator, Sec. 4.3): the same
 * kernel as xattn_block_sparse_attn with every candidate block listed
 * (j <= b causal, all j otherwise), block 128. Bitwise equal to
 * xattn_block_sparse_attn on the lists xattn_select returns for tau >= 1.
 */
int xattn_dense_attn(const void *q, const void *k, const void *v,
                     const xattn_dims *dims, void *o, float *lse, void *stream);

/*
 * The three steps chained on one stream: score -> select -> sparse attention.
 * workspace: at least xattn_forward_workspace_size() bytes. It holds, in
 * order, scores fp32 [HQ][NB][NB], idx int32 [HQ][NB][NB], cnt int32 [HQ][NB]
 * (each at a 256-byte aligned offset reported by xattn_forward_layout) and
 * the scoring scratch; after the call the caller may read scores/idx/cnt there.
 */
int xattn_forward_workspace_size(const xattn_dims *dims, int block, int stride,
                                 size_t *bytes);
int xattn_forward_layout(const xattn_dims *dims, int block, int stride,
                         size_t *scores_off, size_t *idx_off, size_t *cnt_off,
                         size_t *scratch_off);
int xattn_forward(const void *q, const void *k, const void *v, const xattn_dims *dims,
                  int block, int stride, float tau, void *o, float *lse,
                  void *workspace, size_t workspace_bytes, void *stream);

/*
 * xattn_forward without allocation, for callers that cannot allocate device
 * memory: code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc. The workspace of xattn_forward lives in a static device
 * array of XATTN_NOALLOC_SCRATCH_BYTES bytes that the library owns (one per
 * GPU, held until the process ends; its address is looked up once per device
 * on the first call with that device current). The caller passes inputs and
 * outputs only; the call makes no allocation of any kind.
 *   Everything else as xattn_forward (o, lse and their meaning; results
 *   bitwise equal to xattn_forward's on the same inputs).
 * Errors: as xattn_forward, plus XATTN_ERR_UNSUPPORTED when the problem needs
 * more scratch than the static array holds (xattn_forward_workspace_size()
 * > XATTN_NOALLOC_SCRATCH_BYTES), and XATTN_ERR_HIP if the array's address
 * cannot be obtained.
 * Every call on one GPU shares that GPU's array, which keeps the last call's
 * contents: calls that overlap on one GPU (several streams or threads at
 * once) race and must be serialised by the caller.
 */
#define XATTN_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)
int xattn_forward_noalloc(const void *q, const void *k, const void *v, const xattn_dims *dims,
                          int block, int stride, float tau, void *o, float *lse, void *stream);

/*
 * Denoising-step schedule of the video-generation experiment (Sec. 4.2):
 * dense attention for the first warmup_steps steps of a diffusion sampler
 * (step < warmup_steps; the paper uses 5 of 50), XAttention from then on.
 *   step          0-based index of the current denoising step (>= 0)
 *   warmup_steps  number of leading dense steps (>= 0; 0 = never dense)
 * A dense step is exactly xattn_dense_attn (the workspace is not touched and
 * may be NULL); a later step is exactly xattn_forward with the same arguments.
 */
int xattn_forward_scheduled(const void *q, const void *k, const void *v,
                            const xattn_dims *dims, int block, int stride, float tau,
                            int step, int warmup_steps, void *o, float *lse,
                            void *workspace, size_t workspace_bytes, void *stream);

/*
 * Minimum-threshold prediction (Sec. 3.3). The paper fills a table D[h][m],
 * the best performance reachable with exactly m threshold adjustments over
 * the first h heads, each adjustment lowering one head's threshold by 10 %
 * (t <- 0.9 t); head h either keeps D[h-1][m] or takes one more adjustment on
 * top of D[h-1][m-1]. Here a head may take up to max_adjust adjustments
 * (max_adjust = 1 is the paper's recurrence) and performance is additive over
 * heads, given as a table from the caller (for instance minus each head's
 * output error at each adjusted threshold, from xattn_head_error).
 *   perf         host double [heads][max_adjust + 1]: perf[h][a] is head h's
 *                performance after a adjustments; finite
 *   adjustments  M, the total number of adjustments, 0 <= M <= heads * max_adjust
 *   adjust       host int32 [heads] (output): adjustments per head, summing
 *                to M; the threshold of head h becomes t0 * 0.9^adjust[h]
 *   best         host double (output, may be NULL): D[heads][M]
 * On equal performance a head keeps fewer adjustments. Host only (no GPU).
 * XATTN_ERR_ARG for a NULL table or adjust, heads < 1, max_adjust < 1, M
 * outside [0, heads * max_adjust] or a non-finite entry; XATTN_ERR_UNSUPPORTED
 * for tables above 2^26 entries or heads * max_adjust above 2^20.
 */
int xattn_threshold_dp(const double *perf, int heads, int max_adjust, int adjustments,
                       int32_t *adjust, double *best);

/*
 * The thresholds of the minimum-threshold prediction (Sec. 3.3): after a
 * reductions of 10 % from tau0 a head's threshold is tau0 * 0.9^a, computed
 * in fp64 and rounded once to the fp32 value the selection receives.
 *   levels  host float [max_adjust + 1] (output): levels[a] for a = 0 .. max_adjust
 * XATTN_ERR_ARG for a NULL array, tau0 <= 0 / not finite, or max_adjust < 0.
 * Host only (no GPU).
 */
int xattn_threshold_levels(double tau0, int max_adjust, float *levels);

/*
 * The whole prediction step of Sec. 3.3 on a per-head error table: the
 * dynamic program of xattn_threshold_dp with performance = minus the error
 * (the assignment of exactly `adjustments` reductions with the least total
 * error; on equal totals a head keeps fewer adjustments), followed by the
 * thresholds it implies.
 *   err        host double [heads][max_adjust + 1]: err[h][a] is head h's error
 *              after a reductions (e.g. xattn_head_error_mean at levels[a]); finite
 *   tau0       the threshold before any reduction (> 0)
 *   adjust     host int32 [heads] (output), summing to `adjustments`
 *   tau_h      host float [heads] (output): tau0 * 0.9^adjust[h] as in
 *              xattn_threshold_levels, ready for xattn_select_heads
 *   total_err  host double (output, may be NULL): the least total error
 * Errors as xattn_threshold_dp, plus XATTN_ERR_ARG for a bad tau0. Host only.
 */
int xattn_threshold_predict(const double *err, int heads, int max_adjust, int adjustments,
                            double tau0, int32_t *adjust, float *tau_h, double *total_err);

/*
 * Per-head output error, the performance proxy for xattn_threshold_dp:
 * err[h] = sum (o - o_ref)^2 / sum o_ref^2 over head h's [L][D] outputs
 * (bf16 inputs, fp64 accumulation, a fixed order: deterministic).
 *   o, o_ref   bf16 [HQ][L][D] device
 *   err        double [HQ] device (output)
 *   workspace  at least xattn_head_error_workspace_size() bytes of device memory
 */
int xattn_head_error_workspace_size(const xattn_dims *dims, size_t *bytes);
int xattn_head_error(const void *o, const void *o_ref, const xattn_dims *dims, double *err,
                     void *workspace, size_t workspace_bytes, void *stream);

/*
 * xattn_head_error averaged over the batch: err[h] for query head h < hq is
 * (1 / batch) * sum_n of the error of row n * hq + h, added in batch order
 * (the per-head table of the prediction covers heads of the model, not
 * sequences). err is double [hq] device (output); the workspace is the one
 * xattn_head_error_workspace_size() reports. Errors as xattn_head_error.
 */
int xattn_head_error_mean(const void *o, const void *o_ref, const xattn_dims *dims,
                          double *err, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Serving after the prefill: rotary positions, a paged cache of keys and
 * values, the attention of one new token per sequence over it, and the
 * eviction of its lightest tokens. Unlike the prefill these calls take any
 * number of tokens (down to one) and strided inputs.
 *
 * Strides: `x_strides` holds 3 host int64, the distances in ELEMENTS between
 * batch elements, heads and tokens of x[batch][heads][tokens][128]; the 128
 * values of a vector are contiguous. Strides are >= 0 and multiples of 8 (the
 * stride of a dimension of size 1 is not used), those of an output from the smallest
 * on at least what the smaller ones span, so that no two vectors overlap; every
 * array of bfloat16 or cache values is 16-byte aligned. Read during the call only.
 */

/* What a call writes (outputs, weights, workspace; in xattn_cache_append the places
 * of the new tokens) shares no memory with what it reads or with anything else it
 * writes, but where a call says so; XATTN_ERR_ARG where the host can see that it does. */

/* Rotary positions: the 64 pairs of a head are shared out among `axes` position
 * axes (e.g. time, height, width), pairs[a] to axis a in order; the pairs
 * behind them are not rotated.
 *   interleaved  0: pair i is elements (i, i + 64); 1: (2 i, 2 i + 1)
 *   freq         host double [sum of pairs]: radians per position, finite; read
 *                during the call only (copied into the launch) */
typedef struct xattn_rotary_plan {
    int32_t axes;     /* 1 .. 3 */
    int32_t pairs[3]; /* each >= 0 (>= 1 for a < axes, 0 behind), sum <= 64 */
    int32_t interleaved;
    const double *freq;
} xattn_rotary_plan;

/*
 * Rotates every pair (x, y) of every vector by phi = pos * freq:
 * (x cos phi - y sin phi, x sin phi + y cos phi), or by -phi if `inverse`
 * (the inverse rotation, its transpose and therefore its gradient).
 *   x    bf16 [batch][heads][tokens][128], strided   (e.g. a projection's output
 *        [batch][tokens][heads][128])
 *   pos  int32 [axes][batch][tokens] device, any values
 *   out  bf16, same shape, strided; x itself with x's strides, or no memory of x
 *        (which may be another slice of the same buffer)
 * Angles are products in fp64 (off by 2^-52 of themselves), reduced to a turn before
 * they are rounded, so far positions are as exact as near ones; sine and cosine are
 * good to 2.2e-7, the rotation is fp32, rounded once.
 * XATTN_ERR_ARG for a bad plan, stride, alignment or NULL.
 */
int xattn_rotary(const void *x, const int64_t *x_strides, int batch, int heads, int tokens,
                 int head_dim, const int32_t *pos, const xattn_rotary_plan *plan, int inverse,
                 void *out, const int64_t *out_strides, void *stream);

/* A pool of pages that hold the keys and values of `page` tokens each:
 *   k, v              [pages][hkv][page][128], bf16 or OCP e4m3 (device)
 *   k_scale, v_scale  uint8 [pages][hkv][page] (device; e4m3 only, else NULL):
 *                     a vector's values are its e4m3 values times
 *                     2^(byte - 127), byte 1 .. 254
 * A sequence's pages are a row of a page table int32 [batch][table_pages]
 * (device): token t is row t % page of page table[b][t / page]. Entries outside
 * 0 .. pages-1 stand for no page: what they would hold is neither read nor
 * written (its keys are not attended to). Sequences may share pages. */
enum xattn_cache_type { XATTN_CACHE_BF16 = 0, XATTN_CACHE_E4M3 = 1 };
typedef struct xattn_cache {
    int32_t pages;
    int32_t page; /* 16, 32, 64, 128 or 256 */
    int32_t hkv;
    int32_t head_dim; /* 128 */
    int32_t type;
    void *k;
    void *v;
    uint8_t *k_scale;
    uint8_t *v_scale;
} xattn_cache;

/*
 * Writes new tokens into their pages: token t < count[b] of sequence b becomes
 * token start[b] + t of its page table's row, its key rotated on the way if a
 * plan is given. Nothing else is written; tokens whose place is negative or
 * behind the table's row are not stored.
 *   k, v    bf16 [batch][hkv][tokens][128], strided
 *   start   int32 [batch] device
 *   count   int32 [batch] device, or NULL for `tokens` everywhere (larger values
 *           count as `tokens`, negative ones as 0)
 *   pos     int32 [axes][batch][tokens] device, with plan; both NULL: no rotation
 * bf16: a rotated key is rounded once, all else copied. e4m3: the scale is the
 * least power of two (at least 2^-126) that brings the vector's largest finite
 * magnitude to at most 448 (1 for a vector of zeros); a key that is rotated
 * takes the largest length of a pair instead, its square summed in fp32, which bounds
 * it whatever the angle (a pair of which one value is not finite counts with the
 * other); it is turned in fp64. Values are
 * rounded to nearest even; infinities become +-448, NaN stays NaN.
 * No place may be written twice in a call (a page in two tables' rows, for
 * instance): which of the tokens it then holds is not defined.
 */
int xattn_cache_append(const void *k, const int64_t *k_strides, const void *v,
                       const int64_t *v_strides, int batch, int tokens, const int32_t *count,
                       const int32_t *start, const int32_t *table, int table_pages,
                       const int32_t *pos, const xattn_rotary_plan *plan,
                       const xattn_cache *cache, void *stream);

/*
 * Attention of one new token per sequence over its cached tokens
 * t < lens[b] (clamped to 0 .. table_pages * page):
 *   o[b][h]   = sum_t softmax_t(q[b][h] . k_t / sqrt(128)) v_t
 *   lse[b][h] = log sum_t exp(q[b][h] . k_t / sqrt(128))      (natural log)
 * with the head's keys and values (contiguous GQA grouping, any group size).
 * The new token's own key is one of the cached ones: append first. Rows without
 * a key get o = 0 and lse = -inf; keys whose products are -inf have no weight
 * (their values must be finite, as every value with a weight of 0 must). What a
 * page holds behind the last token has no effect, whatever it is.
 * Values (those in 8 bits times their scales) may be of any finite magnitude: the
 * weights' sum is divided by last, but no sum on the way passes the largest value.
 * Values below about 2^-64 lose bits (2^-77 in tables of up to 131,072 tokens). The
 * products q . k, before a key's scale is applied, must be finite in fp32.
 * Several new tokens of one sequence are several rows with the same pages and
 * each its own length.
 *   q        bf16 [batch][hq][128]; o the same (output; may be q itself)
 *   lens     int32 [batch] device
 *   lse      fp32 [batch][hq] (output) or NULL
 *   weights  fp32 [batch][hkv][table_pages * page], 16-byte aligned (updated), or
 *            NULL: entry t of a key head grows by the sum of its query heads'
 *            softmax_t, for t < lens[b]; what lies behind is left as it was
 *   workspace  at least xattn_decode_workspace_size() bytes (`weights`: whether
 *            the call has them; 0 for small calls, then it may be NULL), 16-byte
 *            aligned; its contents on entry are ignored. Calls that may run at the
 *            same time need one each. Its size follows the table's width, not the
 *            lengths, which only the device knows: up to 1536 * 520 bytes times the
 *            query heads of a key head (32 at most) and, with weights, another
 *            batch * hq * (4 * table_pages * page + 8), all in multiples of 256.
 *            (64 sequences of 32 heads in a table of 131,072 tokens: 1 GiB.)
 * QK^T and PV run on the bf16 matrix cores with fp32 accumulation (e4m3 values
 * are exact in bf16); the softmax is fp32, and P goes into PV as the sum of three
 * bf16 values, within 2^-29 of it. The output is rounded once.
 */
int xattn_decode_workspace_size(const xattn_cache *cache, int batch, int hq, int table_pages,
                                int weights, size_t *bytes);
int xattn_decode(const void *q, const xattn_cache *cache, int batch, int hq,
                 const int32_t *table, int table_pages, const int32_t *lens, void *o, float *lse,
                 float *weights, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Eviction by accumulated attention weight: of each sequence and key head the
 * `budget` tokens that are worth most move, in their order, to the pages of
 * another table. Sequences of at most `budget` tokens move whole. Of longer
 * ones the last `recent` tokens stay, and of those before them the
 * budget - recent of the largest weight (equal weights: the earlier token; NaN
 * is below every number). Each key head keeps its own tokens: keys carry their
 * positions, the heads need not agree. The old pages are only read, so they may
 * be shared with other sequences; free them afterwards.
 *   table, lens  the sequences before: int32 [batch][table_pages], [batch];
 *                lens clamped to 0 .. table_pages * page
 *   weights      fp32 [batch][hkv][table_pages * page], e.g. from xattn_decode. A
 *                prompt has none of its own: its last queries give it some, each a
 *                row of xattn_decode with the sequence's pages, its own length and
 *                its own weights, which are then summed
 *   new_table    int32 [batch][new_pages]: distinct pages, none of them in
 *                `table`; new_pages * page >= budget
 *   kept         int32 [batch][hkv][budget] (output): the tokens kept, ascending,
 *                -1 behind them
 *   new_lens     int32 [batch] (output): min(lens, budget)
 *   new_weights  fp32 [batch][hkv][new_pages * page] (output): the kept tokens'
 *                weights, 0 behind them
 *   workspace    as for xattn_decode, xattn_evict_workspace_size() bytes (0 for
 *                tables of up to 16384 tokens, then it may be NULL; else 49,160 for
 *                every 8192 tokens of the table's width and key head)
 * The weights are 16-byte aligned. 1 <= budget, 0 <= recent <= budget. Page rows
 * behind the kept tokens are left as they were. A token without a page takes its
 * place among the kept ones like any other, by its weight, and there is nothing to
 * move: that place is left as it was too, and a later call attends to it. So every
 * token below lens that can be kept should have a page (a weight of NaN is below all
 * others, where those fill the budget).
 */
int xattn_evict_workspace_size(const xattn_cache *cache, int batch, int table_pages, size_t *bytes);
int xattn_cache_evict(const xattn_cache *cache, int batch, const int32_t *table, int table_pages,
                      const int32_t *lens, const float *weights, int budget, int recent,
                      const int32_t *new_table, int new_pages, int32_t *kept, int32_t *new_lens,
                      float *new_weights, void *workspace, size_t workspace_bytes, void *stream);

/* Static description of a status code (never NULL). */
const char *xattn_strerror(int status);
/* Message describing the last failure on the calling thread ("" if none). */
const char *xattn_last_error(void);
/* Library ABI version: major * 10000 + minor * 100 + patch. */
int xattn_version(void);

#ifdef __cplusplus
}
#endif

#endif /* XATTN_H */
