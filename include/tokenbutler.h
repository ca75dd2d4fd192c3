/*
 * tokenbutler.h -- C ABI of the MI355X (gfx950) implementation of TokenButler's decode-time
 * hot path: score every cached token with a low-dimensional importance query against the
 * projected key cache, keep a fixed top-k budget per query head (sink prefix and local window
 * always kept), optionally widen a reused selection with neighbours, and run decode attention
 * over the selected K/V rows only.
 *
 * Conventions shared by every entry point
 *  - All tensor pointers are DEVICE pointers owned by the caller.  The library never
 *    allocates, frees or keeps them.  Scratch memory comes in through `ws` (see
 *    tb_workspace_bytes / tb_workspace_init).
 *  - `stream` is a hipStream_t passed as void* (NULL = the null stream).  Every call only
 *    enqueues work on that stream and returns; nothing synchronises.
 *  - Errors are return codes.  All argument checks happen on the host before anything is
 *    launched; a failing call launches nothing.
 *  - K, V, K_imp, W, q, q_imp share one element type (tb_dtype).  Scores, attention output
 *    and log-sum-exp are always fp32; index lists and counts are int32.
 *  - Query head h reads KV head h / (Hq / Hkv)  (consecutive query heads share a KV head).
 *  - Supported shapes: D in {64, 128}; Dimp in {16, 32, 64}; Hq / Hkv in {1, 2, 4, 8};
 *    N <= 2^20 for selection.  Row starts must be 16-byte aligned: base pointers 16-byte
 *    aligned and all strides multiples of 8 elements.  Anything else -> TB_ERR_UNSUPPORTED.
 */
#ifndef TOKENBUTLER_H_
#define TOKENBUTLER_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum tb_status {
  TB_OK = 0,
  TB_ERR_INVALID_ARG = 1, /* null pointer, negative size, inconsistent shape, capacity too small */
  TB_ERR_UNSUPPORTED = 2, /* well-formed but outside the supported shapes / alignments          */
  TB_ERR_WORKSPACE = 3,   /* ws is NULL or ws_bytes below tb_workspace_bytes()                  */
  TB_ERR_HIP = 4          /* a HIP launch reported an error                                     */
} tb_status;

typedef enum tb_dtype { TB_F32 = 0, TB_BF16 = 1 } tb_dtype;

/* One layer's cache view.  Plain data, read during the call only.
 * K, V   : [B][Hkv][>=N][D]     element (b,h,n,d) at  b*stride_b + h*stride_h + n*stride_n + d
 * K_imp  : [B][Hkv][>=N][Dimp]  same addressing with the ki_ strides
 * Strides are in elements; the innermost dimension is contiguous. */
typedef struct tb_cache_desc {
  int32_t B, Hq, Hkv, D, Dimp;
  int32_t dtype; /* tb_dtype */
  int64_t N;     /* tokens currently valid in the cache */
  int64_t k_stride_b, k_stride_h, k_stride_n;
  int64_t v_stride_b, v_stride_h, v_stride_n;
  int64_t ki_stride_b, ki_stride_h, ki_stride_n;
} tb_cache_desc;

/* Operation selector for tb_workspace_bytes. */
enum { TB_OP_SELECT = 1, TB_OP_ATTN = 2, TB_OP_DECODE_STEP = 3, TB_OP_ATTN_MX = 4, TB_OP_PAGED_ATTN = 5 };

/* Key-cache projection (Sec. 3.1, "Key-cache projection": K_imp = K W_K, W_K in R^{D x Dimp}).
 * Fills K_imp[b,h,n,:] = round(K[b,h,n,:] . W[hw]) for n_begin <= n < n_end, fp32 accumulation,
 * one round-to-nearest-even to the storage type.  Covers both the one-row append and the
 * batched deferred projection of a whole window of rows (Sec. 3.3).
 * W: [Hw][D][Dimp] contiguous; Hw == 1 (one matrix per layer, as the paper writes it) or
 * Hw == Hkv.  Requires 0 <= n_begin <= n_end <= desc->N.  Empty range: no-op, TB_OK. */
tb_status tb_project_keys(const tb_cache_desc* desc, const void* K, const void* W, int32_t Hw, void* Kimp,
                          int64_t n_begin, int64_t n_end, void* stream);

/* Importance scoring (abstract; Sec. 3.4, prediction steps).
 * scores[b,h,n] = scale * sum_j q_imp[b,h,j] * K_imp[b,h/g,n,j]   for 0 <= n < desc->N.
 * q_imp: [B][Hq][Dimp] contiguous.  scores: fp32 [B][Hq][score_stride], score_stride >= N and
 * a multiple of 4.  The paper gives no normalisation of the score; `scale` is explicit. */
tb_status tb_score(const tb_cache_desc* desc, const void* q_imp, const void* Kimp, float scale, float* scores,
                   int64_t score_stride, void* stream);

/* Token selection policy (Sec. 4 "Token Selection Policy").  Per (b,h): candidates are the
 * positions [lo, hi) with lo = min(sink, N), hi = max(lo, N - window); the kk = min(k, hi-lo)
 * candidates with the largest score are kept.  Ordering: larger score first, NaN counts as
 * -inf, -0 equals +0, equal scores -> lower index first.  Output per (b,h), ascending:
 *   idx = [0,lo) ++ ascending(kept) ++ [hi,N),   count = lo + kk + (N - hi).
 * idx: int32 [B][Hq][idx_cap], idx_cap >= lo + kk + (N - hi); entries beyond count are left
 * untouched.  count: int32 [B][Hq].  ws / ws_bytes are optional (NULL / 0 is fine): the selection
 * keeps its scratch on chip, except that long rows (N > 65536 with a budget of at most an
 * eighth of the candidates) are cut into pieces that are filtered by several compute units and
 * then combined, which needs tb_workspace_bytes(TB_OP_SELECT, desc, sink + k + window) bytes
 * (8 bytes per slot for a kept score: at most min(2k + 4096, piece length) slots per piece of
 * 16384 scores, so up to 8 N bytes per (b,h) -- 201 MB for B*Hq = 256, N = 131072, k = 4096);
 * with less, one workgroup selects the whole row (same result, slower).  The batch axis may
 * just as well run over the consumer layers of a producer (Sec. 3.3: their scoring and
 * selection are batched): stack the layers' projected-key caches and queries along B. */
tb_status tb_select_topk(const tb_cache_desc* desc, const float* scores, int64_t score_stride, int32_t k,
                         int32_t sink, int32_t window, int32_t* idx, int32_t* count, int64_t idx_cap, void* ws,
                         size_t ws_bytes, void* stream);

/* Neighbour fetching (Sec. 3.4 "Neighbor fetching").  idx_in lists must be strictly ascending
 * and within [0, N).
 * mode 0: idx_out = ascending, duplicate-free union over the input of [i-radius, i+radius]
 *         clipped to [0, N).  cap_out >= min(N, (2*radius+1) * cap_in) is required.
 * mode 1: cluster-aware fetch: consecutive selected positions form clusters and every
 *         selected token adds the next free position past its cluster (left-to-right; free
 *         positions taken by an earlier cluster are skipped), 2*count positions unless the
 *         sweep reaches N.  radius is ignored.  cap_out >= min(N, 2 * cap_in).
 * Units are the B*Hq lists; count_out[u] receives the output length. */
tb_status tb_expand_neighbors(int32_t B, int32_t Hq, int64_t N, int32_t radius, int32_t mode,
                              const int32_t* idx_in, const int32_t* count_in, int64_t cap_in, int32_t* idx_out,
                              int32_t* count_out, int64_t cap_out, void* stream);

/* Decode attention over the selected rows (Sec. 3.3: attention touches sink, window and
 * important tokens only; with every token selected it is dense decode attention).
 *   out[b,h,:] = sum_i softmax_i(sm_scale * q[b,h] . K[b,h/g,n_i]) * V[b,h/g,n_i]
 * where n_i runs over idx[b,h,0:count[b,h]] followed by the dense range [tail_begin, tail_end)
 * (tokens appended since the list was made, which are always attended while a selection is
 * reused across a prediction interval; pass tail_begin == tail_end for none).
 * q: [B][Hq][D] contiguous.  idx entries must lie in [0, desc->N); tail_end <= desc->N.
 * max_count: host-side upper bound on count[b,h] (<= idx_cap) used to size the launch; a list
 * longer than max_count is truncated to it, and entries from max_count on are not read.  out: fp32 [B][Hq][D]; lse: fp32 [B][Hq] or NULL.
 * An empty list gives out = 0 and lse = -inf.  ws: tb_workspace_bytes(TB_OP_ATTN, ...). */
tb_status tb_sparse_decode_attn(const tb_cache_desc* desc, const void* q, const void* K, const void* V,
                                const int32_t* idx, const int32_t* count, int64_t idx_cap, int64_t max_count,
                                int64_t tail_begin, int64_t tail_end, float sm_scale, float* out, float* lse,
                                void* ws, size_t ws_bytes, void* stream);

/* Head-less form of tb_sparse_decode_attn (Appendix "Additional Efficiency Evaluation": the
 * predictor gives one importance per token per layer, with no head dimension, so one token list
 * serves every head of the layer).  idx: [B][idx_cap], count: [B]; every query head h of batch
 * element b attends over idx[b,0:count[b]] followed by [tail_begin, tail_end).  Such a list is
 * what tb_score and tb_select_topk produce under a descriptor with Hq = Hkv = 1 (one importance
 * head).  All other arguments, results and errors as tb_sparse_decode_attn. */
tb_status tb_sparse_decode_attn_shared(const tb_cache_desc* desc, const void* q, const void* K, const void* V,
                                       const int32_t* idx, const int32_t* count, int64_t idx_cap,
                                       int64_t max_count, int64_t tail_begin, int64_t tail_end, float sm_scale,
                                       float* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/* tb_sparse_decode_attn for callers that cannot allocate device memory or hand over a workspace
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): same
 * arguments minus ws / ws_bytes, same kernels and bit-identical results.  The scratch (arrival
 * counters and split partials) lives in a device array inside the library, 4 MiB per GPU, held
 * from the first call on that GPU until the process ends.  A shape whose scratch would exceed
 * that (tb_workspace_bytes(TB_OP_ATTN, ...) > 4 MiB) is rejected with TB_ERR_WORKSPACE before
 * anything is launched.  The call allocates nothing and enqueues a small fill kernel (the
 * counters are cleared on every call) followed by the attention kernel.  All calls on one GPU
 * share the array: calls that overlap in time on one GPU (different streams) race. */
tb_status tb_sparse_decode_attn_static(const tb_cache_desc* desc, const void* q, const void* K, const void* V,
                                       const int32_t* idx, const int32_t* count, int64_t idx_cap,
                                       int64_t max_count, int64_t tail_begin, int64_t tail_end, float sm_scale,
                                       float* out, float* lse, void* stream);

/* Migration of selected rows into the "Important Buffer" (Sec. 3.3 "Inference Setup": the
 * paper keeps the attended tokens in contiguous buffers and copies the selection there on
 * prediction steps).  Kbuf/Vbuf[b,h,i,:] = K/V[b,h/g,idx[b,h,i],:] for i < min(count[b,h], max_count).
 * Kbuf, Vbuf: [B][Hq][buf_cap][D] contiguous, element type of the cache, buf_cap >= max_count;
 * rows at and beyond the count are left untouched.  The buffers are per *query* head, because
 * every query head selects its own tokens. */
tb_status tb_gather_kv(const tb_cache_desc* desc, const void* K, const void* V, const int32_t* idx,
                       const int32_t* count, int64_t idx_cap, int64_t max_count, void* Kbuf, void* Vbuf,
                       int64_t buf_cap, void* stream);

/* tb_gather_kv for the layout with a Sink Buffer and a Local Window Buffer of their own (Sec. 3.3
 * "Inference Setup"): a list made by tb_select_topk (and widened by tb_expand_neighbors) begins
 * with the sink positions and ends with the local-window positions; those rows live in their own
 * buffers, so only the entries in between are migrated:
 *   Kbuf/Vbuf[b,h,i,:] = K/V[b,h/g,idx[b,h,skip_front + i],:]   for 0 <= i < count_out[b,h],
 *   count_out[b,h] = max(0, min(count[b,h], max_count) - skip_front - skip_back).
 * buf_cap >= max(0, max_count - skip_front - skip_back); count_out: int32 [B][Hq], always written. */
tb_status tb_gather_important(const tb_cache_desc* desc, const void* K, const void* V, const int32_t* idx,
                              const int32_t* count, int64_t idx_cap, int64_t max_count, int32_t skip_front,
                              int32_t skip_back, void* Kbuf, void* Vbuf, int64_t buf_cap, int32_t* count_out,
                              void* stream);

/* Arrival of new rows in a buffer (the Local Window ring of Sec. 3.3): one launch for K and V of every
 * KV head.  Kdst/Vdst[b,h,dst_row + i,:] = K/V[b,h,src_row + i,:] for 0 <= i < rows.  src and dst describe
 * the two places (same B, Hkv, D and dtype; strides as everywhere, rows [0, desc->N)); they must not overlap. */
tb_status tb_append_kv(const tb_cache_desc* src, const void* K, const void* V, int64_t src_row, const tb_cache_desc* dst,
                       void* Kdst, void* Vdst, int64_t dst_row, int64_t rows, void* stream);

/* tb_sparse_decode_attn over rows that tb_gather_kv has migrated: the rows 0 .. count[b,h]-1 of
 * the per-query-head buffers (no index list is read) followed by the dense range
 * [tail_begin, tail_end) of the cache K, V (the local window of tokens appended since the
 * migration).  Same result, bit for bit, as tb_sparse_decode_attn with the list the buffers
 * were filled from.  ws: tb_workspace_bytes(TB_OP_ATTN, ...). */
tb_status tb_buffered_decode_attn(const tb_cache_desc* desc, const void* q, const void* Kbuf, const void* Vbuf,
                                  int64_t buf_cap, const int32_t* count, int64_t max_count, const void* K,
                                  const void* V, int64_t tail_begin, int64_t tail_end, float sm_scale,
                                  float* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/* tb_append_kv of one row (src_row of the cache src, K_src, V_src) into row dst_row of the cache desc, K, V, then
 * tb_buffered_decode_attn over that cache, in one launch: the attention takes the new row from where it comes
 * from while it is copied.  Arguments and results are those of the two calls; src and desc as in tb_append_kv. */
tb_status tb_append_buffered_decode_attn(const tb_cache_desc* src, const void* K_src, const void* V_src, int64_t src_row,
                                         const tb_cache_desc* desc, const void* q, const void* Kbuf, const void* Vbuf,
                                         int64_t buf_cap, const int32_t* count, int64_t max_count, void* K, void* V,
                                         int64_t dst_row, int64_t tail_begin, int64_t tail_end, float sm_scale,
                                         float* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/* tb_gather_important of the lists, from the cache src, K_src, V_src into the buffers, then (src_row >= 0) tb_append_kv of one row
 * into row dst_row of the cache desc, K, V, then tb_buffered_decode_attn over buffers (max_count: the lists', no more than
 * buf_cap) and cache, in one launch: a listed row is attended to on its way into its buffer.  Arguments and results are those of
 * the calls; src and desc agree in all but N and strides, do not overlap, and src->N <= 2^30 (else TB_ERR_UNSUPPORTED). */
tb_status tb_migrate_buffered_decode_attn(const tb_cache_desc* src, const void* K_src, const void* V_src, const int32_t* idx,
                                          const int32_t* count, int64_t idx_cap, int64_t max_count, int32_t skip_front, int32_t skip_back,
                                          int32_t* count_out, int64_t src_row, const tb_cache_desc* desc, const void* q, void* Kbuf,
                                          void* Vbuf, int64_t buf_cap, void* K, void* V, int64_t dst_row, int64_t tail_begin,
                                          int64_t tail_end, float sm_scale, float* out, float* lse, void* ws, size_t ws_bytes,
                                          void* stream);

/* One prediction step in a single enqueue: tb_score -> tb_select_topk -> tb_sparse_decode_attn
 * with one validation pass and one launch plan.  Results (scores, idx, count, out, lse) are
 * identical to calling the three entry points one after the other.
 * ws: tb_workspace_bytes(TB_OP_DECODE_STEP, ...).  For N > 65536, projected rows of at most
 * min(64, 32 Hq / Hkv) bytes and a budget of at most an eighth of the candidates this is about
 * 8 B Hq N bytes whatever the budget (the scoring kernel keeps candidates in lists with room for
 * whole pieces of a row): 547 MB for B*Hq = 512, N = 131072.  With less, down to what
 * TB_OP_SELECT and TB_OP_ATTN ask for (there: 220 MB with a budget of 1311) or TB_OP_ATTN alone,
 * the call takes the same arguments and gives the same results by a slower route. */
tb_status tb_decode_step(const tb_cache_desc* desc, const void* q_imp, const void* Kimp, float score_scale,
                         const void* q, const void* K, const void* V, int32_t k, int32_t sink, int32_t window,
                         float sm_scale, float* scores, int64_t score_stride, int32_t* idx, int32_t* count,
                         int64_t idx_cap, float* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/* Query prediction of a producer layer (Sec. 3.1 "Query prediction"): from the hidden state of
 * the token being decoded, a LayerNorm and a two-layer MLP give one importance query per query
 * head for each of the G consumer layers ("slots") that follow the producer:
 *   x = LN(h) = (h - mean) / sqrt(var + ln_eps) * gamma + beta      (over E, biased variance)
 *   z = gelu(W1 x + b1)          (exact erf form; the paper does not name the nonlinearity)
 *   y = W2 z + b2,   q_imp[s][b][hq][j] = y[(s*Hq + hq)*Dimp + j]
 * h: [B][E]; gamma, beta: [E]; W1: [hidden][E]; b1: [hidden]; W2: [G*Hq*Dimp][hidden];
 * b2: [G*Hq*Dimp] -- all contiguous, all of element type `dtype`; fp32 accumulation, one rounding
 * when q_imp is stored.  q_imp: [G][B][Hq][Dimp] of `dtype`: slot s is the [B][Hq][Dimp] array that
 * tb_score takes for consumer layer s.  hidden_act: fp32 [B][hidden], receives z; ln_act: fp32
 * [B][E], receives LN(h) when B > 2 (both are scratch that the caller owns; 16-byte aligned, as
 * are h, gamma, beta, W1, W2).  E and hidden must be multiples of 8, E <= 8192, hidden <= 2048. */
typedef struct {
  int32_t E, hidden, G, Hq, Dimp;
  tb_dtype dtype;
  float ln_eps;
} tb_predictor_desc;
tb_status tb_predict_queries(const tb_predictor_desc* p, int32_t B, const void* h, const void* gamma,
                             const void* beta, const void* W1, const void* b1, const void* W2, const void* b2,
                             float* hidden_act, float* ln_act, void* q_imp, void* stream);

/* ---- a cache in microscaled 4-bit floating point ------------------------------------------------
 * Rows of K, V and K_imp in OCP's MXFP4 format: a row is cut into blocks of 32 elements, each element a sign and one of
 * 0, 0.5, 1, 1.5, 2, 3, 4, 6 (E2M1), each block with a power of two (E8M0, 2^(byte - 127)) that multiplies its elements; byte 255
 * makes all of them NaN.  4.25 bits an element instead of 16 or 32.
 * codes : [B][Hkv][N][inner/2]   bytes; element 2i of a row in the low half of byte i, element 2i + 1 in the high half
 * scales: [B][Hkv][N][inner/32]  bytes
 * with inner = D (K, V) or Dimp (K_imp; 32 or 64: with 16 there is no whole block -> TB_ERR_UNSUPPORTED).  Strides are in bytes,
 * the innermost dimension is contiguous; codes must be 16-byte aligned with strides that are multiples of 16, scales may lie
 * anywhere.  N: rows that the arrays have room for.  K and V of a token next to each other (one allocation of codes
 * [B][Hkv][N][2][D/2]) are read as one line.
 * The descriptor of a call gives the shape, and the element type of the queries or of the rows that are converted; its strides are
 * those of rows in that type, and are not looked at by calls that have none. */
typedef struct tb_mx_rows {
  void* codes;
  void* scales;
  int64_t N;
  int64_t code_stride_b, code_stride_h, code_stride_n;
  int64_t scale_stride_b, scale_stride_h, scale_stride_n;
} tb_mx_rows;

/* Rows src_row + i of K, V and K_imp (described by desc, rows [0, desc->N)) go to rows dst_row + i of Kq, Vq and Kimpq, 0 <= i <
 * rows, in one launch: a prompt, or the new token of a decode step.  A pair (K, Kq), (V, Vq), (Kimp, Kimpq) of NULLs is left out.
 * Per block: with the largest magnitude in [2^e, 2^(e+1)) the scale is 2^max(e - 2, -127), every element goes to the nearest
 * multiple that a code stands for, halves to the even code, beyond 6 to 6 (OCP Microscaling Formats v1.0); a block of zeros has
 * scale byte 0, and a block with an infinity or a NaN has byte 255 and codes 0.  Sources and destinations must not overlap.
 * rows <= 2^20. */
tb_status tb_quantize_mx(const tb_cache_desc* desc, const void* K, const void* V, const void* Kimp, int64_t src_row, const tb_mx_rows* Kq,
                         const tb_mx_rows* Vq, const tb_mx_rows* Kimpq, int64_t dst_row, int64_t rows, void* stream);

/* The way back: rows dst_row + i of K, V and K_imp receive the values that rows src_row + i of Kq, Vq and Kimpq stand for.  Exact in
 * either element type for all that tb_quantize_mx writes; scale bytes 253 and 254, which it does not, have codes that stand for more than
 * the largest number of either type (4 and 6 under 253, 2 to 6 under 254).  They are infinities here, and scores and attention that they
 * enter are infinite or NaN. */
tb_status tb_dequantize_mx(const tb_cache_desc* desc, const tb_mx_rows* Kq, const tb_mx_rows* Vq, const tb_mx_rows* Kimpq, int64_t src_row,
                           void* K, void* V, void* Kimp, int64_t dst_row, int64_t rows, void* stream);

/* tb_score over projected keys in 4 bits: the queries are taken as they are (fp32 or bf16), products are exact, sums fp32. */
tb_status tb_score_mx(const tb_cache_desc* desc, const void* q_imp, const tb_mx_rows* Kimp, float scale, float* scores, int64_t score_stride,
                      void* stream);

/* tb_sparse_decode_attn over a cache in 4 bits: lists, dense range, results as there.  idx and count may be NULL with max_count = 0
 * (the dense range alone: decode attention over all rows is tail_begin = 0, tail_end = N).  An attended row with a block that stands
 * for NaN makes the row's weight or the block's outputs NaN, as the formula does; rows that are not attended add nothing,
 * whatever they hold.  A head whose scores are all minus infinity has the results of an empty list.  Limits (else
 * TB_ERR_UNSUPPORTED): N <= 2^24, max_count <= 2^29, strides between rows below 2^24 bytes, a head's rows below 4 GiB.
 * ws: tb_workspace_bytes(TB_OP_ATTN_MX, ...). */
tb_status tb_sparse_decode_attn_mx(const tb_cache_desc* desc, const void* q, const tb_mx_rows* K, const tb_mx_rows* V, const int32_t* idx,
                                   const int32_t* count, int64_t idx_cap, int64_t max_count, int64_t tail_begin, int64_t tail_end,
                                   float sm_scale, float* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/* The head-less form: one list per batch element for all of its heads, as tb_sparse_decode_attn_shared. */
tb_status tb_sparse_decode_attn_shared_mx(const tb_cache_desc* desc, const void* q, const tb_mx_rows* K, const tb_mx_rows* V,
                                          const int32_t* idx, const int32_t* count, int64_t idx_cap, int64_t max_count, int64_t tail_begin,
                                          int64_t tail_end, float sm_scale, float* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/* ---- a cache in pages --------------------------------------------------------------------------
 * K and V held as pages of `page` rows of every KV head, handed out to sequences in any order: row n of sequence b is row n % page of
 * page table[b * table_stride + n / page].
 * K, V : [pages][Hkv][page][D]   element (p,h,r,d) at  p*stride_p + h*stride_h + r*stride_n + d, strides in elements (alignment as above)
 * table: int32, on the device, table_len entries a sequence.  An entry outside [0, pages) is a hole: nothing is written there, and its
 *        rows are attended to by nobody.  Sequences may share pages that are only read.
 * page is a power of two from 16 to 65536; page * stride_n stays below 2^29 elements (else TB_ERR_UNSUPPORTED, as for a page of another size).
 * Calls take the element type, B, Hq, Hkv and D from the descriptor, and N, the most rows that a sequence has (at most table_len * page);
 * the descriptor's strides are not looked at. */
typedef struct tb_paged_cache {
  void* K;
  void* V;
  const int32_t* table;
  int32_t pages, page, table_len;
  int64_t table_stride;
  int64_t k_stride_p, k_stride_h, k_stride_n;
  int64_t v_stride_p, v_stride_h, v_stride_n;
} tb_paged_cache;

/* Rows of tokens, [T][heads][D]: element (t,h,d) at t*stride_t + h*stride_h + d, strides in elements (alignment as above), so that
 * queries, keys and values may lie side by side as a projection leaves them. */
typedef struct tb_token_rows {
  void* rows;
  int64_t stride_t, stride_h;
} tb_token_rows;

/* New tokens of the sequences reach the cache, their queries and keys rotated by their positions on the way.
 * The T tokens of a call are those of sequence 0, then of sequence 1, ...: sequence b has the tokens cu[b] .. cu[b+1]-1 (cu: int32 [B+1],
 * cu[0] = 0; NULL: T / B tokens each), which are the last of its lens[b] rows (int32 [B], on the device as cu is): token number i of n
 * is row lens[b] - n + i.  T <= 2^22 (else TB_ERR_UNSUPPORTED).  Tokens whose row is not in [0, N), and those from cu[B] on, take no part:
 * nothing of theirs is read or written.
 *   angle(t, i) = positions[t] * inv_freq[i]   0 <= i < rot / 2; positions: int32 [T], NULL: the token's row; inv_freq: fp32 [rot / 2]
 *   (x[j], x[k]) -> (x[j] cos - x[k] sin, x[k] cos + x[j] sin)   of q and k, (j, k) = (i, i + rot / 2), or (2i, 2i + 1) if interleaved
 * angles (up to 2^50) to 2^-50 of a turn, the rest in 64 (fp32 rows) or in 32 (bf16 rows), rounded at the end; elements from rot on stay as they are.
 * rot: 0 (no rotation) to D, a multiple of 16.
 * k goes to K and, unless NULL, to k_out (what tb_project_keys takes); v to V; q, unless NULL, to q_out.  q_out may be q, and k_out k
 * (the same rows with the same strides); otherwise outputs overlap nothing.  No two tokens of a call may have the same row of the same page. */
tb_status tb_append_paged_kv(const tb_cache_desc* desc, const tb_paged_cache* cache, int64_t T, const int32_t* cu, const int32_t* lens,
                             const int32_t* positions, const float* inv_freq, int32_t rot, int32_t interleaved, const tb_token_rows* q,
                             const tb_token_rows* k, const tb_token_rows* v, const tb_token_rows* q_out, const tb_token_rows* k_out,
                             void* stream);

/* Attention of the new tokens over their sequences, those tokens' own rows among them (tb_append_paged_kv has put them there):
 *   out[t,h,:] = sum_n softmax_n(sm_scale * q[t,h] . K[b,h/g,n]) * V[b,h/g,n],   max(0, p - window + 1) <= n <= p (window = 0: 0 <= n <= p)
 * where p is the token's row; T, cu and lens as above.  One token of every sequence is a dense decode step, many are a prompt or a chunk of
 * one; a call may hold both.  max_new: host-side bound on a sequence's new tokens (tokens past it are left out, as are those past cu[B]:
 * their outputs are not written).
 * out has the element type of q (one rounding).  Weights are rounded to that type, too, before they meet V, except in calls of few tokens
 * (max_new, or T / B without cu, times Hq / Hkv up to 8), which lose at most 2^-16 of each.  lse: fp32 [T][Hq] or NULL.
 * A token that attends to nothing, or with scores of minus infinity alone, has out = 0 and lse = -inf.  Rows that a token does not attend to
 * add nothing to its result, whatever they hold.
 * ws: tb_workspace_bytes(TB_OP_PAGED_ATTN, desc, T); calls that share it have the same Hkv, too. */
tb_status tb_paged_attn(const tb_cache_desc* desc, const tb_paged_cache* cache, int64_t T, const int32_t* cu, const int32_t* lens,
                        int64_t max_new, const tb_token_rows* q, int64_t window, float sm_scale, const tb_token_rows* out, float* lse,
                        void* ws, size_t ws_bytes, void* stream);

/* tb_sparse_decode_attn over a cache in pages: lists and dense range name rows of the sequences, results as there (of a list's entries
 * in holes: as if they were not listed).  K and V may be up to 64 GiB each (else TB_ERR_UNSUPPORTED).  ws: tb_workspace_bytes(TB_OP_ATTN, ...). */
tb_status tb_sparse_decode_attn_paged(const tb_cache_desc* desc, const tb_paged_cache* cache, const void* q, const int32_t* idx,
                                      const int32_t* count, int64_t idx_cap, int64_t max_count, int64_t tail_begin, int64_t tail_end,
                                      float sm_scale, float* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/* Scratch size in bytes for `op` on this cache shape.  max_count is the longest list the
 * attention will see, tail included; for TB_OP_SELECT and TB_OP_DECODE_STEP it is the list
 * length the selection policy produces, lo + kk + N - hi (TB_OP_SELECT returns 0 for every
 * shape whose rows are selected by one workgroup each); for TB_OP_PAGED_ATTN it is the most tokens of a call.  Returns 0 on invalid
 * input.  A workspace of the TB_OP_DECODE_STEP size serves TB_OP_SELECT and TB_OP_ATTN on that
 * shape, too, and a workspace of any of the sizes serves fewer rows and shorter lists as well: make it
 * for a cache's capacity.  The workspace pointer must be 16-byte aligned. */
size_t tb_workspace_bytes(int32_t op, const tb_cache_desc* desc, int64_t max_count);

/* A workspace must be zero-filled once before its first use (this call enqueues that fill;
 * any other device memset does as well).  Every entry point leaves the workspace ready for the
 * next call, provided the calls that share it run one after the other on one stream and use
 * the same B and Hq.  Calls that overlap in time need separate workspaces. */
tb_status tb_workspace_init(void* ws, size_t ws_bytes, void* stream);

/* Measurement aid, not a step of the method: reads `bytes` (rounded down to 16) of device
 * memory at `src` (16-byte aligned) once with plain 128-bit streaming loads and writes nothing
 * (sink: one device word that is written only if the data fold to one particular value).  The
 * rate it reaches is the practical read ceiling of the box for the bandwidth-bound kernels of
 * the path, to be quoted next to the data-sheet HBM bandwidth. */
tb_status tb_read_stream_probe(const void* src, size_t bytes, uint32_t* sink, void* stream);

const char* tb_status_string(tb_status s);

/* Library version: major*10000 + minor*100 + patch. */
int32_t tb_version(void);

#ifdef __cplusplus
}
#endif
#endif /* TOKENBUTLER_H_ */
