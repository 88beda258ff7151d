/*
 * hyq.h - C ABI of libhyq, the MI355X (gfx950) implementation of HyQuant's
 * hybrid-precision prefill attention (HyQuant, arxiv 2608.27875).
 *
 * The prefill operator is three calls, composed as Algorithm 2 (App. A.2):
 *
 *   hyq_select_vertical  Algorithm 1 (App. A.1): vertical-line key positions
 *                        of the non-window prefix, per KV head;
 *   hyq_quantize         Algorithm 2, Stages 1-2: partition of the keys and
 *                        per-block symmetric quantization of Q and of the
 *                        keys/values that are neither vertical lines nor in
 *                        the window;
 *   hyq_attn_prefill     Algorithm 2, Stage 3 / eq. (prefill_hybrid) of
 *                        Section 4.2: one causal online softmax over the
 *                        quantized keys and the full-precision vertical-line
 *                        and window keys;
 *   hyq_prefill          the three in order, as one call.
 *
 * Conventions for every call:
 *  - Tensor pointers are DEVICE pointers owned by the caller.  Nothing is
 *    allocated, nothing is kept between calls, and nothing is read back to
 *    the host: every call only validates its arguments on the host and then
 *    enqueues kernels on `stream` (a hipStream_t; NULL = the null stream).
 *  - Q is [B][Hq][L][D], K and V are [B][Hkv][L][D], all bf16, contiguous.
 *    Query head h uses KV head h / (Hq/Hkv) (consecutive grouping).
 *  - The window is the last `window` keys [L-W, L); the prefix is [0, P) with
 *    P = max(0, L-W).  The vertical budget is k = 0 if budget_ppm = 0 or
 *    P = 0, else min(P, max(1, ceil(P * budget_ppm / 1e6))) (Algorithm 1).
 *  - Arguments are validated before anything is enqueued; on error nothing
 *    is enqueued, the call returns a negative code and hyq_last_error()
 *    describes the problem (thread-local).
 *  - Inputs must be finite.
 */
#ifndef HYQ_H
#define HYQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define HYQ_API __attribute__((visibility("default")))
#else
#define HYQ_API
#endif

/* Return codes. */
#define HYQ_OK            0
#define HYQ_EINVAL       -1   /* bad shape, pointer or argument combination          */
#define HYQ_EUNSUPPORTED -2   /* valid for the method but not built here (D != 128,
                                 block != 64, Hq/Hkv > 8, bits not in {16, 8, 4})   */
#define HYQ_EHIP         -3   /* a HIP launch or runtime error                      */

#define HYQ_KQ_POS_PAD 0x7fffffff   /* kq_pos value of padding slots */

/* Code formats of the quantized path (Algorithm 2 takes B in {INT8, FP8};
   Section 4.2 names INT4/FP4 for the low-precision bulk path as well). */
#define HYQ_FMT_INT 0   /* symmetric integer codes: int8 (c = 127) or int4 (c = 7) */
#define HYQ_FMT_FP8 1   /* OCP FP8 E4M3 codes (c = 448) for Q, K and V; needs
                           bits_kv = 8.  Each code byte is the E4M3 bit pattern of
                           the value nearest to x / s (ties to even, saturating at
                           +-448, zero keeps the sign of x), s = max|x| / 448.     */
#define HYQ_FMT_FP4 2   /* OCP FP4 E2M1 codes (c = 6) for K and V, needs bits_kv =
                           4: the code of x is the E2M1 value nearest to x / s
                           (ties to the even code, saturating at +-6, zero keeps
                           the sign of x), s = max|x| / 6; codes are packed two
                           per byte like int4 (element 2i in the low nibble).  Q
                           keeps 8 bits as E4M3 codes exactly as with
                           HYQ_FMT_FP8.                                          */
#define HYQ_FMT_FP4Q6 3 /* K and V exactly as HYQ_FMT_FP4 (bits_kv = 4); Q as OCP
                           FP6 E2M3 codes (c = 7.5), one per byte (bit 5 sign,
                           bits 4..3 exponent, bits 2..0 mantissa): the E2M3
                           value nearest to x / s, ties to the even code,
                           saturating at +-7.5, zero keeps the sign of x,
                           s = max|x| / 7.5 per 64-row block.  Both operands of
                           the quantized Q.K product are then at most 6 bits
                           wide.  Prefill calls only (decode queries stay bf16;
                           the decode cache rejects this format).             */

/* Readings of the full-precision window (eq. win_def of Section 4.1). */
#define HYQ_WIN_FIXED 0   /* the last W keys [L-W, L), as Algorithms 1, 2 and 4 use it */
#define HYQ_WIN_BAND  1   /* per query row t: keys [t+1-W, t] (eq. win_def with t0 = t+1);
                             quantizable keys older than the band are seen quantized.
                             Affects hyq_attn_prefill only (selection, quantization and
                             the decode cache use the fixed window).                  */

/* Vertical-line scores (Section 4.1). */
#define HYQ_SEL_PROXY   0   /* Algorithm 1: qsum . K, qsum the summed tail queries  */
#define HYQ_SEL_COLMASS 1   /* eq. vl_score: the attention mass the tail queries put
                               on each key (causal softmax, alpha = 1/sqrt(D), summed
                               over the tail rows and the g heads); same budget, top-k
                               and tie rule                                          */

typedef struct hyq_shape {
  int32_t B, Hq, Hkv, L, D;  /* batch, query heads, KV heads, sequence, head dim      */
  int32_t window;            /* W >= 0: full-precision window = last W keys          */
  int32_t budget_ppm;        /* vertical ratio r in parts per million, 0..1000000    */
  int32_t bits_kv;           /* 16 (no quantization), 8 (int8 / E4M3) or 4 (packed
                                int4 / E2M1), see kv_format                          */
  int32_t block;             /* quantization block in tokens (64)                   */
  int32_t kv_format;         /* HYQ_FMT_INT, HYQ_FMT_FP8 (bits 8), HYQ_FMT_FP4 or
                                HYQ_FMT_FP4Q6 (bits 4); ignored when bits = 16      */
  int32_t window_mode;       /* HYQ_WIN_FIXED or HYQ_WIN_BAND                       */
  int32_t selector;          /* HYQ_SEL_PROXY or HYQ_SEL_COLMASS                    */
  int32_t staging;           /* decode only: staging capacity W_s in tokens, 0 for
                                HYQ_DECODE_WS, else a multiple of 64 <= window      */
} hyq_shape;

typedef struct hyq_sizes {
  int32_t P;               /* non-window prefix length                               */
  int32_t k;               /* vertical lines per KV head                             */
  int32_t nQ;              /* quantized keys per KV head: P - k                      */
  int32_t n_qblk;          /* Q blocks per query head: ceil(L / block)               */
  int32_t n_kvblk;         /* K/V blocks per KV head: ceil(nQ / block)               */
  int32_t kv_row_bytes;    /* bytes per K code row: D (8-bit), D/2 (4-bit), 0 (16)   */
  size_t idx_bytes;        /* int32 idx[B][Hkv][k]                                   */
  size_t kq_pos_bytes;     /* int32 kq_pos[B][Hkv][n_kvblk*block]                    */
  size_t q_codes_bytes;    /* q_codes[B][Hq][L][D], one byte per code (int8 or E4M3) */
  size_t q_scale_bytes;    /* float q_scale[B][Hq][n_qblk]                           */
  size_t k_codes_bytes;    /* k_codes[B][Hkv][n_kvblk*block][kv_row_bytes]           */
  size_t v_codes_bytes;    /* v_codes[B][Hkv][n_kvblk][D][block*bits/8]              */
  size_t kv_scale_bytes;   /* float k_scale (and v_scale) [B][Hkv][n_kvblk]          */
  size_t scores_bytes;     /* float scores[B][Hkv][P]                                */
  size_t select_ws_bytes;  /* workspace needed by hyq_select_vertical                */
} hyq_sizes;

/* Pure host arithmetic: the derived sizes of a shape (same formulas as the
 * budget rule of Algorithm 1).  Validates the shape like the calls below.   */
HYQ_API int hyq_sizes_for(const hyq_shape* shape, hyq_sizes* out);

/*
 * Algorithm 1 (Vertical Token Identification), GQA-native, per KV head:
 *   qsum[b][j] = sum over the g query heads of group j and the last
 *                t = min(W, L) rows of Q (float32; per head, rows ascending
 *                from +0, then heads in order);
 *   S[b][j][p] = qsum . K[b][j][p] for p < P (float32 products, then the
 *                upper half of the 128 products folded onto the lower half
 *                repeatedly: 64, 32, ..., 1);
 *   idx[b][j]  = the k positions with the largest S, ties to the lowest
 *                position (-0 == +0), written in ascending order.
 * Q, K:    bf16 device tensors as above.
 * idx:     int32 [B][Hkv][k] (output).  Untouched when k = 0.
 * scores:  optional float [B][Hkv][P] output of S (NULL: not written).
 * ws:      device workspace of at least sizes.select_ws_bytes bytes (may be
 *          NULL when that is 0); its contents are scratch.
 * With selector = HYQ_SEL_COLMASS, S[b][j][p] is instead the column mass of
 * eq. vl_score: the sum over the tail rows i in [L-t, L) and the g heads of
 * group j of softmax_{k <= i}(alpha <Q[i], K[k]>)[p], computed with bf16
 * MFMA products and float32 exponentials and sums (not bit-reproducible
 * against another summation order; the top-k is the same kernel).
 * Errors:  HYQ_EINVAL also when W = 0 and k > 0 (no tail queries).
 */
HYQ_API int hyq_select_vertical(const hyq_shape* shape, const void* Q, const void* K,
                        int32_t* idx, float* scores, void* ws, size_t ws_bytes,
                        void* stream);

/*
 * Algorithm 2, Stages 1-2.  No-op (returns HYQ_OK) when bits_kv = 16.
 *   kq_pos[b][j][n]  the n-th quantized key position ([0, P) minus idx,
 *                    ascending); slots n >= nQ hold HYQ_KQ_POS_PAD.
 *   Q blocks:        rows [i*64, i*64+64) of each query head (ragged last);
 *   K/V blocks:      compacted rows [c*64, c*64+64) (K and V at kq_pos),
 *                    ragged last block; padding rows get code 0.
 *   scale s = fl32(max|x| / c), code = clamp(rint(fl32(x / s)), -c, c),
 *   c = 127 for Q and 8-bit K/V, c = 7 for 4-bit K/V; s = 0 gives codes 0
 *   (HYQ_FMT_INT; the floating-point formats round as described at
 *   HYQ_FMT_FP8 and HYQ_FMT_FP4, Q then in E4M3 with c = 448).
 * Layouts (all outputs written in full, padding included):
 *   q_codes int8 [B][Hq][L][D];           q_scale float [B][Hq][n_qblk]
 *   k_codes [B][Hkv][n_kvblk*64][row]:    8-bit: one code byte per channel;
 *            4-bit: byte i = channel 2i (low nibble) | channel 2i+1 (high
 *            nibble), two's-complement int4 or E2M1 nibbles;
 *   v_codes [B][Hkv][n_kvblk][D][64*bits/8]: each block stored channel-major
 *            (transposed): row d lists the block's 64 keys; 4-bit: byte i =
 *            key 2i (low nibble) | key 2i+1 (high nibble);
 *   k_scale, v_scale float [B][Hkv][n_kvblk].
 * idx: the output of hyq_select_vertical (ignored when k = 0).
 */
HYQ_API int hyq_quantize(const hyq_shape* shape, const void* Q, const void* K, const void* V,
                 const int32_t* idx, int8_t* q_codes, float* q_scale,
                 void* k_codes, float* k_scale, void* v_codes, float* v_scale,
                 int32_t* kq_pos, void* stream);

/*
 * Algorithm 2, Stage 3 and eq. (prefill_hybrid), causal by original key
 * position:
 *   out[b][h][t] = sum_k w_k value_k / sum_k w_k over keys k <= t, with
 *   w_k = exp(z_k - max z), and
 *   - quantized key (position kq_pos[n], block c = n/64):
 *       z = alpha * q_scale[t/64] * k_scale[c] * <q_code[t], k_code[n]>,
 *       value = v_scale[c] * v_code[n];
 *   - vertical-line key (idx) or window key ([P, L)), and every key when
 *     bits_kv = 16:  z = alpha * <Q[t], K[k]>, value = V[k] (bf16 inputs).
 * With window_mode = HYQ_WIN_BAND the window of row t is [t+1-W, t]: a
 * quantizable key k is taken in full precision (as above) when t+1-W <= k
 * and quantized when k <= t - W; vertical lines and keys >= P as above.
 * alpha = softmax_scale (1/sqrt(D) for the paper's operator).
 * out: [B][Hq][L][D], float32 (out_dtype 0) or bf16 (out_dtype 1).
 * The quantization buffers (q_codes ... kq_pos) are the outputs of
 * hyq_quantize for the same shape; they are not read when bits_kv = 16.
 * Precision: quantized logits are exact int32 dot products scaled in
 * float32 (int codes) or the float32 results of the E4M3 / E2M1 x E4M3
 * MFMA; full-precision logits are bf16 x bf16 products accumulated in
 * float32; softmax weights enter the P.V products as f16, against exact
 * f16 codes (quantized keys) or against V / sVref in f16 (full-precision
 * keys: exact for bf16 V within 2^16 of the reference sVref, a power of two
 * the kernel raises when a tile's V exceeds that range); all accumulation is
 * float32.
 */
HYQ_API int hyq_attn_prefill(const hyq_shape* shape, const void* Q, const void* K, const void* V,
                     const int32_t* idx, const int8_t* q_codes, const float* q_scale,
                     const void* k_codes, const float* k_scale,
                     const void* v_codes, const float* v_scale,
                     const int32_t* kq_pos, float softmax_scale,
                     void* out, int32_t out_dtype, void* stream);

/* hyq_prefill - Algorithm 2 as one call: hyq_select_vertical (with no
 * scores output), hyq_quantize and hyq_attn_prefill on `stream`, with the
 * results of that order (the selection and the quantization share
 * launches).  Arguments, layouts, ownership and sizes are those of the three
 * calls (ws / ws_bytes: the selection workspace); the arguments of all
 * three are validated before the first launch, so an invalid argument
 * returns HYQ_EINVAL with nothing launched.  Allocates nothing and keeps no
 * state, so the call can be captured in a HIP graph.
 */
HYQ_API int hyq_prefill(const hyq_shape* shape, const void* Q, const void* K, const void* V,
                        int32_t* idx, int8_t* q_codes, float* q_scale, void* k_codes,
                        float* k_scale, void* v_codes, float* v_scale, int32_t* kq_pos,
                        float softmax_scale, void* out, int32_t out_dtype, void* ws,
                        size_t ws_bytes, void* stream);

/* ======================================================================
 * Decode: Algorithm 4 (Freeze, App. A.4) and Algorithm 3 (HyQuant Decode,
 * App. A.3).
 *
 * Freeze turns a prefill of N tokens into the hybrid KV cache of decode:
 *   - vertical-line tokens (Algorithm 1 on the prefill's tail queries, held
 *     fixed from then on): K and V kept in bf16;
 *   - the other non-window tokens [0, N-W) minus the vertical lines:
 *     per-block quantized exactly as hyq_quantize quantizes K_Q and V_Q;
 *   - the last W tokens (the window): kept in bf16;
 *   - an empty staging buffer of W_s tokens (shape.staging, default
 *     HYQ_DECODE_WS), kept in bf16.
 * Each decode step appends one token.  When it arrives with the staging
 * buffer full, the W_s oldest window tokens are first quantized into W_s/64
 * new blocks of the quantized prefix (same formula, c_B and format, 64
 * tokens per block, oldest first) and the staged tokens join the window,
 * which stays W tokens long.
 * Decode attention of one query row per (b, h) is one softmax over every
 * cached key (no mask): quantized keys enter as scale * code, all other
 * keys as their bf16 values; the query is used in full precision.
 *
 * Memory: the window and the staging buffer share one ring of
 * ring_rows = roundup(W, 64) + W_s bf16 rows per KV head (window = the W
 * oldest valid rows from ring_head on, staging = the rest), so a merge
 * moves no full-precision data.  Vertical-line rows and the ring are stored
 * together: fp_k row i < vl_rows is vertical line i (rows >= n_vl are zero
 * padding), row vl_rows + s is ring slot s.  fp_v holds the same rows
 * transposed (channel-major), the layout the P.V matrix product reads.
 * The caller owns every buffer; state lives in the struct, which
 * hyq_decode_append advances on the host.
 * ==================================================================== */

#define HYQ_DECODE_WS 64   /* default staging buffer capacity W_s (tokens)    */

typedef struct hyq_dcache {
  /* geometry, set by hyq_dcache_init */
  int32_t B, Hq, Hkv, D;
  int32_t window;        /* W, 64 <= W <= N                                      */
  int32_t bits_kv;       /* 8 or 4                                               */
  int32_t kv_format;     /* HYQ_FMT_INT, HYQ_FMT_FP8 (bits 8) or HYQ_FMT_FP4 (bits 4)*/
  int32_t n_vl;          /* k: vertical-line tokens per KV head                  */
  int32_t vl_rows;       /* k rounded up to a multiple of 64                     */
  int32_t ring_rows;     /* roundup(W, 64) + staging                             */
  int32_t n_frozen;      /* quantized tokens written by Freeze (nQ of the prefill)*/
  int32_t cap_blocks;    /* quantized blocks the buffers hold (Freeze + merges)  */
  /* state, set by hyq_freeze and advanced by hyq_decode_append */
  int32_t n_merged;      /* merged blocks, stored after the ceil(nQ/64) frozen ones */
  int32_t ring_head;     /* ring slot of the oldest window token                 */
  int32_t n_staged;      /* tokens in the staging buffer, 0..staging             */
  int32_t staging;       /* W_s: staging capacity, a multiple of 64, <= window   */
  int64_t t;             /* tokens cached: N + appended tokens                   */
  /* caller-owned device buffers (byte sizes from hyq_dcache_init) */
  void* k_codes;         /* [B][Hkv][cap_blocks*64][row] row-major, as hyq_quantize */
  void* v_codes;         /* [B][Hkv][cap_blocks][D][64*bits/8] channel-major blocks */
  float* k_scale;        /* [B][Hkv][cap_blocks]                                 */
  float* v_scale;        /* [B][Hkv][cap_blocks]                                 */
  int32_t* q_pos;        /* [B][Hkv][cap_blocks*64]: original position of each
                            quantized token; HYQ_KQ_POS_PAD in padding slots     */
  void* fp_k;            /* bf16 [B][Hkv][vl_rows + ring_rows][D]                */
  void* fp_v;            /* bf16 [B][Hkv][D][vl_rows + ring_rows]                */
  int32_t* vl_pos;       /* [B][Hkv][n_vl]: vertical-line positions, ascending   */
} hyq_dcache;

typedef struct hyq_dcache_sizes {
  size_t k_codes_bytes, v_codes_bytes, k_scale_bytes, v_scale_bytes, q_pos_bytes;
  size_t fp_k_bytes, fp_v_bytes, vl_pos_bytes;
  size_t freeze_ws_bytes;   /* workspace of hyq_freeze                              */
  size_t attn_ws_bytes;     /* workspace of hyq_decode_attn (any state of the cache)*/
} hyq_dcache_sizes;

/*
 * Pure host arithmetic: fills the geometry of a decode cache for a prefill
 * of shape `prefill` (L = N tokens; window, budget, bits and format as for
 * the prefill calls; bits_kv must be 8 or 4) that will hold up to
 * max_tokens tokens (>= N), zeroes its state and buffer pointers, and
 * returns the byte size of every buffer.
 * Errors: HYQ_EINVAL if W < W_s, N < W or max_tokens < N, or if
 * prefill->staging is neither 0 nor a multiple of 64.
 */
HYQ_API int hyq_dcache_init(const hyq_shape* prefill, int64_t max_tokens, hyq_dcache* cache,
                            hyq_dcache_sizes* sizes);

/*
 * Algorithm 4 (Freeze).  Q, K, V: the prefill's bf16 tensors (shape as for
 * the prefill calls); only the last min(W, N) query rows are read.  Fills
 * every buffer of `cache` (whose pointers the caller has set) and sets its
 * state: no merged blocks, ring_head 0, nothing staged, t = N.
 * ws: device workspace of at least freeze_ws_bytes (scratch).
 */
HYQ_API int hyq_freeze(const hyq_shape* prefill, const void* Q, const void* K, const void* V,
                       hyq_dcache* cache, void* ws, size_t ws_bytes, void* stream);

/*
 * One decode step's key and value rows, k_new and v_new bf16 [B][Hkv][D],
 * enter the staging buffer; when the staging buffer is full they are
 * preceded by the merge of the W_s oldest window tokens into quantized
 * blocks ceil(n_frozen/64) + n_merged, ... (W_s/64 of them).  Advances the state in
 * `cache` (host memory).
 * Errors: HYQ_EINVAL when a merge is due and all cap_blocks blocks are in
 * use (nothing is enqueued and the state is unchanged).
 */
HYQ_API int hyq_decode_append(hyq_dcache* cache, const void* k_new, const void* v_new,
                              void* stream);

/*
 * Algorithm 3: attention of one query row per (b, h) over every token of
 * the cache, split over the sequence axis and merged as in its
 * ReduceSoftmax step:
 *   out[b][h] = sum_k w_k value_k / sum_k w_k,  w_k = exp(z_k - max z),
 *   z_k = alpha * <q[b][h], key_k>, with key/value = scale * code for
 *   quantized tokens and the bf16 rows for vertical-line, window and staged
 *   tokens.  alpha = softmax_scale.
 * q: bf16 [B][Hq][D]; out: [B][Hq][D], float32 (out_dtype 0) or bf16 (1).
 * ws: device workspace of at least attn_ws_bytes (scratch).
 * Precision: the query enters the products with quantized keys as f16
 * after an exact power-of-two scaling per head (exact unless an entry is
 * below 2^-29 of the head's largest), codes as exact f16; full-precision
 * keys as bf16 x bf16; float32 accumulation; weights as f16 against
 * quantized values and as a high + low bf16 pair against bf16 values.
 */
HYQ_API int hyq_decode_attn(const hyq_dcache* cache, const void* q, float softmax_scale,
                            void* out, int32_t out_dtype, void* ws, size_t ws_bytes,
                            void* stream);

/*
 * hyq_decode_attn without a workspace, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, runtimes
 * that forbid hipMalloc): the same kernels and result, bit for bit, with
 * the split partials in a scratch array of HYQ_NOALLOC_SCRATCH_BYTES that
 * the library holds on each GPU (from its first use there until the process
 * ends).  Nothing is allocated by this call or by the library for it.
 * The scratch is shared by every call on a GPU: calls that overlap on one
 * GPU (different streams, or host threads without ordering) race and give
 * wrong results; calls ordered on one stream are fine.  The first call on
 * a device looks up the scratch's address (once per device, with that
 * device current), so make it outside graph capture.
 * Errors: as hyq_decode_attn; HYQ_EUNSUPPORTED when this launch's partials
 * (B * Hkv * splits * (Hq/Hkv) * 132 floats; about 9 MB for batch 16 at a
 * 32k-token cache) exceed the scratch.  Nothing is enqueued on error.
 */
#define HYQ_NOALLOC_SCRATCH_BYTES ((size_t)16 << 20)
HYQ_API int hyq_decode_attn_noalloc(const hyq_dcache* cache, const void* q, float softmax_scale,
                                    void* out, int32_t out_dtype, void* stream);

/* ======================================================================
 * Paged serving: the calls that stand before and beside the ones above in a
 * server of many sequences.
 *
 *   hyq_norm_rope     per-head RMS norms of queries and keys and the position
 *                     rotation in one pass, from token-major projections to
 *                     the [B][H][L][D] tensors of the prefill and decode calls;
 *   hyq_paged_append  the same pass for the new tokens of a ragged batch; keys
 *                     and values go into the pages of a cache;
 *   hyq_paged_attn    causal attention of each sequence's new tokens (one, a
 *                     few, or a chunk) over its pages; on request, the
 *                     attention weight that every cached key received;
 *   hyq_evict         eviction by that weight, per KV head, into new pages.
 *
 * A paged cache is a pool of n_pages pages of `page` slots for each of the
 * Hkv heads.  A sequence owns the pages that its row of a block table lists:
 * its slot n is slot n % page of page table[n / page].  One table serves all
 * heads.  Keys and values are rows of D channels, bf16, or 8-bit codes with
 * one float32 scale per row (s = max|x| / c, code = the value nearest to
 * fl32(x / s), c = 127 for int8 and 448 for E4M3, rounding as at
 * hyq_quantize; s = 0 gives codes 0).
 *
 * What a device array says is not checked on the host, but bounded in the
 * kernels: a table entry outside [0, n_pages) is a hole, whose keys nobody
 * sees and whose rows are not written; lengths are taken as at most the
 * bounds given with them.  No such value makes a kernel leave its buffers.
 * Slots behind a sequence may hold anything (NaN too); the rows of its own
 * slots must be finite.  Buffers must be aligned to 16 bytes, and what a call
 * writes must lie apart from all that it reads and from what else it writes
 * (refused with HYQ_EINVAL otherwise).
 * ==================================================================== */

typedef struct hyq_rope {
  int32_t rot_dim;        /* channels [0, rot_dim) are rotated: a multiple of 16, 0..D */
  int32_t interleaved;    /* pairs of frequency f: 0 channels (f, f + rot_dim/2),
                             1 channels (2f, 2f + 1)                              */
  float eps;              /* added to the mean square, >= 0                       */
  const void* q_weight;   /* bf16 [D], NULL: queries are not normalized           */
  const void* k_weight;   /* bf16 [D], NULL: keys are not normalized              */
  const float* inv_freq;  /* [rot_dim/2] radians per position (not read if rot_dim = 0) */
} hyq_rope;

/*
 * For every row x of q (weight w = q_weight) and k (k_weight):
 *   y = x * w / sqrt(mean(x^2) + eps)        (y = x where w is NULL; y = 0
 *                                             for a row of zeros, eps = 0 too)
 *   the pair (a, c) of frequency f becomes (a cos - c sin, c cos + a sin) of
 *   the angle pos * inv_freq[f]
 * in float32 (the angle in float64), rounded to bf16 once; v is copied.
 * Token t = b * L + i of shape (its B, Hq, Hkv, L, D count here; the other
 * fields only have to be valid).  q: bf16 rows [B*L][Hq][D] with q_stride
 * elements from token to token (a multiple of 8, >= Hq * D), k and v the same
 * with Hkv heads (three slices of one packed projection, or three tensors).
 * pos: int32 [B*L], any value.  Q [B][Hq][L][D], K and V [B][Hkv][L][D] bf16,
 * apart from the inputs and each other.  v and V may be NULL together; so may k and K.
 * At most 2^24 - 1 tokens and 2^30 head rows (B * L * (Hq + 2 Hkv)).
 * With L = 1 the outputs are the rows of hyq_decode_append / hyq_decode_attn.
 */
HYQ_API int hyq_norm_rope(const hyq_shape* shape, const hyq_rope* rope, const void* q,
                          int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                          int64_t v_stride, const int32_t* pos, void* Q, void* K, void* V,
                          void* stream);

typedef struct hyq_pcache {
  int32_t Hq, Hkv, D;    /* query heads that read it, KV heads, head dim (128)     */
  int32_t page;          /* slots per page: 16, 32, 64, 128 or 256                 */
  int32_t n_pages;       /* pages in the pool                                      */
  int32_t bits_kv;       /* 16 (bf16) or 8                                         */
  int32_t kv_format;     /* 8 bits: HYQ_FMT_INT or HYQ_FMT_FP8                     */
  /* caller-owned device buffers (byte sizes from hyq_pcache_init) */
  void* k;               /* [n_pages][Hkv][page][D] bf16 or code bytes             */
  void* v;               /* the same                                               */
  float* k_scale;        /* [n_pages][Hkv][page], 8 bits only                      */
  float* v_scale;
  float* mass;           /* [n_pages][Hkv][page] attention weight received; NULL if
                            nobody collects it                                     */
} hyq_pcache;

typedef struct hyq_pcache_sizes {
  size_t kv_bytes;       /* of k and of v                                          */
  size_t scale_bytes;    /* of k_scale and of v_scale (0 with 16 bits)             */
  size_t mass_bytes;     /* of mass                                                */
} hyq_pcache_sizes;

/* Most head rows of a step: T * (Hq + 2 Hkv). */
#define HYQ_PAGED_MAX_ROWS (1 << 24)

/* One step of B sequences with T token rows in all: tokens [cu_new[b],
   cu_new[b+1]) are the new ones of sequence b (none is fine), which go to its
   slots lens[b], lens[b] + 1, ...  Rows from cu_new[B] on belong to nobody:
   they are neither read nor written.  A page that the step writes (its new
   slots, or mass) must belong to one sequence only; pages that are only read
   may be shared.                                                            */
typedef struct hyq_pbatch {
  int32_t B, T;
  int32_t max_new;         /* no sequence has more new tokens                      */
  int32_t max_len;         /* no lens[b] is larger                                 */
  int32_t max_pages;       /* entries per table row                                */
  const int32_t* cu_new;   /* device [B + 1], ascending from 0                     */
  const int32_t* lens;     /* device [B]: slots in use before the step             */
  const int32_t* table;    /* device [B][max_pages]                                */
} hyq_pbatch;

/* Pure host arithmetic: checks the geometry, fills it in (buffers NULL) and
   returns the buffer sizes (sizes may be NULL).                              */
HYQ_API int hyq_pcache_init(int32_t Hq, int32_t Hkv, int32_t D, int32_t page, int32_t n_pages,
                            int32_t bits_kv, int32_t kv_format, hyq_pcache* cache,
                            hyq_pcache_sizes* sizes);

/*
 * hyq_norm_rope for the new tokens of a batch: q rows to q_out [T][Hq][D]
 * bf16, k and v rows into their slots (codes are taken of the float32 values,
 * not of bf16 ones); mass, where there is one, is 0 in those slots.
 * q, k, v: bf16 rows [T][heads][D] with strides as for hyq_norm_rope; pos
 * int32 [T].  q and q_out may be NULL together (keys and values only).
 * lens is not changed: hyq_paged_attn of the same step takes the same batch.
 */
HYQ_API int hyq_paged_append(const hyq_pcache* cache, const hyq_pbatch* batch,
                             const hyq_rope* rope, const void* q, int64_t q_stride, const void* k,
                             int64_t k_stride, const void* v, int64_t v_stride,
                             const int32_t* pos, void* q_out, void* stream);

#define HYQ_MASS_NONE 0   /* the weights are not collected                         */
#define HYQ_MASS_ADD  1   /* added to cache.mass                                   */
#define HYQ_MASS_SET  2   /* cache.mass = the weights of this call                 */

/* Workspace of hyq_paged_attn for this cache and these bounds (host only; the
   device arrays of the batch are not read and may be NULL).  0: none needed.
   One for T token rows serves fewer.  With masses it holds a float32 logit of
   every slot up to max_len + max_new in min(max_new * Hq/Hkv, 16) rows of every
   sequence and KV head (256 sequences of 32768 slots with 8 KV heads and a chunk
   among them: 4.3 GB).                                                       */
HYQ_API int hyq_paged_ws_bytes(const hyq_pcache* cache, const hyq_pbatch* batch, int32_t mass,
                               size_t* bytes);

/*
 * For new token i of sequence b, query head h and its KV head j:
 *   z_n = softmax_scale * <q, K[n]> over the slots n <= lens[b] + i,
 *   out = sum_n w_n V[n] / sum_n w_n, w_n = exp(z_n - max z);
 * a row that sees no key (all holes) gives 0.  Scores (and softmax_scale) may be
 * of any size that float32 holds, log2(e) times them too.  The new tokens' rows
 * must be in their slots (hyq_paged_append).
 * With mass, for every slot n < lens[b] + new of a sequence with new tokens:
 *   mass[b][j][n] (+)= sum over its new tokens i and the g heads of group j of
 *                      the weight w_n / sum w that they give n.
 * q: bf16 [T][Hq][D]; out: [T][Hq][D], float32 (out_dtype 0) or bf16 (1).
 * Precision: bf16 products (8-bit codes are exact in bf16, their scales are
 * applied in float32), float32 sums; the weights enter the products with V as
 * a high + low bf16 pair where a sequence has at most 16 query rows per KV
 * head (new tokens * Hq/Hkv; of a single sequence, max_new * Hq/Hkv), and as
 * bf16 where it has more (which adds an error of the size of a bf16 output's own
 * rounding: 0.0024 in all, relative, where that is 0.0017; up to 0.003 where few
 * keys in 8-bit pages hold the weight).  Values of up to 2^80 keep their weighted
 * sums within float32.  Every result is the same from run to run: nothing is
 * added atomically.
 * Allocates nothing and keeps no state; it can be captured in a HIP graph
 * (lens, tables and token counts may change between replays, within the
 * bounds).  ws: scratch of hyq_paged_ws_bytes; calls that overlap need one each.
 */
HYQ_API int hyq_paged_attn(const hyq_pcache* cache, const hyq_pbatch* batch, const void* q,
                           float softmax_scale, int32_t mass, void* out, int32_t out_dtype,
                           void* ws, size_t ws_bytes, void* stream);

/*
 * Eviction by accumulated attention weight.  Of the n = min(lens[b], max_len)
 * slots of sequence b, every KV head keeps min(n, budget): the last `recent`
 * ones, and of the others those with the largest cache.mass (ties: the lowest
 * slot; -0 equals +0, NaN counts as less than any number), in ascending order:
 *   keep[b][j][i] = the i-th kept slot (entries i >= min(n, budget) hold
 *                   HYQ_KQ_POS_PAD),
 * whose key, value, scales and mass go to slot i of the pages of row b of
 * new_table; new_lens[b] = min(n, budget).  Slots behind that are left as they
 * were, and so are the old pages: the caller may free them.  The new pages
 * must be no one else's, old pages of this call among them.  Old pages may be
 * shared (by sequences, or with readers).
 * B sequences; table int32 [B][max_pages], new_table int32 [B][new_pages] with
 * new_pages * page >= budget >= recent >= 0, budget >= 1; keep int32
 * [B][Hkv][budget], new_lens int32 [B] (another array than lens).
 */
HYQ_API int hyq_evict(const hyq_pcache* cache, int32_t B, const int32_t* lens,
                      const int32_t* table, int32_t max_pages, int32_t max_len, int32_t budget,
                      int32_t recent, const int32_t* new_table, int32_t new_pages, int32_t* keep,
                      int32_t* new_lens, void* stream);

/* Static description of a return code. */
HYQ_API const char* hyq_strerror(int code);

/* Message of the last failing call on this thread ("" if none). */
HYQ_API const char* hyq_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* HYQ_H */
