/*
 * qm_attn.h - fused scaled-dot-product attention forward for AMD MI355X (gfx950),
 * and the operators around it that serve a model (from "Serving" on, at the end).
 *
 * The operation is the paper's statement of the attention problem (Background,
 * subsection "Attention Operators and acceleration"): for queries Q, keys K and
 * values V holding N tokens of head dimension d,
 *
 *     O = softmax(Mask(scale * Q K^T)) V,     lse_i = ln sum_{j visible} exp(scale * q_i . k_j)
 *
 * evaluated independently for every (batch, head), the way the paper's kernels
 * give each thread block a fixed batch and head of Q (Method, "Parameter
 * Analysis and Reasoning").  The N x N score matrix is never stored: scores are
 * formed block by block on chip with an online softmax that keeps a running row
 * maximum and row sum (the paper's Appendix B listings: "Softmax S with Smax and
 * Ssum" between the two fused GEMMs).
 *
 * Conventions shared by every entry point:
 *   - All tensor pointers are DEVICE pointers owned by the caller.  The library
 *     never allocates, frees, retains or synchronises them.
 *   - q and o are contiguous row-major [B][H][N][d] arrays, k and v
 *     [B][Hkv][N][d] (Hkv = H except in qm_attn_fwd_gqa and the _layout
 *     calls; in qm_attn_fwd_mla v and o have their own head dimension; the
 *     _layout calls also take [B][N][heads][d]), of the 16-bit type named by
 *     `dtype` (FP8 calls: one-byte E4M3 codes, bf16 o); otherwise o has the
 *     input type.  lse is a contiguous [B][H][N] float32 array.  Base
 *     pointers must be 16-byte aligned.
 *   - The call validates its arguments on the host, then enqueues one kernel
 *     (qm_attn_decode: one or two) on
 *     `stream` (NULL = the null stream) and returns; results are valid once the
 *     caller has synchronised that stream.  On any error nothing is enqueued and
 *     no output is written.
 *   - Calls are thread-safe; calls on different streams may run concurrently,
 *     and calls may be captured into a HIP graph (nothing but the kernel
 *     launches is enqueued).
 *   - Input elements are expected to be finite.  An infinite or NaN element
 *     gives unspecified values in the outputs that read it: its own query row
 *     (an element of q), or every row of the query heads that use its
 *     key/value head (an element of k or v).  All other outputs are unaffected,
 *     and the addresses the kernel touches, its barriers and its loop trip
 *     counts never depend on element values.
 *   - Range: the kernel forms each dot product q_i . k_j in fp32 and works in
 *     base 2, multiplying it by |scale| * log2(e) in fp32; lse is fp32 too.
 *     Every q_i . k_j (of the stored codes, for the FP8 calls) and every
 *     |scale * q_i . k_j| * log2(e) (FP8: with scale * q_scale * k_scale)
 *     must therefore be finite in fp32, i.e. below 3.4e38.  A row with a
 *     larger one gets unspecified O and lse (in practice NaN or infinity);
 *     the other rows are unaffected.  The front end rejects a combined scale
 *     whose fp32 value overflows (QM_ERR_SCALE); it cannot see the inputs.
 */
#ifndef QM_ATTN_H
#define QM_ATTN_H

#include <hip/hip_runtime_api.h>
#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

/* 16-bit storage types of q, k, v and o. */
typedef enum {
  QM_F16 = 0,  /* IEEE binary16 */
  QM_BF16 = 1, /* bfloat16 (top half of an IEEE binary32) */
  QM_E4M3 = 2  /* cached keys and values only: OCP E4M3 codes with one scale per tensor */
} qm_dtype_t;

/* Memory layouts of q, k, v and o (the _layout entry points; lse is always [B][H][N]). */
typedef enum {
  QM_BHND = 0,  /* [B][heads][N][width]: each head a contiguous N x width slab */
  QM_BNHD = 1   /* [B][N][heads][width]: each token's heads side by side */
} qm_layout_t;

/* Status codes returned by every qm_attn_fwd* entry point. */
enum {
  QM_OK = 0,
  QM_ERR_NULL = -1,        /* q, k, v, o or lse is NULL */
  QM_ERR_SHAPE = -2,       /* B, H or N < 1, Hkv not a divisor of H, B*H*N*d
                              does not fit in 62 bits, or (N + 256) * d (QM_BNHD:
                              times the heads, in bytes of q, k and v) does not fit
                              in 31 (32) bits */
  QM_ERR_HEADDIM = -3,     /* d is not 64 or 128 (qm_attn_fwd_mla: (d_qk, d_v) is not
                              (64, 64), (128, 128) or (192, 128)) */
  QM_ERR_DTYPE = -4,       /* dtype is not QM_F16 or QM_BF16 */
  QM_ERR_SCALE = -5,       /* scale (or an FP8 tensor scale) is infinite or NaN, or the
                              combined scale times log2(e) overflows fp32 */
  QM_ERR_ALIAS = -6,       /* o or lse overlaps q, k, v or each other */
  QM_ERR_CAUSAL = -7,      /* causal is neither 0 nor 1 */
  QM_ERR_LAUNCH = -8,      /* the HIP runtime rejected the kernel launch */
  QM_ERR_UNSUPPORTED = -9, /* a pointer is not 16-byte aligned */
  QM_ERR_LAYOUT = -10,     /* layout is not QM_BHND or QM_BNHD, or QM_BNHD with
                              d_qk = 192 */
  QM_ERR_TILE = -11,       /* qm_attn_set_tile_rows: rows is not 0, 128 or 256 */
  QM_ERR_WINDOW = -12,     /* window is below 1 (qm_attn_decode: below 0), or sinks below 0 */
  QM_ERR_PAGE = -13,       /* page_size is not a multiple of 16 from 16 to 65536, num_pages,
                              table_cols or max_length is below 1, table_cols * page_size is above
                              2^29 tokens, or the cache is 2^62 bytes or more */
  QM_ERR_ROTARY = -14,     /* rotary is not a multiple of 16 from 0 to d, its table is missing or
                              (starts NULL) shorter than N, eps is negative, infinite or NaN, or
                              interleaved is neither 0 nor 1 */
  QM_ERR_STRIDE = -15,     /* a stride is negative or not a multiple of 8 elements */
  QM_ERR_WORKSPACE = -16   /* workspace is NULL or smaller than the call needs */
};

/*
 * qm_attn_fwd - attention forward for B batches x H heads of N tokens.
 *
 *   q, k, v  [in]  device, [B][H][N][d] of `dtype`.  May alias one another.
 *   o        [out] device, [B][H][N][d] of `dtype`: the attention output,
 *                  rounded to the storage type (round-to-nearest-even).
 *   lse      [out] device, [B][H][N] float32: natural-log log-sum-exp of the
 *                  visible scaled scores of each query row.
 *   B, H, N        batch, heads, tokens (any N >= 1; tails are masked on chip).
 *   d              head dimension: 64 or 128 (the paper's head dimensions,
 *                  Evaluation section, "Benchmark setting").
 *   scale          any finite float multiplying q_i . k_j (usually 1/sqrt(d)).
 *                  It is applied to the fp32 dot product, never to 16-bit Q.
 *   causal         0: every key is visible; 1: key j is visible to query i
 *                  iff j <= i (the paper's causal mask; fully masked key blocks
 *                  are skipped, not computed).
 *   stream         HIP stream to enqueue on (NULL = null stream).
 *   dtype          a qm_dtype_t.
 *
 * Arithmetic: 16-bit products with fp32 accumulation on the matrix cores; the
 * softmax in fp32; probabilities rounded to `dtype` before the second product.
 * Results are deterministic: the same inputs give byte-identical outputs on the
 * same device.  A head's bytes may depend on how many heads the call has and on
 * the device's CU count, within the rounding of fp32 sums: calls whose query
 * blocks all fit the device at once may sum their keys in two or four groups
 * (see qm_attn_set_tile_rows).
 *
 * Returns QM_OK or one of the QM_ERR_* codes above; every check except
 * QM_ERR_LAUNCH happens before anything is enqueued.
 */
int qm_attn_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
                int B, int H, int N, int d, float scale, int causal,
                hipStream_t stream, int dtype);

/*
 * qm_attn_fwd_gqa - attention forward where H query heads share Hkv key/value
 * heads: multi-query (Hkv = 1) and grouped-query attention, the variants the
 * paper names beside multi-head attention in its Background and evaluates in
 * its Evaluation section ("Attention variants"; the appendix table of LLM
 * configurations: 64 query / 8 key-value heads, 128 / 8).  Query head h of a
 * batch attends with key/value head h / (H / Hkv) of that batch: consecutive
 * query heads form a group.  Every query head is otherwise exactly the
 * qm_attn_fwd operation.
 *
 *   q, o     [B][H][N][d] of `dtype` (o [out]).
 *   k, v     [in] device, [B][Hkv][N][d] of `dtype`.
 *   lse      [out] device, [B][H][N] float32.
 *   Hkv      key/value heads: 1 <= Hkv <= H and H % Hkv == 0, else
 *            QM_ERR_SHAPE.  Hkv = H is exactly qm_attn_fwd.
 *   all other arguments, the arithmetic, determinism and the status codes are
 *   those of qm_attn_fwd.
 */
int qm_attn_fwd_gqa(const void* q, const void* k, const void* v, void* o, float* lse,
                    int B, int H, int Hkv, int N, int d, float scale, int causal,
                    hipStream_t stream, int dtype);

/*
 * qm_attn_fwd_mla - attention forward with a wider query/key head than value
 * head: the multi-head latent attention shape the paper evaluates (its MLA
 * table: DeepSeek-V3's configuration, head dimension 128 plus a 64-wide RoPE
 * part, so d_qk = 192 and d_v = 128, with the causal mask), taken in its
 * explicit form where every head has its own keys and values.
 *
 *   q, k     [in]  device, [B][H][N][d_qk] of `dtype`.
 *   v        [in]  device, [B][H][N][d_v] of `dtype`.
 *   o        [out] device, [B][H][N][d_v] of `dtype`.
 *   lse      [out] device, [B][H][N] float32.
 *   d_qk, d_v      (192, 128); (64, 64) and (128, 128) are qm_attn_fwd.
 *                  Any other pair: QM_ERR_HEADDIM.
 *   scale          multiplies q_i . k_j over all d_qk columns (usually
 *                  1/sqrt(d_qk)).
 *   all other arguments, the arithmetic, determinism and the status codes are
 *   those of qm_attn_fwd.
 */
int qm_attn_fwd_mla(const void* q, const void* k, const void* v, void* o, float* lse,
                    int B, int H, int N, int d_qk, int d_v, float scale, int causal,
                    hipStream_t stream, int dtype);

/*
 * qm_attn_fwd_fp8 - attention forward on FP8 inputs, the variant the paper's
 * case study generates (its FP8 table: MHA with the causal mask at head
 * dimension 128).  q, k and v hold OCP E4M3 codes (1 sign, 4 exponent bits
 * with bias 7, 3 mantissa bits; the largest value 448), each with one scale
 * factor for the whole tensor: the operation is qm_attn_fwd's on the real
 * tensors q_scale*Q, k_scale*K and v_scale*V.  The products run on the FP8
 * matrix cores with fp32 accumulation; the probabilities are rounded to E4M3
 * (to nearest even) before the second product; per output row i that bounds
 * the error by 2^-4 sum_j P_ij |v_j| + 2^-10 exp(m_i - lse_i) sum_j |v_j| (P the
 * exact probabilities, m_i the row's largest score, v the real values), and the
 * row sums and lse stay in fp32.  The matrix cores sum each group of 8
 * products after truncating them to multiples of 2^-13 of the group's
 * largest, which adds at most 7 * 2^-13 of sum_j P_ij |v_j| to O and of
 * |scale| sum_c |q_ic k_jc| to each score.
 *
 *   q, k, v  [in]  device, [B][H][N][d] uint8 E4M3 codes.
 *   o        [out] device, [B][H][N][d] bfloat16 (round to nearest even).
 *   lse      [out] device, [B][H][N] float32, of the scaled scores.
 *   d              128; any other value: QM_ERR_HEADDIM.
 *   q_scale, k_scale, v_scale   finite per-tensor factors (QM_ERR_SCALE otherwise).
 *   scale          finite, multiplies the dot product of the real tensors.
 *   B, H, N, causal, stream: as for qm_attn_fwd; there is no dtype argument.
 */
int qm_attn_fwd_fp8(const void* q, const void* k, const void* v, void* o, float* lse,
                    int B, int H, int N, int d, float q_scale, float k_scale, float v_scale,
                    float scale, int causal, hipStream_t stream);

/*
 * qm_attn_fwd_layout - the 16-bit entry points in one call, with the memory
 * layout as an argument.  Computes exactly what qm_attn_fwd_gqa (Hkv < H) and
 * qm_attn_fwd_mla (d_qk = 192, d_v = 128) compute, on tensors stored as
 * `layout`:
 *
 *   QM_BHND  q [B][H][N][d_qk], k [B][Hkv][N][d_qk], v [B][Hkv][N][d_v],
 *            o [B][H][N][d_v] (the other entry points' layout);
 *   QM_BNHD  q [B][N][H][d_qk], k [B][N][Hkv][d_qk], v [B][N][Hkv][d_v],
 *            o [B][N][H][d_v]: the layout a projection writes before any
 *            transpose.
 *
 *   lse      [out] device, [B][H][N] float32 in either layout.
 *   (d_qk, d_v)    (64, 64), (128, 128) or (192, 128); QM_ERR_HEADDIM otherwise.
 *   layout         a qm_layout_t; QM_BNHD takes (d_qk, d_v) = (64, 64) or
 *                  (128, 128).  QM_ERR_LAYOUT otherwise.
 *   all other arguments, the arithmetic, determinism and the status codes are
 *   those of qm_attn_fwd.  Both layouts give byte-identical results.
 */
int qm_attn_fwd_layout(const void* q, const void* k, const void* v, void* o, float* lse,
                       int B, int H, int Hkv, int N, int d_qk, int d_v, float scale,
                       int causal, hipStream_t stream, int dtype, int layout);

/*
 * qm_attn_fwd_fp8_layout - qm_attn_fwd_fp8 with grouped-query key/value heads
 * and the memory layout as arguments: k and v hold Hkv heads (H % Hkv == 0;
 * query head h reads key/value head h / (H / Hkv), as in qm_attn_fwd_gqa),
 * and q, k, v and o are stored as `layout` (QM_BHND or QM_BNHD, as in
 * qm_attn_fwd_layout).  The arithmetic, its error bound and the status codes
 * are those of qm_attn_fwd_fp8, plus QM_ERR_SHAPE for an Hkv that is below 1,
 * above H or not a divisor of H, and QM_ERR_LAYOUT for any other layout.
 * Hkv = H with QM_BHND is exactly qm_attn_fwd_fp8; both layouts give
 * byte-identical results.
 */
int qm_attn_fwd_fp8_layout(const void* q, const void* k, const void* v, void* o, float* lse,
                           int B, int H, int Hkv, int N, int d, float q_scale, float k_scale,
                           float v_scale, float scale, int causal, hipStream_t stream,
                           int layout);

/*
 * qm_attn_fwd_window - causal attention forward in which a query sees a sliding
 * window of the latest keys and a few first keys that stay visible (attention
 * sinks): key j is visible to query i iff
 *
 *     j <= i  and  (i - j < window  or  j < sinks).
 *
 * Every row sees at least its own key.  Key blocks that no row of a query block
 * sees are neither loaded nor computed, so a call costs about
 * N * (window + sinks) pairs.  lse is over the visible keys.
 *
 *   window         keys a query sees counting its own, at least 1; any value of
 *                  N - sinks or more hides nothing and gives exactly the causal
 *                  qm_attn_fwd_layout (byte-identical).
 *   sinks          first keys of each sequence that all later queries see, 0 or
 *                  more (QM_ERR_WINDOW otherwise).
 *   all other arguments, the arithmetic, determinism and the status codes are
 *   those of qm_attn_fwd_layout with causal = 1.  Both layouts give
 *   byte-identical results.
 */
int qm_attn_fwd_window(const void* q, const void* k, const void* v, void* o, float* lse,
                       int B, int H, int Hkv, int N, int d_qk, int d_v, float scale,
                       int window, int sinks, hipStream_t stream, int dtype, int layout);

/*
 * qm_attn_set_tile_rows - a tuning control: the query rows one workgroup
 * owns, for every later call in the process.
 *
 *   rows = 0 (the default): chosen per call from the shape.  256-row
 *            workgroups (eight wavefronts, one per CU) keep each K/V block in
 *            LDS for the most rows; 128-row workgroups (four wavefronts, two
 *            per CU) overlap one workgroup's start and end with the other's
 *            work, and run for short sequences (N <= 1024, causal 2048, d = 64
 *            and FP8 4096) or when the 256-row workgroups, dealt out in rounds
 *            over the device's CUs, would leave too many of them idle.
 *   rows = 128 or 256: that size.
 *
 * Calls whose query blocks all fit the device at once (a few heads, equal head
 * dimensions) split the keys between the wavefronts of 64- or 128-row
 * workgroups, whatever this setting is: into four groups from N = 384 on
 * (d = 64 and FP8), into two from N = 768 (d = 64) or 1536 (d = 128 and FP8).
 * qm_attn_fwd_window has rules of its own for the same choices, with 128-row
 * workgroups always at d = 64.
 *
 * Results do not depend on the setting: every query row takes the same
 * arithmetic in the same order under each, so outputs are byte-identical;
 * only speed changes.  Returns QM_OK, or QM_ERR_TILE for any other value (the setting is
 * then unchanged).  Thread-safe; a call racing with attention calls on other
 * threads may or may not apply to them.
 */
int qm_attn_set_tile_rows(int rows);

/*
 * ---------------------------------------------------------------------------
 * Serving: what makes the queries and keys that the calls above take, a paged
 * cache of keys and values, and attention of new tokens over it.
 *
 * The cache is two arrays of pages, k_cache and v_cache, of `cache_layout`
 *
 *   QM_BHND  [num_pages][Hkv][page_size][d]
 *   QM_BNHD  [num_pages][page_size][Hkv][d]
 *
 * and of `cache_dtype`: the call's own dtype, or QM_E4M3 codes.  Either way the
 * real tensor is k_scale (v_scale) times what is stored.  page_table
 * [B][table_cols] int32 holds each sequence's pages in order: token t of
 * sequence b is row t % page_size of page page_table[b][t / page_size].
 * page_size is a multiple of 16.  The table, lengths, starts and counts are device
 * arrays that the host does not read; entries of the table past a sequence's
 * tokens are never used.  A page number outside 0 .. num_pages - 1 among those in
 * use is not followed: see each call for what it gives instead.
 *
 * The arrays of numbers (page_table, lengths, starts, counts) must be 4-byte
 * aligned, all others 16-byte aligned.
 */

/*
 * qm_qk_norm_rope - the norm of each query and key head and the rotation by its
 * token's position, in one pass.  Per row x of d columns:
 *
 *   y_c = x_c w_c / sqrt(mean(x^2) + eps)     where the weight is given, else y = x;
 *   pairs (a, b) of the first `rotary` columns, pair j at angle index j:
 *     a' = a cos[p][j] - b sin[p][j],  b' = b cos[p][j] + a sin[p][j]
 *   with p the token's position starts[b] + t, and pair j = columns
 *   (j, j + rotary / 2), or with interleaved = 1 columns (2 j, 2 j + 1);
 *
 * in fp32, rounded once (to nearest even) into the output.
 *
 *   q, k         [in]  device, of `dtype`.  q_strides and k_strides (host arrays,
 *                      read during the call) give the elements from one batch,
 *                      token and head to the next, in this order: multiples of 8,
 *                      0 or more, so q and k may be parts of one projection's
 *                      output, in any order of dimensions; the d columns are
 *                      contiguous.  NULL: contiguous, in `layout`.
 *   q_out, k_out [out] device, contiguous, of `dtype` in `layout` (as
 *                      qm_attn_fwd_layout takes them).  They overlap no input.
 *   q_weight, k_weight   [in] device, [d] of `dtype`, or NULL.
 *   cos, sin     [in]  device, [table_rows][rotary / 2] float32; not read when
 *                      rotary is 0.
 *   starts       [in]  device, [B] int32: the position of each sequence's first
 *                      token, or NULL for 0.
 *   counts       [in]  device, [B] int32: tokens that each sequence holds, or NULL
 *                      for N.  Rows of a padded batch from there on are written as
 *                      zeros, whatever their input holds.
 *   d            64 or 128.       rotary   0, or a multiple of 16 up to d.
 *   A token whose position is outside the table gets NaN rows.
 *   Hkv need not divide H.  B * N * (H + 2 Hkv) is below 2^27 (QM_ERR_SHAPE).
 *   stream, errors, capture: as for the calls above (one kernel, nothing else).
 */
int qm_qk_norm_rope(const void* q, const void* k, void* q_out, void* k_out,
                    const void* q_weight, const void* k_weight, const float* cos,
                    const float* sin, const int* starts, const int* counts, int B, int H,
                    int Hkv, int N, int d, int rotary, int table_rows, float eps,
                    int interleaved, const long long* q_strides, const long long* k_strides,
                    hipStream_t stream, int dtype, int layout);

/*
 * qm_qk_norm_rope_append - qm_qk_norm_rope, with the keys and the values v
 * written to the cache: token t of sequence b to position starts[b] + t.
 *
 *   v            [in]  device, of `dtype`, Hkv heads, v_strides as for k.
 *   k_out        [out] may be NULL: the keys then go to the cache only.
 *   k_cache, v_cache   [in, out] device.  Stored is key / k_scale and value /
 *                      v_scale (the quotient as a product with the fp32
 *                      reciprocal), from the fp32 result, to nearest even; E4M3
 *                      values beyond 448 become 448, NaN stays NaN.
 *   starts       [in]  tokens that each sequence's cache holds so far (NULL: 0).
 *   k_scale, v_scale   finite, with a finite reciprocal (QM_ERR_SCALE otherwise).
 *   cos, sin, the weights and rotary = 0 are as above: without them keys are
 *   stored as they are.
 *   Rows past a sequence's count store nothing.  A token whose position is outside
 *   the rotation's table or the page table, or whose page number is out of range,
 *   is not stored.  Pages that hold a written position must belong to one sequence and
 *   stand once in its row of the table (else either token's bytes may stay there).
 */
int qm_qk_norm_rope_append(const void* q, const void* k, const void* v, void* q_out, void* k_out,
                           void* k_cache, void* v_cache, const int* page_table,
                           const void* q_weight, const void* k_weight, const float* cos,
                           const float* sin, const int* starts, const int* counts, int B, int H,
                           int Hkv, int N, int d, int rotary, int table_rows, float eps,
                           int interleaved, int num_pages, int page_size, int table_cols,
                           float k_scale, float v_scale, const long long* q_strides,
                           const long long* k_strides, const long long* v_strides,
                           hipStream_t stream, int dtype, int layout, int cache_dtype,
                           int cache_layout);

/*
 * qm_attn_decode - attention of one new token per sequence over the cache.  Query
 * head h of sequence b sees the cached tokens j < lengths[b] of key/value head
 * h / (H / Hkv), and with window > 0 of those only
 *
 *     j >= lengths[b] - window  or  j < sinks
 *
 * (the last row of qm_attn_fwd_window on the same tokens; the new token's own key
 * is already in the cache).
 *
 *   q            [in]  device, [B][H][d] of `dtype`.
 *   o            [out] device, [B][H][d] of `dtype`.
 *   lse          [out] device, [B][H] float32, over the visible scaled scores.
 *   lengths      [in]  device, [B] int32: cached tokens of each sequence, which
 *                      must not change while the call runs.  0: o is
 *                      0 and lse -infinity.  Below 0, above max_length or beyond the
 *                      page table, or with a page number out of range among the
 *                      visible tokens' pages: that sequence's o and lse are NaN.
 *   d            64 or 128.  H % Hkv == 0.  B * H is below 2^22 (QM_ERR_SHAPE).
 *   max_length   a bound on lengths that the host knows; the call's split of the
 *                cache is chosen for it (and for the number of sequences), so a close
 *                one is faster.
 *   window       0: every cached token is visible.  sinks: 0 or more.
 *   k_scale, v_scale   as given to qm_qk_norm_rope_append (finite).
 *   workspace    [out] device, 16-byte aligned, at least as many bytes as
 *                qm_attn_decode_workspace says (NULL where that is 0).  Its content
 *                before the call does not matter, and after it is unspecified; calls
 *                that may run at once must not share one.
 *
 * Arithmetic in fp32 (E4M3 codes are widened exactly; the probabilities enter the
 * second product as two values of `dtype`, which lose 2^-16 (bf16) or 2^-22 (fp16) of
 * them).  What the cache holds in places that are not visible does not matter, NaN
 * included.  Results are deterministic; a sequence's bytes may depend on B, the other
 * sequences' lengths, max_length and the device's CU count, within the rounding of fp32
 * sums (where its cache is cut between workgroups).  One kernel is enqueued, or two.
 */
int qm_attn_decode(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse,
                   const int* page_table, const int* lengths, int B, int H, int Hkv, int d,
                   int num_pages, int page_size, int table_cols, int max_length, float scale,
                   float k_scale, float v_scale, int window, int sinks, void* workspace,
                   size_t workspace_bytes, hipStream_t stream, int dtype, int cache_dtype,
                   int cache_layout);

/*
 * qm_attn_decode_workspace - the workspace of a qm_attn_decode call with these
 * arguments on the current device, in bytes, into *bytes (0: none).  max_length is
 * cut to table_cols * page_size as there.  Returns a status.
 */
int qm_attn_decode_workspace(int B, int H, int Hkv, int d, int page_size, int table_cols,
                             int max_length, int window, int sinks, size_t* bytes);

/* qm_attn_strerror - a static, human-readable string for a status code. */
const char* qm_attn_strerror(int status);

#ifdef __cplusplus
}
#endif

#endif /* QM_ATTN_H */
