/*
 * loco_layer.h -- C ABI of the operators of a decoder layer's training step on B200 (sm_100a).
 *
 * loco.h compresses, exchanges and averages the gradients of Llama / Mixtral shaped models; the operators declared
 * here are the ones between the matrix products of such a layer that produce those gradients:
 *
 *   rotary      rotary positions on query and key heads (half and interleaved pairs, part of the head, tables scaled
 *               for long contexts) and the transposed rotation of their gradients;
 *   attention   softmax attention forward (o and the log-sum-exp of every row) and backward, which recomputes the
 *               probabilities; grouped heads, causal, padded or packed samples;
 *   router      the top-k router of a mixture of experts: chosen experts and weights, per-expert counts, balance and
 *               z loss, and their gradient.  An expert whose count is zero has an all-zero gradient segment;
 *   norm        root-mean-square norm with the residual's addition, its output in the type of the heads or in 8 bits
 *               with scales, and its gradient;
 *   experts     the router's choices sorted by expert, tokens laid out in that order and summed back with their weights,
 *               the product of every expert's rows with its matrix, and all their gradients;
 *   gradient    the sum of squares of a list of gradients, and the list scaled down to a largest norm.
 *
 * The conventions are those of loco.h: d_* are DEVICE pointers owned by the caller, `stream` is a cudaStream_t, work
 * is asynchronous, nothing allocates or synchronises unless stated, every call returns a loco_status_t and launches
 * nothing on an error.  Buffers of one call must not overlap except where stated.  The functions live in
 * libloco_layer_b200.so.
 */
#ifndef LOCO_B200_LAYER_H
#define LOCO_B200_LAYER_H

#include "loco.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Heads of a [batch, row, head, dim] tensor: element (b, t, h, i) lies at ptr + b*batch_stride + t*row_stride +
 * h*head_stride + i, strides in elements, so that heads may be cut out of one projection's output.  The stride of a
 * dimension of extent one is ignored; a zero stride repeats an input over its dimension and is refused (ARG) in an output. */
typedef struct {
    void   *ptr;
    int64_t batch_stride, row_stride, head_stride;
} loco_heads_t;

/* ---- rotary positions ----------------------------------------------------------------------
 * A token at position p rotates r/2 pairs of every head:  y_a = x_a c - x_b s,  y_b = x_b c + x_a s  with
 * (c, s) = row p of a table: r/2 cosines, then r/2 sines (fp32).  inverse != 0 applies the transposed rotation (the
 * gradient with respect to x, given the one with respect to y).  Dimensions from r on are copied.
 */
typedef enum { LOCO_ROTARY_HALF = 0,          /* pair j is (j, j + r/2)   */
               LOCO_ROTARY_INTERLEAVED = 1    /* pair j is (2j, 2j + 1)   */ } loco_rotary_layout_t;

typedef enum { LOCO_ROTARY_PLAIN = 0,         /* w_j = base^(-2j/r)                                             */
               LOCO_ROTARY_LINEAR = 1,        /* w_j / factor: positions divided                                */
               LOCO_ROTARY_PARTS = 2          /* a pair that turns at least `fast` times within `trained` tokens
                                                 keeps w_j, one that turns at most `slow` times takes w_j / factor,
                                                 linear in the number of turns between                          */
} loco_rotary_scaling_t;

typedef struct {
    int32_t rotary_dim;      /* r, even, 2 .. 1024                                      */
    int32_t positions;       /* rows of the table, >= 1                                 */
    int32_t scaling;         /* loco_rotary_scaling_t                                   */
    float   base, factor;    /* > 0; factor is ignored by PLAIN                         */
    float   trained, slow, fast;   /* PARTS only: trained > 0, 0 <= slow < fast         */
    float   magnitude;       /* multiplies every cosine and sine (1 = a pure rotation)  */
} loco_rotary_table_t;

/* Fill d_table (positions x r fp32, 16-byte aligned) with magnitude * cos(p w_j), magnitude * sin(p w_j), evaluated in
 * 64 bits and rounded once.  One launch.  Errors: ARG, ALIGN, CUDA. */
int loco_rotary_table(const loco_rotary_table_t *cfg, float *d_table, void *stream);

typedef struct {
    int32_t dtype;           /* loco_dtype_t of all heads                                                        */
    int32_t layout;          /* loco_rotary_layout_t                                                             */
    int32_t head_dim;        /* d, 1 .. 1024                                                                     */
    int32_t rotary_dim;      /* r <= d, even                                                                     */
    int32_t batch, seq;      /* tokens: batch * seq < 2^31                                                       */
    int32_t positions;       /* rows of the table                                                                */
    int32_t position_bytes;  /* 4 or 8: signed integers in d_positions; ignored without them                     */
    int32_t inverse;
} loco_rotary_t;

/*
 * Rotate the heads of `count` (1 or 2: queries and keys) tensors x[i] of heads[i] heads each into y[i].
 *   d_positions  one position per token [batch, seq], contiguous; NULL: token t of every sample is at position t
 *                (then seq <= positions).  A position outside the table gives NaN in the rotated dimensions of that token.
 *   x and y      any strides; y[i] may be x[i] itself with the same strides (in place), else they must not overlap.
 *                16-byte vector accesses are used where the base addresses, strides and dimensions allow them.
 * One launch.  Errors: ARG, ALIGN (d_table not 16-byte aligned, a pointer not aligned to its element), CUDA.
 */
int loco_rotary_apply(const loco_rotary_t *cfg, const float *d_table, const void *d_positions, const loco_heads_t *x,
                      const loco_heads_t *y, const int32_t *heads, int32_t count, void *stream);

/* ---- attention -----------------------------------------------------------------------------
 *   s_ij = scale * q_i . k_j   for the keys j < length_k that query i sees (causal: j <= i + length_k - length_q)
 *   lse_i = log sum_j exp(s_ij)          o_i = sum_j exp(s_ij - lse_i) v_j
 *   backward:  D_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - D_i)
 *              dq_i = scale * sum_j ds_ij k_j,  dk_j = scale * sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i
 * bf16 heads, fp32 statistics.  Query head h reads key head h / (heads_q / heads_kv); the gradients of a shared key head
 * are summed over its query heads.  A query that sees no key has o = 0, lse = -inf and no gradient; one whose scores are all
 * -inf has o = 0 and lse = -inf.  A score of +inf or NaN makes its query's o NaN (lse: +inf or NaN).  Keys and values that
 * only the causal mask hides have to be finite: zero times what they hold is added where they share a tile.
 */
typedef struct {
    int32_t batch, heads_q, heads_kv;   /* heads_kv divides heads_q, batch * heads_q < 2^31                     */
    int32_t head_dim;                   /* a multiple of 8, 8 .. 128                                            */
    int32_t packed;                     /* 0: padded samples, 1: samples one after the other                    */
    int32_t seq_q, seq_k;               /* rows: of every sample (padded), of all samples together (packed)     */
    int32_t max_q, max_k;               /* packed: no sample is longer; ignored when padded                     */
    int32_t causal;
    float   scale;                      /* finite                                                               */
    const int32_t *d_len_q, *d_len_k;   /* padded: length of each sample [batch], NULL = seq.  Rows past it are
                                           not read as numbers (they may hold anything) and get zeros (lse: -inf)
                                           packed: batch + 1 ascending offsets each, from 0 to seq              */
} loco_attention_t;

/* o: as q.  d_lse: fp32 [batch, heads_q, seq_q], packed [heads_q, seq_q].
 * Errors: ARG, ALIGN (a pointer not 16-byte aligned or a stride not a multiple of 8 elements), UNSUPPORTED, CUDA. */
int loco_attention_forward(const loco_attention_t *cfg, const loco_heads_t *q, const loco_heads_t *k, const loco_heads_t *v,
                           const loco_heads_t *o, float *d_lse, void *stream);

/* Bytes of device memory loco_attention_backward needs beside its operands. */
uint64_t loco_attention_backward_workspace_bytes(const loco_attention_t *cfg);

/* dq as q, dk as k, dv as v; every row is written.  d_work: 16-byte aligned, contents irrelevant before and after.
 * No atomics: the same inputs give the same bits.  Errors: as forward, plus SIZE (d_work_bytes too small). */
int loco_attention_backward(const loco_attention_t *cfg, const loco_heads_t *q, const loco_heads_t *k, const loco_heads_t *v,
                            const loco_heads_t *o, const float *d_lse, const loco_heads_t *d_o, const loco_heads_t *dq,
                            const loco_heads_t *dk, const loco_heads_t *dv, void *d_work, uint64_t d_work_bytes, void *stream);

/* ---- router --------------------------------------------------------------------------------
 * Logits z [tokens, experts].  An expert is available to a token where z is not -inf; a token is active where its mask
 * byte is not 0 (no mask: all are) and some expert is available to it.  N = number of active tokens.
 *   p_t = softmax over the available experts, 0 elsewhere;  lse_t = log sum exp z_t
 *   choice: the top_k largest logits, ties to the lowest index; a choice that finds no available expert is -1, weight 0
 *   weight: p / (sum of the chosen p) with normalize, else p
 *   n_e = tokens that chose e;  P_e = (1/N) sum_t p_te
 *   balance loss = balance_coef * E * sum_e n_e / (N top_k) * P_e        z loss = z_coef / N * sum_t lse_t^2
 * The counts are constants of the gradient.  A NaN logit counts as +infinity in the choice and makes both losses NaN.
 */
typedef struct {
    int32_t dtype;           /* loco_dtype_t of the logits and of their gradient          */
    int32_t experts;         /* E, 1 .. 512                                               */
    int32_t top_k;           /* 1 .. min(E, 16)                                           */
    int32_t normalize;
    float   balance_coef, z_coef;
} loco_router_t;

/* Device workspace of the forward call for any number of tokens (0 on a bad configuration). */
uint64_t loco_router_workspace_bytes(const loco_router_t *cfg);

/*
 *   d_logits      element (t, e) at t*row_stride + e            d_mask   uint8 [tokens] or NULL
 *   d_index       int32 [tokens, top_k]                         d_weight fp32 [tokens, top_k]
 *   d_counts      int32 [E + 1]: n_e, then N                    d_mean   fp32 [E]: P_e (0 where N = 0)
 *   d_losses      fp32 [2]: balance, z (0 where N = 0)
 *   d_work        16-byte aligned; its first 256 bytes must be zero before the first call, and every call leaves them
 *                 zero.  Calls that may run at the same time need workspaces of their own.
 * tokens * top_k < 2^31.  No floating-point atomics: the same inputs give the same bits.  One launch.
 * Errors: ARG, ALIGN, SIZE, CUDA.
 */
int loco_router_forward(const loco_router_t *cfg, int64_t tokens, const void *d_logits, int64_t row_stride,
                        const uint8_t *d_mask, int32_t *d_index, float *d_weight, int32_t *d_counts, float *d_mean,
                        float *d_losses, void *d_work, uint64_t d_work_bytes, void *stream);

/*
 * Gradient with respect to the logits of  d_dlosses[0] * balance + d_dlosses[1] * z + sum d_dweight * weight, from the
 * forward call's d_index and d_counts (an index outside 0 .. E - 1 is no choice).  d_dlosses (fp32 [2]) or d_dweight (fp32
 * [tokens, top_k]) may be NULL (zero).  d_dlogits: element (t, e) at t*drow_stride + e; rows of inactive tokens get zeros.
 * One launch.  Errors: ARG, ALIGN, CUDA.
 */
int loco_router_backward(const loco_router_t *cfg, int64_t tokens, const void *d_logits, int64_t row_stride,
                         const uint8_t *d_mask, const int32_t *d_index, const int32_t *d_counts, const float *d_dlosses,
                         const float *d_dweight, void *d_dlogits, int64_t drow_stride, void *stream);

/* ---- norm ----------------------------------------------------------------------------------
 *   h = x + residual, rounded to the type of x (no residual: h = x)
 *   r = 1 / sqrt(mean_i h_i^2 + eps)         y_i = h_i r w_i   (no weight: w = 1)
 *   8 bits: per row, or per run of `block` columns of a row,  scale = max(max_i |y_i| / 448, 2^-126),  y_i / scale as e4m3
 *   (y_i not rounded before; the weight times h_i has to stay within fp32)
 *   backward, from h:  g = dy w,  n = h r:   dx = r (g - n mean(g n)) + dtotal,   dw = sum over rows of dy n
 * dx is the gradient of x and of the residual alike; dtotal is the one that reaches h past the norm.  Through the 8-bit
 * output it is passed as if nothing had been rounded.  The norm is that of h as it is kept, so that y of a kept h has the
 * same bits.  Squares are summed in fp32.  A row with NaN or an infinity has NaN in y there; its 8-bit scale is NaN.
 */
typedef struct {
    void   *ptr;             /* element (t, i) of a [rows, dim] tensor lies at ptr + t*row_stride + i             */
    int64_t row_stride;      /* in elements; ignored with one row, zero repeats an input, >= dim in an output     */
} loco_rows_t;

typedef struct {
    int32_t dtype;           /* loco_dtype_t of x, residual, h, weight, y and their gradients                     */
    int32_t dim;             /* 1 .. 16384                                                                        */
    int32_t bits8;           /* forward: y is e4m3 with scales                                                    */
    int32_t block;           /* with bits8: columns that share a scale, 0 (the whole row) or 128                  */
    float   eps;             /* >= 0                                                                              */
} loco_norm_t;

/*
 *   residual, weight    NULL: none                    total   h; needed with a residual, NULL without: it would be x
 *   d_scale             with bits8: fp32 [rows, ceil(dim / block)], one a row with block = 0
 * total may be x or the residual itself, with its stride; y may too, without bits8 and where total is not there as well.
 * One launch.  Errors: ARG, ALIGN, CUDA.
 */
int loco_norm_forward(const loco_norm_t *cfg, int64_t rows, const loco_rows_t *x, const loco_rows_t *residual, const void *d_weight,
                      const loco_rows_t *total, const loco_rows_t *y, float *d_scale, void *stream);

/* Bytes of device memory loco_norm_backward needs for the gradient of the weight. */
uint64_t loco_norm_backward_workspace_bytes(const loco_norm_t *cfg);

/*
 *   h        what the norm was taken of               dtotal    NULL: none
 *   d_dweight  NULL: not wanted (d_work may be NULL then); else [dim], the type of x.  d_work: 16-byte aligned, contents
 *              irrelevant before and after; calls that may run at the same time need workspaces of their own.
 * dx may be dy or dtotal itself, with its stride.  No atomics on values: the same inputs give the same bits.  One launch, two
 * with d_dweight.  Errors: ARG, ALIGN, SIZE, CUDA.
 */
int loco_norm_backward(const loco_norm_t *cfg, int64_t rows, const loco_rows_t *h, const loco_rows_t *dy, const void *d_weight,
                       const loco_rows_t *dtotal, const loco_rows_t *dx, void *d_dweight, void *d_work, uint64_t d_work_bytes, void *stream);

/* ---- experts -------------------------------------------------------------------------------
 * Choices index [tokens, top_k] (the router's; outside 0 .. experts - 1: none) are sorted by expert, then token, then slot:
 *   offsets[e]  first row of expert e, offsets[experts] the number of rows in use       place[t, j]  row of a choice, or -1
 *   dispatch    rows[place[t, j]] = x[t]
 *   combine     y[t] = sum_j weight[t, j] rows[place[t, j]]     (no weight: 1; no choice: nothing)
 * Dispatch's gradient is combine without weights, combine's without weights is dispatch.  With weights:
 *   drows[place[t, j]] = weight[t, j] dy[t]      dweight[t, j] = dy[t] . rows[place[t, j]]   (0 where there is no choice)
 * Rows that no choice has are not written; a place outside the rows is none.  Sums in fp32, in the order of the slots; dweight's in fp32 too,
 * at most max(64, dim / 64) products one after the other, then some ten sums of those.  No output may overlap an input.
 */

/* Device workspace of loco_experts_sort for any number of tokens (0 for a bad number of experts). */
uint64_t loco_experts_sort_workspace_bytes(int32_t experts);

/* d_index, d_place: int32 [tokens, top_k]; d_offsets: int32 [experts + 1]; experts 1 .. 512, tokens * top_k < 2^31.  d_work:
 * 16-byte aligned, contents irrelevant before and after; calls that may run at the same time need workspaces of their own.
 * One or two launches.  Errors: ARG, ALIGN, SIZE, CUDA. */
int loco_experts_sort(int32_t experts, int64_t tokens, int32_t top_k, const int32_t *d_index, int32_t *d_offsets, int32_t *d_place,
                      void *d_work, uint64_t d_work_bytes, void *stream);

typedef struct {
    int32_t dtype;           /* loco_dtype_t of the tokens and rows                       */
    int32_t dim;             /* 1 .. 2^30                                                 */
    int32_t top_k;           /* 1 .. 16                                                   */
    int64_t tokens;          /* tokens * top_k < 2^31                                     */
    int64_t rows;            /* rows of the sorted tensors: places are below, < 2^31      */
} loco_experts_t;

/* x [tokens, dim], rows [rows, dim]; d_place, d_weight (fp32), d_dweight (fp32): [tokens, top_k].  No place may come twice in
 * dispatch and combine_backward, which write it.  One launch each.  Errors: ARG, ALIGN, CUDA. */
int loco_experts_dispatch(const loco_experts_t *cfg, const loco_rows_t *x, const int32_t *d_place, const loco_rows_t *rows, void *stream);
int loco_experts_combine(const loco_experts_t *cfg, const loco_rows_t *rows, const int32_t *d_place, const float *d_weight,
                         const loco_rows_t *y, void *stream);
int loco_experts_combine_backward(const loco_experts_t *cfg, const loco_rows_t *dy, const loco_rows_t *rows, const int32_t *d_place,
                                  const float *d_weight, const loco_rows_t *drows, float *d_dweight, void *stream);

/* Zeros in rows [rows, dim] from offsets[experts] on (d_offsets: int32 [experts + 1]), which the calls here leave as they were: for
 * what goes on with all rows.  One launch.  Errors: ARG, ALIGN, CUDA. */
int loco_experts_clear(int32_t dtype, int32_t dim, int64_t rows_count, const loco_rows_t *rows, int32_t experts, const int32_t *d_offsets, void *stream);

/* The same for all rows that no expert has, the offsets being read as loco_experts_product reads them: those ahead of offsets[0] too, and
 * those from the largest offset on. */
int loco_experts_clear_others(int32_t dtype, int32_t dim, int64_t rows_count, const loco_rows_t *rows, int32_t experts, const int32_t *d_offsets, void *stream);

/* The experts' matrices, [experts, first, second]: element (e, i, j) at ptr + e*expert_stride + i*row_stride + j. */
typedef struct {
    void   *ptr;
    int64_t expert_stride, row_stride;
} loco_matrices_t;

typedef struct {
    int32_t experts;         /* 1 .. 512                                                                          */
    int64_t rows;            /* of x and y, < 2^31; expert e has rows offsets[e] .. offsets[e + 1] - 1            */
    int32_t d_in, d_out;     /* multiples of 8, to 2^30                                                           */
    int32_t transposed;      /* product: the matrices are [experts, d_out, d_in]; else [experts, d_in, d_out]     */
} loco_product_t;

/*
 * y_t = x_t W_e, transposed: x_t W_e^T, for the rows t of every expert e; x [rows, d_in], y [rows, d_out]; bfloat16, fp32
 * sums.  The gradient of x is the same call on dy with `transposed` the other way round (d_in and d_out change places).
 * d_offsets: int32 [experts + 1], ascending; they are read on the device, as the largest so far and within the rows.  Rows outside every expert
 * are neither read as numbers nor written.  A NaN or infinity in a row or matrix reaches that row's or expert's outputs only.
 * y may not overlap x or the matrices.  One launch.  Errors: ARG, ALIGN (a pointer not 16-byte aligned or a stride not a multiple of 8
 * elements), UNSUPPORTED, CUDA.
 */
int loco_experts_product(const loco_product_t *cfg, const loco_rows_t *x, const loco_matrices_t *w, const int32_t *d_offsets,
                         const loco_rows_t *y, void *stream);

/* dw_e = sum over the rows t of expert e of a_t^T b_t; a [rows, d_in], b [rows, d_out], dw [experts, d_in, d_out]; an expert
 * without rows gets zeros.  The gradient of the matrices: a = x, b = dy, or, where they are transposed, a = dy, b = x.
 * `transposed` is ignored.  No atomics: the same inputs give the same bits.  One launch.  Errors: as loco_experts_product. */
int loco_experts_product_weights(const loco_product_t *cfg, const loco_rows_t *a, const loco_rows_t *b, const int32_t *d_offsets,
                                 const loco_matrices_t *dw, void *stream);

/* ---- gradient ------------------------------------------------------------------------------
 * Of a list of gradients g:   squares = sum over all elements of g^2,   norm = sqrt(squares),
 *   out = c g  with  c = max_norm / norm where norm > max_norm, else 1   (a norm that is infinite: c = 0; NaN: c = NaN)
 * Between the two calls the squares of the ranks that hold the other shards can be added.  Groups of 32 squares (fp32 gradients: 16) are added
 * in fp32, six roundings in a row at most, and the groups in 64 bits: squares is off by at most 6 * 2^-24 of itself.  A group that leaves
 * fp32's range is squared and added in 64 bits.
 */
typedef struct {
    const void *x;           /* n elements, any alignment to their own size                                       */
    void       *y;           /* the same, or x itself; ignored by loco_gradient_squares                           */
    uint64_t    n;
    int32_t     dtype;       /* loco_dtype_t                                                                      */
} loco_span_t;

/* Device workspace of loco_gradient_squares for any list. */
uint64_t loco_gradient_squares_workspace_bytes(void);

/* d_squares: one double.  d_work: 16-byte aligned; its first 256 bytes must be zero before the first call, and every call
 * leaves them zero; calls that may run at the same time need workspaces of their own.  The same list gives the same bits.
 * One launch for every 768 spans.  Errors: ARG, ALIGN, SIZE, CUDA. */
int loco_gradient_squares(const loco_span_t *spans, int32_t count, double *d_squares, void *d_work, uint64_t d_work_bytes, void *stream);

/* d_norm: one fp32, or NULL.  max_norm >= 0.  No output may overlap another, another's gradient, or its own unless it is that.  Where c is 1
 * nothing is written to a y that is x.  One launch for every 768 spans.  Errors: ARG, ALIGN, CUDA. */
int loco_gradient_clip(const loco_span_t *spans, int32_t count, const double *d_squares, double max_norm, float *d_norm, void *stream);

/*
 * Flags raised on the current device since the library was loaded; SYNCHRONISES `stream`.  The attention and product kernels
 * wait on their own copies and products, never on another launch; a wait that exceeds two seconds gives up, the outputs of
 * its block are meaningless and the flag is raised.
 */
#define LOCO_LAYER_FLAG_TIMEOUT 1u
int loco_layer_status(uint32_t *flags, void *stream);

/* Number of kernels launched by the functions of this header in the calling process. */
uint64_t loco_layer_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* LOCO_B200_LAYER_H */
