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
 *               z loss, and their gradient.  An expert whose count is zero has an all-zero gradient segment.
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

/*
 * Flags raised on the current device since the library was loaded; SYNCHRONISES `stream`.  The attention kernels wait on
 * their own copies and products, never on another block; a wait that exceeds two seconds gives up, the outputs of its
 * block are meaningless and the flag is raised.
 */
#define LOCO_LAYER_FLAG_TIMEOUT 1u
int loco_layer_status(uint32_t *flags, void *stream);

/* Number of kernels launched by the functions of this header in the calling process. */
uint64_t loco_layer_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* LOCO_B200_LAYER_H */
