/*
 * alpa_blocks.h — C ABI of what a block has between its products (gfx950): attention, rotary positions, layer norm.
 *
 * With the products of alpa_layers.h they make the blocks whose times the planner of alpa_dp.h plans with.
 *
 * Conventions: those of alpa_layers.h (device pointers of the caller, work memory, no synchronisation, no allocation, the same bits from
 * two calls, errors as negative codes with alpa_dp_last_error()).  Beside matrices there are tensors [rows][heads][dim] whose elements of
 * a head are contiguous, heads and rows any distance apart that keeps them from overlapping (in results) and in 2^40 bytes.
 */
#ifndef ALPA_BLOCKS_H
#define ALPA_BLOCKS_H

#include "alpa_layers.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ALPA_BLOCK_MAX_HEADS      4096
#define ALPA_BLOCK_MAX_DIM        4096      /* rotary positions                                  */
#define ALPA_ATTENTION_MAX_DIM    256
#define ALPA_ATTENTION_MAX_SEQS   65536
#define ALPA_ATTENTION_MAX_ITEMS  (1 << 30) /* rows x heads, of queries and of keys              */

typedef struct { void *p; int64_t row, head; } alpa_heads_t;    /* first element; elements from row to row, from head to head */

/*
 * Attention of packed sequences.  Sequence s has the query rows offsets[s] .. offsets[s + 1] - 1 and the key rows
 * k_offsets[s * k_step] .. k_offsets[s * k_step + 1] - 1: with k_step 1 keys are packed like queries, with k_step 2 each sequence has a first key and an end of
 * its own, which may leave gaps (a cache with room for more keys) or meet (a beginning that sequences share).  Documents that are packed
 * in one row of a batch are sequences.  Query i of n stands at place p = i + m - n of its m keys: the last query at the last key.
 *     r_ij = scale q_i . k_j
 *     a_ij = cap tanh(r_ij / cap) - slope |p - j|      (cap 0: r_ij itself; slopes NULL: no bias)
 *     y_i  = sum_j exp(a_ij - lse_i) v_j,   lse_i = log sum_j exp(a_ij)     over the keys j that i sees
 * A row sees all keys of its sequence; with `causal` those up to its own place, and those in front of prefix[s].  A row that sees none, and
 * a row of no sequence, gets zeros and an lse of -infinity.
 * Query head h reads kv head h / (heads / kv_heads).
 * Offsets are taken as they come, cut to the tensors' rows, as in alpa_experts_forward; sequences must not overlap in queries.
 * exp(a - lse) is rounded to `dtype` as an operand of the product with v (in float16 times 2^12 of the row's largest, about, so that small ones keep their bits).  Values that are not finite in q, k, v or dy may reach all rows and keys of
 * their sequence and kv head, also where the mask hides them (zero times infinity); keys and rows of no sequence are not read.
 */
typedef struct {
    int32_t dtype;
    int32_t seqs, heads, kv_heads, dim;      /* heads a multiple of kv_heads                                        */
    int32_t causal, k_step;
    float scale, cap;                        /* finite; cap 0 or positive                                            */
    int64_t rows, k_rows;                    /* of q and y, of k and v                                               */
    const int32_t *offsets, *k_offsets;      /* DEVICE [seqs + 1]; DEVICE [seqs + 1] or [seqs][2]; NULL with one      *
                                              * sequence: all rows, all keys                                           */
    const int32_t *prefix;                   /* DEVICE [seqs], or NULL; read where causal                            */
    const float *slopes;                     /* DEVICE [heads], or NULL                                              */
} alpa_attention_t;

/*
 * lse: DEVICE float [rows][heads], or NULL: not kept (the backward pass takes it).
 * Work memory: parts of results where few rows meet many keys (the keys are split then), and copies of q, k, v that are not aligned to 16 bytes.
 */
int64_t alpa_attention_forward_work(const alpa_attention_t *how, alpa_heads_t q, alpa_heads_t k, alpa_heads_t v);
int alpa_attention_forward(const alpa_attention_t *how, alpa_heads_t q, alpa_heads_t k, alpa_heads_t v, alpa_heads_t y,
                           float *lse, void *work, int64_t work_bytes, void *hip_stream);

/*
 * Its gradients, any of dq, dk, dv NULL (p NULL).  Keys have to be packed (k_step 1).  Slopes are constants.
 *     P = exp(a - lse),  dA = P (dy . v - dy . y),  dR = dA (1 - tanh^2)
 *     dv_j = sum_i P_ij dy_i,   dq_i = scale sum_j dR_ij k_j,   dk_j = scale sum_i dR_ij q_i    (kv heads: over their query heads too)
 * P and dR are rounded to `dtype` as operands of the products (in float16 P times 2^14, so that the weights of many keys keep their bits, dR times powers of two that keep it
 * from overflowing and small ones from losing bits); y is taken as it was rounded.  Rows and keys of no sequence get zeros.
 */
int64_t alpa_attention_backward_work(const alpa_attention_t *how, alpa_heads_t dy, alpa_heads_t q, alpa_heads_t k,
                                     alpa_heads_t v, alpa_heads_t y);
int alpa_attention_backward(const alpa_attention_t *how, alpa_heads_t dy, alpa_heads_t q, alpa_heads_t k, alpa_heads_t v,
                            alpa_heads_t y, const float *lse, alpa_heads_t dq, alpa_heads_t dk, alpa_heads_t dv, void *work,
                            int64_t work_bytes, void *hip_stream);

/*
 * Rotary positions: the first `rot` (even) elements of each head are pairs, (t, t + rot / 2), or (2 t, 2 t + 1) if `interleaved`, and pair (a, b) of
 * index t in a row at position p becomes
 *     scale (a cos u - b sin u),  scale (a sin u + b cos u),   u = p frequencies[t];
 * the other elements are copied.  The angle is reduced in 64 bits.  y may be x itself (all three of its members equal): rows are turned in
 * place then.  The backward call turns the other way, by the same scale.
 *   positions    DEVICE int64 [rows]
 *   frequencies  DEVICE double [rot / 2], radians a position
 */
int alpa_rotary_forward(int dtype, int64_t rows, int heads, int dim, int rot, int interleaved, float scale,
                        const int64_t *positions, const double *frequencies, alpa_heads_t x, alpa_heads_t y,
                        void *hip_stream);
int alpa_rotary_backward(int dtype, int64_t rows, int heads, int dim, int rot, int interleaved, float scale,
                         const int64_t *positions, const double *frequencies, alpa_heads_t dy, alpa_heads_t dx,
                         void *hip_stream);
/*
 * Frequencies base^(-2 t / rot) for contexts `factor` times longer than those that a model was trained on, `context` positions (into HOST memory, no
 * device is touched): pairs that turn `high` times and more over `context` stay, those that turn `low` times and less are divided by factor,
 * those between linearly in between.  context 0: all are divided.
 * Errors: EINVAL (rot not in 2, 4 .. ALPA_BLOCK_MAX_DIM, base or factor not positive, context negative, not low < high, null pointer).
 */
int alpa_rotary_frequencies(int rot, double base, double factor, double context, double low, double high, double *frequencies);

/*
 * Layer norm of rows of n:   y = (x - mean) rstd weight + bias,   rstd = 1 / sqrt(variance + eps).
 *   weight, bias  [n] of type `dtype`, or NULL (1, 0);  mean, rstd  DEVICE float [rows], or both NULL: not kept.
 */
int alpa_norm_forward(int dtype, int64_t rows, int64_t n, float eps, alpa_mat_t x, const void *weight, const void *bias,
                      alpa_mat_t y, float *mean, float *rstd, void *hip_stream);
/*
 * Its gradients, any of dx, dweight, dbias NULL:  h = (x - mean) rstd,  g = dy weight,
 *     dx = rstd (g - mean(g) - h mean(g h)),   dweight = sum over rows of dy h,   dbias = sum over rows of dy.
 * With rows == 0 dweight and dbias are zero.
 */
int64_t alpa_norm_backward_work(int dtype, int64_t rows, int64_t n);
int alpa_norm_backward(int dtype, int64_t rows, int64_t n, alpa_mat_t dy, alpa_mat_t x, const float *mean,
                       const float *rstd, const void *weight, alpa_mat_t dx, void *dweight, void *dbias, void *work,
                       int64_t work_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ALPA_BLOCKS_H */
