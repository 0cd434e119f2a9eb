/*
 * alpa_layers.h — C ABI of the layer operators (gfx950).
 *
 * What the planner of alpa_dp.h needs to know of a stage is how long its layers take on a submesh (the profiled
 * options of alpa_dp_create_from_profiles; "Profile" in Alg. 1).  These are the layers' products themselves, forward
 * and backward: the product of a dense layer with its epilogue, the products of an expert layer, and the loss of the
 * last layer over a vocabulary.
 *
 * Conventions
 *   - all tensors are DEVICE pointers owned by the caller, row-major, rows `ld` elements apart (ld >= row length); weights are
 *     [out][in]; x, w, bias, residual, y, z and their gradients have the type `dtype`, sums are held in 32 bits or
 *     more, results are rounded once;
 *   - a call only queues kernels on `hip_stream` (a hipStream_t, NULL = the null stream) and returns: it allocates nothing, copies
 *     nothing to or from the host and does not synchronise, so that it may be recorded into a HIP graph.  It must be made with the tensors'
 *     device current.  Calls that may overlap need work memory of their own each;
 *   - work memory: `work` of at least the bytes that the `_work` call of the same arguments returns (0 for arguments that are
 *     refused), aligned to 256 bytes; NULL if that is 0.  Nothing in it needs to be kept or cleared between calls;
 *   - an output must not overlap any other tensor of the call;
 *   - results do not depend on the launch: two calls on the same arguments give the same bits.
 *
 * Limits: sizes of a row up to ALPA_LAYER_MAX_WIDTH, strides up to 2^22 bytes, rows up to ALPA_LAYER_MAX_ROWS (0 is allowed),
 * words and experts as below.  Tensors need no more than the alignment of one element; operands whose address, stride or row length is no
 * multiple of 16 bytes are first copied to work memory.
 *
 * All functions return ALPA_DP_OK or a negative code of alpa_dp.h and never throw or abort; alpa_dp_last_error() has the message.
 */
#ifndef ALPA_LAYERS_H
#define ALPA_LAYERS_H

#include "alpa_dp.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ALPA_F32   0
#define ALPA_F16   1
#define ALPA_BF16  2

#define ALPA_ACT_NONE       0
#define ALPA_ACT_RELU       1
#define ALPA_ACT_GELU       2     /* z * normal distribution function(z)                           */
#define ALPA_ACT_GELU_TANH  3     /* z / 2 * (1 + tanh(sqrt(2 / pi) * (z + 0.044715 z^3)))         */
#define ALPA_ACT_SILU       4     /* z / (1 + exp(-z))                                             */

#define ALPA_LAYER_MAX_WIDTH    (1 << 20)
#define ALPA_LAYER_MAX_ROWS     (1 << 28)
#define ALPA_LAYER_MAX_EXPERTS  4096
#define ALPA_LAYER_MAX_WORDS    (1 << 24)

typedef struct { void *p; int64_t ld; } alpa_mat_t;    /* first element; elements from row to row */

/*
 * Product with its epilogue:   z = x w^T + bias,   y = act(z) + residual.
 *   x [rows][n_in], w [n_out][n_in], bias [n_out] or NULL, residual [rows][n_out] (p NULL: none), y [rows][n_out], z [rows][n_out] (p
 *   NULL: not kept; what the backward pass of an activation needs).
 * An activation reads z before it is rounded.
 * Errors: EINVAL (null pointer, size, type, activation or stride out of range, pointer not aligned to an element, work memory too small),
 * EHIP.
 */
int64_t alpa_linear_forward_work(int dtype, int64_t rows, int64_t n_in, int64_t n_out, alpa_mat_t x, alpa_mat_t w);
int alpa_linear_forward(int dtype, int act, int64_t rows, int64_t n_in, int64_t n_out, alpa_mat_t x, alpa_mat_t w,
                        const void *bias, alpa_mat_t residual, alpa_mat_t y, alpa_mat_t z, void *work,
                        int64_t work_bytes, void *hip_stream);

/*
 * Its gradients:   dz = dy * act'(z),   dx = dz w,   dw = dz^T x,   dbias = column sums of dz.
 *   Any of dx, dw, dbias may be NULL (p NULL).  z is needed unless act is ALPA_ACT_NONE, x for dw, w for dx.  dz is rounded to
 *   `dtype` as an operand of the two products (in float16, with a smooth activation, times a power of two found from the largest |dy|, so that it
 *   neither overflows nor loses bits of small dy); dbias is summed from the 32-bit values.  The slope of ALPA_ACT_RELU at 0 is 0.  (The residual's gradient is dy.)
 * With rows == 0, dw and dbias are zero.  Work memory has room for dbias's sums, wanted or not.
 */
int64_t alpa_linear_backward_work(int dtype, int act, int64_t rows, int64_t n_in, int64_t n_out, alpa_mat_t dy,
                                  alpa_mat_t x, alpa_mat_t w);
int alpa_linear_backward(int dtype, int act, int64_t rows, int64_t n_in, int64_t n_out, alpa_mat_t dy, alpa_mat_t z,
                         alpa_mat_t x, alpa_mat_t w, alpa_mat_t dx, alpa_mat_t dw, void *dbias, void *work,
                         int64_t work_bytes, void *hip_stream);

/*
 * The same grouped by expert: rows offsets[e] .. offsets[e + 1] - 1 go through w[e] and bias[e].
 *   offsets   DEVICE int32 [experts + 1], non-decreasing, within 0 .. rows; groups may be empty.  (Values outside that give
 *             unspecified results, but no access outside the tensors.)  Rows of no group get zeros in y, z and dx.
 *   w, dw     [experts][n_out][n_in], an expert's rows `ld` apart and the next expert's behind them (n_out * ld elements).
 *   bias, dbias  [experts][n_out].
 * dw and dbias of an empty group are zero.
 */
int64_t alpa_experts_forward_work(int dtype, int64_t rows, int experts, int64_t n_in, int64_t n_out, alpa_mat_t x,
                                  alpa_mat_t w);
int alpa_experts_forward(int dtype, int act, int64_t rows, int experts, int64_t n_in, int64_t n_out,
                         const int32_t *offsets, alpa_mat_t x, alpa_mat_t w, const void *bias, alpa_mat_t residual,
                         alpa_mat_t y, alpa_mat_t z, void *work, int64_t work_bytes, void *hip_stream);
int64_t alpa_experts_backward_work(int dtype, int act, int64_t rows, int experts, int64_t n_in, int64_t n_out,
                                   alpa_mat_t dy, alpa_mat_t x, alpa_mat_t w);
int alpa_experts_backward(int dtype, int act, int64_t rows, int experts, int64_t n_in, int64_t n_out,
                          const int32_t *offsets, alpa_mat_t dy, alpa_mat_t z, alpa_mat_t x, alpa_mat_t w,
                          alpa_mat_t dx, alpa_mat_t dw, void *dbias, void *work, int64_t work_bytes,
                          void *hip_stream);

/*
 * Softmax cross entropy of l = x w^T over `words` words, piece by piece: l is never in memory as a whole.
 *   target  DEVICE int64 [rows]; negative: the row has no loss (0) and no gradient; words or above: its loss is NaN, and so
 *           are the gradients it has a part in.
 *   loss    DEVICE float [rows]: log(sum_v exp(l_v)) - l_target.
 *   lse     DEVICE float [rows]: the logarithm, which the backward pass takes back.
 * Work memory holds two floats for every row and 64 words, an eighth of a byte a logit.
 */
int64_t alpa_vocab_loss_forward_work(int dtype, int64_t rows, int64_t n_in, int64_t words, alpa_mat_t x, alpa_mat_t w);
int alpa_vocab_loss_forward(int dtype, int64_t rows, int64_t n_in, int64_t words, alpa_mat_t x, alpa_mat_t w,
                            const int64_t *target, float *loss, float *lse, void *work, int64_t work_bytes,
                            void *hip_stream);

/*
 * Its gradients for loss gradients dloss (DEVICE float [rows]):   g = (softmax(l) - onehot(target)) * dloss,   dx = g w,   dw = g^T x.
 *   l is computed again, a piece of the words at a time, and with many rows a block of them: 256 MiB of work memory at most, beside what it takes to
 *   sum dx, and dw of a piece, in 32 bits over several of them.  g is rounded to `dtype` as an operand of the two products, divided by the
 *   largest |dloss| (found on the device) so that small probabilities keep their bits in 16-bit floats.  dx or dw may be NULL.  A row without a
 *   loss is not read into dx; in dw it counts as 0 times its x.
 */
int64_t alpa_vocab_loss_backward_work(int dtype, int64_t rows, int64_t n_in, int64_t words, alpa_mat_t x,
                                      alpa_mat_t w);
int alpa_vocab_loss_backward(int dtype, int64_t rows, int64_t n_in, int64_t words, const float *dloss, alpa_mat_t x,
                             alpa_mat_t w, const int64_t *target, const float *lse, alpa_mat_t dx, alpa_mat_t dw,
                             void *work, int64_t work_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ALPA_LAYERS_H */
