// What the layer operators' kernels take, and how they are launched (device code: product_kernel.hpp, kernels_layers.hip).
#pragma once
#include "internal.hpp"

namespace alpa {

// What becomes of a tile of the product.
enum Epilogue : int {
    EPI_LINE,       // act(v) + residual with act none or relu:  v < low ? low : v
    EPI_SIGMOID,    // v / (1 + exp(-v (c1 + c3 v^2))): silu, and gelu in its tanh form
    EPI_ERF,        // gelu
    EPI_SUM,        // 32-bit sums, added to what is there or put down, and rounded into the result by the last of several
    EPI_LOSS,       // logits: per row and stripe of columns a maximum, a sum of exponentials, and the target's logit
    EPI_GRAD,       // logits: (softmax - onehot) * coef
};

// How rows are dealt to weights.
enum Grouping : int { GROUP_NONE, GROUP_ROWS, GROUP_STEPS };     // ragged in the result's rows, or in the contraction

struct ProductArgs {
    const char *a, *b;              // operands; strides in bytes
    int64_t lda, ldb;
    int M, N, K;                    // result rows (all groups together), columns, contraction (all groups together)
    int a_k, b_k, a_len, b_len;     // extents of the contraction, and of rows where those are contiguous, with their padding to 16 bytes
    int grouping, experts;
    const int32_t *offsets;
    int64_t b_expert;               // GROUP_ROWS: bytes from an expert's b to the next one's; GROUP_STEPS: result elements
    int row_tiles, col_tiles;       // grid: row tiles (GROUP_ROWS: slots), column tiles; GROUP_STEPS: times experts
    int before;                     // of each XCD's tiles, those that earlier launches took
    int splits, split_steps;        // of the contraction, 128 bytes a step, all of them if it is not split (GROUP_NONE only)
    // epilogue
    char *out;                      // result, strides in elements
    int64_t ldo;
    const char *bias, *residual;
    int64_t ldr;
    char *z;
    int64_t ldz;
    int wide;                       // pointers, strides and row length allow 16-byte accesses in the epilogue
    float low, c1, c3;
    float *sum;                     // EPI_SUM: [split][M][N]
    int first, last;
    float *total;                   // EPI_SUM: where `sum` goes on from product to product, if one that is split may be joined to it (NULL: none is split)
    const float *scale;             // EPI_SUM, EPI_LINE: result times *scale (NULL: 1)
    const int64_t *target;          // EPI_LOSS, EPI_GRAD
    int64_t word0;                  // EPI_GRAD: the first column's word
    float2 *stat;                   // EPI_LOSS: [stripe][M]
    float *at_target;
    const float *lse, *coef;        // EPI_GRAD: [M]
};

constexpr int SMALL_TILE = 64, TILE = 128, BIG_TILE = 256;         // rows and columns of a workgroup's tile
constexpr int COMPUTE_UNITS = 256;
constexpr int STEP_BYTES = 128;
constexpr int STRIPE = 64;                        // columns of a stripe of EPI_LOSS, in all tiles

// Form of the two operands: both with their contraction contiguous (x wT), the second one's rows contiguous (dz w), or both (dzT x).
enum Forms : int { FORM_RR, FORM_RC, FORM_CC };

// tile: one of the three; the large one only where results are aligned (`wide`) and their rows multiples of eight elements.  Addresses, strides and contiguous extents of the operands are multiples of 16 bytes.
hipError_t launch_product(hipStream_t st, int dtype, Forms forms, Epilogue epi, int tile, const ProductArgs &a);
hipError_t launch_product_f32(hipStream_t, Forms, Epilogue, int, const ProductArgs &);
hipError_t launch_product_f16(hipStream_t, Forms, Epilogue, int, const ProductArgs &);
hipError_t launch_product_bf16(hipStream_t, Forms, Epilogue, int, const ProductArgs &);

// Copies matrices, [rows][len], to rows of `to_len` elements (a multiple of 16 bytes), zeros behind len: what an operand needs that is not aligned to 16 bytes.
struct PackArgs {
    struct { const char *from; char *to; int64_t ld, rows; int len, to_len; } mats[3];
    int count;
};
hipError_t launch_pack(hipStream_t st, int dtype, const PackArgs &g);

// dz = dy * act'(z), and sums of dz over the rows of each slot of `slot_rows` rows
struct SlopeArgs {
    const char *dy, *z;             // strides in elements
    int64_t lddy, ldz;
    char *dz;                       // [rows][ldd], zeros behind N, or NULL
    int64_t ldd;
    float *part;                    // [slots][N], or NULL
    int rows, N, slots, slot_rows, experts;    // experts 0: no groups
    const int32_t *offsets;
    int act, bytes;                 // bytes: of dy and z that may be read at once, 16, 8 or 0 (one element)
    float *tops, *scale;            // float16: dz is kept divided by *scale, a power of two found here (tops, [TOP_PARTS]: room for that; NULL: as it is)
    int top_count;
};
constexpr int TOP_PARTS = 1024;
hipError_t launch_slope(hipStream_t st, int dtype, const SlopeArgs &a);
// dbias[e][n] = sum over the expert's slots
hipError_t launch_bias_sum(hipStream_t st, int dtype, const float *part, char *dbias, int rows, int N, int slots, int slot_rows, int experts,
                           const int32_t *offsets);
// result = act(sum over splits + bias) + residual, and z (epi: EPI_LINE, EPI_SIGMOID or EPI_ERF)
hipError_t launch_join(hipStream_t st, int dtype, Epilogue epi, const ProductArgs &a);
// loss and lse of each row from its stripes
hipError_t launch_loss(hipStream_t st, const float2 *stat, int stripes, int rows, const float *at_target, const int64_t *target,
                       int64_t words, float *loss, float *lse);
// coef = dloss / *scale for counted rows, 0 for others; *scale = largest |dloss| / 2^14
hipError_t launch_coef(hipStream_t st, const float *dloss, const int64_t *target, int64_t words, int rows, float *coef, float *scale);

// slots of `tile` rows that the groups of `rows` rows can make at most, rows of no group among them
inline int64_t slots_at_most(int64_t rows, int experts, int tile)
{
    const int64_t groups = (int64_t)experts + 2;
    return rows / tile + (groups < rows ? groups : rows);
}

}  // namespace alpa
