// What the kernels between a block's products take, and how they are launched (device code: attention_kernel.hpp, kernels_blocks.hip).
#pragma once
#include "layers.hpp"

namespace alpa {

// A tensor [rows][heads][dim]; strides in bytes.
struct Heads {
    char *p;
    int64_t row, head;
};

struct AttentionArgs {
    Heads q, k, v, dy, y;           // operands; a head's `bytes` are aligned to 16 and padded with zeros (y: read in the backward pass)
    Heads out, out2;                // results: y; dq; dk and dv
    int wide;                       // results may be written four elements at a time
    float *lse;                     // [rows][heads]; NULL in the forward pass: not kept
    float *delta;                   // backward: [rows][heads], sum over a head of dy y
    int rows, k_rows, seqs, heads, kv_heads, group, dim, bytes;
    const int32_t *offsets, *k_offsets, *prefix;
    const float *slopes;
    int k_step, causal;
    float scale, cap, twice;        // twice: 2 scale / cap, times the binary logarithm of e
    int tiles;                      // grid: row tiles of all sequences, at most
    uint32_t before;                // of the grid, workgroups of earlier launches
    int key_tile;                   // dk, dv: keys of a workgroup
    int unit;                       // keys of a step: what parts of them are multiples of
    int splits;                     // parts, at most, of the keys (y, dq) or of the rows (dk, dv)
    float *part;                    // splits > 1: [part][item][dim] sums, of dk or else; items: rows x heads, or key rows x kv heads
    float2 *stat;                   // forward: [part][item] (maximum, sum)
    float *part2;                   // of dv
};

constexpr int ATTENTION_TILE = 128, FEW_TILE = 32;     // packed rows, or keys, of a workgroup

// An element type's kernels (one file each, to build them side by side).
#define ALPA_ATTENTION_LAUNCHES(type)                                                 \
    hipError_t launch_attention_##type(hipStream_t, int few, const AttentionArgs &);       \
    hipError_t launch_attention_dq_##type(hipStream_t, int few, const AttentionArgs &); \
    hipError_t launch_attention_dkv_##type(hipStream_t, const AttentionArgs &);
ALPA_ATTENTION_LAUNCHES(f32)
ALPA_ATTENTION_LAUNCHES(f16)
ALPA_ATTENTION_LAUNCHES(bf16)

// rows of a head's dim padded to blocks of 32, as the kernels are compiled for them: 2, 3, 4 or 8
inline int dim_blocks(int dim) { return dim <= 64 ? 2 : dim <= 96 ? 3 : dim <= 128 ? 4 : 8; }


// Copies tensors to [rows][heads][to_len] elements (a multiple of 16 bytes), zeros behind len.
struct HeadPack {
    struct { const char *from; char *to; int64_t row, head, rows; int heads; } t[5];      // strides in elements
    int count, len, to_len;
};
hipError_t launch_head_pack(hipStream_t st, int dtype, const HeadPack &g);

struct RotaryArgs {
    Heads x, y;                     // strides in elements
    int64_t rows;
    int heads, dim, rot, interleaved, wide, copy;      // copy: elements behind rot are copied
    float scale, sign;
    const int64_t *positions;
    const double *frequencies;
};
hipError_t launch_rotary(hipStream_t st, int dtype, const RotaryArgs &a);

struct NormArgs {
    const char *x, *dy, *weight, *bias;
    char *y;                        // y, or dx
    int64_t ldx, lddy, ldy;         // elements
    int rows, n, wide;
    float eps;
    float *mean, *rstd;
    float *part_w, *part_b;         // backward: [groups][n], or NULL
    int groups;
    char *dweight, *dbias;
};
hipError_t launch_norm(hipStream_t st, int dtype, const NormArgs &a);
hipError_t launch_norm_backward(hipStream_t st, int dtype, const NormArgs &a);
int norm_groups(int64_t rows);

}  // namespace alpa
