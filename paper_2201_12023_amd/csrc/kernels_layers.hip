// The small kernels around the products of the layer operators: the activation's slope with the bias gradient's sums, the join of a
// product that was split over its contraction, and the statistics of the loss.
#include "epilogue.hpp"
#include "slots.hpp"

#include <type_traits>

namespace alpa {

// ---------------------------------------------------------------- rows in 16-byte units

// A thread writes sixteen bytes; reads of one row are consecutive, so the lines they share come from the cache.  All of a call's matrices go in one
// launch (two launches took 5 us more where both are small).
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(const PackArgs g)
{
    constexpr int V = 16 / sizeof(T);
    const auto &mat = g.mats[blockIdx.y];
    const int per_row = mat.to_len / V;
    const int64_t total = mat.rows * per_row;
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < total; c += (int64_t)gridDim.x * 256) {
        const int64_t r = c / per_row;
        const int n = (int)(c - r * per_row) * V;
        float v[V];
        load_row<T>(mat.from, r * mat.ld + n, mat.len - n, 0, v);
        store_row<T>(mat.to, r * mat.to_len + n, V, 1, v);
    }
}

hipError_t launch_pack(hipStream_t st, int dtype, const PackArgs &g)
{
    int64_t chunks = 0;
    for (int k = 0; k < g.count; ++k) chunks = std::max(chunks, g.mats[k].rows * g.mats[k].to_len * (dtype == 0 ? 4 : 2) / 16);
    const dim3 grid((unsigned)std::min<int64_t>((chunks + 255) / 256, 8192), (unsigned)g.count);
    if (dtype == 0) pack_kernel<float><<<grid, 256, 0, st>>>(g);
    else if (dtype == 1) pack_kernel<f16><<<grid, 256, 0, st>>>(g);
    else pack_kernel<bf16><<<grid, 256, 0, st>>>(g);
    return hipGetLastError();
}

// ---------------------------------------------------------------- dz = dy * act'(z), sums of its columns

// act'(z); at infinities the limits
template <class T>
__device__ __forceinline__ float slope_of(float z, int act)
{
    if (act == 1) return z > 0.0f ? 1.0f : (z == z ? 0.0f : z);
    if (act == 2) {
        if (fabsf(z) == INFINITY) return z > 0.0f ? 1.0f : 0.0f;
        const float e = exp_for<T>(-0.5f * z * z);
        return normal_integral<T>(z, e) + z * 0.39894228040143268f * e;
    }
    // z s(u) with u = c1 z + c3 z^3:  s + z s (1 - s) u'
    const float c1 = act == 3 ? 1.5957691216057308f : 1.0f, c3 = act == 3 ? 0.071354816272600257f : 0.0f;
    if (fabsf(z) > 1e4f) return z > 0.0f ? 1.0f : 0.0f;          // (there 1 - s or s is 0 in 32 bits, and z^3 may not be finite)
    const float zz = z * z, e = exp_for<T>(-z * (c1 + c3 * zz)), s = divide_for<T>(1.0f, 1.0f + e);
    return s + z * s * (1.0f - s) * (c1 + 3.0f * c3 * zz);
}

// Float16 has room for neither end: a slope of 1.13 takes a dy of 6e4 past its largest value, and a dy of 1e-6 has four bits left, which dz would lose.
// So dz is kept times a power of two that brings the largest |dy| to 2^13 .. 2^14, and the products' results are given the inverse: powers of two
// are exact, so no other result changes.  (bfloat16 has the exponents of 32 bits; relu's slopes are 0 and 1, dz is a dy then.)  The largest value is
// looked for in a pass of its own (3001 x 1500 in 16 bits: 7 us of a backward pass of 75; 8192 x 16384: 71 of 1930).  Here its parts: a wave takes every so-many-th row, a lane V consecutive columns; rows of no
// expert and values that are not finite do not count.
template <int V>
__global__ __launch_bounds__(256) void top_kernel(const SlopeArgs g)
{
    __shared__ float tops[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int first = 0, end = g.rows;
    if (g.experts) {
        first = min(max(g.offsets[0], 0), g.rows);
        end = min(max(g.offsets[g.experts], 0), g.rows);
    }
    float top = 0.0f;
    for (int n = (blockIdx.y * 64 + lane) * V; n < g.N; n += gridDim.y * 64 * V) {
#pragma unroll 4
        for (int m = first + blockIdx.x * 4 + wave; m < end; m += gridDim.x * 4) {
            float d[V];
            load_row<f16>(g.dy, (int64_t)m * g.lddy + n, g.N - n, V > 1, d);
#pragma unroll
            for (int j = 0; j < V; ++j) top = fabsf(d[j]) < INFINITY ? fmaxf(top, fabsf(d[j])) : top;
        }
    }
#pragma unroll
    for (int off = 32; off; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    if (threadIdx.x == 0) g.tops[blockIdx.y * gridDim.x + blockIdx.x] = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
}

// The power of two that dz is multiplied with, found by a workgroup from the parts' largest values.
__device__ __forceinline__ float factor_of(const float *parts, int count)
{
    __shared__ float tops[4];
    float top = 0.0f;
    for (int k = threadIdx.x; k < count; k += 256) top = fmaxf(top, parts[k]);
#pragma unroll
    for (int off = 32; off; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    int e = 14;
    if (top > 0.0f) (void)frexpf(top, &e);
    return ldexpf(1.0f, 14 - e);
}

// A workgroup takes a slot of rows and 64 * V columns; a wave every fourth row, a lane V consecutive columns.  One pass: dy
// and z are read once, dz written once, and the sums of a slot go to `part`, to be added in the order of the slots.
template <class T, int V, bool HAS_Z>
__global__ __launch_bounds__(256) void slope_kernel(const SlopeArgs g)
{
    __shared__ float sums[4][64 * V];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = (blockIdx.y * 64 + lane) * V, cnt = g.N - n;
    int first = blockIdx.x * g.slot_rows, end = min(first + g.slot_rows, g.rows);
    bool skip = false;
    if (g.experts) {
        const Slot s = find_slot(g.offsets, g.experts, g.rows, g.slot_rows, blockIdx.x);
        first = s.first;
        end = s.end;
        skip = s.expert < 0 || s.expert >= g.experts;      // rows of no expert: their dz is read by nobody
    }
    float by = 1.0f;
    if constexpr (std::is_same_v<T, f16> && HAS_Z) {
        if (g.tops) {
            by = factor_of(g.tops, g.top_count);
            if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *g.scale = 1.0f / by;
        }
    }
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.0f;
    if (!skip && n < (g.dz ? (int)g.ldd : g.N)) {
#pragma unroll 4
        for (int m = first + wave; m < end; m += 4) {
            float d[V];
            load_row<T>(g.dy, (int64_t)m * g.lddy + n, cnt, V > 1, d);
            if (HAS_Z) {
                float z[V];
                load_row<T>(g.z, (int64_t)m * g.ldz + n, cnt, V > 1, z);
#pragma unroll
                for (int j = 0; j < V; ++j) d[j] *= slope_of<T>(z[j], g.act);
                if (g.dz) {                                                           // (behind N: zeros)
                    float kept[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) kept[j] = d[j] * by;
                    store_row<T>(g.dz, (int64_t)m * g.ldd + n, V, 1, kept);
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += d[j];
        }
    }
    if (!g.part) return;
#pragma unroll
    for (int j = 0; j < V; ++j) sums[wave][j * 64 + lane] = sum[j];
    __syncthreads();
    for (int c = threadIdx.x; c < 64 * V; c += 256) {
        const int col = blockIdx.y * 64 * V + c;
        if (col >= g.N) continue;
        const int at = (c % V) * 64 + c / V;
        g.part[(int64_t)blockIdx.x * g.N + col] = (sums[0][at] + sums[1][at]) + (sums[2][at] + sums[3][at]);
    }
}

template <class T, int V>
hipError_t slope_wide(hipStream_t st, const SlopeArgs &g)
{
    const int per = 64 * V, columns = g.dz ? (int)g.ldd : g.N;
    const dim3 grid((unsigned)g.slots, (unsigned)((columns + per - 1) / per));
    if (g.act) slope_kernel<T, V, true><<<grid, 256, 0, st>>>(g);
    else slope_kernel<T, V, false><<<grid, 256, 0, st>>>(g);
    return hipGetLastError();
}

// TOP_PARTS workgroups at most, each with four rows and more
dim3 top_grid(const SlopeArgs &g)
{
    const int per = 64 * (g.bytes ? g.bytes / 2 : 1), columns = std::min((g.N + per - 1) / per, TOP_PARTS);
    return dim3((unsigned)std::min((g.rows + 15) / 16, TOP_PARTS / columns), (unsigned)columns);
}

hipError_t launch_top(hipStream_t st, const SlopeArgs &g)
{
    const dim3 grid = top_grid(g);
    if (g.bytes == 16) top_kernel<8><<<grid, 256, 0, st>>>(g);
    else if (g.bytes == 8) top_kernel<4><<<grid, 256, 0, st>>>(g);
    else top_kernel<1><<<grid, 256, 0, st>>>(g);
    return hipGetLastError();
}

// (3001 x 1500 in 16 bits, rows aligned to 8 bytes: 12.4 us by 8 bytes, 18 by elements)
template <class T>
hipError_t slope_typed(hipStream_t st, const SlopeArgs &g)
{
    return g.bytes == 16 ? slope_wide<T, 16 / sizeof(T)>(st, g) : g.bytes == 8 ? slope_wide<T, 8 / sizeof(T)>(st, g) : slope_wide<T, 1>(st, g);
}

hipError_t launch_slope(hipStream_t st, int dtype, const SlopeArgs &args)
{
    SlopeArgs g = args;
    if (g.tops) {
        const dim3 grid = top_grid(g);
        g.top_count = (int)(grid.x * grid.y);
        const hipError_t e = launch_top(st, g);
        if (e != hipSuccess) return e;
    }
    return dtype == 0 ? slope_typed<float>(st, g) : dtype == 1 ? slope_typed<f16>(st, g) : slope_typed<bf16>(st, g);
}

// Sixty-four columns a workgroup, four waves each adding a quarter of the expert's slots; the quarters are joined in their order.
template <class T>
__global__ __launch_bounds__(256) void bias_sum_kernel(const float *part, T *dbias, int rows, int N, int slots, int slot_rows, int experts,
                                                       const int32_t *offsets)
{
    __shared__ float sums[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.y;
    int first = 0, count = slots;
    if (experts) {
        int a, b;
        group_rows(offsets, experts, rows, e, a, b);
        first = slots_before(offsets, experts, rows, slot_rows, e);
        count = min((b - a + slot_rows - 1) / slot_rows, max(slots - first, 0));
    }
    const int n = blockIdx.x * 64 + lane, quarter = (count + 3) / 4;
    float sum = 0.0f;
    if (n < N) {
#pragma unroll 8
        for (int s = wave * quarter; s < min((wave + 1) * quarter, count); ++s) sum += part[(int64_t)(first + s) * N + n];
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && n < N) dbias[(int64_t)e * N + n] = (T)((sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]));
}

hipError_t launch_bias_sum(hipStream_t st, int dtype, const float *part, char *dbias, int rows, int N, int slots, int slot_rows, int experts,
                           const int32_t *offsets)
{
    const dim3 grid((unsigned)((N + 63) / 64), (unsigned)(experts ? experts : 1));
    if (dtype == 0) bias_sum_kernel<float><<<grid, 256, 0, st>>>(part, (float *)dbias, rows, N, slots, slot_rows, experts, offsets);
    else if (dtype == 1) bias_sum_kernel<f16><<<grid, 256, 0, st>>>(part, (f16 *)dbias, rows, N, slots, slot_rows, experts, offsets);
    else bias_sum_kernel<bf16><<<grid, 256, 0, st>>>(part, (bf16 *)dbias, rows, N, slots, slot_rows, experts, offsets);
    return hipGetLastError();
}

// ---------------------------------------------------------------- join of a split product

// Four columns a thread; the splits are added in their order.
template <class T, int EPI>
__global__ __launch_bounds__(256) void join_kernel(const ProductArgs g)
{
    const int per_row = (g.N + 3) / 4;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = t / per_row;
    if (m >= g.M) return;
    const int n = (int)(t - m * per_row) * 4, cnt = g.N - n, aligned = (g.N & 3) == 0;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < g.splits; ++s) {
        float part[4];
        load_row<float>((const char *)g.sum, ((int64_t)s * g.M + m) * g.N + n, cnt, aligned, part);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += part[j];
    }
    if (g.total) {
        if (!g.first) {
            float old[4];
            load_row<float>((const char *)g.total, m * g.N + n, cnt, aligned, old);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += old[j];
        }
        if (!g.last) {
            store_row<float>((char *)g.total, m * g.N + n, cnt, aligned, v);
            return;
        }
    }
    const float scale = g.scale ? *g.scale : 1.0f;
    if (EPI == EPI_LINE) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= scale;
    }
    float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (g.bias) load_row<T>(g.bias, n, cnt, g.wide, bias);
    put_row<T, EPI>(g, 0, bias, m, n, cnt, g.wide, false, v);
}

template <class T>
hipError_t join_typed(hipStream_t st, Epilogue epi, const ProductArgs &g)
{
    const int64_t threads = (int64_t)g.M * ((g.N + 3) / 4);
    const unsigned blocks = (unsigned)((threads + 255) / 256);
    if (epi == EPI_SIGMOID) join_kernel<T, EPI_SIGMOID><<<blocks, 256, 0, st>>>(g);
    else if (epi == EPI_ERF) join_kernel<T, EPI_ERF><<<blocks, 256, 0, st>>>(g);
    else join_kernel<T, EPI_LINE><<<blocks, 256, 0, st>>>(g);
    return hipGetLastError();
}

hipError_t launch_join(hipStream_t st, int dtype, Epilogue epi, const ProductArgs &g)
{
    return dtype == 0 ? join_typed<float>(st, epi, g) : dtype == 1 ? join_typed<f16>(st, epi, g) : join_typed<bf16>(st, epi, g);
}

// ---------------------------------------------------------------- the loss's statistics

// (top, sum of exp(l - top)) of two sets of logits; of none: (-inf, 0)
__device__ __forceinline__ float2 join_stat(float2 a, float2 b)
{
    const float top = fmaxf(a.x, b.x), ref = top == -INFINITY ? 0.0f : top;
    return make_float2(top, a.y * expf(a.x - ref) + b.y * expf(b.x - ref));
}

// Sixteen rows at a time; sixty-four threads a row take every sixty-fourth stripe, in order, and are joined in order by eights.
constexpr int LOSS_GROUPS = 1 << 21;               // (a grid's threads are counted in 32 bits)

__global__ __launch_bounds__(1024) void loss_kernel(const float2 *stat, int stripes, int rows, const float *at_target,
                                                    const int64_t *target, int64_t words, float *loss, float *lse)
{
    __shared__ float2 share[64][17], eights[8][17];
    const int r = threadIdx.x & 15, part = threadIdx.x >> 4;
    for (int first = blockIdx.x * 16; first < rows; first += gridDim.x * 16) {
        const int m = first + r;
        float2 s = make_float2(-INFINITY, 0.0f);
        if (m < rows) {
#pragma unroll 4
            for (int j = part; j < stripes; j += 64) s = join_stat(s, stat[(int64_t)j * rows + m]);
        }
        __syncthreads();                           // (the rows before have been joined)
        share[part][r] = s;
        __syncthreads();
        if (part < 8) {
            s = share[part * 8][r];
            for (int j = 1; j < 8; ++j) s = join_stat(s, share[part * 8 + j][r]);
            eights[part][r] = s;
        }
        __syncthreads();
        if (part != 0 || m >= rows) continue;
        for (int j = 1; j < 8; ++j) s = join_stat(s, eights[j][r]);
        const float l = s.x + logf(s.y);
        const int64_t word = target[m];
        lse[m] = l;
        loss[m] = word < 0 ? 0.0f : word >= words ? NAN : l - at_target[m];
    }
}

hipError_t launch_loss(hipStream_t st, const float2 *stat, int stripes, int rows, const float *at_target, const int64_t *target,
                       int64_t words, float *loss, float *lse)
{
    loss_kernel<<<(unsigned)std::min((rows + 15) / 16, LOSS_GROUPS), 1024, 0, st>>>(stat, stripes, rows, at_target, target, words, loss, lse);
    return hipGetLastError();
}

// One workgroup.  The largest |dloss| of a counted row becomes 2^14: |g| is no larger, so it fits in a 16-bit float, and a probability of
// 2^-28 beside it is still a normal one.  The divisor is that largest value itself and no power of two near it: rows mostly have one weight,
// the mean's, and what they add at their target, (1 - p) times it with small p, would be rounded the same way in all of them (measured
// with 8192 rows: errors of the gradients 0.0035 relative with a power of two, 0.0017 being the least a 16-bit result can have).
__global__ __launch_bounds__(1024) void coef_kernel(const float *dloss, const int64_t *target, int64_t words, int rows, float *coef,
                                                    float *scale)
{
    __shared__ float tops[16];
    float top = 0.0f;
    for (int m = threadIdx.x; m < rows; m += 1024) {
        const float d = fabsf(dloss[m]);
        if (target[m] >= 0 && d < INFINITY) top = fmaxf(top, d);
    }
#pragma unroll
    for (int off = 32; off; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = tops[0];
    for (int j = 1; j < 16; ++j) top = fmaxf(top, tops[j]);
    const float most = top > 0.0f ? fmaxf(top, 0x1p-100f) : 16384.0f, by = 16384.0f / most;
    if (threadIdx.x == 0) *scale = most * 0x1p-14f;
    for (int m = threadIdx.x; m < rows; m += 1024)
        coef[m] = target[m] < 0 ? 0.0f : target[m] >= words ? NAN : dloss[m] * by;
}

hipError_t launch_coef(hipStream_t st, const float *dloss, const int64_t *target, int64_t words, int rows, float *coef, float *scale)
{
    coef_kernel<<<1, 1024, 0, st>>>(dloss, target, words, rows, coef, scale);
    return hipGetLastError();
}

}  // namespace alpa
