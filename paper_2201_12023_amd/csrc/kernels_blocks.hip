// The kernels between a block's products beside attention itself: copies to aligned memory, rotary positions, layer norm.
#include "blocks.hpp"
#include "epilogue.hpp"

namespace alpa {

template <class Call>
hipError_t by_type(int dtype, Call call)
{
    if (dtype == 0) call(float{});
    else if (dtype == 1) call(f16{});
    else call(bf16{});
    return hipGetLastError();
}

// (a grid's threads are counted in 32 bits)
unsigned blocks_for(int64_t work, int64_t most) { return (unsigned)std::max<int64_t>(std::min(work, most), 1); }

// ---------------------------------------------------------------- heads in 16-byte units

// A thread writes sixteen bytes; all of a call's tensors in one launch.
template <class T>
__global__ __launch_bounds__(256) void head_pack_kernel(const HeadPack g)
{
    constexpr int V = 16 / sizeof(T);
    const auto &t = g.t[blockIdx.y];
    const int per = g.to_len / V;
    const int64_t total = t.rows * t.heads * per;
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < total; c += (int64_t)gridDim.x * 256) {
        const int64_t item = c / per, row = item / t.heads;
        const int n = (int)(c - item * per) * V;
        float v[V];
        load_row<T>(t.from, row * t.row + (item - row * t.heads) * t.head + n, g.len - n, 0, v);
        store_row<T>(t.to, item * g.to_len + n, V, 1, v);
    }
}

hipError_t launch_head_pack(hipStream_t st, int dtype, const HeadPack &g)
{
    int64_t chunks = 0;
    for (int k = 0; k < g.count; ++k) chunks = std::max(chunks, g.t[k].rows * g.t[k].heads * (g.to_len * (dtype == 0 ? 4 : 2) / 16));
    const dim3 grid(blocks_for((chunks + 255) / 256, 8192), (unsigned)g.count);
    return by_type(dtype, [&](auto t) { head_pack_kernel<decltype(t)><<<grid, 256, 0, st>>>(g); });
}

// ---------------------------------------------------------------- rotary positions

// A workgroup takes `per` rows: their sines and cosines once, for all heads, then the heads.  The angle is counted in turns in 64 bits, where a position of
// 2^40 still leaves 13 bits behind the point; what is left of it after whole turns is exact enough in 32 for results of 16 bits.
template <class T, int V>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs g, int per)
{
    extern __shared__ float2 turns[];                              // [per][rot / 2] (cos, sin)
    const int half = g.rot / 2;
    // a unit: V pairs of a head (their two halves, or 2 V elements that follow each other), or 2 V elements behind rot
    const int turned = (half + V - 1) / V, units = turned + (g.copy ? (g.dim - g.rot + 2 * V - 1) / (2 * V) : 0);
    for (int64_t row0 = (int64_t)blockIdx.x * per; row0 < g.rows; row0 += (int64_t)gridDim.x * per) {
        const int rows = (int)min((int64_t)per, g.rows - row0);
        __syncthreads();                                               // (the rows before are done with)
        for (int c = threadIdx.x; c < rows * half; c += 256) {
            const int r = c / half;
            const double u = (double)g.positions[row0 + r] * g.frequencies[c - r * half] * 0.15915494309189533577;
            const double part = u - rint(u);
            const float near = (float)part;
            float sin, cos;
            sincospif(2.0f * near, &sin, &cos);
            if constexpr (sizeof(T) == 4) {
                // (what 32 bits of the turn leave out, up to 9e-8 of a radian: the rest of a sine of float32 is off by less)
                const float rest = 6.2831853071795865f * (float)(part - near), c = cos;
                cos = fmaf(-sin, rest, cos);
                sin = fmaf(c, rest, sin);
            }
            turns[c] = make_float2(cos * g.scale, sin * g.scale * g.sign);
        }
        __syncthreads();
        for (int c = threadIdx.x + blockIdx.y * 256; c < rows * g.heads * units; c += 256 * gridDim.y) {
            const int item = c / units, unit = c - item * units, r = item / g.heads, head = item - r * g.heads;
            const char *x = g.x.p + ((row0 + r) * g.x.row + head * g.x.head) * (int64_t)sizeof(T);
            char *y = g.y.p + ((row0 + r) * g.y.row + head * g.y.head) * (int64_t)sizeof(T);
            float a[V], b[V];
            if (unit >= turned) {
                const int d = g.rot + (unit - turned) * 2 * V;
                load_row<T>(x, d, g.dim - d, g.wide, a);
                load_row<T>(x, d + V, g.dim - d - V, g.wide, b);
                store_row<T>(y, d, g.dim - d, g.wide, a);
                store_row<T>(y, d + V, g.dim - d - V, g.wide, b);
                continue;
            }
            const int t = unit * V, cnt = half - t;
            const float2 *u = turns + r * half + t;
            if (g.interleaved) {
                load_row<T>(x, 2 * t, 2 * cnt, g.wide, a);
                load_row<T>(x, 2 * t + V, 2 * cnt - V, g.wide, b);
                float p[2 * V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    p[j] = a[j];
                    p[V + j] = b[j];
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float2 w = j < cnt ? u[j] : make_float2(0.0f, 0.0f);
                    const float m = p[2 * j], n = p[2 * j + 1];
                    p[2 * j] = m * w.x - n * w.y;
                    p[2 * j + 1] = m * w.y + n * w.x;
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    a[j] = p[j];
                    b[j] = p[V + j];
                }
                store_row<T>(y, 2 * t, 2 * cnt, g.wide, a);
                store_row<T>(y, 2 * t + V, 2 * cnt - V, g.wide, b);
            } else {
                load_row<T>(x, t, cnt, g.wide, a);
                load_row<T>(x, half + t, cnt, g.wide, b);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float2 w = j < cnt ? u[j] : make_float2(0.0f, 0.0f);
                    const float m = a[j], n = b[j];
                    a[j] = m * w.x - n * w.y;
                    b[j] = m * w.y + n * w.x;
                }
                store_row<T>(y, t, cnt, g.wide, a);
                store_row<T>(y, half + t, cnt, g.wide, b);
            }
        }
    }
}

hipError_t launch_rotary(hipStream_t st, int dtype, const RotaryArgs &g)
{
    // (a workgroup's units are counted in 32 bits)
    const int half = g.rot / 2, per = (int)std::max<int64_t>(1, std::min<int64_t>(256 / half, (1 << 24) / ((int64_t)g.heads * g.dim)));
    const int64_t groups = (g.rows + per - 1) / per;
    const int64_t work = (int64_t)per * g.heads * ((g.dim + 15) / 16);
    const dim3 grid(blocks_for(groups, 1 << 20), groups < 512 ? blocks_for(work / 256, 8) : 1);
    const size_t bytes = (size_t)per * half * sizeof(float2);
    return by_type(dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int ES = sizeof(T);
        if (g.wide == 16) rotary_kernel<T, 16 / ES><<<grid, 256, bytes, st>>>(g, per);
        else if (g.wide == 8) rotary_kernel<T, 8 / ES><<<grid, 256, bytes, st>>>(g, per);
        else rotary_kernel<T, 1><<<grid, 256, bytes, st>>>(g, per);
    });
}

// ---------------------------------------------------------------- layer norm

// Sums over the threads of a row: a wave, or several.  `lds`: a float for each wave of the workgroup and each of N, not those of the sums before.
template <int THREADS, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float *lds)
{
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int off = 32; off; off >>= 1) v[k] += __shfl_xor(v[k], off, 64);
    if constexpr (THREADS > 64) {
        constexpr int WAVES = THREADS / 64;
        lds += threadIdx.x / THREADS * (WAVES * N);
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) lds[k * WAVES + (threadIdx.x % THREADS >> 6)] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v[k] += lds[k * WAVES + w];
        }
    }
}

// A row's elements as THREADS threads hold them, C times V each, as they were read, so that a row can be under way while another one is worked on.
// WIDE: V at once.
template <class T, int THREADS, int C, bool WIDE>
struct RowOf {
    static constexpr int V = 16 / sizeof(T), N = C * V;
    u32x4 raw[WIDE ? C : 1];
    T one[WIDE ? 1 : N];

    static __device__ __forceinline__ int column(int c, int j, int t) { return WIDE ? (c * THREADS + t) * V + j : (c * V + j) * THREADS + t; }
    __device__ __forceinline__ void load(const char *p, int n, int t)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (WIDE) {
                const int at = column(c, 0, t);
                raw[c] = u32x4{0, 0, 0, 0};
                if (at < n) raw[c] = *(const u32x4 *)((const T *)p + at);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int at = column(c, j, t);
                    one[c * V + j] = at < n ? ((const T *)p)[at] : (T)0.0f;
                }
            }
        }
    }
    __device__ __forceinline__ void values(float (&v)[N]) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            T e[V];
            if constexpr (WIDE) __builtin_memcpy(e, &raw[c], 16);
#pragma unroll
            for (int j = 0; j < V; ++j) v[c * V + j] = (float)(WIDE ? e[j] : one[WIDE ? 0 : c * V + j]);
        }
    }
    static __device__ __forceinline__ void store(char *p, int n, int t, const float (&v)[N])
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (WIDE) {
                float e[V];
                const int at = column(c, 0, t);
#pragma unroll
                for (int j = 0; j < V; ++j) e[j] = v[c * V + j];
                if (at < n) store_row<T>(p, at, V, 1, e);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int at = column(c, j, t);
                    if (at < n) ((T *)p)[at] = (T)v[c * V + j];
                }
            }
        }
    }
};

// Rows one after the other, the next one under way; weight and bias stay in registers.  The variance is summed from the differences to the mean, which is known
// by then, as the row is in registers.  Memory bounds it: 8192 rows of 4096 in 16 bits 24 us with
// inputs in the caches behind the L2s, 36 with one row a workgroup.
template <class T, int THREADS, int C, bool WIDE>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_kernel(const NormArgs g)
{
    using R = RowOf<T, THREADS, C, WIDE>;
    constexpr int AT_ONCE = THREADS < 256 ? 256 / THREADS : 1;
    __shared__ float lds[2][16];
    const int t = threadIdx.x % THREADS;
    const int64_t apart = (int64_t)gridDim.x * AT_ONCE;
    int64_t row = (int64_t)blockIdx.x * AT_ONCE + threadIdx.x / THREADS;
    if (row >= g.rows) return;                                     // (whole waves, where a wave has a row)
    R next, weight, bias;
    next.load(g.x + row * g.ldx * (int64_t)sizeof(T), g.n, t);
    if (g.weight) weight.load(g.weight, g.n, t);
    if (g.bias) bias.load(g.bias, g.n, t);
    for (; row < g.rows; row += apart) {
        float x[R::N];
        next.values(x);
        if (row + apart < g.rows) next.load(g.x + (row + apart) * g.ldx * (int64_t)sizeof(T), g.n, t);
        float sum[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < R::N; ++j) sum[0] += x[j];
        row_sums<THREADS>(sum, lds[0]);
        const float mean = sum[0] / (float)g.n;
        sum[0] = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < R::V; ++j) {
                const float d = R::column(c, j, t) < g.n ? x[c * R::V + j] - mean : 0.0f;
                x[c * R::V + j] = d;
                sum[0] += d * d;
            }
        row_sums<THREADS>(sum, lds[1]);
        const float rstd = 1.0f / sqrtf(sum[0] / (float)g.n + g.eps);
        float v[R::N];
#pragma unroll
        for (int j = 0; j < R::N; ++j) x[j] *= rstd;
        if (g.weight) {
            weight.values(v);
#pragma unroll
            for (int j = 0; j < R::N; ++j) x[j] *= v[j];
        }
        if (g.bias) {
            bias.values(v);
#pragma unroll
            for (int j = 0; j < R::N; ++j) x[j] += v[j];
        }
        R::store(g.y + row * g.ldy * (int64_t)sizeof(T), g.n, t, x);
        if (g.mean && t == 0) {
            g.mean[row] = mean;
            g.rstd[row] = rstd;
        }
    }
}

// Rows that the registers do not hold are read three times, from the caches.
template <class T>
__global__ __launch_bounds__(1024) void norm_long_kernel(const NormArgs g)
{
    __shared__ float lds[2][16];
    for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
        const T *x = (const T *)g.x + row * g.ldx;
        float sum[1] = {0.0f};
        for (int k = threadIdx.x; k < g.n; k += 1024) sum[0] += (float)x[k];
        row_sums<1024>(sum, lds[0]);
        const float mean = sum[0] / (float)g.n;
        sum[0] = 0.0f;
        for (int k = threadIdx.x; k < g.n; k += 1024) {
            const float d = (float)x[k] - mean;
            sum[0] += d * d;
        }
        row_sums<1024>(sum, lds[1]);
        const float rstd = 1.0f / sqrtf(sum[0] / (float)g.n + g.eps);
        T *y = (T *)g.y + row * g.ldy;
        for (int k = threadIdx.x; k < g.n; k += 1024) {
            float v = ((float)x[k] - mean) * rstd;
            if (g.weight) v *= (float)((const T *)g.weight)[k];
            if (g.bias) v += (float)((const T *)g.bias)[k];
            y[k] = (T)v;
        }
        if (g.mean && threadIdx.x == 0) {
            g.mean[row] = mean;
            g.rstd[row] = rstd;
        }
    }
}

// Rows that a workgroup of the backward pass works on at once.  (Two of 256 threads with four times 16 bytes each need more registers than there are.)
constexpr int rows_at_once(int threads, int c) { return threads == 64 ? 4 : threads == 256 && c <= 2 ? 2 : 1; }

// A workgroup's rows, some at once, the next ones under way: dx, and the sums for dweight and dbias in registers, as a thread has the same columns of all of
// them.  The rows' sums are joined through LDS, so that few parts go to memory: bound by memory, 8192 rows of 4096 in 16 bits take 38 us and 65536 of 768 59, and the
// sums of parts 5 (with a part to memory for each of the rows at once 57 and 105, those among them).
template <class T, int THREADS, int C, bool WIDE>
__global__ __launch_bounds__(THREADS * rows_at_once(THREADS, C)) void norm_backward_kernel(const NormArgs g)
{
    using R = RowOf<T, THREADS, C, WIDE>;
    constexpr int AT_ONCE = rows_at_once(THREADS, C);
    __shared__ float lds[2][32];
    __shared__ float joined[AT_ONCE > 1 ? (AT_ONCE - 1) * THREADS * R::N : 1];
    const int t = threadIdx.x % THREADS, sub = threadIdx.x / THREADS;
    const int64_t apart = (int64_t)g.groups * AT_ONCE, own = (int64_t)g.groups * sub;
    R next_x, next_dy, weight;
    float dw[R::N], db[R::N], next_mean = 0.0f, next_rstd = 0.0f;
    const auto ask = [&](int64_t row) {
        if (row >= g.rows) return;
        next_x.load(g.x + row * g.ldx * (int64_t)sizeof(T), g.n, t);
        next_dy.load(g.dy + row * g.lddy * (int64_t)sizeof(T), g.n, t);
        next_mean = g.mean[row];
        next_rstd = g.rstd[row];
    };
    ask(blockIdx.x + own);
    if (g.weight) weight.load(g.weight, g.n, t);
#pragma unroll
    for (int j = 0; j < R::N; ++j) dw[j] = db[j] = 0.0f;
    int turn = 0;
    for (int64_t at = blockIdx.x; at < g.rows; at += apart, turn ^= 1) {
        const int64_t row = at + own;
        const bool here = row < g.rows;                            // (the others only take part in the sums)
        float x[R::N], dy[R::N], w[R::N];
        float sum[2] = {0.0f, 0.0f};
        const float mean = next_mean, rstd = next_rstd;
        if (here) {
            next_x.values(x);
            next_dy.values(dy);
        }
        ask(row + apart);
        if (here) {
            if (g.weight) weight.values(w);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < R::V; ++j) {
                    const int k = c * R::V + j;
                    x[k] = R::column(c, j, t) < g.n ? (x[k] - mean) * rstd : 0.0f;
                    dw[k] += dy[k] * x[k];
                    db[k] += dy[k];
                    if (g.weight) dy[k] *= w[k];
                    sum[0] += dy[k];
                    sum[1] += dy[k] * x[k];
                }
        }
        if (!g.y) continue;
        row_sums<THREADS>(sum, lds[turn]);
        if (!here) continue;
        const float a = sum[0] / (float)g.n, b = sum[1] / (float)g.n;
#pragma unroll
        for (int k = 0; k < R::N; ++k) x[k] = rstd * (dy[k] - a - x[k] * b);
        R::store(g.y + row * g.ldy * (int64_t)sizeof(T), g.n, t, x);
    }
    const auto finish = [&](float (&v)[R::N], float *part) {
        if (!part) return;
        if constexpr (AT_ONCE > 1) {
            __syncthreads();                                       // (the other sums have been read)
            if (sub)
#pragma unroll
                for (int k = 0; k < R::N; ++k) joined[((sub - 1) * R::N + k) * THREADS + t] = v[k];
            __syncthreads();
            if (sub) return;
#pragma unroll
            for (int k = 0; k < R::N; ++k)
                for (int o = 0; o < AT_ONCE - 1; ++o) v[k] += joined[(o * R::N + k) * THREADS + t];
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (WIDE) {
                float e[R::V];
                const int at = R::column(c, 0, t);
#pragma unroll
                for (int j = 0; j < R::V; ++j) e[j] = v[c * R::V + j];
                if (at < g.n)
#pragma unroll
                    for (int j = 0; j < R::V; j += 4) *(f32x4 *)(part + (int64_t)blockIdx.x * g.n + at + j) = f32x4{e[j], e[j + 1], e[j + 2], e[j + 3]};
            } else {
#pragma unroll
                for (int j = 0; j < R::V; ++j) {
                    const int at = R::column(c, j, t);
                    if (at < g.n) part[(int64_t)blockIdx.x * g.n + at] = v[c * R::V + j];
                }
            }
        }
    };
    finish(dw, g.part_w);
    finish(db, g.part_b);
}

// Long rows: dx alone, and the sums by columns.
template <class T>
__global__ __launch_bounds__(1024) void norm_backward_long_kernel(const NormArgs g)
{
    __shared__ float lds[2][32];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x, turn ^= 1) {
        const T *x = (const T *)g.x + row * g.ldx, *dy = (const T *)g.dy + row * g.lddy, *w = (const T *)g.weight;
        const float mean = g.mean[row], rstd = g.rstd[row];
        float sum[2] = {0.0f, 0.0f};
        for (int k = threadIdx.x; k < g.n; k += 1024) {
            const float d = (float)dy[k] * (w ? (float)w[k] : 1.0f);
            sum[0] += d;
            sum[1] += d * ((float)x[k] - mean) * rstd;
        }
        row_sums<1024>(sum, lds[turn]);
        const float a = sum[0] / (float)g.n, b = sum[1] / (float)g.n;
        T *dx = (T *)g.y + row * g.ldy;
        for (int k = threadIdx.x; k < g.n; k += 1024) {
            const float d = (float)dy[k] * (w ? (float)w[k] : 1.0f);
            dx[k] = (T)(rstd * (d - a - ((float)x[k] - mean) * rstd * b));
        }
    }
}
template <class T>
__global__ __launch_bounds__(256) void norm_columns_kernel(const NormArgs g)
{
    const int k = blockIdx.x * 256 + threadIdx.x;
    if (k >= g.n) return;
    float dw = 0.0f, db = 0.0f;
#pragma unroll 4
    for (int64_t row = blockIdx.y; row < g.rows; row += g.groups) {
        const float d = (float)((const T *)g.dy)[row * g.lddy + k];
        db += d;
        dw += d * (((float)((const T *)g.x)[row * g.ldx + k] - g.mean[row]) * g.rstd[row]);
    }
    if (g.part_w) g.part_w[(int64_t)blockIdx.y * g.n + k] = dw;
    if (g.part_b) g.part_b[(int64_t)blockIdx.y * g.n + k] = db;
}

// Sixty-four columns a workgroup, sixteen waves each adding a sixteenth of the groups; these are joined in their order.
template <class T>
__global__ __launch_bounds__(1024) void norm_sum_kernel(const NormArgs g)
{
    __shared__ float sums[16][64];
    const float *part = blockIdx.y ? g.part_b : g.part_w;
    char *out = blockIdx.y ? g.dbias : g.dweight;
    if (!out) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = blockIdx.x * 64 + lane, share = (g.groups + 15) / 16;
    float sum = 0.0f;
    if (n < g.n) {
#pragma unroll 8
        for (int k = wave * share; k < min(wave * share + share, g.groups); ++k) sum += part[(int64_t)k * g.n + n];
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || n >= g.n) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += sums[w][lane];
    ((T *)out)[n] = (T)sum;
}

// Threads of a row and elements of each: as few threads as hold it, sixteen bytes to eight times that each.  (v: elements of 16 bytes)
// MOST: elements of a thread at most, where a row has 1024.
template <class T, int MOST, class Call>
bool with_shape(int n, Call call)
{
    constexpr int V = 16 / sizeof(T);
    using std::integral_constant;
    const auto try_one = [&](auto threads, auto c) {
        if constexpr (threads() == 1024 && c() * V > MOST) return false;
        else {
            if (n > threads() * c() * V) return false;
            call(threads, c);
            return true;
        }
    };
    return try_one(integral_constant<int, 64>{}, integral_constant<int, 1>{}) || try_one(integral_constant<int, 64>{}, integral_constant<int, 2>{}) ||
           try_one(integral_constant<int, 256>{}, integral_constant<int, 1>{}) || try_one(integral_constant<int, 256>{}, integral_constant<int, 2>{}) ||
           try_one(integral_constant<int, 256>{}, integral_constant<int, 4>{}) || try_one(integral_constant<int, 1024>{}, integral_constant<int, 2>{}) ||
           try_one(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

hipError_t launch_norm(hipStream_t st, int dtype, const NormArgs &g)
{
    return by_type(dtype, [&](auto type) {
        using T = decltype(type);
        const bool done = with_shape<T, 16>(g.n, [&](auto threads, auto c) {
            constexpr int THREADS = threads(), AT_ONCE = THREADS < 256 ? 256 / THREADS : 1;
            const unsigned blocks = blocks_for((g.rows + AT_ONCE - 1) / AT_ONCE, THREADS == 1024 ? 512 : 2048);
            if (g.wide) norm_kernel<T, THREADS, c(), true><<<blocks, THREADS * AT_ONCE, 0, st>>>(g);
            else norm_kernel<T, THREADS, c(), false><<<blocks, THREADS * AT_ONCE, 0, st>>>(g);
        });
        if (!done) norm_long_kernel<T><<<blocks_for(g.rows, 1 << 20), 1024, 0, st>>>(g);
    });
}

int norm_groups(int64_t rows) { return (int)std::min<int64_t>(std::max<int64_t>(rows, 1), 512); }

hipError_t launch_norm_backward(hipStream_t st, int dtype, const NormArgs &g)
{
    return by_type(dtype, [&](auto type) {
        using T = decltype(type);
        const bool done = with_shape<T, sizeof(T) == 4 ? 8 : 16>(g.n, [&](auto threads, auto c) {
            constexpr int THREADS = threads();
            if (g.wide) norm_backward_kernel<T, THREADS, c(), true><<<(unsigned)g.groups, THREADS * rows_at_once(THREADS, c()), 0, st>>>(g);
            else norm_backward_kernel<T, THREADS, c(), false><<<(unsigned)g.groups, THREADS * rows_at_once(THREADS, c()), 0, st>>>(g);
        });
        if (!done) {
            if (g.y) norm_backward_long_kernel<T><<<blocks_for(g.rows, 1 << 20), 1024, 0, st>>>(g);
            if (g.part_w || g.part_b) norm_columns_kernel<T><<<dim3((unsigned)((g.n + 255) / 256), (unsigned)g.groups), 256, 0, st>>>(g);
        }
        if (g.part_w || g.part_b) norm_sum_kernel<T><<<dim3((unsigned)((g.n + 63) / 64), 2), 1024, 0, st>>>(g);
    });
}

}  // namespace alpa
