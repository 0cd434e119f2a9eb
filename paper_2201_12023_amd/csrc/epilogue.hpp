// Elements, activations, and what becomes of a product's results (device code).
#pragma once
#include "layers.hpp"
#include "product.hpp"

namespace alpa {

// N consecutive elements as floats; `wide`: they are aligned to 16 bytes, or to their size if that is less; `n`: how many exist
template <class T, int N>
__device__ __forceinline__ void load_row(const char *base, int64_t at, int n, int wide, float (&v)[N])
{
    const T *p = (const T *)base + at;
    if (wide && n >= N) {
        struct __align__(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack { T e[N]; };
        const Pack k = *(const Pack *)p;
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = (float)k.e[j];
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = j < n ? (float)p[j] : 0.0f;
    }
}

// the one rounding of a result to its type (to nearest, ties to even)
template <class T, int N>
__device__ __forceinline__ void store_row(char *base, int64_t at, int n, int wide, const float (&v)[N])
{
    T *p = (T *)base + at;
    if (wide && n >= N) {
        struct __align__(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack { T e[N]; };
        Pack k;
#pragma unroll
        for (int j = 0; j < N; ++j) k.e[j] = (T)v[j];
        *(Pack *)p = k;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < n) p[j] = (T)v[j];
    }
}

// exp for values that end in 32 bits, and the faster one (its error grows with the exponent: 2^-24 |x|) for those rounded to 16
template <class T>
__device__ __forceinline__ float exp_for(float x)
{
    return sizeof(T) == 4 ? expf(x) : __expf(x);
}

// n / d: correctly rounded for values that end in 32 bits, within two units in the last place for those rounded to 16
template <class T>
__device__ __forceinline__ float divide_for(float n, float d)
{
    return sizeof(T) == 4 ? n / d : n * __builtin_amdgcn_rcpf(d);
}

// z * logistic(z (c1 + c3 z^2)).  An infinite z is given the limit: the formula would have inf / inf or 0 * inf there.
template <class T>
__device__ __forceinline__ float gated(float z, float c1, float c3)
{
    const float y = divide_for<T>(z, 1.0f + exp_for<T>(-z * (c1 + c3 * z * z)));
    return fabsf(z) == INFINITY ? (z > 0.0f ? z : -0.0f) : y;
}

// The normal distribution's integral up to z; e = exp(-z^2 / 2).  For values rounded to 16 bits erfc(x) = exp(-x^2) t P(t), t = 1 / (1 + 0.46 x), x >= 0,
// P of least relative error in its class (7e-7, fitted here): an eighth of erfcf's instructions and one exponential for it and the slope.  Either
// way very negative z keep their relative error.
template <class T>
__device__ __forceinline__ float normal_integral(float z, float e)
{
    if (sizeof(T) == 4) return 0.5f * erfcf(-0.70710678118654752f * z);
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.46f * 0.70710678118654752f, 1.0f));
    float p = 0.06771395355463028f;
    p = fmaf(p, t, -0.22664865851402283f);
    p = fmaf(p, t, 0.16924932599067688f);
    p = fmaf(p, t, 0.05254606902599335f);
    p = fmaf(p, t, 0.18688102066516876f);
    p = fmaf(p, t, 0.23117370903491974f);
    p = fmaf(p, t, 0.25955814123153687f);
    p = fmaf(p, t, 0.2595270276069641f);
    const float below = 0.5f * e * t * p;
    return z < 0.0f ? below : 1.0f - below;
}

template <class T>
__device__ __forceinline__ float gelu(float z)
{
    const float y = z * normal_integral<T>(z, exp_for<T>(-0.5f * z * z));
    return z == -INFINITY ? -0.0f : y;
}

template <class T, int EPI>
__device__ __forceinline__ float activate(float z, const ProductArgs &g)
{
    if (EPI == EPI_SIGMOID) return gated<T>(z, g.c1, g.c3);
    if (EPI == EPI_ERF) return gelu<T>(z);
    return z < g.low ? g.low : z;              // (a NaN stays)
}

// Columns n .. n + N - 1 of row m, `cnt` of them real: z = v + bias, result act(z) (+ residual).  `skip`: a row of no expert, zeros.
template <class T, int EPI, int N>
__device__ __forceinline__ void put_row(const ProductArgs &g, int64_t out_base, const float (&bias)[N], int64_t m, int n, int cnt, int wide,
                                        bool skip, float (&v)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] += bias[j];
    if (g.z) store_row<T>(g.z, m * g.ldz + n, cnt, wide, v);
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = activate<T, EPI>(v[j], g);
    if (g.residual && !skip) {
        float r[N];
        load_row<T>(g.residual, m * g.ldr + n, cnt, wide, r);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] += r[j];
    }
    store_row<T>(g.out, out_base + m * g.ldo + n, cnt, wide, v);
}

}  // namespace alpa
