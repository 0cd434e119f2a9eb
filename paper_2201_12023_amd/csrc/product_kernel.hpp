// The tiled product with its epilogues, instantiated per element type (kernels_product_*.hip).
#pragma once
#include "epilogue.hpp"
#include "slots.hpp"

namespace alpa {

// Place of a workgroup among the tiles.  Workgroups are dealt to the eight XCDs in turn; each XCD gets a run of consecutive places, and places
// go through bands of eight row tiles, so that what an XCD works on at one time shares its operands' tiles in its L2.
__device__ __forceinline__ int xcd_place(int block, int total)
{
    const int x = block & 7, per = total >> 3, rem = total & 7;
    return x * per + min(x, rem) + (block >> 3);
}
__device__ __forceinline__ void tile_at(int place, int row_tiles, int col_tiles, int &tm, int &tn)
{
    constexpr int BAND = 8;
    const int band = place / (BAND * col_tiles), first = band * BAND, rows = min(BAND, row_tiles - first);
    const int in = place - band * BAND * col_tiles;
    tm = first + in % rows;
    tn = in / rows;
}

// Statistics of a wave's columns, by stripes: a lane has four rows' worth of blocks of one row, the four lanes of a row are joined.
template <class T, class P, int SPAN>
__device__ __forceinline__ void loss_stripes(const ProductArgs &g, const typename P::Acc &acc, int m_first, int m_end, int n_first, int i, int q)
{
    constexpr int CW = P::TB::PAIRED ? 8 : 4, PER = SPAN / STRIPE, IN = P::NTL * 4 / CW / PER;
    static_assert(SPAN % STRIPE == 0, "stripes do not lie in waves");
#pragma unroll
    for (int a = 0; a < P::MT; ++a) {
        // every lane of the wave takes part; rows behind the last one are not written
        const int m = m_first + P::TA::row_of(i, a);
        const int64_t word = m < m_end ? g.target[m] : -1;
#pragma unroll
        for (int s = 0; s < PER; ++s) {
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int c = s * IN; c < (s + 1) * IN; ++c)
#pragma unroll
                for (int j = 0; j < CW; ++j) {
                    const int n = n_first + c * CW * 4 + q * CW + j;
                    const float v = acc[a][c * CW / 4 + j / 4][j & 3];
                    if (n < g.N) top = fmaxf(top, v);
                    if (n < g.N && word == n) g.at_target[m] = v;
                }
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int c = s * IN; c < (s + 1) * IN; ++c)
#pragma unroll
                for (int j = 0; j < CW; ++j) {
                    const int n = n_first + c * CW * 4 + q * CW + j;
                    const float v = acc[a][c * CW / 4 + j / 4][j & 3];
                    if (n < g.N) sum += exp_for<T>(v - ref);
                }
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            const int stripe = n_first / STRIPE + s;
            if (q == 0 && m < m_end && stripe * STRIPE < g.N) g.stat[(int64_t)stripe * g.M + m] = make_float2(top, sum);
        }
    }
}

// The other epilogues: each wave's rows, half of them at a time where they are many, go through LDS, from where a thread takes eight consecutive columns of a row, row after
// row.  So the code is a short loop (unrolled over the accumulators it was 60 KB, fetched anew for every tile: at 512 rows an expert a
// tile of the weights' gradient took 41 us, with this NN), and a row's columns are written as one piece whatever the operands' form was.
template <class T, class P, int BM, int BN, int WM, int WN, int EPI>
__device__ __forceinline__ void through_lds(const ProductArgs &g, const typename P::Acc &acc, char *lds, int m0, int m_end, int n0, int wm, int wn,
                                            int i, int q, int64_t out_base, int64_t bias_base, bool skip)
{
    constexpr int PARTS = P::MT > 1 ? 2 : 1, LDT = BN + 4, PART = BM / WM / PARTS, CW = 8, THREADS = BN / CW, AT_ONCE = WM * WN * 64 / THREADS;      // (four columns more: no bank twice)
    static_assert(BM / PARTS * LDT * 4 <= P::LDS_BYTES, "the tile's part does not fit in LDS");
    float *const tile = (float *)lds;
    const int col = threadIdx.x % THREADS * CW, n = n0 + col, cnt = g.N - n;
    const float scale = (EPI == EPI_LINE || EPI == EPI_SUM) && g.scale ? *g.scale : 1.0f;
    float bias[CW];
#pragma unroll
    for (int j = 0; j < CW; ++j) bias[j] = 0.0f;
    if (g.bias && !skip && cnt > 0) load_row<T>(g.bias, bias_base + n, cnt, g.wide, bias);
#pragma unroll
    for (int h = 0; h < PARTS; ++h) {
        lds_barrier();
#pragma unroll
        for (int a = h * P::MT / PARTS; a < (h + 1) * P::MT / PARTS; ++a)
#pragma unroll
            for (int b = 0; b < P::NTL; ++b) {
                const int row = wm / PARTS + P::TA::row_of(i, a) - h * PART;
                *(f32x4 *)(tile + row * LDT + wn + P::TB::row_of(q * 4, b)) = acc[a][b];
            }
        lds_barrier();
        if (cnt <= 0) continue;
#pragma unroll 2
        for (int row = threadIdx.x / THREADS; row < BM / PARTS; row += AT_ONCE) {
            const int m = m0 + row / PART * (PARTS * PART) + h * PART + row % PART;
            if (m >= m_end) continue;
            float v[CW];
            *(f32x4 *)v = *(const f32x4 *)(tile + row * LDT + col);
            *(f32x4 *)(v + 4) = *(const f32x4 *)(tile + row * LDT + col + 4);
            if constexpr (EPI == EPI_GRAD) {
                const float lse = g.lse[m], coef = g.coef[m];
                const int64_t word = g.target[m] - g.word0;
#pragma unroll
                for (int j = 0; j < CW; ++j)
                    v[j] = coef == 0.0f || j >= cnt ? 0.0f : (exp_for<T>(v[j] - lse) - (word == n + j ? 1.0f : 0.0f)) * coef;
                store_row<T>(g.out, (int64_t)m * g.ldo + n, CW, 1, v);         // (work memory, with zeros up to the next 16 bytes)
            } else if constexpr (EPI == EPI_SUM) {
                char *sum = (char *)g.sum;
                const int64_t at = ((int64_t)blockIdx.y * g.M + m) * g.N + n;
                const int aligned = (g.N & 3) == 0;
#pragma unroll
                for (int k = 0; k < CW; k += 4) {
                    float part[4] = {v[k], v[k + 1], v[k + 2], v[k + 3]};
                    if (!g.first) {
                        float old[4];
                        load_row<float>(sum, at + k, cnt - k, aligned, old);
#pragma unroll
                        for (int j = 0; j < 4; ++j) part[j] += old[j];
                    }
                    if (!g.last) store_row<float>(sum, at + k, cnt - k, aligned, part);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[k + j] = part[j] * scale;
                }
                if (g.last) store_row<T>(g.out, (int64_t)m * g.ldo + n, cnt, g.wide, v);
            } else {
                if (EPI == EPI_LINE) {
#pragma unroll
                    for (int j = 0; j < CW; ++j) v[j] *= scale;
                }
                put_row<T, EPI>(g, out_base, bias, m, n, cnt, skip, v);
            }
        }
    }
}

template <class T, int FA, int FB, int BM, int BN, int WM, int WN, int EPI>
__global__ __launch_bounds__(WM *WN * 64, 2) void product_kernel(const ProductArgs g)
{
    using P = Product<T, FA, FB, BM, BN, WM, WN>;
    __shared__ __align__(1024) char lds[P::LDS_BYTES];
    constexpr int ES = sizeof(T), BK = STEP_BYTES / ES;

    int per_expert = g.row_tiles * g.col_tiles;
    int place = xcd_place(blockIdx.x, gridDim.x), expert = 0;
    if (g.grouping == GROUP_STEPS) {
        expert = place / per_expert;
        place -= expert * per_expert;
    }
    int tm, tn;
    tile_at(place, g.row_tiles, g.col_tiles, tm, tn);
    int m0 = tm * BM, m_end = min(m0 + BM, g.M), k0 = 0, k_end = g.K;
    bool skip = false;
    int64_t out_base = 0, bias_base = 0;
    const char *b = g.b;
    if (g.grouping == GROUP_ROWS) {
        const Slot s = find_slot(g.offsets, g.experts, g.M, BM, tm);
        if (s.expert < 0) return;
        skip = s.expert >= g.experts;
        m0 = s.first;
        m_end = s.end;
        if (skip) {
            k_end = 0;
        } else {
            b += (int64_t)s.expert * g.b_expert;
            bias_base = (int64_t)s.expert * g.N;
        }
    } else if (g.grouping == GROUP_STEPS) {
        group_rows(g.offsets, g.experts, g.K, expert, k0, k_end);
        out_base = (int64_t)expert * g.b_expert;
    } else if (g.splits > 1) {
        k0 = min((int)blockIdx.y * g.split_steps * BK, g.K);
        k_end = min(k0 + g.split_steps * BK, g.K);
    }
    const int n0 = tn * BN;
    // (a contiguous contraction is padded with zeros to 16 bytes, the other operand's may end before)
    const int a_rows = FA == ROWS ? m_end - m0 : min(BM, g.a_len - m0), a_k = min(k_end, g.a_k) - k0;
    const int b_rows = min(BN, (FB == ROWS ? g.N : g.b_len) - n0), b_k = min(k_end, g.b_k) - k0;
    const Operand A{g.a + (FA == ROWS ? (int64_t)m0 * g.lda + (int64_t)k0 * ES : (int64_t)k0 * g.lda + (int64_t)m0 * ES), g.lda, a_rows, a_k};
    const Operand B{b + (FB == ROWS ? (int64_t)n0 * g.ldb + (int64_t)k0 * ES : (int64_t)k0 * g.ldb + (int64_t)n0 * ES), g.ldb, b_rows, b_k};
    typename P::Acc acc;
    P::run(A, B, lds, acc);

    const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    if constexpr (EPI == EPI_LOSS) loss_stripes<T, P, BN / WN>(g, acc, m0 + wm, m_end, n0 + wn, i, q);
    else through_lds<T, P, BM, BN, WM, WN, EPI>(g, acc, lds, m0, m_end, n0, wm, wn, i, q, out_base, bias_base, skip);
}

template <class T, int FA, int FB, int EPI>
hipError_t launch_tiles(hipStream_t st, int tile, const ProductArgs &g)
{
    const int64_t tiles = (int64_t)g.row_tiles * g.col_tiles * (g.grouping == GROUP_STEPS ? g.experts : 1);
    const dim3 grid((unsigned)tiles, (unsigned)g.splits);
    if (tile == BIG_TILE) product_kernel<T, FA, FB, 256, 256, 2, 4, EPI><<<grid, 512, 0, st>>>(g);
    else if (tile == TILE) product_kernel<T, FA, FB, 128, 128, 2, 2, EPI><<<grid, 256, 0, st>>>(g);
    else product_kernel<T, FA, FB, 64, 64, 4, 1, EPI><<<grid, 256, 0, st>>>(g);
    return hipGetLastError();
}

template <class T>
hipError_t launch_forms(hipStream_t st, Forms forms, Epilogue epi, int tile, const ProductArgs &g)
{
    if (forms == FORM_RR) {
        switch (epi) {
        case EPI_LINE: return launch_tiles<T, ROWS, ROWS, EPI_LINE>(st, tile, g);
        case EPI_SIGMOID: return launch_tiles<T, ROWS, ROWS, EPI_SIGMOID>(st, tile, g);
        case EPI_ERF: return launch_tiles<T, ROWS, ROWS, EPI_ERF>(st, tile, g);
        case EPI_SUM: return launch_tiles<T, ROWS, ROWS, EPI_SUM>(st, tile, g);
        case EPI_LOSS: return launch_tiles<T, ROWS, ROWS, EPI_LOSS>(st, tile, g);
        case EPI_GRAD: return launch_tiles<T, ROWS, ROWS, EPI_GRAD>(st, tile, g);
        }
    } else if (forms == FORM_RC) {
        if (epi == EPI_LINE) return launch_tiles<T, ROWS, COLS, EPI_LINE>(st, tile, g);
        if (epi == EPI_SUM) return launch_tiles<T, ROWS, COLS, EPI_SUM>(st, tile, g);
    } else {
        if (epi == EPI_LINE) return launch_tiles<T, COLS, COLS, EPI_LINE>(st, tile, g);
        if (epi == EPI_SUM) return launch_tiles<T, COLS, COLS, EPI_SUM>(st, tile, g);
    }
    return hipErrorInvalidValue;
}

}  // namespace alpa
