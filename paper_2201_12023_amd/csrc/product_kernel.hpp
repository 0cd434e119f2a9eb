// The tiled product with its epilogues, instantiated per element type (kernels_product_*.hip).
#pragma once
#include "epilogue.hpp"
#include "slots.hpp"

namespace alpa {

// One tile's part of a product.
struct Job {
    Operand A, B;
    int m0, m_end, n0;             // rows m0 .. m_end - 1, columns n0 ..
    int skip;                      // 1: rows of no expert
    int64_t out_base, bias_base;   // elements in front of an expert's result and bias
};

// The tiles in an order of their own, for a workgroup's walk.  Workgroups are dealt to the eight XCDs in turn (blockIdx & 7).  Each XCD gets a run of
// consecutive tiles, or, where the contraction is ragged, an eighth of every expert's tiles, as experts differ in length; tiles go through
// bands of eight row tiles, so that what an XCD works on at one time shares its operands' tiles in its L2.  Slots of ragged rows that do not
// exist are not dealt at all.
template <class T, int FA, int FB, int BM, int BN, int GROUPING>
struct Walk {
    int row_tiles, tiles, per, first, count;    // tiles of the result (of one expert's), of an XCD's in each expert, the XCD's first, its number

    __device__ __forceinline__ Walk(const ProductArgs &g)
    {
        const int x = blockIdx.x & 7;
        row_tiles = GROUPING == GROUP_ROWS ? min(slots_before(g.offsets, g.experts, g.M, BM, g.experts + 2), g.row_tiles) : g.row_tiles;
        tiles = row_tiles * g.col_tiles;
        per = (tiles + 7) / 8;
        first = GROUPING == GROUP_STEPS ? x * per : x * (tiles >> 3) + min(x, tiles & 7);
        count = GROUPING == GROUP_STEPS ? per * g.experts : (tiles >> 3) + (x < (tiles & 7) ? 1 : 0);
    }
    // The XCD's i-th tile, i < count (an eighth of an expert's tiles may end with places that are no tiles: nothing is read or written there).
    __device__ __forceinline__ Job at(const ProductArgs &g, int i) const
    {
        constexpr int ES = sizeof(T), BK = STEP_BYTES / ES, BAND = 8;
        const int expert = GROUPING == GROUP_STEPS ? i / per : 0, place = first + i - expert * per;
        const int band = place / (BAND * g.col_tiles), top = band * BAND, high = max(min(BAND, row_tiles - top), 1);
        const int in = place - top * g.col_tiles, tm = top + in % high;
        Job job;
        job.n0 = in / high * BN;
        job.m0 = tm * BM;
        job.m_end = min(job.m0 + BM, g.M);
        job.skip = 0;
        job.out_base = job.bias_base = 0;
        int k0 = 0, k_end = g.K;
        const char *b = g.b;
        if constexpr (GROUPING == GROUP_ROWS) {
            const Slot s = find_slot(g.offsets, g.experts, g.M, BM, tm);
            const int e = s.expert < 0 || s.expert >= g.experts ? 0 : s.expert;
            job.skip = s.expert != e;
            job.m0 = s.first;
            job.m_end = s.end;
            k_end = job.skip ? 0 : k_end;
            b += (int64_t)e * g.b_expert;
            job.bias_base = (int64_t)e * g.N;
        }
        if constexpr (GROUPING == GROUP_STEPS) {
            group_rows(g.offsets, g.experts, g.K, expert, k0, k_end);
            job.m0 = place < tiles ? job.m0 : 0;
            job.m_end = place < tiles ? job.m_end : 0;
            k_end = place < tiles ? k_end : k0;
            job.out_base = (int64_t)expert * g.b_expert;
        }
        if constexpr (GROUPING == GROUP_NONE) {
            const int part = g.split_steps * BK;
            k0 = min((int)blockIdx.y * part, k_end);
            k_end = min(k0 + part, k_end);
        }
        const int m0 = job.m0, n0 = job.n0;
        // (a contiguous contraction is padded with zeros to 16 bytes, the other operand's may end before)
        job.A = Operand{g.a + (FA == ROWS ? (int64_t)m0 * g.lda + (int64_t)k0 * ES : (int64_t)k0 * g.lda + (int64_t)m0 * ES), g.lda,
                        FA == ROWS ? job.m_end - m0 : min(BM, g.a_len - m0), min(k_end, g.a_k) - k0};
        job.B = Operand{b + (FB == ROWS ? (int64_t)n0 * g.ldb + (int64_t)k0 * ES : (int64_t)k0 * g.ldb + (int64_t)n0 * ES), g.ldb,
                        min(BN, (FB == ROWS ? g.N : g.b_len) - n0), min(k_end, g.b_k) - k0};
        return job;
    }
};

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

// What becomes of columns n .. n + CW - 1 of row m, `cnt` of them real, in the other epilogues.  BARE: gradients, which have no bias, activation,
// z or residual.
template <class T, int EPI, bool BARE, int CW>
__device__ __forceinline__ void finish_row(const ProductArgs &g, const Job &job, float scale, const float (&bias)[CW], int m, int n, int cnt,
                                           int wide, float (&v)[CW])
{
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
        if (g.last) store_row<T>(g.out, (int64_t)m * g.ldo + n, cnt, wide, v);
    } else {
        if (EPI == EPI_LINE) {
#pragma unroll
            for (int j = 0; j < CW; ++j) v[j] *= scale;
        }
        if (BARE) store_row<T>(g.out, job.out_base + (int64_t)m * g.ldo + n, cnt, wide, v);
        else put_row<T, EPI>(g, job.out_base, bias, m, n, cnt, wide, job.skip, v);
    }
}

// The small tiles: each wave's rows, half of them at a time where they are many, go through LDS, from where a thread takes eight consecutive columns
// of a row, row after row.  So the code is a short loop, whatever is aligned and whatever is not (unrolled over the accumulators it was 60 KB,
// fetched anew for every tile), and a row's columns are written as one piece whatever the operands' form was.
template <class T, class P, int BM, int BN, int WM, int WN, int EPI, bool BARE>
__device__ __forceinline__ void through_lds(const ProductArgs &g, const typename P::Acc &acc, char *lds, const Job &job, int wm, int wn, int i, int q)
{
    constexpr int PARTS = P::MT > 1 ? 2 : 1, LDT = BN + 4, PART = BM / WM / PARTS, CW = 8, THREADS = BN / CW, AT_ONCE = WM * WN * 64 / THREADS;      // (four columns more: no bank twice)
    static_assert(BM / PARTS * LDT * 4 <= P::LDS_BYTES, "the tile's part does not fit in LDS");
    float *const tile = (float *)lds;
    const int col = threadIdx.x % THREADS * CW, n = job.n0 + col, cnt = g.N - n;
    const float scale = (EPI == EPI_LINE || EPI == EPI_SUM) && g.scale ? *g.scale : 1.0f;
    float bias[CW];
#pragma unroll
    for (int j = 0; j < CW; ++j) bias[j] = 0.0f;
    if (!BARE && g.bias && job.skip == 0 && cnt > 0) load_row<T>(g.bias, job.bias_base + n, cnt, g.wide, bias);
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
            const int m = job.m0 + row / PART * (PARTS * PART) + h * PART + row % PART;
            if (m >= job.m_end) continue;
            float v[CW];
            *(f32x4 *)v = *(const f32x4 *)(tile + row * LDT + col);
            *(f32x4 *)(v + 4) = *(const f32x4 *)(tile + row * LDT + col + 4);
            finish_row<T, EPI, BARE>(g, job, scale, bias, m, n, cnt, g.wide, v);
        }
    }
}

// The large tile, whose LDS holds the next tile's operands: straight from the accumulators.  Everything is aligned and rows are multiples of eight
// elements, so a lane's columns exist or do not and the code stays short.
template <class T, class P, int EPI, bool BARE>
__device__ __forceinline__ void straight(const ProductArgs &g, const typename P::Acc &acc, const Job &job, int wm, int wn, int i, int q)
{
    // With w in COLS a lane has four columns of each block: of two blocks lanes of even q take the first one's from their neighbour of odd q, whose
    // share of the second they give, so that every lane has eight consecutive ones (stores of 8 bytes, 32 a row, instead: products by
    // w in COLS 2 % slower, and with the contraction ragged 4 %).
    constexpr bool TAKE = sizeof(T) == 2 && !P::TB::PAIRED;
    constexpr int CW = 16 / sizeof(T), GROUPS = P::NTL * 4 / CW;
    const int at = TAKE ? (q & 1) * 16 + (q >> 1) * 8 : q * CW;
    const float scale = (EPI == EPI_LINE || EPI == EPI_SUM) && g.scale ? *g.scale : 1.0f;
    float bias[GROUPS][CW];
#pragma unroll
    for (int c = 0; c < GROUPS; ++c) {
        const int n = job.n0 + wn + c * CW * 4 + at;
#pragma unroll
        for (int j = 0; j < CW; ++j) bias[c][j] = 0.0f;
        if (!BARE && g.bias && job.skip == 0 && n < g.N) load_row<T>(g.bias, job.bias_base + n, CW, 1, bias[c]);
    }
    // Waited for here: to the compiler a load that no row may use is under way until its register is used again, which is in the steps of the next
    // tile, and there it would wait for all loads in every step.
    asm volatile("" ::"v"(scale));
#pragma unroll
    for (int c = 0; c < GROUPS; ++c)
#pragma unroll
        for (int j = 0; j < CW; ++j) asm volatile("" ::"v"(bias[c][j]));
#pragma unroll
    for (int a = 0; a < P::MT; ++a) {
        const int m = job.m0 + wm + P::TA::row_of(i, a);
        if (!TAKE && m >= job.m_end) continue;
#pragma unroll
        for (int c = 0; c < GROUPS; ++c) {
            const int n = job.n0 + wn + c * CW * 4 + at;
            if (!TAKE && n >= g.N) continue;
            float v[CW];
#pragma unroll
            for (int j = 0; j < CW; ++j) v[j] = acc[a][c * CW / 4 + j / 4][j & 3];
            if constexpr (TAKE) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const u32x2 both = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[j]), __float_as_uint(v[j + 4]), false, false);
                    v[j] = __uint_as_float(both.x);
                    v[j + 4] = __uint_as_float(both.y);
                }
                if (m >= job.m_end || n >= g.N) continue;
            }
            finish_row<T, EPI, BARE>(g, job, scale, bias[c], m, n, CW, 1, v);
        }
    }
}

template <class T, class P, int BM, int BN, int WM, int WN, int EPI, bool BARE>
__device__ __forceinline__ void epilogue(const ProductArgs &g, const typename P::Acc &acc, char *lds, const Job &job)
{
    const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    if constexpr (EPI == EPI_LOSS) loss_stripes<T, P, BN / WN>(g, acc, job.m0 + wm, job.m_end, job.n0 + wn, i, q);
    else if constexpr (P::DEEP) straight<T, P, EPI, BARE>(g, acc, job, wm, wn, i, q);
    else through_lds<T, P, BM, BN, WM, WN, EPI, BARE>(g, acc, lds, job, wm, wn, i, q);
}

template <class T, int FA, int FB, int BM, int BN, int WM, int WN, int EPI, int GROUPING>
__global__ __launch_bounds__(WM *WN * 64, 2) void product_kernel(const ProductArgs g)
{
    using P = Product<T, FA, FB, BM, BN, WM, WN>;
    __shared__ __align__(1024) char lds[P::LDS_BYTES];
    const Walk<T, FA, FB, BM, BN, GROUPING> walk(g);
    int i = (P::DEEP ? 0 : g.before) + (blockIdx.x >> 3);
    if (i >= walk.count) return;
    Job job = walk.at(g, i);
    typename P::Acc acc;
    if constexpr (P::DEEP) {
        // as many workgroups as compute units, each with every so-many-th tile of its XCD's
        const int apart = ((int)gridDim.x - (int)(blockIdx.x & 7) + 7) >> 3;
        int steps = max((max(job.A.k, job.B.k) + P::TA::BK - 1) / P::TA::BK, P::Deep::LEAST);
        typename P::Deep deep;
        deep.begin(job.A, job.B, steps, lds);
        for (;;) {
            i += apart;
            const bool more = i < walk.count;
            // (behind the last tile: that tile once more, with no rows)
            Job next = walk.at(g, more ? i : i - apart);
            next.A.rows = more ? next.A.rows : 0;
            next.B.rows = more ? next.B.rows : 0;
            const int steps_next = max((max(next.A.k, next.B.k) + P::TA::BK - 1) / P::TA::BK, P::Deep::LEAST);
            deep.la.follow(next.A, steps_next);
            deep.lb.follow(next.B, steps_next);
            deep.run(steps, acc);
            epilogue<T, P, BM, BN, WM, WN, EPI, FB == COLS>(g, acc, lds, job);
            if (!more) break;
            job = next;
            steps = steps_next;
        }
        deep.end();
    } else {
        P::run(job.A, job.B, lds, acc);
        epilogue<T, P, BM, BN, WM, WN, EPI, FB == COLS>(g, acc, lds, job);
    }
}

template <class T, int FA, int FB, int EPI, int GROUPING>
hipError_t launch_tiles(hipStream_t st, int tile, const ProductArgs &g)
{
    const int64_t tiles = (int64_t)g.row_tiles * g.col_tiles;
    const int64_t all = GROUPING == GROUP_STEPS ? (tiles + 7) / 8 * 8 * g.experts : tiles;
    if (tile == BIG_TILE) {
        const dim3 grid((unsigned)std::min<int64_t>(all, COMPUTE_UNITS), (unsigned)g.splits);
        product_kernel<T, FA, FB, 256, 256, 2, 4, EPI, GROUPING><<<grid, 512, 0, st>>>(g);
        return hipGetLastError();
    }
    // (a grid's threads are counted in 32 bits)
    constexpr int64_t MOST = 1 << 23;
    ProductArgs part = g;
    for (int64_t done = 0; done < all; done += MOST) {
        part.before = (int)(done / 8);
        const dim3 grid((unsigned)std::min(all - done, MOST), (unsigned)g.splits);
        if (tile == TILE) product_kernel<T, FA, FB, 128, 128, 2, 2, EPI, GROUPING><<<grid, 256, 0, st>>>(part);
        else product_kernel<T, FA, FB, 64, 64, 4, 1, EPI, GROUPING><<<grid, 256, 0, st>>>(part);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T>
hipError_t launch_forms(hipStream_t st, Forms forms, Epilogue epi, int tile, const ProductArgs &g)
{
    if (forms == FORM_RR && g.grouping == GROUP_NONE) {
        switch (epi) {
        case EPI_LINE: return launch_tiles<T, ROWS, ROWS, EPI_LINE, GROUP_NONE>(st, tile, g);
        case EPI_SIGMOID: return launch_tiles<T, ROWS, ROWS, EPI_SIGMOID, GROUP_NONE>(st, tile, g);
        case EPI_ERF: return launch_tiles<T, ROWS, ROWS, EPI_ERF, GROUP_NONE>(st, tile, g);
        case EPI_SUM: return launch_tiles<T, ROWS, ROWS, EPI_SUM, GROUP_NONE>(st, tile, g);
        case EPI_LOSS: return launch_tiles<T, ROWS, ROWS, EPI_LOSS, GROUP_NONE>(st, tile, g);
        case EPI_GRAD: return launch_tiles<T, ROWS, ROWS, EPI_GRAD, GROUP_NONE>(st, tile, g);
        }
    } else if (forms == FORM_RR && g.grouping == GROUP_ROWS) {
        if (epi == EPI_LINE) return launch_tiles<T, ROWS, ROWS, EPI_LINE, GROUP_ROWS>(st, tile, g);
        if (epi == EPI_SIGMOID) return launch_tiles<T, ROWS, ROWS, EPI_SIGMOID, GROUP_ROWS>(st, tile, g);
        if (epi == EPI_ERF) return launch_tiles<T, ROWS, ROWS, EPI_ERF, GROUP_ROWS>(st, tile, g);
    } else if (forms == FORM_RC && g.grouping == GROUP_NONE) {
        if (epi == EPI_LINE) return launch_tiles<T, ROWS, COLS, EPI_LINE, GROUP_NONE>(st, tile, g);
        if (epi == EPI_SUM) return launch_tiles<T, ROWS, COLS, EPI_SUM, GROUP_NONE>(st, tile, g);
    } else if (forms == FORM_RC && g.grouping == GROUP_ROWS) {
        if (epi == EPI_LINE) return launch_tiles<T, ROWS, COLS, EPI_LINE, GROUP_ROWS>(st, tile, g);
    } else if (forms == FORM_CC && g.grouping == GROUP_NONE) {
        if (epi == EPI_LINE) return launch_tiles<T, COLS, COLS, EPI_LINE, GROUP_NONE>(st, tile, g);
        if (epi == EPI_SUM) return launch_tiles<T, COLS, COLS, EPI_SUM, GROUP_NONE>(st, tile, g);
    } else if (forms == FORM_CC && g.grouping == GROUP_STEPS) {
        if (epi == EPI_LINE) return launch_tiles<T, COLS, COLS, EPI_LINE, GROUP_STEPS>(st, tile, g);
    }
    return hipErrorInvalidValue;
}

}  // namespace alpa
