// Matrix products of the layer operators (gfx950): D[m][n] = sum_k A(m, k) B(n, k), accumulated in 32 bits.
//
// An operand lies in memory either with its contraction contiguous (ROWS: p[row * ld + k]) or with its rows contiguous
// (COLS: p[k * ld + row]).  x wT has both in ROWS, dz w has w in COLS, dzT x has both in COLS, so no operand is ever transposed in
// memory: a tile of COLS goes to LDS as it lies and is read with the transposing LDS read (16-bit types) or word by word (32 bits).
//
// A workgroup computes a BM x BN tile.  A step of the contraction is 128 bytes of each row: 64 elements of 16 bits, 32 of 32 bits.
#pragma once
#include "internal.hpp"

namespace alpa {

enum : int { ROWS = 0, COLS = 1 };

using f32x4 = float __attribute__((ext_vector_type(4)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));
using i16x4 = short __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));
using bf16 = __bf16;
using f16 = _Float16;

#define ALPA_LDS __attribute__((address_space(3)))

// Sixteen bytes of one row's contraction in each lane: lane (i, q) = (lane & 15, lane >> 4) holds row i, elements
// q * 8 .. q * 8 + 7 of 32 (16 bits), or q * 4 .. q * 4 + 3 of 16 (32 bits; four products of four elements each, the j-th taking
// element j of every lane: the order of a sum's terms is free as long as both operands have the same one).
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c, bf16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c, f16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c, float)
{
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
    return c;
}

// One operand's place in memory, as a tile sees it: the tile's first row and step are at `p`.
struct Operand {
    const char *p;          // bytes
    int64_t ld;             // bytes between rows (ROWS) or between steps of the contraction (COLS)
    int rows;               // rows of this tile that exist
};

constexpr uint32_t OUT_OF_RANGE = 0x80000000u;       // a buffer offset beyond every range used here: such loads give zero

// How a tile's R rows lie in LDS, and how they get there and into registers.
//   ROWS: 128 bytes a row; the 16-byte chunk c of row r is stored at place c ^ swz(r), so that the sixteen rows that a read takes
//   at one chunk are spread over all banks.
//   COLS: R * es bytes a step; chunks are permuted within a step, so that the steps that a read takes at one column are.
template <class T, int FORM, int R, int NT>
struct Tile {
    static constexpr int ES = sizeof(T), BK = 128 / ES, BYTES = R * 128, CHUNKS = R * 8 / NT, CPS = R * ES / 16;
    // rows of two 16-row blocks are dealt to the product's rows so that a lane ends with eight consecutive columns of the result
    static constexpr bool PAIRED = FORM == ROWS && ES == 2;

    static __device__ __forceinline__ int row_of(int i, int t)
    {
        return PAIRED ? (t >> 1) * 32 + (i >> 2) * 8 + (t & 1) * 4 + (i & 3) : t * 16 + i;
    }
    static __device__ __forceinline__ int swz(int row)
    {
        return PAIRED ? (row & 3) | (row >> 1 & 4) : row & 7;
    }
    static __device__ __forceinline__ int swz_step(int k)        // in 16-byte chunks
    {
        return ES == 2 ? ((k & 3) | (k >> 1 & 4)) << 1 : (k >> 2 & 3) << 2;
    }
    // chunk `c` of the tile: its row (ROWS) or step (COLS), and which 16 bytes of that it holds
    static __device__ __forceinline__ void place(int c, int &major, int &chunk)
    {
        if (FORM == ROWS) { major = c >> 3; chunk = (c & 7) ^ swz(major); }
        else { major = c / CPS; chunk = (c % CPS) ^ swz_step(major); }
    }
    // the rows of block t as lane (i, q) holds them, elements of step ks (of two)
    static __device__ __forceinline__ u32x4 fragment(const char *lds, int row0, int t, int ks, int i, int q)
    {
        if (FORM == ROWS) {
            const int row = row_of(i, t);
            return *(const u32x4 *)(lds + (row0 + row) * 128 + ((ks * 4 + q) ^ swz(row)) * 16);
        } else if (ES == 2) {
            const int k = ks * 32 + q * 8 + (i >> 2), col = (row0 >> 4) + t;
            const int at = k * (R * 2) + ((col ^ (swz_step(k) >> 1)) * 32) + (i & 3) * 8;
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ALPA_LDS i16x4 *)(lds + at));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ALPA_LDS i16x4 *)(lds + at + 4 * (R * 2)));
            const u32x2 l = __builtin_bit_cast(u32x2, lo), h = __builtin_bit_cast(u32x2, hi);
            return u32x4{l.x, l.y, h.x, h.y};
        } else {
            u32x4 r;
            const int col = row0 + t * 16 + i;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = ks * 16 + q * 4 + j;
                r[j] = *(const uint32_t *)(lds + k * (R * 4) + (((col >> 2) ^ swz_step(k)) << 4) + (col & 3) * 4);
            }
            return r;
        }
    }
};

// Sixteen bytes from an address of any alignment, of which the first `n` elements exist.
template <class T>
__device__ __forceinline__ u32x4 load_some(const char *p, int n)
{
    constexpr int V = 16 / sizeof(T);
    u32x4 r = {0, 0, 0, 0};
    if (n >= V) {
        __builtin_memcpy(&r, p, 16);
    } else if (n > 0) {
        T e[V];
#pragma unroll
        for (int j = 0; j < V; ++j) e[j] = j < n ? ((const T *)p)[j] : (T)0.0f;
        __builtin_memcpy(&r, e, 16);
    }
    return r;
}

// Brings an operand's tiles to LDS with the load unit writing there itself.  Addresses, strides and the contiguous extent are multiples of 16
// bytes, so every chunk exists or does not; those that do not are out of the buffer's range and arrive as zeros.  The loads are written as
// assembly without a result register because the compiler, for the load's builtin, waits for all loads before the next transposing LDS
// read (measured at 8192 x 16384 x 4096 in 16 bits, operands in COLS: 1340 us, and 1060 without those waits); what has arrived is
// known here by counting (arrived()).
template <class T, int FORM, int R, int NT>
struct DirectLoader {
    using TL = Tile<T, FORM, R, NT>;
    static constexpr int N = TL::CHUNKS, ES = TL::ES, BK = TL::BK;
    const char *p;                          // the next step
    int64_t advance;
    int rows, ld, left, chunk0;             // left: of the contraction
    uint32_t off[N], cut;
    u32x4 range;

    __device__ __forceinline__ void init(const Operand &o, int k, int tid)
    {
        p = o.p;
        rows = o.rows;
        ld = (int)o.ld;
        left = k;
        advance = FORM == ROWS ? BK * ES : BK * o.ld;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            int major, chunk;
            TL::place(j * NT + tid, major, chunk);
            const bool in = FORM == ROWS ? major < rows : chunk * (16 / ES) < rows;
            off[j] = in ? (uint32_t)(major * ld + chunk * 16) : OUT_OF_RANGE;
            if (j == 0) chunk0 = chunk;     // (ROWS: the same for all j, as rows NT / 8 apart are permuted alike)
        }
    }
    // goes to the next step; behind the last one nothing is in range
    __device__ __forceinline__ void step()
    {
        const int n = min(left, BK);
        const int span = FORM == ROWS ? (rows - 1) * ld + n * ES : (n - 1) * ld + rows * ES;
        const uint64_t at = (uint64_t)p;
        range = u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, (uint32_t)(rows > 0 && n > 0 ? span : 0), 0x00020000u};
        cut = FORM == ROWS && chunk0 * (16 / ES) >= n ? OUT_OF_RANGE : 0;
        p += advance;
        left -= BK;
    }
    __device__ __forceinline__ void load(int j, char *lds, int wave) const
    {
        const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(ALPA_LDS char *)lds + (j * NT + wave * 64) * 16);
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"         // (m0 is reserved, and said to be overwritten all the same)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :
                     : "s"(to), "v"(FORM == ROWS ? off[j] | cut : off[j]), "s"(range)
                     : "m0");
#pragma clang diagnostic pop
    }
};

// The same through registers, from any address, element by element at the edges.
template <class T, int FORM, int R, int NT>
struct AnyLoader {
    using TL = Tile<T, FORM, R, NT>;
    static constexpr int N = TL::CHUNKS, ES = TL::ES, BK = TL::BK;
    Operand o;
    int K;
    u32x4 held[N];

    __device__ __forceinline__ void fetch(int kt, int tid)
    {
        const int k0 = kt * BK, left = K - k0;
        const char *base = o.p + (FORM == ROWS ? (int64_t)k0 * ES : (int64_t)k0 * o.ld);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            int major, chunk;
            TL::place(j * NT + tid, major, chunk);
            int n = FORM == ROWS ? left - chunk * (16 / ES) : o.rows - chunk * (16 / ES);
            if (FORM == ROWS ? major >= o.rows : major >= left) n = 0;
            held[j] = load_some<T>(base + (int64_t)major * o.ld + chunk * 16, n);
        }
    }
    __device__ __forceinline__ void store(char *lds, int tid) const
    {
#pragma unroll
        for (int j = 0; j < N; ++j) *(u32x4 *)(lds + (j * NT + tid) * 16) = held[j];
    }
};

// All but the last N loads to LDS of this wave have arrived, its LDS reads are done, and every wave is here.
template <int N>
__device__ __forceinline__ void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A workgroup of WM x WN waves computes the BM x BN tile.  The product's first operand is B, so that a lane's four results of a
// 16 x 16 block are consecutive columns n of one row m: acc[mt][nt][r] is row row_of(i, mt), column (of block nt) 4 q + r.
template <class T, int FA, int FB, int BM, int BN, int WM, int WN, bool DIRECT>
struct Product {
    static constexpr int NT = WM * WN * 64, MT = BM / WM / 16, NTL = BN / WN / 16, ES = sizeof(T);
    using TA = Tile<T, FA, BM, NT>;
    using TB = Tile<T, FB, BN, NT>;
    // The large tile: three stages of A and two of B, all the LDS there is.  The small one: two of each, two workgroups in a compute unit.
    static constexpr bool DEEP = DIRECT && BM == 256;
    static constexpr int A_STAGES = DEEP ? 3 : 2, LDS_BYTES = A_STAGES * TA::BYTES + 2 * TB::BYTES;
    using Acc = f32x4[MT][NTL];
    struct Fragments { u32x4 a[MT], b[NTL]; };

    static __device__ __forceinline__ void clear(Acc &acc)
    {
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < NTL; ++b) acc[a][b] = f32x4{0, 0, 0, 0};
    }

    static __device__ __forceinline__ void run(const Operand &A, const Operand &B, int K, char *lds, Acc &acc)
    {
        clear(acc);
        const int steps = (K + TA::BK - 1) / TA::BK;
        if (steps == 0) return;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int m0 = wave / WN * (BM / WM), n0 = wave % WN * (BN / WN);
        if constexpr (DEEP) run_deep(A, B, K, steps, lds, acc, wave, m0, n0, lane & 15, lane >> 4);
        else if constexpr (DIRECT) run_direct(A, B, K, steps, lds, acc, wave, m0, n0, lane & 15, lane >> 4);
        else run_any(A, B, K, steps, lds, acc, m0, n0, lane & 15, lane >> 4);
    }

private:
    static __device__ __forceinline__ void half_step(const char *a_lds, const char *b_lds, int ks, Acc &acc, int m0, int n0, int i, int q)
    {
        Fragments f;
#pragma unroll
        for (int b = 0; b < NTL; ++b) f.b[b] = TB::fragment(b_lds, n0, b, ks, i, q);
#pragma unroll
        for (int a = 0; a < MT; ++a) f.a[a] = TA::fragment(a_lds, m0, a, ks, i, q);
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < NTL; ++b) acc[a][b] = mma(f.b[b], f.a[a], acc[a][b], T{});
    }

    // The next step's loads are under way while this one is multiplied; the other workgroup of the compute unit fills what is left.
    static __device__ __forceinline__ void run_direct(const Operand &A, const Operand &B, int K, int steps, char *lds, Acc &acc, int wave,
                                                      int m0, int n0, int i, int q)
    {
        DirectLoader<T, FA, BM, NT> la;
        DirectLoader<T, FB, BN, NT> lb;
        la.init(A, K, threadIdx.x);
        lb.init(B, K, threadIdx.x);
        char *here = lds, *next = lds + TA::BYTES + TB::BYTES;
        auto fetch = [&](char *to) {
            la.step();
            lb.step();
#pragma unroll
            for (int j = 0; j < la.N; ++j) la.load(j, to, wave);
#pragma unroll
            for (int j = 0; j < lb.N; ++j) lb.load(j, to + TA::BYTES, wave);
        };
        fetch(here);
        for (int kt = 0; kt < steps; ++kt) {
            arrived<0>();
            fetch(next);
            half_step(here, here + TA::BYTES, 0, acc, m0, n0, i, q);
            half_step(here, here + TA::BYTES, 1, acc, m0, n0, i, q);
            char *t = here;
            here = next;
            next = t;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // (the loads of nothing behind the last step)
    }

    static __device__ __forceinline__ void run_any(const Operand &A, const Operand &B, int K, int steps, char *lds, Acc &acc, int m0, int n0,
                                                   int i, int q)
    {
        AnyLoader<T, FA, BM, NT> la{A, K};
        AnyLoader<T, FB, BN, NT> lb{B, K};
        char *here = lds, *next = lds + TA::BYTES + TB::BYTES;
        la.fetch(0, threadIdx.x);
        lb.fetch(0, threadIdx.x);
        la.store(here, threadIdx.x);
        lb.store(here + TA::BYTES, threadIdx.x);
        for (int kt = 0; kt < steps; ++kt) {
            arrived<0>();
            if (kt + 1 < steps) {
                la.fetch(kt + 1, threadIdx.x);
                lb.fetch(kt + 1, threadIdx.x);
            }
            half_step(here, here + TA::BYTES, 0, acc, m0, n0, i, q);
            half_step(here, here + TA::BYTES, 1, acc, m0, n0, i, q);
            if (kt + 1 < steps) {
                la.store(next, threadIdx.x);
                lb.store(next + TA::BYTES, threadIdx.x);
            }
            char *t = here;
            here = next;
            next = t;
        }
    }

    // A step is sixteen groups of four products, eight for each half of its contraction; a group also issues a share of the LDS reads of the
    // next half and every second one a load, so that matrix unit, LDS and load unit have work all the time (eight loads together take the load
    // unit as long as half a step's products).  A's and B's stages of step kt are read by group 3 (barrier) and then hold loads of
    // A's step kt + 3 and B's step kt + 2, which gives A nearly two steps to arrive and B one; the last six loads may be under way when step
    // kt + 1 is looked at (group 8).  At 8192 x 4096 x 16384 in 16 bits a step takes 2490 to 2650 cycles of the 2048 its products need, against
    // 2810 with loads one step ahead, and the clock that the power limit leaves is 1.65 GHz.
    static __device__ __forceinline__ void run_deep(const Operand &A, const Operand &B, int K, int steps, char *lds, Acc &acc, int wave,
                                                    int m0, int n0, int i, int q)
    {
        DirectLoader<T, FA, BM, NT> la;
        DirectLoader<T, FB, BN, NT> lb;
        static_assert(la.N == 4 && lb.N == 4 && MT == 8 && NTL == 4, "loads and reads are dealt to groups for these");
        la.init(A, K, threadIdx.x);
        lb.init(B, K, threadIdx.x);
        char *a0 = lds, *a1 = lds + TA::BYTES, *a2 = lds + 2 * TA::BYTES, *b0 = lds + 3 * TA::BYTES, *b1 = b0 + TB::BYTES;
        la.step();
        lb.step();
#pragma unroll
        for (int j = 0; j < 4; ++j) la.load(j, a0, wave);
#pragma unroll
        for (int j = 0; j < 4; ++j) lb.load(j, b0, wave);
        la.step();
        lb.step();
#pragma unroll
        for (int j = 0; j < 4; ++j) la.load(j, a1, wave);
#pragma unroll
        for (int j = 0; j < 4; ++j) lb.load(j, b1, wave);
        la.step();
        la.load(0, a2, wave);
        la.load(1, a2, wave);
        arrived<10>();
        Fragments f[2];
        auto read = [&](int half, int a, const char *a_lds, const char *b_lds) {
            if (a & 1) f[half].b[a >> 1] = TB::fragment(b_lds, n0, a >> 1, half, i, q);
            f[half].a[a] = TA::fragment(a_lds, m0, a, half, i, q);
        };
#pragma unroll
        for (int a = 0; a < 8; ++a) read(0, a, a0, b0);
        for (int kt = 0; kt < steps; ++kt) {
#pragma unroll
            for (int g = 0; g < 16; ++g) {
                const int half = g >> 3, a = g & 7;
                if (g == 0) la.load(2, a2, wave);
                if (g == 2) la.load(3, a2, wave);
                if (g < 4) {
                    read(1, 2 * g, a0, b0);
                    read(1, 2 * g + 1, a0, b0);
                }
                if (g == 4) {
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    lb.step();
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (g == 8) {
                    arrived<6>();
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (g >= 4 && g <= 10 && g % 2 == 0) lb.load((g - 4) / 2, b0, wave);
                if (g == 12) {
                    la.step();
                    la.load(0, a0, wave);
                }
                if (g == 14) la.load(1, a0, wave);
                if (g >= 8) read(0, a, a1, b1);
#pragma unroll
                for (int b = 0; b < 4; ++b) acc[a][b] = mma(f[half].b[b], f[half].a[a], acc[a][b], T{});
                __builtin_amdgcn_sched_barrier(0);
            }
            char *t = a0;
            a0 = a1;
            a1 = a2;
            a2 = t;
            t = b0;
            b0 = b1;
            b1 = t;
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");       // (the loads and reads of nothing behind the last step)
    }
};

}  // namespace alpa
