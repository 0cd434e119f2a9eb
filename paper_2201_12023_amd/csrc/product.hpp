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
    int k;                  // extent of the contraction; a multiple of 16 bytes if it is the contiguous one, as is `rows` otherwise
};

constexpr uint32_t OUT_OF_RANGE = 0x80000000u;       // a buffer offset beyond every range used here: such loads give zero

// How a tile's R rows lie in LDS, and how they get there and into registers.
//   ROWS: 128 bytes a row; the 16-byte chunk c of row r is stored at place c ^ swz(r), so that the sixteen rows that a read takes
//   at one chunk are spread over all banks.
//   COLS: R * es bytes a step; chunks are permuted within a step, so that the steps that a read takes at one column are.
template <class T, int FORM, int R, int NT, bool COLUMNS>
struct Tile {
    static constexpr int ES = sizeof(T), BK = 128 / ES, BYTES = R * 128, CHUNKS = R * 8 / NT, CPS = R * ES / 16;
    // COLUMNS: the tile's rows are the result's columns; those of two blocks of sixteen are dealt to the product's rows so that a lane
    // ends with eight consecutive ones
    static constexpr bool PAIRED = COLUMNS && FORM == ROWS && ES == 2;

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
        if (ES == 4) return (k >> 2 & 3) << 2;
        return R == 64 ? ((k >> 1 & 1) | (k >> 2 & 2)) << 1 : ((k & 3) | (k >> 1 & 4)) << 1;      // (R == 64: two steps cover all banks)
    }
    // chunk `c` of the tile: its row (ROWS) or step (COLS), and which 16 bytes of that it holds
    static __device__ __forceinline__ void place(int c, int &major, int &chunk)
    {
        if (FORM == ROWS) { major = c >> 3; chunk = (c & 7) ^ swz(major); }
        else { major = c / CPS; chunk = (c % CPS) ^ swz_step(major); }
    }
    static __device__ __forceinline__ int first_major(int c) { return FORM == ROWS ? c >> 3 : c / CPS; }

    // Where lane (i, q) reads, in the tile: from there, blocks and halves of the step are an exclusive or and a constant away, so that one
    // register serves all of a wave's reads.
    static __device__ __forceinline__ uint32_t lane_at(int row0, int i, int q)
    {
        if (FORM == ROWS) return (row0 + row_of(i, 0)) * 128 + (q ^ swz(row_of(i, 0))) * 16;
        if (ES == 2) {
            const int k = q * 8 + (i >> 2);
            return k * (R * 2) + (((row0 >> 3) ^ swz_step(k)) << 4) + (i & 3) * 8;
        }
        return q * 4 * (R * 4) + (((row0 >> 2) ^ swz_step(q * 4)) + (i >> 2)) * 16 + (i & 3) * 4;
    }
    // the rows of block t as lane (i, q) holds them, elements of half ks of the step; `at`: lane_at() behind the stage's first byte
    static __device__ __forceinline__ u32x4 fragment(uint32_t at, int t, int ks)
    {
        if (FORM == ROWS) {
            return *(const ALPA_LDS u32x4 *)(uintptr_t)((at ^ (ks * 64)) + row_of(0, t) * 128);
        } else if (ES == 2) {
            const uint32_t from = (at ^ (t * 32)) + ks * 32 * (R * 2);
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ALPA_LDS i16x4 *)(uintptr_t)from);
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ALPA_LDS i16x4 *)(uintptr_t)(from + 4 * (R * 2)));
            const u32x2 l = __builtin_bit_cast(u32x2, lo), h = __builtin_bit_cast(u32x2, hi);
            return u32x4{l.x, l.y, h.x, h.y};
        } else {
            u32x4 r;
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = *(const ALPA_LDS uint32_t *)(uintptr_t)((at ^ (t * 64)) + (ks * 16 + j) * (R * 4));
            return r;
        }
    }
};

// Brings an operand's tiles to LDS with the load unit writing there itself.  Addresses, strides and the contiguous extent are multiples of 16
// bytes, so every chunk exists or does not; those that do not are out of the buffer's range and arrive as zeros.  The loads are written as
// assembly without a result register because the compiler, for the load's builtin, waits for all loads before the next transposing LDS
// read (measured at 8192 x 16384 x 4096 in 16 bits, operands in COLS: 1340 us, and 1060 without those waits); what has arrived is
// known here by counting (arrived()).
template <class T, class TL, int FORM, int NT>
struct DirectLoader {
    static constexpr int N = TL::CHUNKS, ES = TL::ES, BK = TL::BK;
    const char *p;                          // the next step
    int64_t advance;
    int rows, ld, left, chunk;              // left: of the contraction
    // A thread's chunks lie at the same place of rows or steps that are NT / 8 or NT / CPS apart, which are permuted alike; steps of 32-bit
    // elements, eight apart, are so every second time.
    static constexpr int KINDS = FORM == COLS && ES == 4 ? 2 : 1;
    uint32_t first[KINDS], off[KINDS], apart;      // this thread's first chunks, as they are in this step, and how far chunks are apart
    u32x4 range;

    __device__ __forceinline__ void init(const Operand &o, int tid)
    {
        p = o.p;
        rows = o.rows;
        ld = (int)o.ld;
        left = o.k;
        advance = FORM == ROWS ? BK * ES : BK * o.ld;
#pragma unroll
        for (int j = 0; j < KINDS; ++j) {
            int major, c;
            TL::place(j * NT + tid, major, c);
            if (j == 0) chunk = c;
            first[j] = FORM == COLS && c * (16 / ES) >= rows ? OUT_OF_RANGE : (uint32_t)(TL::first_major(tid) * ld + c * 16);
        }
        apart = (uint32_t)(ld * (FORM == ROWS ? NT / 8 : NT / TL::CPS));
    }
    // Goes to the next step; behind the last one nothing is in range.  The range ends with the last row's (or step's) last byte, so rows and steps
    // that do not exist are behind it; chunks behind a row's end but in front of the next row are cut.
    __device__ __forceinline__ void step()
    {
        const int n = min(left, BK);
        const int span = FORM == ROWS ? (rows - 1) * ld + n * ES : (n - 1) * ld + rows * ES;
        const uint64_t at = (uint64_t)p;
        range = u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, (uint32_t)(rows > 0 && n > 0 ? span : 0), 0x00020000u};
#pragma unroll
        for (int j = 0; j < KINDS; ++j) off[j] = FORM == ROWS && chunk * (16 / ES) >= n ? first[j] | OUT_OF_RANGE : first[j];
        p += advance;
        left -= BK;
    }
    __device__ __forceinline__ void load(int j, uint32_t lds, int wave) const
    {
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (j * NT + wave * 64) * 16);
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"         // (m0 is reserved, and said to be overwritten all the same)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :
                     : "s"(to), "v"(off[j % KINDS] + j * apart), "s"(range)
                     : "m0");
#pragma clang diagnostic pop
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
template <class T, int FA, int FB, int BM, int BN, int WM, int WN>
struct Product {
    static constexpr int NT = WM * WN * 64, MT = BM / WM / 16, NTL = BN / WN / 16, ES = sizeof(T);
    using TA = Tile<T, FA, BM, NT, false>;
    using TB = Tile<T, FB, BN, NT, true>;
    using LoaderA = DirectLoader<T, TA, FA, NT>;
    using LoaderB = DirectLoader<T, TB, FB, NT>;
    // The large tile: three stages of A and two of B, all the LDS there is.  The others: as many stages as leave room for a second workgroup.
    static constexpr bool DEEP = BM == 256;
    static constexpr int STAGE = TA::BYTES + TB::BYTES, STAGES = BM == 128 ? 2 : 5;
    static constexpr int LDS_BYTES = DEEP ? 3 * TA::BYTES + 2 * TB::BYTES : STAGES * STAGE;
    using Acc = f32x4[MT][NTL];
    struct Fragments { u32x4 a[MT], b[NTL]; };

    static __device__ __forceinline__ void clear(Acc &acc)
    {
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < NTL; ++b) acc[a][b] = f32x4{0, 0, 0, 0};
    }

    // a wave's place: its rows and columns in the tile, where its lanes read
    struct Wave { int id; uint32_t a_at, b_at; };

    static __device__ __forceinline__ void run(const Operand &A, const Operand &B, char *lds_memory, Acc &acc)
    {
        clear(acc);
        const int steps = (max(A.k, B.k) + TA::BK - 1) / TA::BK;
        if (steps == 0) return;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const Wave w{wave, TA::lane_at(wave / WN * (BM / WM), lane & 15, lane >> 4), TB::lane_at(wave % WN * (BN / WN), lane & 15, lane >> 4)};
        const uint32_t lds = (uint32_t)(uintptr_t)(ALPA_LDS char *)lds_memory;
        if constexpr (DEEP) run_deep(A, B, steps, lds, acc, w);
        else run_ring(A, B, steps, lds, acc, w);
    }

private:
    static __device__ __forceinline__ void half_step(uint32_t a_at, uint32_t b_at, int ks, Acc &acc)
    {
        Fragments f;
#pragma unroll
        for (int b = 0; b < NTL; ++b) f.b[b] = TB::fragment(b_at, b, ks);
#pragma unroll
        for (int a = 0; a < MT; ++a) f.a[a] = TA::fragment(a_at, a, ks);
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < NTL; ++b) acc[a][b] = mma(f.b[b], f.a[a], acc[a][b], T{});
    }

    // STAGES - 1 steps' loads are under way; a stage is loaded again when every wave has read it, one barrier later.  The other workgroup of
    // the compute unit fills what is left.
    static __device__ __forceinline__ void run_ring(const Operand &A, const Operand &B, int steps, uint32_t lds, Acc &acc, const Wave &w)
    {
        LoaderA la;
        LoaderB lb;
        la.init(A, threadIdx.x);
        lb.init(B, threadIdx.x);
        auto fetch = [&](uint32_t to) {
            la.step();
            lb.step();
#pragma unroll
            for (int j = 0; j < la.N; ++j) la.load(j, to, w.id);
#pragma unroll
            for (int j = 0; j < lb.N; ++j) lb.load(j, to + TA::BYTES, w.id);
        };
        const uint32_t end = lds + STAGES * STAGE;
        uint32_t here = lds, to = lds;
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k, to += STAGE) fetch(to);
        for (int kt = 0; kt < steps; ++kt) {
            arrived<(STAGES - 2) * (la.N + lb.N)>();
            fetch(to);
            half_step(here + w.a_at, here + TA::BYTES + w.b_at, 0, acc);
            half_step(here + w.a_at, here + TA::BYTES + w.b_at, 1, acc);
            here = here + STAGE == end ? lds : here + STAGE;
            to = to + STAGE == end ? lds : to + STAGE;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // (the loads of nothing behind the last step)
    }

    // A step is sixteen groups of four products, eight for each half of its contraction; a group also issues a share of the LDS reads of the
    // next half and every second one a load, so that matrix unit, LDS and load unit have work all the time (eight loads together take the load
    // unit as long as half a step's products).  A's and B's stages of step kt are read by group 3 (barrier) and then hold loads of
    // A's step kt + 3 and B's step kt + 2, which gives A nearly two steps to arrive and B one; the last six loads may be under way when step
    // kt + 1 is looked at (group 8).  At 8192 x 4096 x 16384 in 16 bits a step takes 2490 to 2650 cycles of the 2048 its products need, against
    // 2810 with loads one step ahead, and the clock that the power limit leaves is 1.65 GHz.
    static __device__ __forceinline__ void run_deep(const Operand &A, const Operand &B, int steps, uint32_t lds, Acc &acc, const Wave &w)
    {
        LoaderA la;
        LoaderB lb;
        static_assert(la.N == 4 && lb.N == 4 && MT == 8 && NTL == 4, "loads and reads are dealt to groups for these");
        la.init(A, threadIdx.x);
        lb.init(B, threadIdx.x);
        uint32_t a0 = lds, a1 = lds + TA::BYTES, a2 = lds + 2 * TA::BYTES, b0 = lds + 3 * TA::BYTES, b1 = b0 + TB::BYTES;
        la.step();
        lb.step();
#pragma unroll
        for (int j = 0; j < 4; ++j) la.load(j, a0, w.id);
#pragma unroll
        for (int j = 0; j < 4; ++j) lb.load(j, b0, w.id);
        la.step();
        lb.step();
#pragma unroll
        for (int j = 0; j < 4; ++j) la.load(j, a1, w.id);
#pragma unroll
        for (int j = 0; j < 4; ++j) lb.load(j, b1, w.id);
        la.step();
        la.load(0, a2, w.id);
        la.load(1, a2, w.id);
        arrived<10>();
        Fragments f[2];
        auto read = [&](int half, int a, uint32_t a_at, uint32_t b_at) {
            if (a & 1) f[half].b[a >> 1] = TB::fragment(b_at, a >> 1, half);
            f[half].a[a] = TA::fragment(a_at, a, half);
        };
#pragma unroll
        for (int a = 0; a < 8; ++a) read(0, a, a0 + w.a_at, b0 + w.b_at);
        for (int kt = 0; kt < steps; ++kt) {
#pragma unroll
            for (int g = 0; g < 16; ++g) {
                const int half = g >> 3, a = g & 7;
                if (g == 0) la.load(2, a2, w.id);
                if (g == 2) la.load(3, a2, w.id);
                if (g < 4) {
                    read(1, 2 * g, a0 + w.a_at, b0 + w.b_at);
                    read(1, 2 * g + 1, a0 + w.a_at, b0 + w.b_at);
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
                if (g >= 4 && g <= 10 && g % 2 == 0) lb.load((g - 4) / 2, b0, w.id);
                if (g == 12) {
                    la.step();
                    la.load(0, a0, w.id);
                }
                if (g == 14) la.load(1, a0, w.id);
                if (g >= 8) read(0, a, a1 + w.a_at, b1 + w.b_at);
#pragma unroll
                for (int b = 0; b < 4; ++b) acc[a][b] = mma(f[half].b[b], f[half].a[a], acc[a][b], T{});
                __builtin_amdgcn_sched_barrier(0);
            }
            uint32_t t = a0;
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
