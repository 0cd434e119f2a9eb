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
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c, int, bf16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c, int, f16)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// `parts` instructions make the product: the parts of several go in turn, so that none waits for the one in front.
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c, int j, float)
{
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, a)[j], __builtin_bit_cast(f32x4, b)[j], c, 0, 0, 0);
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
template <class T, class TL, int FORM, int NT, bool FOLLOWED>
struct DirectLoader {
    static constexpr int N = TL::CHUNKS, ES = TL::ES, BK = TL::BK;
    const char *p, *p_next;                 // the next step; the operand that follows
    int64_t advance;
    int ld, rows, left, steps;              // left, steps: of the contraction
    int rows_next, left_next, steps_next;
    // A thread's chunks lie at the same place of rows or steps that are NT / 8 or NT / CPS apart, which are permuted alike; steps of 32-bit
    // elements, eight apart, are so every second time.
    static constexpr int KINDS = FORM == COLS && ES == 4 ? 2 : 1;
    int chunk[KINDS];
    uint32_t first, off[KINDS], apart;      // this thread's first row or step, its first chunks in this step, and how far chunks are apart
    u32x4 range;

    __device__ __forceinline__ void init(int64_t ld_bytes, int tid)
    {
        ld = (int)ld_bytes;
        advance = FORM == ROWS ? BK * ES : BK * ld_bytes;
#pragma unroll
        for (int j = 0; j < KINDS; ++j) {
            int major;
            TL::place(j * NT + tid, major, chunk[j]);
        }
        first = (uint32_t)(TL::first_major(tid) * ld);
        apart = (uint32_t)(ld * (FORM == ROWS ? NT / 8 : NT / TL::CPS));
        steps = 0;
    }
    // The only operand (not FOLLOWED).
    __device__ __forceinline__ void begin(const Operand &o)
    {
        p = o.p;
        rows = o.rows;
        left = o.k;
    }
    // The operand whose first step follows the present one's last: `n` steps, of which those behind its extent are empty.
    __device__ __forceinline__ void follow(const Operand &o, int n)
    {
        p_next = o.p;
        rows_next = o.rows;
        left_next = o.k;
        steps_next = n;
    }
    // Goes to the next step.  The range ends with the last row's (or step's) last byte, so rows and steps that do not exist are behind it; chunks
    // behind a row's end but in front of the next row are cut.
    __device__ __forceinline__ void step()
    {
        if constexpr (FOLLOWED) {
            const bool over = steps == 0;
            p = over ? p_next : p;
            rows = over ? rows_next : rows;
            left = over ? left_next : left;
            steps = (over ? steps_next : steps) - 1;
        }
        const int n = min(left, BK);
        const int span = FORM == ROWS ? (rows - 1) * ld + n * ES : (n - 1) * ld + rows * ES;
        const uint64_t at = (uint64_t)p;
        range = u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, (uint32_t)(rows > 0 && n > 0 ? span : 0), 0x00020000u};
#pragma unroll
        for (int j = 0; j < KINDS; ++j)
            off[j] = chunk[j] * (16 / ES) >= (FORM == ROWS ? n : rows) ? OUT_OF_RANGE : first + chunk[j] * 16;
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
    static constexpr int NT = WM * WN * 64, MT = BM / WM / 16, NTL = BN / WN / 16, ES = sizeof(T), MMA_PARTS = ES == 4 ? 4 : 1;
    using TA = Tile<T, FA, BM, NT, false>;
    using TB = Tile<T, FB, BN, NT, true>;
    // The large tile: three stages of A and two of B, all the LDS there is.  The others: as many stages as leave room for a second workgroup.
    static constexpr bool DEEP = BM == 256;
    using LoaderA = DirectLoader<T, TA, FA, NT, DEEP>;
    using LoaderB = DirectLoader<T, TB, FB, NT, DEEP>;
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
    struct Wave {
        int id;
        uint32_t a_at, b_at;
        __device__ __forceinline__ Wave()
        {
            const int lane = threadIdx.x & 63;
            id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
            a_at = TA::lane_at(id / WN * (BM / WM), lane & 15, lane >> 4);
            b_at = TB::lane_at(id % WN * (BN / WN), lane & 15, lane >> 4);
        }
    };

    // The smaller tiles' share g of four: of the reads of a half step, and of its products.
    static __device__ __forceinline__ void read(uint32_t stage, const Wave &w, int ks, int g, Fragments &f)
    {
        f.b[g] = TB::fragment(stage + TA::BYTES + w.b_at, g, ks);
        if (g < MT) f.a[g] = TA::fragment(stage + w.a_at, g, ks);
    }
    static __device__ __forceinline__ void multiply(const Fragments &f, int g, Acc &acc)
    {
#pragma unroll
        for (int j = 0; j < MMA_PARTS; ++j)
#pragma unroll
            for (int a = 0; a < MT; ++a)
#pragma unroll
                for (int b = 0; b < NTL; ++b)
                    if (g == (MT > 1 ? a : MMA_PARTS > 1 ? j : b)) acc[a][b] = mma(f.b[b], f.a[a], acc[a][b], j, T{});
        __builtin_amdgcn_sched_barrier(0);
    }

    // The smaller tiles.  The products of a step's first half run while its second half is read and the next loads are prepared; then the stage that
    // all have read is loaded again and the next step's first half is read while the products of the second half run.  STAGES - 1 steps' loads
    // are under way, and the other workgroup of the compute unit fills what is left.  Against reads and loads in front of a step's products: one row,
    // 16384 x 4096 in 16 bits, 24 -> 21.5 us (its weights, largely from the caches there, at 6.2 TB/s); 777 x 1001 x 1335 in 32 bits, both products of the
    // backward pass, 80 -> 72, of which 36 are the matrix unit's.
    static __device__ __forceinline__ void run(const Operand &A, const Operand &B, char *lds_memory, Acc &acc)
    {
        static_assert(NTL == 4 && (MT == 1 || MT == 4) && LoaderA::N == LoaderB::N, "reads, loads and products are dealt to four groups for these");
        constexpr int LOADS = LoaderA::N;
        clear(acc);
        const int steps = (max(A.k, B.k) + TA::BK - 1) / TA::BK;
        if (steps <= 0) return;
        const Wave w;
        const uint32_t lds = (uint32_t)(uintptr_t)(ALPA_LDS char *)lds_memory, end = lds + STAGES * STAGE;
        LoaderA la;
        LoaderB lb;
        la.init(A.ld, threadIdx.x);
        lb.init(B.ld, threadIdx.x);
        la.begin(A);
        lb.begin(B);
        auto load = [&](int j, uint32_t to) {
            if (j < LOADS) la.load(j, to, w.id);
            else lb.load(j - LOADS, to + TA::BYTES, w.id);
        };
#pragma unroll
        for (int k = 0; k < STAGES; ++k) {
            la.step();
            lb.step();
#pragma unroll
            for (int j = 0; j < 2 * LOADS; ++j) load(j, lds + k * STAGE);
        }
        arrived<(STAGES - 1) * 2 * LOADS>();
        Fragments first, second;
#pragma unroll
        for (int g = 0; g < 4; ++g) read(lds, w, 0, g, first);
        uint32_t here = lds;
        for (int kt = 0; kt < steps; ++kt) {
            const uint32_t next = here + STAGE == end ? lds : here + STAGE;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                read(here, w, 1, g, second);
                if (g == 1) la.step();
                if (g == 2) lb.step();
                multiply(first, g, acc);
            }
            arrived<(STAGES - 2) * 2 * LOADS>();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
#pragma unroll
                for (int j = g * LOADS / 2; j < (g + 1) * LOADS / 2; ++j) load(j, here);
                read(next, w, 0, g, first);
                multiply(second, g, acc);
            }
            here = next;
        }
        // (the loads of nothing and the reads behind the last step)
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    }

    // The large tile: tile after tile as one row of steps, so that the loads of a tile's first steps are under way during the steps and the
    // epilogue of the tile in front (against one tile a workgroup: ragged rows of 32 experts, 16384 x 8192 x 2048 with z, 770 -> 665 us, 8192 x 16384 x 4096 910
    // -> 881).
    //
    // A step is sixteen groups of four products, eight for each half of its contraction; a group also issues a share of the LDS reads of the
    // next half and every second one a load, so that matrix unit, LDS and load unit have work all the time (eight loads together take the load
    // unit as long as half a step's products).  A's and B's stages of step kt are read by group 3 (barrier) and then hold loads of
    // A's step kt + 3 and B's step kt + 2, which gives A nearly two steps to arrive and B one; the last six loads may be under way when step
    // kt + 1 is looked at (group 8).  At 8192 x 4096 x 16384 in 16 bits a step takes 2490 to 2650 cycles of the 2048 its products need, against
    // 2810 with loads one step ahead, and the clock that the power limit leaves is 1.65 GHz.
    struct Deep {
        static constexpr int LEAST = 3;        // steps of a tile at least: loads run into the next tile, but not past it
        LoaderA la;
        LoaderB lb;
        Wave w;
        uint32_t a0, a1, a2, b0, b1;           // stages: of this step, the next one and the one after that
        Fragments f[2];

        // A stage's first byte plus a lane's place in it, as one opaque value: the reads' constants then go into the instructions and not, added to
        // the lane's place in front of the loop, into registers of their own.
        static __device__ __forceinline__ uint32_t place(uint32_t stage, uint32_t lane)
        {
            uint32_t at;
            asm("v_add_u32 %0, %1, %2" : "=v"(at) : "s"(stage), "v"(lane));
            return at;
        }
        // fragments of group a: a block of rows, and every second time one of columns
        __device__ __forceinline__ void read(int half, int a, uint32_t a_at, uint32_t b_at)
        {
            if (a & 1) f[half].b[a >> 1] = TB::fragment(b_at, a >> 1, half);
            f[half].a[a] = TA::fragment(a_at, a, half);
        }
        // the first tile's operands, `steps` steps
        __device__ __forceinline__ void begin(const Operand &A, const Operand &B, int steps, char *lds_memory)
        {
            static_assert(LoaderA::N == 4 && LoaderB::N == 4 && MT == 8 && NTL == 4, "loads and reads are dealt to groups for these");
            const uint32_t lds = (uint32_t)(uintptr_t)(ALPA_LDS char *)lds_memory;
            a0 = lds;
            a1 = a0 + TA::BYTES;
            a2 = a1 + TA::BYTES;
            b0 = a2 + TA::BYTES;
            b1 = b0 + TB::BYTES;
            la.init(A.ld, threadIdx.x);
            lb.init(B.ld, threadIdx.x);
            la.follow(A, steps);
            lb.follow(B, steps);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                la.step();
                lb.step();
#pragma unroll
                for (int j = 0; j < 4; ++j) la.load(j, k ? a1 : a0, w.id);
#pragma unroll
                for (int j = 0; j < 4; ++j) lb.load(j, k ? b1 : b0, w.id);
            }
            la.step();
            la.load(0, a2, w.id);
            la.load(1, a2, w.id);
            arrived<10>();
#pragma unroll
            for (int a = 0; a < 8; ++a) read(0, a, place(a0, w.a_at), place(b0, w.b_at));
        }
        // One tile's steps; la and lb follow into the next tile's.  (Stores of the tile before may be under way: they only make vmcnt(6) wait
        // for more.)
        __device__ __forceinline__ void run(int steps, Acc &acc)
        {
            clear(acc);
            for (int kt = 0; kt < steps; ++kt) {
                const uint32_t a_here = place(a0, w.a_at), b_here = place(b0, w.b_at), a_next = place(a1, w.a_at), b_next = place(b1, w.b_at);
#pragma unroll
                for (int g = 0; g < 16; ++g) {
                    const int half = g >> 3, a = g & 7;
                    if (g == 0) la.load(2, a2, w.id);
                    if (g == 2) la.load(3, a2, w.id);
                    if (g < 4) {
                        read(1, 2 * g, a_here, b_here);
                        read(1, 2 * g + 1, a_here, b_here);
                    }
                    if (g == 4) {
                        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                        __builtin_amdgcn_s_barrier();
                        asm volatile("" ::: "memory");
                        lb.step();
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    if (g == 8) {
                        asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
                        __builtin_amdgcn_s_barrier();
                        asm volatile("" ::: "memory");
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    if (g >= 4 && g <= 10 && g % 2 == 0) lb.load((g - 4) / 2, b0, w.id);
                    if (g == 12) {
                        la.step();
                        la.load(0, a0, w.id);
                    }
                    if (g == 14) la.load(1, a0, w.id);
                    if (g >= 8) read(0, a, a_next, b_next);
#pragma unroll
                    for (int j = 0; j < MMA_PARTS; ++j)
#pragma unroll
                        for (int b = 0; b < 4; ++b) acc[a][b] = mma(f[half].b[b], f[half].a[a], acc[a][b], j, T{});
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
        }
        // (loads of nothing and reads behind the last tile)
        __device__ __forceinline__ void end() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
    };
};

}  // namespace alpa
