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

// Brings an operand's tiles to LDS.  DIRECT: the load unit writes LDS itself (addresses, strides and the contiguous extent are
// multiples of 16 bytes, so every chunk exists or does not); otherwise through registers, element by element at the edges.
template <class T, int FORM, int R, int NT, bool DIRECT>
struct Loader {
    using TL = Tile<T, FORM, R, NT>;
    static constexpr int N = TL::CHUNKS, ES = TL::ES, BK = TL::BK;
    Operand o;
    int K;                                  // extent of the contraction
    uint32_t off[DIRECT ? N : 1];
    u32x4 held[DIRECT ? 1 : N];

    __device__ __forceinline__ void init(const Operand &op, int k_extent, int tid)
    {
        o = op;
        K = k_extent;
        if constexpr (DIRECT) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                int major, chunk;
                TL::place(j * NT + tid, major, chunk);
                const bool in = FORM == ROWS ? major < o.rows : chunk * (16 / ES) < o.rows;
                off[j] = in ? (uint32_t)(major * (int)o.ld + chunk * 16) : OUT_OF_RANGE;
            }
        }
    }
    // starts the loads of step kt (into LDS at `lds` if DIRECT)
    __device__ __forceinline__ void start(int kt, char *lds, int tid)
    {
        const int k0 = kt * BK, left = K - k0;
        const char *base = o.p + (FORM == ROWS ? (int64_t)k0 * ES : (int64_t)k0 * o.ld);
        if constexpr (DIRECT) {
            // what of the operand lies behind `base`; more than a tile can reach is cut to what a range holds
            const int64_t span = FORM == ROWS ? (int64_t)(o.rows - 1) * o.ld + (int64_t)left * ES
                                              : (int64_t)(left - 1) * o.ld + (int64_t)o.rows * ES;
            const int range = o.rows > 0 ? (int)(span < 0x7fffffffll ? span : 0x7fffffffll) : 0;
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, range, 0x00020000);
            const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                uint32_t v = off[j];
                if (FORM == ROWS) {
                    int major, chunk;
                    TL::place(j * NT + tid, major, chunk);
                    if (left < BK && chunk * (16 / ES) >= left) v = OUT_OF_RANGE;
                }
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (ALPA_LDS void *)(lds + (j * NT + wave * 64) * 16), 16, v, 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                int major, chunk;
                TL::place(j * NT + tid, major, chunk);
                int n = FORM == ROWS ? left - chunk * (16 / ES) : o.rows - chunk * (16 / ES);
                if (FORM == ROWS ? major >= o.rows : major >= left) n = 0;
                held[j] = load_some<T>(base + (int64_t)major * o.ld + chunk * 16, n);
            }
        }
    }
    __device__ __forceinline__ void finish(char *lds, int tid)
    {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int j = 0; j < N; ++j) *(u32x4 *)(lds + (j * NT + tid) * 16) = held[j];
        }
    }
};

// Every load to LDS of this wave has arrived, and every wave is here.
__device__ __forceinline__ void loads_and_barrier()
{
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
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
    static constexpr int STAGE = TA::BYTES + TB::BYTES, LDS_BYTES = 2 * STAGE;

    static __device__ __forceinline__ void run(const Operand &A, const Operand &B, int K, char *lds, f32x4 (&acc)[MT][NTL])
    {
        const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, q = lane >> 4;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int m0 = wave / WN * (BM / WM), n0 = wave % WN * (BN / WN);
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < NTL; ++b) acc[a][b] = f32x4{0, 0, 0, 0};
        Loader<T, FA, BM, NT, DIRECT> la;
        Loader<T, FB, BN, NT, DIRECT> lb;
        la.init(A, K, tid);
        lb.init(B, K, tid);
        const int steps = (K + TA::BK - 1) / TA::BK;
        if (steps == 0) return;
        la.start(0, lds, tid);
        lb.start(0, lds + TA::BYTES, tid);
        la.finish(lds, tid);
        lb.finish(lds + TA::BYTES, tid);
        for (int kt = 0; kt < steps; ++kt) {
            char *here = lds + (kt & 1) * STAGE, *next = lds + (~kt & 1) * STAGE;
            loads_and_barrier();
            if (kt + 1 < steps) {
                la.start(kt + 1, next, tid);
                lb.start(kt + 1, next + TA::BYTES, tid);
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                u32x4 fa[MT], fb[NTL];
#pragma unroll
                for (int b = 0; b < NTL; ++b) fb[b] = TB::fragment(here + TA::BYTES, n0, b, ks, i, q);
#pragma unroll
                for (int a = 0; a < MT; ++a) fa[a] = TA::fragment(here, m0, a, ks, i, q);
#pragma unroll
                for (int a = 0; a < MT; ++a)
#pragma unroll
                    for (int b = 0; b < NTL; ++b) acc[a][b] = mma(fb[b], fa[a], acc[a][b], T{});
            }
            if (kt + 1 < steps) {
                la.finish(next, tid);
                lb.finish(next + TA::BYTES, tid);
            }
        }
    }
};

}  // namespace alpa
