// Attention forward and backward, instantiated per element type (kernels_attention_*.hip).
//
// Everything is computed transposed: a block of 32 keys x 32 rows of scores is K Qt, so that a lane holds 16 keys' scores of one row.  A row's maximum
// and sum are then a lane's own numbers, joined once with the lane that has the row's other 16 keys, and the rounded exponentials are the second operand of
// yt = Vt Pt as they lie in the registers: no weight goes through LDS.  The gradients are built alike: dqt = Kt dRt with a lane per row, dvt = dyt P
// and dkt = Qt dR with a lane per key.
//
// The query heads that share a kv head are rows of one product: packed row r of a sequence's kv head is query r / group, head r % group.
#pragma once
#include "blocks.hpp"
#include "epilogue.hpp"
#include "slots.hpp"

namespace alpa {

using f32x16 = float __attribute__((ext_vector_type(16)));

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.69314718055994531f;

__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c, bf16)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c, f16)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c, float)
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(f32x4, a)[j], __builtin_bit_cast(f32x4, b)[j], c, 0, 0, 0);
    return c;
}

// the row (first operand) that register i of a lane's 32 x 32 block holds
__device__ __forceinline__ int block_row(int i, int h) { return (i >> 2) * 8 + h * 4 + (i & 3); }

// Rows of a head in LDS: 16-byte chunk c of row r lies at place c ^ swz(r), so that both reads are spread over all banks: 32 rows at one chunk
// (products over the head's elements), and four rows at four chunks that follow each other (transposed).
template <class T, int DB>
struct Rows {
    static constexpr int ES = sizeof(T), WIDTH = DB <= 2 ? 64 : DB <= 4 ? 128 : 256, ROWB = WIDTH * ES, CHUNKS = ROWB / 16;
    static constexpr int STEPS = DB * ES;              // 32 bytes of a head: 16 elements of 16 bits, 8 of 32
    static constexpr int PER = ES == 2 ? 16 : 8;       // rows of a transposed fragment
    static constexpr int FRAGS = 32 / PER;

    static __device__ __forceinline__ int swz(int r)
    {
        return CHUNKS == 8 ? ((r >> 1 & 1) << 2) | (r >> 2 & 3) : ((r & 3) << 2) | (r >> 2 & 3);
    }
    static __device__ __forceinline__ uint32_t at(int r, int chunk) { return r * ROWB + ((chunk ^ swz(r)) << 4); }

    // Lane (i, h) = (lane & 31, lane >> 5): row i, bytes 32 step + 16 h of it.
    struct Place {
        uint32_t row, col, col2;
        __device__ __forceinline__ Place()
        {
            const int lane = threadIdx.x & 63, i = lane & 31, h = lane >> 5;
            row = at(i, h);
            if (ES == 2) {
                const int r = 4 * h + ((lane & 15) >> 2), c = 2 * (lane >> 4 & 1) + ((lane & 3) >> 1);
                col = at(r, c) + (lane & 1) * 8;
                col2 = at(r + 8, c) + (lane & 1) * 8;
            } else {
                col = h * 4 * ROWB + (i & 3) * 4;
                col2 = i >> 2;
            }
        }
    };
    // rows row0 + i, step; row0 a multiple of 32
    static __device__ __forceinline__ u32x4 along(const char *lds, const Place &p, int row0, int step)
    {
        return *(const u32x4 *)(lds + ((p.row ^ (step * 32)) + row0 * ROWB));
    }
    // Elements d0 + i (d0 a multiple of 32) of the rows that a lane's fragment `t` of a 32 x 32 block stands for: row0 + block_row(PER / 2 * t + e, h).
    static __device__ __forceinline__ u32x4 across(const char *lds, const Place &p, int row0, int t, int d0)
    {
        if constexpr (ES == 2) {
            const uint32_t from = (uint32_t)(uintptr_t)(const ALPA_LDS char *)lds + (row0 + t * 16) * ROWB;
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ALPA_LDS i16x4 *)(uintptr_t)(from + (p.col ^ (d0 * 2))));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ALPA_LDS i16x4 *)(uintptr_t)(from + (p.col2 ^ (d0 * 2))));
            const u32x2 l = __builtin_bit_cast(u32x2, lo), g = __builtin_bit_cast(u32x2, hi);
            return u32x4{l.x, l.y, g.x, g.y};
        } else {
            u32x4 r;
            const int h = threadIdx.x >> 5 & 1;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int s = (e << 2) | ((2 * t + h) & 3);
                r[e] = *(const uint32_t *)(lds + p.col + (row0 + 8 * t + e) * ROWB + ((((d0 >> 2) + p.col2) ^ s) << 4));
            }
            return r;
        }
    }
    // s + the sum of a fragment's eight values of 16 bits.  (Assembly, as the compiler's builtin read one of the four registers four times; the three wait states
    // that the hardware wants between such a sum and another instruction that uses it are in it.)
    static __device__ __forceinline__ float added(u32x4 f, float s)
    {
        constexpr uint32_t ONES = std::is_same_v<T, bf16> ? 0x3f803f80u : 0x3c003c00u;
        if constexpr (std::is_same_v<T, bf16>)
            asm("v_dot2c_f32_bf16 %0, %1, %5\n\tv_dot2c_f32_bf16 %0, %2, %5\n\tv_dot2c_f32_bf16 %0, %3, %5\n\tv_dot2c_f32_bf16 %0, %4, %5\n\ts_nop 2"
                : "+v"(s) : "v"(f.x), "v"(f.y), "v"(f.z), "v"(f.w), "v"(ONES));
        else
            asm("v_dot2c_f32_f16 %0, %1, %5\n\tv_dot2c_f32_f16 %0, %2, %5\n\tv_dot2c_f32_f16 %0, %3, %5\n\tv_dot2c_f32_f16 %0, %4, %5\n\ts_nop 2"
                : "+v"(s) : "v"(f.x), "v"(f.y), "v"(f.z), "v"(f.w), "v"(ONES));
        return s;
    }
    // A block's values, rounded to the type, as the second operand of fragment t.
    static __device__ __forceinline__ u32x4 packed(const f32x16 &v, int t)
    {
        if constexpr (ES == 2) {
            T e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = (T)v[8 * t + j];
            return __builtin_bit_cast(u32x4, *(i16x8 *)e);
        } else {
            return u32x4{__float_as_uint(v[4 * t]), __float_as_uint(v[4 * t + 1]), __float_as_uint(v[4 * t + 2]), __float_as_uint(v[4 * t + 3])};
        }
    }
    using i16x8 = short __attribute__((ext_vector_type(8)));
};

// acc += (32 rows in LDS from row0 on) x (a fragment a step): reads go ahead of the products by groups of four.
template <class R, class T>
__device__ __forceinline__ void along_product(const char *lds, const typename R::Place &p, int row0, const u32x4 (&b)[R::STEPS], f32x16 &acc)
{
    constexpr int GROUP = 4;
    u32x4 f[2][GROUP];
#pragma unroll
    for (int c = 0; c < GROUP && c < R::STEPS; ++c) f[0][c] = R::along(lds, p, row0, c);
#pragma unroll
    for (int k = 0; k < R::STEPS; k += GROUP) {
#pragma unroll
        for (int c = 0; c < GROUP; ++c)
            if (k + GROUP + c < R::STEPS) f[(k / GROUP + 1) & 1][c] = R::along(lds, p, row0, k + GROUP + c);
#pragma unroll
        for (int c = 0; c < GROUP; ++c)
            if (k + c < R::STEPS) acc = mma32(f[(k / GROUP) & 1][c], b[k + c], acc, T{});
    }
}

// A sequence's share of the tensors.
struct Span {
    int seq;                        // seqs and above: rows of no sequence, seqs + 2: none
    int first, n;                   // its rows
    int r0;                         // a tile's first packed row
    int k_first, m;                 // its keys
    int ahead;                      // m - n: the place of row 0
    int prefix;
};

// group_rows() of slots.hpp; without offsets there is one sequence of all rows
__device__ __forceinline__ void sequence_rows(const int32_t *offsets, int seqs, int rows, int group, int &first, int &end)
{
    if (offsets) return group_rows(offsets, seqs, rows, group, first, end);
    first = 0;
    end = group == 0 ? rows : 0;
}

__device__ __forceinline__ void find_keys(const AttentionArgs &g, Span &s)
{
    s.k_first = s.m = s.prefix = 0;
    if (s.seq < g.seqs) {
        const int32_t *at = g.k_offsets + (int64_t)s.seq * g.k_step;
        const int a = g.k_offsets ? min(max(at[0], 0), g.k_rows) : 0, b = g.k_offsets ? min(max(at[1], 0), g.k_rows) : g.k_rows;
        s.k_first = a;
        s.m = max(b - a, 0);
        if (g.prefix && g.causal) s.prefix = g.prefix[s.seq];
    }
    s.ahead = s.m - s.n;
}

// The index-th run of up to `tile` packed rows of one group of rows (slots.hpp), `group` of them a row.  LAST_FIRST: a sequence's runs from its last one on.
// With a causal mask the last rows have most keys, and the first keys most rows: those go first, and the short ones fill up the end.
template <bool LAST_FIRST>
__device__ __forceinline__ Span find_span(const int32_t *offsets, int seqs, int rows, int group, int tile, int index)
{
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int base = 0; base < seqs + 2; base += 64) {
        int first, end;
        sequence_rows(offsets, seqs, rows, base + lane, first, end);
        const int n = ((end - first) * group + tile - 1) / tile;
        int sum = n;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(sum, off, 64);
            if (lane >= off) sum += o;
        }
        const unsigned long long past = __ballot(before + sum > index);
        if (past) {
            const int l = __ffsll(past) - 1;
            const int f = __builtin_amdgcn_readlane(first, l), e = __builtin_amdgcn_readlane(end, l), count = __builtin_amdgcn_readlane(n, l);
            const int s = before + __builtin_amdgcn_readlane(sum, l) - count;
            if (index < s || index - s >= count) break;          // (offsets that are none)
            return Span{base + l, f, e - f, (LAST_FIRST ? count - 1 - (index - s) : index - s) * tile, 0, 0, 0, 0};
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return Span{seqs + 2, 0, 0, 0, 0, 0, 0, 0};
}

// keys that row `i` of a sequence sees: those in front of this one
__device__ __forceinline__ int limit_of(const AttentionArgs &g, const Span &s, int i)
{
    return min(s.m, g.causal ? max(max(i + s.ahead + 1, s.prefix), 0) : s.m);
}

// A capped score from the product of q and k, in units of the binary logarithm, and the slope of the cap.  1 - tanh(x) = 2 / (1 + exp(2 x)) = 2 u, and the
// slope is 4 u^2 exp(2 x), which keeps its relative error where the cap is reached; tanh is off by a few units of 2^-24 absolute so, and the score by as much of the cap.
// EXACT, for float32 and for caps above 256 (where that would be more than 2^-15 of a weight): the score's error goes with the score.
// The score itself takes the exponential as it is, infinite ones (u = 0) and no numbers among them: a minimum, which gives the other operand for a NaN, may
// only stand in the slope.
template <bool EXACT>
__device__ __forceinline__ float capped(const AttentionArgs &g, float s, float &bent)
{
    if constexpr (EXACT) {
        const float x = s * g.scale / g.cap, u = 1.0f / (1.0f + expf(2.0f * fabsf(x)));
        bent = 4.0f * u * (1.0f - u);
        return g.cap * tanhf(x) * LOG2E;
    } else {
        const float e = __builtin_amdgcn_exp2f(s * g.twice), u = __builtin_amdgcn_rcpf(1.0f + e);
        bent = 4.0f * fminf(e, 0x1p60f) * u * u;
        return fmaf(-2.0f * LOG2E * g.cap, u, LOG2E * g.cap);
    }
}

// The maximum and the sum with the lane that has the row's other half, by exchanging the halves of the wave (through LDS it would take a hundred cycles more).
__device__ __forceinline__ float max_halves(float v)
{
    const u32x2 both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(both.x), __uint_as_float(both.y));
}
__device__ __forceinline__ float add_halves(float v)
{
    const u32x2 both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(both.x) + __uint_as_float(both.y);
}

// Sixteen bytes a lane from memory to LDS, written there by the load unit itself: the wave's go to `lds` and the 1008 bytes behind, in the order of its lanes; those
// whose offset is out of range are zeros.  Assembly without a result register, as in product.hpp: what has arrived is known by counting.  (The hardware wants five
// wait states between a vector instruction that writes a scalar register and a load that reads it, which the compiler does not see: the move and the wait.)
__device__ __forceinline__ void load_chunk(uint32_t lds, uint32_t off, u32x4 range)
{
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"         // (m0 is reserved, and said to be overwritten all the same)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"(range)
                 : "m0");
#pragma clang diagnostic pop
}
// Four of them, `APART` bytes apart in LDS.
template <int APART>
__device__ __forceinline__ void load_chunks(uint32_t lds, uint32_t a, uint32_t b, uint32_t c, uint32_t d, u32x4 range)
{
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
                 "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %5, 0 offen lds\n\t"
                 "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %5, 0 offen lds\n\t"
                 "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, 0 offen lds"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(a), "v"(b), "v"(c), "v"(d), "s"(range), "n"(APART)
                 : "m0", "scc");
#pragma clang diagnostic pop
}
__device__ __forceinline__ u32x4 range_of(const char *p, uint32_t bytes)
{
    const uint64_t at = (uint64_t)p;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(at >> 32) & 0xffffu)),
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}
__device__ __forceinline__ uint32_t lds_at(const char *p) { return (uint32_t)(uintptr_t)(const ALPA_LDS char *)p; }

// The COUNT rows of a tile that follow each other in memory, brought to LDS by NT threads: keys or values.
template <class R, int COUNT, int NT>
struct KeyLoader {
    static constexpr int N = COUNT * R::CHUNKS / NT, APART = NT / R::CHUNKS;          // a thread's chunks are so many rows apart
    static constexpr int KINDS = APART >= 16 ? 1 : 16 / APART < N ? 16 / APART : N;       // and lie at the same place of rows sixteen apart
    static_assert(COUNT * R::CHUNKS % NT == 0 && (APART & (APART - 1)) == 0 && APART > 0, "chunks are dealt evenly");
    const char *p;
    int64_t stride;
    int bytes;
    uint32_t off[KINDS];

    __device__ __forceinline__ KeyLoader(const char *first, int64_t row, int head_bytes) : p(first), stride(row), bytes(head_bytes)
    {
        const int t = threadIdx.x % NT;
#pragma unroll
        for (int j = 0; j < KINDS; ++j) {
            const int r = t / R::CHUNKS + j * APART, chunk = (t % R::CHUNKS) ^ R::swz(r);
            off[j] = chunk * 16 < bytes ? (uint32_t)(r * (int)row + chunk * 16) : OUT_OF_RANGE;
        }
    }
    // rows j0 .. of which those from `end` on do not exist
    __device__ __forceinline__ void load(uint32_t lds, int j0, int end) const
    {
        const int rows = min(end - j0, COUNT);
        const u32x4 range = range_of(p + j0 * stride, rows > 0 ? (uint32_t)((rows - 1) * (int)stride + bytes) : 0u);
        const uint32_t to = lds + __builtin_amdgcn_readfirstlane(threadIdx.x % NT / 64) * 1024;
        const auto from = [&](int j) { return off[j % KINDS] + (uint32_t)(j / KINDS * KINDS * APART * (int)stride); };
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int j = 0; j < N; j += 4) load_chunks<NT * 16>(to + j * NT * 16, from(j), from(j + 1), from(j + 2), from(j + 3), range);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) load_chunk(to + j * NT * 16, from(j), range);
        }
    }
};

// COUNT packed rows of two tensors of queries.
template <class R, int COUNT, int NT>
struct PackedLoader {
    static constexpr int N = COUNT * R::CHUNKS / NT, APART = NT / R::CHUNKS;
    static_assert(COUNT * R::CHUNKS % NT == 0, "chunks are dealt evenly");
    const char *a, *b;              // the kv head's first head of the sequence's row 0
    int a_row, a_head, b_row, b_head, group, bytes;
    int64_t a_long, b_long;
    uint32_t inverse;

    __device__ __forceinline__ PackedLoader(const AttentionArgs &g, const Heads &x, const Heads &y, int first, int kv)
        : a(x.p + (int64_t)first * x.row + (int64_t)kv * g.group * x.head), b(y.p + (int64_t)first * y.row + (int64_t)kv * g.group * y.head), a_row((int)x.row),
          a_head((int)x.head), b_row((int)y.row), b_head((int)y.head), group(g.group), bytes(g.bytes), a_long(x.row), b_long(y.row),
          inverse(0xffffffffu / (uint32_t)g.group + 1)
    {
    }
    // packed row r0 + t as row and head of the group
    __device__ __forceinline__ void place(int r0, int t, int &row, int &head) const
    {
        const int i0 = r0 / group, x = r0 - i0 * group + t, i = group == 1 ? x : (int)__umulhi((uint32_t)x, inverse);
        row = i0 + i;
        head = x - i * group;
    }
    __device__ __forceinline__ void load(uint32_t a_lds, uint32_t b_lds, int r0, int end) const
    {
        const int i0 = r0 / group, rest = r0 - i0 * group, t = threadIdx.x % NT;
        const u32x4 ra = range_of(a + i0 * a_long, 0x7fffffffu), rb = range_of(b + i0 * b_long, 0x7fffffffu);
        const uint32_t to = __builtin_amdgcn_readfirstlane(t / 64) * 1024;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int r = t / R::CHUNKS + j * APART, chunk = (t % R::CHUNKS) ^ R::swz(r);
            // (a quotient of at most 4160 by at most 4096; one head a row: the inverse has no room)
            const int x = rest + r, i = group == 1 ? x : (int)__umulhi((uint32_t)x, inverse), h = x - i * group;
            const bool here = r0 + r < end && chunk * 16 < bytes;
            load_chunk(a_lds + to + j * NT * 16, here ? (uint32_t)(i * a_row + h * a_head + chunk * 16) : OUT_OF_RANGE, ra);
            load_chunk(b_lds + to + j * NT * 16, here ? (uint32_t)(i * b_row + h * b_head + chunk * 16) : OUT_OF_RANGE, rb);
        }
    }
};

// Fragments that are waited for here: to the compiler a load is under way until its register is used, which is in the loop, where it would wait for the loads to
// LDS as well (a tenth of a forward pass's time).
template <int N>
__device__ __forceinline__ void settle(const u32x4 (&f)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("" ::"v"(f[k]));
}

// Where packed row r of a sequence's kv head lies in a tensor of queries.
__device__ __forceinline__ const char *packed_row(const AttentionArgs &g, const Heads &t, const Span &s, int kv, int r)
{
    const int i = r / g.group;
    return t.p + (int64_t)(s.first + i) * t.row + (int64_t)(kv * g.group + r - i * g.group) * t.head;
}
__device__ __forceinline__ int64_t packed_item(const AttentionArgs &g, const Span &s, int kv, int r)
{
    const int i = r / g.group;
    return (int64_t)(s.first + i) * g.heads + kv * g.group + r - i * g.group;
}

// The results of one row or key, times `by`, as a lane holds them of each block; `at` the head's first element.  With several waves that have the same rows
// (WAVES) each writes every so-many-th block.
template <class T, int DB, int WAVES = 1>
__device__ __forceinline__ void store_head(char *at, const f32x16 (&acc)[DB], float by, int dim, int wide)
{
    const int h = threadIdx.x >> 5 & 1, wave = WAVES > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (WAVES > 1 && b % WAVES != wave) continue;
            const int d = b * 32 + j * 8 + h * 4;
            const float v[4] = {acc[b][4 * j] * by, acc[b][4 * j + 1] * by, acc[b][4 * j + 2] * by, acc[b][4 * j + 3] * by};
            if (d < dim) store_row<T>(at, d, dim - d, wide, v);
        }
}

template <int DB>
__device__ __forceinline__ void clear(f32x16 (&acc)[DB])
{
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[b][j] = 0.0f;
}

struct Nothing {
    __device__ __forceinline__ void operator()() const {}
};

// One row a lane, twice: what has been seen of the keys so far.
template <class T, int DB, bool EXTRA, bool FAR_CAP>
struct Running {
    using R = Rows<T, DB>;
    static constexpr bool EXACT = sizeof(T) == 4 || FAR_CAP;
    u32x4 q[R::STEPS];
    f32x16 y[DB];
    float top, sum;                 // in units of the binary logarithm; of this lane's half of the keys
    // The sum of the exponentials as they were rounded for the product with v, which y is divided by: with few keys that count the roundings of a sum and of
    // its weights cancel then (one key: none is left).  lse takes the sum of those that were not rounded.
    float rounded;
    int limit, place;
    float slope;

    __device__ __forceinline__ void begin(const AttentionArgs &g, const Span &s, int kv, int r)
    {
        const int h = threadIdx.x >> 5 & 1, last = s.n * g.group - 1, i = min(r, last);
        const char *p = packed_row(g, g.q, s, kv, i);
#pragma unroll
        for (int k = 0; k < R::STEPS; ++k) {
            const int at = k * 32 + h * 16;
            q[k] = at < g.bytes ? *(const u32x4 *)(p + at) : u32x4{0, 0, 0, 0};
        }
        settle(q);
        clear(y);
        top = -INFINITY;
        sum = rounded = 0.0f;
        limit = limit_of(g, s, i / g.group);
        place = i / g.group + s.ahead;
        slope = EXTRA && g.slopes ? g.slopes[kv * g.group + i % g.group] * LOG2E : 0.0f;
        asm volatile("" ::"v"(slope));
    }

    // Float16 has exponentials up to 2^15, and 2^-14 as its smallest normal number: with 2^12 for the largest one, weights of 2^-26 of it keep their bits (with 1, those
    // below 2^-25 were zeros, however many).
    static constexpr float LEAD = std::is_same_v<T, f16> ? 3.0f : 8.0f, ROOM = std::is_same_v<T, f16> ? 12.0f : 0.0f;

    // The fragments that products of 16-bit types read go through two sets of DB registers of four, in the order of their use: a set is read from LDS
    // while the products of the other one run (read as they were needed, a product waited for LDS three times as long as it takes).
    static constexpr bool AHEAD = sizeof(T) == 2 && DB <= 4;

    // NB blocks of 32 keys from j0 on; `between` runs once the keys have been read and before the values are
    template <int NB, class Between = Nothing>
    __device__ __forceinline__ void step(const AttentionArgs &g, const char *k_lds, const char *v_lds, const typename R::Place &p, int j0, const Between &between = {})
    {
        static_assert(!AHEAD || std::is_same<Between, Nothing>::value, "the values are read among the keys");
        const int h = threadIdx.x >> 5 & 1;
        f32x16 s[NB];
        clear(s);
        u32x4 f[2][DB];
        const auto k_read = [&](int n) {                           // the n-th set of DB steps
#pragma unroll
            for (int c = 0; c < DB; ++c) f[n & 1][c] = R::along(k_lds, p, n / 2 * 32, n % 2 * DB + c);
        };
        const auto v_read = [&](int n) {                           // the n-th fragment of a block's weights, all blocks of y
#pragma unroll
            for (int c = 0; c < DB; ++c) f[n & 1][c] = R::across(v_lds, p, n / 2 * 32, n % 2, c * 32);
        };
        if constexpr (AHEAD) {
            k_read(0);
#pragma unroll
            for (int n = 0; n < 2 * NB; ++n) {
                if (n + 1 < 2 * NB) k_read(n + 1);
                else v_read(0);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int c = 0; c < DB; ++c) s[n / 2] = mma32(f[n & 1][c], q[n % 2 * DB + c], s[n / 2], T{});
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int k = 0; k < R::STEPS; ++k) s[b] = mma32(R::along(k_lds, p, b * 32, k), q[k], s[b], T{});
            between();
        }
        const float by = EXTRA ? 1.0f : g.scale * LOG2E;
        if constexpr (EXTRA) {
            float bent;
            const float far = (float)(place - j0 - 4 * h);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (g.cap != 0.0f) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] = capped<EXACT>(g, s[b][i], bent);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] *= g.scale * LOG2E;
                }
                if (g.slopes) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] = fmaf(-slope, fabsf(far - (float)(b * 32 + block_row(i, 0))), s[b][i]);
                }
            }
        }
        if (__any(j0 + NB * 32 > limit)) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = j0 + b * 32 + block_row(i, h) < limit ? s[b][i] : -INFINITY;
        }
        float most = s[0][0];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, s[b][i]);
        most = max_halves(most) * by;
        // Exponents are taken from a reference, ROOM below a maximum, that follows the maximum once that is LEAD ahead: exponentials up to 2^(LEAD + ROOM) round to the type like
        // those up to 1
        if (__any(most > top + (LEAD + ROOM))) {
            const float next = fmaxf(top, most - ROOM), down = exp2f(top - (next == -INFINITY ? 0.0f : next));
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) y[b][i] *= down;
            sum *= down;
            rounded *= down;
            top = next;
        }
        const float ref = top == -INFINITY ? 0.0f : top;
        if constexpr (AHEAD) {
            // the exponentials of the next eight keys go between the products of these
            const auto weigh = [&](int n, int from, int to) {
#pragma unroll
                for (int i = from; i < to; ++i) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(s[n / 2][n % 2 * 8 + i], by, -ref));
                    s[n / 2][n % 2 * 8 + i] = e;
                    sum += e;
                }
            };
            weigh(0, 0, 8);
#pragma unroll
            for (int n = 0; n < 2 * NB; ++n) {
                const u32x4 w = R::packed(s[n / 2], n % 2);
                rounded = R::added(w, rounded);
                if (n + 1 < 2 * NB) v_read(n + 1);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    y[d] = mma32(f[n & 1][d], w, y[d], T{});
                    if (n + 1 < 2 * NB) weigh(n + 1, d * 8 / DB, (d + 1) * 8 / DB);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        } else {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], by, -ref));
                    sum += s[b][i];
                }
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int t = 0; t < R::FRAGS; ++t) {
                    const u32x4 w = R::packed(s[b], t);
                    if constexpr (sizeof(T) == 2) rounded = R::added(w, rounded);
#pragma unroll
                    for (int d = 0; d < DB; ++d) y[d] = mma32(R::across(v_lds, p, b * 32, t, d * 32), w, y[d], T{});
                }
        }
    }

    // what makes of the sum over the rounded exponentials one over all
    __device__ __forceinline__ float evened() const
    {
        if constexpr (sizeof(T) == 4) return 1.0f;
        const float all = add_halves(sum), r = add_halves(rounded);
        return r > 0.0f ? all / r : 1.0f;
    }

    // y and lse, or this part of them
    template <int WAVES = 1>
    __device__ __forceinline__ void end(const AttentionArgs &g, const Span &s, int kv, int r, int part, int parts)
    {
        const float all = add_halves(sum), even = WAVES > 1 ? 1.0f : evened();      // (of several waves that has been done)
        if (r >= s.n * g.group) return;
        const int64_t item = packed_item(g, s, kv, r);
        const bool first = (threadIdx.x & (WAVES > 1 ? ~31u : 32u)) == 0;
        if (parts > 1) {
            const int64_t at = (int64_t)part * g.rows * g.heads + item;
            store_head<float, DB, WAVES>((char *)(g.part + at * g.dim), y, even, g.dim, (g.dim & 3) == 0);
            if (first) g.stat[at] = make_float2(top, all);
            return;
        }
        char *out = (char *)packed_row(g, g.out, s, kv, r);
        store_head<T, DB, WAVES>(out, y, all == 0.0f ? 0.0f : even / all, g.dim, g.wide);
        if (g.lse && first) g.lse[item] = all == 0.0f ? -INFINITY : (top + log2f(all)) * LN2;
    }
};

// zeros for rows that belong to no sequence, packed rows r0 .. r0 + count - 1
template <class T>
__device__ __forceinline__ void no_rows(const AttentionArgs &g, const Heads &out, const Span &s, int kv, int r0, int count, float *lse)
{
    for (int r = r0 + (threadIdx.x >> 6); r < min(r0 + count, s.n * g.group) && blockIdx.y == 0; r += blockDim.x >> 6) {
        T *to = (T *)packed_row(g, out, s, kv, r);
        for (int d = threadIdx.x & 63; d < g.dim; d += 64) to[d] = (T)0.0f;
        if (lse && (threadIdx.x & 63) == 0) lse[packed_item(g, s, kv, r)] = -INFINITY;
    }
}

// The keys that a tile of rows sees, `most`, and the parts they are dealt in: of a causal sequence the last rows have most keys, and their tiles alone would be
// what the call waits for; of one new token a tile is all there is.  Parts are `chunk` keys, an even share of the sequence's in steps of the
// kernel, so that a tile with few
// keys is one part and needs no join.
struct KeyParts {
    int most, chunk, count;

    // the tile's packed rows are those from s.r0 on, `rows` at most
    __device__ __forceinline__ KeyParts(const AttentionArgs &g, const Span &s, int rows)
    {
        most = limit_of(g, s, (min(s.r0 + rows, s.n * g.group) - 1) / g.group);
        chunk = max(((s.m + g.unit - 1) / g.unit + g.splits - 1) / g.splits, 1) * g.unit;
        count = max((most + chunk - 1) / chunk, 1);
    }
};

// Many rows: a wave has 32 packed rows, the waves share tiles of keys, of which one is worked on and the next one under way.
template <class T, int DB, bool EXTRA, int WAVES, bool FAR_CAP>
__global__ __launch_bounds__(WAVES * 64, 2) void attention_kernel(const AttentionArgs g)
{
    using R = Rows<T, DB>;
    constexpr int KEYS = R::ROWB <= 256 ? 64 : 32, NT = WAVES * 64, HALF = KEYS * R::ROWB;
    __shared__ __align__(1024) char lds[4 * HALF];
    const int kv = (int)((blockIdx.x + g.before) % g.kv_heads);
    Span s = find_span<true>(g.offsets, g.seqs, g.rows, g.group, WAVES * 32, (int)((blockIdx.x + g.before) / g.kv_heads));
    if (s.seq >= g.seqs) {
        if (s.n > 0) no_rows<T>(g, g.out, s, kv, s.r0, WAVES * 32, g.lse);
        return;
    }
    find_keys(g, s);
    const KeyParts part(g, s, WAVES * 32);
    const int index = g.splits - 1 - (int)blockIdx.y, from = index * part.chunk, to = min(from + part.chunk, part.most);
    if (index >= part.count) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = s.r0 + wave * 32 + (threadIdx.x & 31);
    const KeyLoader<R, KEYS, NT> k(g.k.p + (int64_t)s.k_first * g.k.row + (int64_t)kv * g.k.head, g.k.row, g.bytes);
    const KeyLoader<R, KEYS, NT> v(g.v.p + (int64_t)s.k_first * g.v.row + (int64_t)kv * g.v.head, g.v.row, g.bytes);
    uint32_t here = 0;
    if (from < to) {
        k.load(lds_at(lds), from, s.m);
        v.load(lds_at(lds) + HALF, from, s.m);
    }
    Running<T, DB, EXTRA, FAR_CAP> run;
    run.begin(g, s, kv, r);
    const typename R::Place place;
    const int mine = __builtin_amdgcn_readlane(run.limit, 31);
    for (int j0 = from; j0 < to; j0 += KEYS, here ^= 2 * HALF) {
        arrived<0>();
        if (j0 + KEYS < to) {
            k.load(lds_at(lds) + (here ^ 2 * HALF), j0 + KEYS, s.m);
            v.load(lds_at(lds) + (here ^ 2 * HALF) + HALF, j0 + KEYS, s.m);
        }
        if (j0 < mine) run.template step<KEYS / 32>(g, lds + here, lds + here + HALF, place, j0);
    }
    run.end(g, s, kv, r, index, part.count);
}

// A workgroup's rows: one tile of a sequence's (g.tiles of them), or all rows of one sequence, without a search; the rows of none are one sequence more then,
// with those in front of the first sequence in `other`.
struct Share {
    Span s, other;
    int begin, end;

    __device__ __forceinline__ Share(const AttentionArgs &g, int tile)
    {
        const int index = (int)((blockIdx.x + g.before) / g.kv_heads);
        if (g.tiles) {
            s = find_span<true>(g.offsets, g.seqs, g.rows, g.group, tile, index);
            begin = s.r0;
            end = min(s.r0 + tile, s.n * g.group);
            return;
        }
        const auto rows_of = [&](int k, Span &to) {
            int last;
            sequence_rows(g.offsets, g.seqs, g.rows, k, to.first, last);
            to.seq = k;
            to.n = last - to.first;
            to.r0 = 0;
        };
        rows_of(index, s);
        if (index == g.seqs) rows_of(index + 1, other);
        begin = 0;
        end = s.n * g.group;
    }
};

// Few rows: the waves of a workgroup have the same 32 packed rows and take tiles of 32 keys in turn, each from its own part of LDS; in the end their sums
// are joined.  A wave has room for two tiles of keys and two of values; or, where rows are wide (STAGES 1), for one, so that there are twice as many waves: the
// next keys are under way while the values are worked on, and the other way round (32 bits, heads of 75: y 43 and 28 us, dq 53 and 36; of 128, 64 rows on 2048
// keys each: 170 and 111; 16 bits, heads of 256, a row on 4095 keys: 41 and 29).
template <class T, int DB>
struct FewShape {
    using R = Rows<T, DB>;
    static constexpr int STAGES = R::ROWB <= 256 ? 2 : 1, WAVES = R::ROWB <= 512 ? 4 : 2, TILE = 32 * R::ROWB, LDS = WAVES * STAGES * 2 * TILE;
    using Loader = KeyLoader<R, 32, 64>;
};

// Waits until the loads have arrived that came before the last LEFT, and what was asked of LDS.
template <int LEFT>
__device__ __forceinline__ void arrived_but()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
}

// A wave's tiles of 32 keys, each with room for one tile of `a` and one of `b`: work(j0, between) reads `a`, calls between, and reads `b` (or `a` no more
// before it ends).  Both loads of the first tile are under way.
template <class Loader, class Work>
__device__ __forceinline__ void in_turn(const Loader &a, uint32_t a_lds, const Loader &b, uint32_t b_lds, int j0, int to, int apart, int end, const Work &work)
{
    for (; j0 < to; j0 += apart) {
        const int next = j0 + apart;
        arrived_but<Loader::N>();
        work(j0, [&] {
            // (a's reads have ended before its place is written to)
            arrived_but<63>();
            if (next < to) {
                a.load(a_lds, next, end);
                arrived_but<Loader::N>();
            } else {
                arrived_but<0>();
            }
        });
        arrived_but<63>();
        if (next < to) b.load(b_lds, next, end);
    }
}

// Adds up the waves' blocks, each times `by`: a wave has every so-many-th one then.  What was in LDS has been read; the sums' 16 KB a wave for heads of 128 lie in the
// room of the tiles.
template <int WAVES, int DB>
__device__ __forceinline__ void join_waves(char *lds, f32x16 (&acc)[DB], float by)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    f32x4 *const all = (f32x4 *)lds + (threadIdx.x & 63), *const mine = all + wave * DB * 256;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[(b * 4 + i) * 64] = f32x4{acc[b][4 * i] * by, acc[b][4 * i + 1] * by, acc[b][4 * i + 2] * by, acc[b][4 * i + 3] * by};
    __syncthreads();
#pragma unroll
    for (int b = 0; b < DB; ++b) {
        if (b % WAVES != wave) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v += all[(w * DB * 4 + b * 4 + i) * 64];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[b][4 * i + j] = v[j];
        }
    }
}

template <class T, int DB, bool EXTRA, bool FAR_CAP>
__global__ __launch_bounds__((FewShape<T, DB>::WAVES * 64)) void attention_few_kernel(const AttentionArgs g)
{
    using F = FewShape<T, DB>;
    using R = Rows<T, DB>;
    constexpr int WAVES = F::WAVES;
    __shared__ __align__(1024) char lds[F::LDS];
    __shared__ float tops[WAVES][32], sums[WAVES][32];
    const int kv = (int)((blockIdx.x + g.before) % g.kv_heads), lane = threadIdx.x & 63;
    const Share share(g, 32);
    Span s = share.s;
    if (s.seq >= g.seqs) {
        no_rows<T>(g, g.out, s, kv, share.begin, share.end - share.begin, g.lse);
        if (s.seq == g.seqs && !g.tiles) no_rows<T>(g, g.out, share.other, kv, 0, share.other.n * g.group, g.lse);
        return;
    }
    find_keys(g, s);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const typename R::Place place;
    const char *const own = lds + wave * F::STAGES * 2 * F::TILE;
    const uint32_t mine = lds_at(lds) + wave * F::STAGES * 2 * F::TILE;
    const typename F::Loader k(g.k.p + (int64_t)s.k_first * g.k.row + (int64_t)kv * g.k.head, g.k.row, g.bytes);
    const typename F::Loader v(g.v.p + (int64_t)s.k_first * g.v.row + (int64_t)kv * g.v.head, g.v.row, g.bytes);
    for (int r0 = share.begin; r0 < share.end; r0 += 32) {
        const int r = r0 + (lane & 31);
        s.r0 = r0;
        const KeyParts part(g, s, 32);
        const int index = g.splits - 1 - (int)blockIdx.y, from = index * part.chunk, to = min(from + part.chunk, part.most);
        if (index >= part.count) continue;
        // each wave waits for its own loads alone
        const int j1 = from + wave * 32;
        __syncthreads();                                   // (the rows before are done with)
        if (j1 < to) {
            k.load(mine, j1, s.m);
            v.load(mine + F::TILE, j1, s.m);
        }
        Running<T, DB, EXTRA, FAR_CAP> run;
        run.begin(g, s, kv, r);
        if constexpr (F::STAGES == 1) {
            in_turn(k, mine, v, mine + F::TILE, j1, to, 32 * WAVES, s.m, [&](int j0, auto between) { run.template step<1>(g, own, own + F::TILE, place, j0, between); });
        } else {
            uint32_t here = 0;
            for (int j0 = j1; j0 < to; j0 += 32 * WAVES, here ^= 2 * F::TILE) {
                arrived_but<0>();
                if (j0 + 32 * WAVES < to) {
                    k.load(mine + (here ^ 2 * F::TILE), j0 + 32 * WAVES, s.m);
                    v.load(mine + (here ^ 2 * F::TILE) + F::TILE, j0 + 32 * WAVES, s.m);
                }
                run.template step<1>(g, own + here, own + here + F::TILE, place, j0);
            }
        }
        if constexpr (WAVES > 1) {
            // the waves' sums, each brought to the common maximum; wave 0 goes on with them
            __syncthreads();
            const float all = add_halves(run.sum);
            if (lane < 32) {
                tops[wave][lane] = run.top;
                sums[wave][lane] = all;
            }
            __syncthreads();
            float top = tops[0][lane & 31];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) top = fmaxf(top, tops[w][lane & 31]);
            const float ref = top == -INFINITY ? 0.0f : top, down = exp2f(run.top - ref);
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) total += sums[w][lane & 31] * exp2f(tops[w][lane & 31] - ref);
            join_waves<WAVES>(lds, run.y, down * run.evened());
            run.top = top;
            run.sum = (threadIdx.x & 32) ? 0.0f : total;
        }
        run.template end<WAVES>(g, s, kv, r, index, part.count);
    }
}

// The packed rows that see a tile's keys, and the parts they are dealt in: of a causal sequence the first keys have most rows, and their tiles alone would
// be what the call waits for.  Parts are `chunk` rows, counted from the last one, so that a tile with few rows is one part and needs no join.
struct RowParts {
    int all, begin, chunk, count;

    // `s` as find_span() gives it for keys; it is turned into rows and keys
    __device__ __forceinline__ RowParts(const AttentionArgs &g, Span &s, int key0)
    {
        s.k_first = s.first;
        s.m = s.n;
        int first, stop;
        sequence_rows(g.offsets, g.seqs, g.rows, s.seq, first, stop);
        s.first = first;
        s.n = stop - first;
        s.ahead = s.m - s.n;
        s.prefix = g.prefix && g.causal ? g.prefix[s.seq] : 0;
        all = s.n * g.group;
        // row i sees key j in front of the prefix or where j <= i + ahead
        begin = !g.causal || key0 < s.prefix ? 0 : min(max(key0 - s.ahead, 0), s.n) * g.group;
        chunk = max((all + g.splits * 32 - 1) / (g.splits * 32) * 32, 32);
        count = (all - begin + chunk - 1) / chunk;
    }
};

// In float16 dR has neither room for large gradients nor bits for small ones.  A lane's dR are kept times a power of two (its row's, or its key's), found from
// the largest |dR| so far; when a larger one comes, what has been summed is brought to the new one.  The two lanes of a row go together.
template <class T, int DB>
__device__ __forceinline__ void keep_in_range(f32x16 &d, f32x16 (&acc)[DB], float &by)
{
    if constexpr (std::is_same_v<T, f16>) {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(d[i]));
        most = max_halves(most);
        most = most < INFINITY ? most : 0.0f;
        if (__any(most * by > 32768.0f)) {
            // the new factor leaves room for 2^4 more
            int e;
            (void)frexpf(most, &e);
            const float next = most * by > 32768.0f ? ldexpf(1.0f, max(11 - e, -100)) : by, down = next / by;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[b][i] *= down;
            by = next;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) d[i] *= by;
    }
}
template <class T>
__device__ __forceinline__ float first_factor() { return std::is_same_v<T, f16> ? 0x1p60f : 1.0f; }

// One row a lane, twice: what of its gradient the keys so far have given; the sum of dy y on the way.
template <class T, int DB, bool EXTRA, bool FAR_CAP>
struct Backward {
    using R = Rows<T, DB>;
    static constexpr bool EXACT = sizeof(T) == 4 || FAR_CAP;
    u32x4 q[R::STEPS], dy[R::STEPS];
    f32x16 dq[DB];
    float delta, lse, slope, by;
    int limit, where;

    __device__ __forceinline__ void begin(const AttentionArgs &g, const Span &s, int kv, int r)
    {
        const int h = threadIdx.x >> 5 & 1, i = min(r, s.n * g.group - 1);          // (of several parts each puts down the sum of dy y, the same bits)
        const char *qp = packed_row(g, g.q, s, kv, i), *dp = packed_row(g, g.dy, s, kv, i), *yp = packed_row(g, g.y, s, kv, i);
        delta = 0.0f;
#pragma unroll
        for (int k = 0; k < R::STEPS; ++k) {
            const int at = k * 32 + h * 16;
            const bool here = at < g.bytes;
            const u32x4 none = {0, 0, 0, 0}, y = here ? *(const u32x4 *)(yp + at) : none;
            q[k] = here ? *(const u32x4 *)(qp + at) : none;
            dy[k] = here ? *(const u32x4 *)(dp + at) : none;
            T a[16 / sizeof(T)], b[16 / sizeof(T)];
            __builtin_memcpy(a, &dy[k], 16);
            __builtin_memcpy(b, &y, 16);
#pragma unroll
            for (int j = 0; j < (int)(16 / sizeof(T)); ++j) delta += (float)a[j] * (float)b[j];
        }
        settle(q);
        settle(dy);
        delta = add_halves(delta);
        const int64_t item = packed_item(g, s, kv, i);
        if (h == 0 && r == i) g.delta[item] = delta;
        lse = g.lse[item] * LOG2E;
        lse = lse == -INFINITY ? INFINITY : lse;           // (no key seen: all exponentials are zero)
        limit = limit_of(g, s, i / g.group);
        where = i / g.group + s.ahead;
        slope = EXTRA && g.slopes ? g.slopes[kv * g.group + i % g.group] * LOG2E : 0.0f;
        by = first_factor<T>();
        asm volatile("" ::"v"(lse), "v"(slope));
        clear(dq);
    }

    // 32 keys from j0 on, in LDS from row `at` on; `between`, if there is one, runs once the values have been read and before the keys are
    template <class Between = Nothing>
    __device__ __forceinline__ void step(const AttentionArgs &g, const char *k_lds, const char *v_lds, const typename R::Place &place, int j0, int at,
                                         const Between &between = {})
    {
        const int h = threadIdx.x >> 5 & 1;
        f32x16 a, d;
#pragma unroll
        for (int j = 0; j < 16; ++j) a[j] = d[j] = 0.0f;
        if constexpr (std::is_same<Between, Nothing>::value) {
            along_product<R, T>(k_lds, place, at, q, a);
            along_product<R, T>(v_lds, place, at, dy, d);
        } else {
            along_product<R, T>(v_lds, place, at, dy, d);
            between();
            along_product<R, T>(k_lds, place, at, q, a);
        }
        const float by_log = EXTRA ? 1.0f : g.scale * LOG2E;
        if constexpr (EXTRA) {
            if (g.cap != 0.0f) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    float bent;
                    a[j] = capped<EXACT>(g, a[j], bent);
                    d[j] = (d[j] - delta) * bent;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    a[j] *= g.scale * LOG2E;
                    d[j] -= delta;
                }
            }
            if (g.slopes) {
                const float far = (float)(where - j0 - 4 * h);
#pragma unroll
                for (int j = 0; j < 16; ++j) a[j] = fmaf(-slope, fabsf(far - (float)block_row(j, 0)), a[j]);
            }
        }
        if (__any(j0 + 32 > limit)) {
#pragma unroll
            for (int j = 0; j < 16; ++j) a[j] = j0 + block_row(j, h) < limit ? a[j] : -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float p = __builtin_amdgcn_exp2f(fmaf(a[j], by_log, -lse));
            d[j] = p * (EXTRA ? d[j] : d[j] - delta);
        }
        keep_in_range<T>(d, dq, by);
#pragma unroll
        for (int t = 0; t < R::FRAGS; ++t) {
            const u32x4 w = R::packed(d, t);
#pragma unroll
            for (int b = 0; b < DB; ++b) dq[b] = mma32(R::across(k_lds, place, at, t, b * 32), w, dq[b], T{});
        }
    }

    template <int WAVES = 1>
    __device__ __forceinline__ void end(const AttentionArgs &g, const Span &s, int kv, int r, float scale, int part, int parts)
    {
        if (r >= s.n * g.group) return;
        if (parts > 1) store_head<float, DB, WAVES>((char *)(g.part + ((int64_t)part * g.rows * g.heads + packed_item(g, s, kv, r)) * g.dim), dq, scale, g.dim, (g.dim & 3) == 0);
        else store_head<T, DB, WAVES>((char *)packed_row(g, g.out, s, kv, r), dq, scale, g.dim, g.wide);
    }
};

// dq of many rows: a wave has 32 packed rows, the waves share tiles of keys.
template <class T, int DB, bool EXTRA, int WAVES, bool FAR_CAP>
__global__ __launch_bounds__(WAVES * 64, sizeof(T) == 2 && DB <= 4 ? 2 : 1) void attention_dq_kernel(const AttentionArgs g)
{
    using R = Rows<T, DB>;
    constexpr int KEYS = R::ROWB <= 256 ? 64 : 32, NT = WAVES * 64, HALF = KEYS * R::ROWB;
    __shared__ __align__(1024) char lds[4 * HALF];
    const int kv = (int)((blockIdx.x + g.before) % g.kv_heads), lane = threadIdx.x & 63;
    Span s = find_span<true>(g.offsets, g.seqs, g.rows, g.group, WAVES * 32, (int)((blockIdx.x + g.before) / g.kv_heads));
    if (s.seq >= g.seqs) {
        if (s.n > 0 && g.out.p) no_rows<T>(g, g.out, s, kv, s.r0, WAVES * 32, nullptr);
        return;
    }
    find_keys(g, s);
    const KeyParts part(g, s, WAVES * 32);
    const int index = g.splits - 1 - (int)blockIdx.y, from = index * part.chunk, to = min(from + part.chunk, part.most);
    if (index >= part.count) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = s.r0 + wave * 32 + (lane & 31);
    const KeyLoader<R, KEYS, NT> k(g.k.p + (int64_t)s.k_first * g.k.row + (int64_t)kv * g.k.head, g.k.row, g.bytes);
    const KeyLoader<R, KEYS, NT> v(g.v.p + (int64_t)s.k_first * g.v.row + (int64_t)kv * g.v.head, g.v.row, g.bytes);
    uint32_t here = 0;
    const bool wanted = g.out.p != nullptr;
    if (wanted && from < to) {
        k.load(lds_at(lds), from, s.m);
        v.load(lds_at(lds) + HALF, from, s.m);
    }
    Backward<T, DB, EXTRA, FAR_CAP> run;
    run.begin(g, s, kv, r);
    if (!wanted) return;
    const int mine = __builtin_amdgcn_readlane(run.limit, 31);
    const typename R::Place place;
    for (int j0 = from; j0 < to; j0 += KEYS, here ^= 2 * HALF) {
        arrived<0>();
        if (j0 + KEYS < to) {
            k.load(lds_at(lds) + (here ^ 2 * HALF), j0 + KEYS, s.m);
            v.load(lds_at(lds) + (here ^ 2 * HALF) + HALF, j0 + KEYS, s.m);
        }
#pragma unroll
        for (int at = 0; at < KEYS; at += 32)
            if (j0 + at < mine) run.step(g, lds + here, lds + here + HALF, place, j0 + at, at);
    }
    run.end(g, s, kv, r, g.scale / run.by, index, part.count);
}

// dq of few rows: as in attention_few_kernel, the waves have the same 32 packed rows and take tiles of 32 keys in turn.
template <class T, int DB, bool EXTRA, bool FAR_CAP>
__global__ __launch_bounds__((FewShape<T, DB>::WAVES * 64)) void attention_dq_few_kernel(const AttentionArgs g)
{
    using F = FewShape<T, DB>;
    using R = Rows<T, DB>;
    constexpr int WAVES = F::WAVES;
    __shared__ __align__(1024) char lds[F::LDS];
    const int kv = (int)((blockIdx.x + g.before) % g.kv_heads), lane = threadIdx.x & 63;
    Span s = find_span<true>(g.offsets, g.seqs, g.rows, g.group, 32, (int)((blockIdx.x + g.before) / g.kv_heads));
    if (s.seq >= g.seqs) {
        if (s.n > 0 && g.out.p) no_rows<T>(g, g.out, s, kv, s.r0, 32, nullptr);
        return;
    }
    find_keys(g, s);
    const KeyParts part(g, s, 32);
    const int index = g.splits - 1 - (int)blockIdx.y, from = index * part.chunk, to = min(from + part.chunk, part.most);
    if (index >= part.count) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = s.r0 + (lane & 31);
    const typename F::Loader k(g.k.p + (int64_t)s.k_first * g.k.row + (int64_t)kv * g.k.head, g.k.row, g.bytes);
    const typename F::Loader v(g.v.p + (int64_t)s.k_first * g.v.row + (int64_t)kv * g.v.head, g.v.row, g.bytes);
    const char *const own = lds + wave * F::STAGES * 2 * F::TILE;
    const uint32_t mine = lds_at(lds) + wave * F::STAGES * 2 * F::TILE;
    const bool wanted = g.out.p != nullptr;
    const int j1 = from + wave * 32;
    if (wanted && j1 < to) {
        v.load(mine + F::TILE, j1, s.m);
        k.load(mine, j1, s.m);
    }
    Backward<T, DB, EXTRA, FAR_CAP> run;
    run.begin(g, s, kv, r);
    if (!wanted) return;
    const typename R::Place place;
    if constexpr (F::STAGES == 1) {
        in_turn(v, mine + F::TILE, k, mine, j1, to, 32 * WAVES, s.m, [&](int j0, auto between) { run.step(g, own, own + F::TILE, place, j0, 0, between); });
    } else {
        uint32_t here = 0;
        for (int j0 = j1; j0 < to; j0 += 32 * WAVES, here ^= 2 * F::TILE) {
            arrived_but<0>();
            if (j0 + 32 * WAVES < to) {
                k.load(mine + (here ^ 2 * F::TILE), j0 + 32 * WAVES, s.m);
                v.load(mine + (here ^ 2 * F::TILE) + F::TILE, j0 + 32 * WAVES, s.m);
            }
            run.step(g, own + here, own + here + F::TILE, place, j0, 0);
        }
    }
    const float scale = g.scale / run.by;
    if constexpr (WAVES > 1) {
        __syncthreads();
        join_waves<WAVES>(lds, run.dq, scale);
        run.template end<WAVES>(g, s, kv, r, 1.0f, index, part.count);
    } else {
        run.end(g, s, kv, r, scale, index, part.count);
    }
}

// dk and dv: a wave has 32 keys, the waves share tiles of 32 packed rows of the kv head.
// DK, DV: which of the two; heads of 256 elements have no registers for both at once.
template <class T, int DB, bool EXTRA, int WAVES, bool DK, bool DV, bool FAR_CAP>
__global__ __launch_bounds__(WAVES * 64, sizeof(T) == 2 && (DB <= 4 || !DK) ? 2 : 1) void attention_dkv_kernel(const AttentionArgs g)
{
    using R = Rows<T, DB>;
    constexpr int TILE = WAVES == 8 ? 64 : 32, NT = WAVES * 64, HALF = TILE * R::ROWB;
    constexpr bool EXACT = sizeof(T) == 4 || FAR_CAP;
    // Weights are up to 1, and 1 / keys where rows weigh their keys alike, less than float16's smallest normal number from 2^14 keys on: there they, and dR with them,
    // are kept times 2^14.
    constexpr float WEIGHT_BITS = std::is_same_v<T, f16> ? 14.0f : 0.0f, WEIGHT_UNIT = std::is_same_v<T, f16> ? 0x1p-14f : 1.0f;
    // (in registers the keys would leave room for one wave a SIMD)
    constexpr bool K_IN_LDS = sizeof(T) == 2 && DB == 4;
    struct RowsInfo { float lse[TILE], delta[TILE], slope[TILE]; int limit[TILE], place[TILE]; };
    __shared__ __align__(1024) char lds[4 * HALF + (K_IN_LDS ? WAVES * 32 * R::ROWB : 0)];
    __shared__ __align__(16) RowsInfo infos[2];
    const char *const k_lds = lds + 4 * HALF;
    const int kv = (int)((blockIdx.x + g.before) % g.kv_heads), lane = threadIdx.x & 63, h = lane >> 5;
    Span s = find_span<false>(g.k_offsets, g.seqs, g.k_rows, 1, WAVES * 32, (int)((blockIdx.x + g.before) / g.kv_heads));
    const int key0 = s.r0;
    if (s.seq >= g.seqs) {
        for (int c = threadIdx.x / 64; c < min(WAVES * 32, s.n - key0) && blockIdx.y == 0; c += WAVES)
            for (int d = lane; d < g.dim; d += 64) {
                const int64_t row = s.first + key0 + c;
                if (DK && g.out.p) *((T *)(g.out.p + row * g.out.row + kv * g.out.head) + d) = (T)0.0f;
                if (DV && g.out2.p) *((T *)(g.out2.p + row * g.out2.row + kv * g.out2.head) + d) = (T)0.0f;
            }
        return;
    }
    // (the parts of the last rows, which end with the shortest ones, go last and fill up the end)
    const int index = g.splits - 1 - (int)blockIdx.y;
    const RowParts part(g, s, key0);
    if (index >= max(part.count, 1)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), key_w = key0 + wave * 32, key = key_w + (lane & 31);
    const int64_t key_row = s.k_first + min(key, s.m - 1);
    const char *kp = g.k.p + key_row * g.k.row + kv * g.k.head, *vp = g.v.p + key_row * g.v.row + kv * g.v.head;
    u32x4 k[K_IN_LDS ? 1 : R::STEPS], v[R::STEPS];
#pragma unroll
    for (int c = 0; c < R::STEPS; ++c) {
        const int at = c * 32 + h * 16;
        const bool here = at < g.bytes;
        if (!K_IN_LDS) k[K_IN_LDS ? 0 : c] = here ? *(const u32x4 *)(kp + at) : u32x4{0, 0, 0, 0};
        if (DK) v[c] = here ? *(const u32x4 *)(vp + at) : u32x4{0, 0, 0, 0};
    }
    if constexpr (!K_IN_LDS) settle(k);
    if constexpr (DK) settle(v);
    f32x16 dk[DB], dv[DB];
    if (DK) clear(dk);
    if (DV) clear(dv);
    const typename R::Place place;
    float by = first_factor<T>();
    const int to = part.all - index * part.chunk, from = max(part.begin, to - part.chunk);
    // From the last tile of rows to the first one: all workgroups of a sequence begin at the same rows, so that what is under way is shared in the
    // caches, and end where their keys are no longer seen.
    const int top = from + (max(to - from, 1) - 1) / TILE * TILE;
    const PackedLoader<R, TILE, NT> loader(g, g.q, g.dy, s.first, kv);
    // What is known of a tile's rows, by one thread each: asked for in front of a step, put to LDS behind it.
    float lse_next = 0.0f, delta_next = 0.0f;
    int row_next = 0, head_next = 0;
    const auto ask = [&](int r0) {
        if (threadIdx.x >= TILE) return;
        loader.place(r0, min((int)threadIdx.x, to - 1 - r0), row_next, head_next);
        const int64_t item = (int64_t)(s.first + row_next) * g.heads + kv * g.group + head_next;
        lse_next = g.lse[item];
        delta_next = g.delta[item];
    };
    const auto put = [&](int r0, RowsInfo &info) {
        if (threadIdx.x >= TILE) return;
        const int t = threadIdx.x;
        const bool none = r0 + t >= to;
        info.lse[t] = none || lse_next == -INFINITY ? INFINITY : fmaf(lse_next, LOG2E, -WEIGHT_BITS);
        info.delta[t] = none ? 0.0f : delta_next;
        info.limit[t] = limit_of(g, s, row_next);
        info.place[t] = row_next + s.ahead;
        info.slope[t] = EXTRA && g.slopes ? g.slopes[kv * g.group + head_next] * LOG2E : 0.0f;
    };
    int here = 0;
    if (from < to) {
        if constexpr (K_IN_LDS) {
            const KeyLoader<R, WAVES * 32, NT> keys(g.k.p + (int64_t)s.k_first * g.k.row + (int64_t)kv * g.k.head, g.k.row, g.bytes);
            keys.load(lds_at(k_lds), key0, s.m);
        }
        ask(top);
        loader.load(lds_at(lds), lds_at(lds) + HALF, top, to);
        put(top, infos[0]);
    }
    for (int r0 = from < to ? top : from - 1; r0 >= from; r0 -= TILE, here ^= 1) {
        arrived<0>();
        if (r0 > from) {
            ask(r0 - TILE);
            loader.load(lds_at(lds) + (here ^ 1) * 2 * HALF, lds_at(lds) + (here ^ 1) * 2 * HALF + HALF, r0 - TILE, to);
        }
        const RowsInfo &info = infos[here];
        const char *const q_lds = lds + here * 2 * HALF, *const dy_lds = q_lds + HALF;
#pragma unroll
        for (int at = 0; at < TILE; at += 32) {
            if (info.limit[at + 31] <= key_w) continue;          // (no row of these sees a key of this wave)
            f32x16 a, d;
#pragma unroll
            for (int j = 0; j < 16; ++j) a[j] = d[j] = 0.0f;
            if constexpr (K_IN_LDS) {
#pragma unroll
                for (int c = 0; c < R::STEPS; ++c) a = mma32(R::along(q_lds, place, at, c), R::along(k_lds, place, wave * 32, c), a, T{});
            } else {
                along_product<R, T>(q_lds, place, at, k, a);
            }
            if constexpr (DK) along_product<R, T>(dy_lds, place, at, v, d);
            const float by_log = EXTRA ? 1.0f : g.scale * LOG2E;
            if constexpr (EXTRA) {
                if (g.cap != 0.0f) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float bent;
                        a[j] = capped<EXACT>(g, a[j], bent);
                        d[j] = (d[j] - info.delta[at + block_row(j, h)]) * bent;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        a[j] *= g.scale * LOG2E;
                        d[j] -= info.delta[at + block_row(j, h)];
                    }
                }
                if (g.slopes) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int r = at + block_row(j, h);
                        a[j] = fmaf(-info.slope[r], fabsf((float)(info.place[r] - key)), a[j]);
                    }
                }
            }
            if (info.limit[at] < key_w + 32) {
#pragma unroll
                for (int j = 0; j < 16; ++j) a[j] = key < info.limit[at + block_row(j, h)] ? a[j] : -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int r = at + block_row(j, h);
                a[j] = __builtin_amdgcn_exp2f(fmaf(a[j], by_log, -info.lse[r]));
                d[j] = a[j] * (EXTRA ? d[j] : d[j] - info.delta[r]);
            }
            if constexpr (DV) {
#pragma unroll
                for (int t = 0; t < R::FRAGS; ++t) {
                    const u32x4 w = R::packed(a, t);
#pragma unroll
                    for (int b = 0; b < DB; ++b) dv[b] = mma32(R::across(dy_lds, place, at, t, b * 32), w, dv[b], T{});
                }
            }
            if constexpr (DK) {
                keep_in_range<T>(d, dk, by);
#pragma unroll
                for (int t = 0; t < R::FRAGS; ++t) {
                    const u32x4 w = R::packed(d, t);
#pragma unroll
                    for (int b = 0; b < DB; ++b) dk[b] = mma32(R::across(q_lds, place, at, t, b * 32), w, dk[b], T{});
                }
            }
        }
        if (r0 > from) put(r0 - TILE, infos[here ^ 1]);
    }
    if (key >= s.m) return;
    const float dk_unit = g.scale / by * WEIGHT_UNIT;
    const int64_t row = s.k_first + key;
    if (part.count > 1) {
        const int64_t at = ((int64_t)index * g.k_rows + row) * g.kv_heads + kv;
        const int wide = (g.dim & 3) == 0;
        if constexpr (DK) if (g.out.p) store_head<float, DB>((char *)(g.part + at * g.dim), dk, dk_unit, g.dim, wide);
        if constexpr (DV) if (g.out2.p) store_head<float, DB>((char *)(g.part2 + at * g.dim), dv, WEIGHT_UNIT, g.dim, wide);
        return;
    }
    if constexpr (DK) if (g.out.p) store_head<T, DB>(g.out.p + row * g.out.row + kv * g.out.head, dk, dk_unit, g.dim, g.wide);
    if constexpr (DV) if (g.out2.p) store_head<T, DB>(g.out2.p + row * g.out2.row + kv * g.out2.head, dv, WEIGHT_UNIT, g.dim, g.wide);
}

// Rows of tiles whose keys went in several parts, eight a workgroup and a wave each: y and lse, each part brought to the common maximum, or (SUM) dq.  Four
// elements a lane, the parts in their order.
template <class T, bool SUM>
__global__ __launch_bounds__(256) void attention_join_kernel(const AttentionArgs g, int tile)
{
    const int kv = (int)((blockIdx.x + g.before) % g.kv_heads), lane = threadIdx.x & 63;
    const Share share(g, tile);
    Span s = share.s;
    if (s.seq >= g.seqs) return;
    find_keys(g, s);
    const int64_t items = (int64_t)g.rows * g.heads;
    // (a head's elements take 16, 32 or 64 lanes; the others go through other parts)
    const int lanes = g.dim <= 64 ? 16 : g.dim <= 128 ? 32 : 64, sub = lane / lanes, subs = 64 / lanes;
    const int d = lane % lanes * 4, cnt = g.dim - d, wide = (g.dim & 3) == 0;
    for (int r0 = share.begin; r0 < share.end; r0 += tile)
    for (int r = r0 + blockIdx.y * 8 + (threadIdx.x >> 6); r < min(r0 + (int)blockIdx.y * 8 + 8, share.end); r += 4) {
        s.r0 = r0;
        const KeyParts part(g, s, tile);
        if (part.count < 2) break;
        const int64_t item = packed_item(g, s, kv, r);
        float weight = 1.0f, sum = 1.0f, top = 0.0f;
        if constexpr (!SUM) {
            const float2 mine = lane < part.count ? g.stat[lane * items + item] : make_float2(-INFINITY, 0.0f);
            top = mine.x;
#pragma unroll
            for (int off = 32; off; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
            weight = mine.y == 0.0f ? 0.0f : exp2f(mine.x - (top == -INFINITY ? 0.0f : top));
            sum = mine.y * weight;
#pragma unroll
            for (int off = 32; off; off >>= 1) sum += __shfl_xor(sum, off, 64);
        }
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int k0 = 0; k0 < part.count; k0 += subs) {
            const int k = k0 + sub;
            const float w = SUM ? 1.0f : __shfl(weight, min(k, 63), 64);
            if (cnt <= 0 || k >= part.count) continue;
            float one[4];
            load_row<float>((const char *)g.part, (k * items + item) * g.dim + d, cnt, wide, one);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += w == 0.0f ? 0.0f : w * one[j];
        }
        for (int off = lanes; off < 64; off <<= 1)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += __shfl_xor(v[j], off, 64);
        const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= by;
        if (cnt > 0 && sub == 0) store_row<T>((char *)packed_row(g, g.out, s, kv, r), d, cnt, g.wide, v);
        if (!SUM && g.lse && lane == 0) g.lse[item] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * LN2;
    }
}

// dk and dv of tiles whose rows went in several parts, which are added in their order: four elements a thread, `keys_each` keys a workgroup.
template <class T>
__global__ __launch_bounds__(256) void attention_sum_kernel(const AttentionArgs g, int keys_each)
{
    const int kv = (int)((blockIdx.x + g.before) % g.kv_heads);
    Span s = find_span<false>(g.k_offsets, g.seqs, g.k_rows, 1, g.key_tile, (int)((blockIdx.x + g.before) / g.kv_heads));
    if (s.seq >= g.seqs) return;
    const int key0 = s.r0;
    const RowParts part(g, s, key0);
    const Heads &out = blockIdx.y & 1 ? g.out2 : g.out;
    const float *const sums = blockIdx.y & 1 ? g.part2 : g.part;
    if (part.count < 2 || !out.p) return;
    const int per = (g.dim + 3) / 4, key1 = key0 + (blockIdx.y >> 1) * keys_each, keys = min(keys_each, s.m - key1);
    const int64_t items = (int64_t)g.k_rows * g.kv_heads;
    for (int c = threadIdx.x; c < keys * per; c += 256) {
        const int key = c / per, d = (c - key * per) * 4, cnt = g.dim - d, wide = (g.dim & 3) == 0;
        const int64_t row = s.k_first + key1 + key;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int k = 0; k < part.count; ++k) {
            float one[4];
            load_row<float>((const char *)sums, (k * items + row * g.kv_heads + kv) * g.dim + d, cnt, wide, one);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] += one[j];
        }
        store_row<T>(out.p + row * out.row + kv * out.head, d, cnt, g.wide, v);
    }
}

inline bool extra(const AttentionArgs &g) { return g.cap != 0.0f || g.slopes || !(g.scale > 0.0f); }

// (a grid's threads are counted in 32 bits)
template <class Launch>
hipError_t in_launches(const AttentionArgs &g, int64_t workgroups, Launch launch)
{
    constexpr int64_t MOST = 1 << 22;
    AttentionArgs part = g;
    for (int64_t done = 0; done < workgroups; done += MOST) {
        part.before = (uint32_t)done;
        launch(part, dim3((unsigned)std::min(workgroups - done, MOST), (unsigned)g.splits));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, bool SUM>
hipError_t launch_join(hipStream_t st, int few, const AttentionArgs &g)
{
    const int tile = few ? FEW_TILE : ATTENTION_TILE;
    return in_launches(g, (g.tiles ? g.tiles : (int64_t)g.seqs) * g.kv_heads,
                       [&](const AttentionArgs &p, dim3 grid) { attention_join_kernel<T, SUM><<<dim3(grid.x, tile / 8), 256, 0, st>>>(p, tile); });
}
// keys of a step of the kernels of rows
template <class T, int DB>
AttentionArgs with_unit(int few, AttentionArgs g)
{
    g.unit = few ? 32 * FewShape<T, DB>::WAVES : 64;
    return g;
}
template <class T, int DB, bool EXTRA, bool FAR_CAP>
hipError_t launch_rows(hipStream_t st, int few, const AttentionArgs &args)
{
    const AttentionArgs g = with_unit<T, DB>(few, args);
    const hipError_t e = in_launches(g, (g.tiles ? g.tiles : (int64_t)g.seqs + 1) * g.kv_heads, [&](const AttentionArgs &p, dim3 grid) {
        if (few) attention_few_kernel<T, DB, EXTRA, FAR_CAP><<<grid, FewShape<T, DB>::WAVES * 64, 0, st>>>(p);
        else attention_kernel<T, DB, EXTRA, 4, FAR_CAP><<<grid, 256, 0, st>>>(p);
    });
    return e != hipSuccess || g.splits == 1 ? e : launch_join<T, false>(st, few, g);
}
template <class T, int DB, bool EXTRA, bool FAR_CAP>
hipError_t launch_dq(hipStream_t st, int few, const AttentionArgs &args)
{
    const AttentionArgs g = with_unit<T, DB>(few, args);
    const hipError_t e = in_launches(g, (int64_t)g.tiles * g.kv_heads, [&](const AttentionArgs &p, dim3 grid) {
        if (few) attention_dq_few_kernel<T, DB, EXTRA, FAR_CAP><<<grid, FewShape<T, DB>::WAVES * 64, 0, st>>>(p);
        else attention_dq_kernel<T, DB, EXTRA, 4, FAR_CAP><<<grid, 256, 0, st>>>(p);
    });
    return e != hipSuccess || g.splits == 1 || !g.out.p ? e : launch_join<T, true>(st, few, g);
}
template <class T, int DB, bool EXTRA, bool FAR_CAP>
hipError_t launch_dkv(hipStream_t st, const AttentionArgs &g)
{
    const int64_t tiles = (int64_t)g.tiles * g.kv_heads;
    const hipError_t e = in_launches(g, tiles, [&](const AttentionArgs &p, dim3 grid) {
        if constexpr (DB <= 4) {
            if constexpr (sizeof(T) == 2) {
                if (p.key_tile == 256) {
                    attention_dkv_kernel<T, DB, EXTRA, 8, true, true, FAR_CAP><<<grid, 512, 0, st>>>(p);
                    return;
                }
            }
            attention_dkv_kernel<T, DB, EXTRA, 4, true, true, FAR_CAP><<<grid, 256, 0, st>>>(p);
        } else {
            if (p.out.p) attention_dkv_kernel<T, DB, EXTRA, 4, true, false, FAR_CAP><<<grid, 256, 0, st>>>(p);
            if (p.out2.p) attention_dkv_kernel<T, DB, EXTRA, 4, false, true, FAR_CAP><<<grid, 256, 0, st>>>(p);
        }
    });
    if (e != hipSuccess || g.splits == 1) return e;
    const int keys_each = tiles >= COMPUTE_UNITS ? 64 : 16;
    return in_launches(g, tiles, [&](const AttentionArgs &p, dim3 grid) {
        attention_sum_kernel<T><<<dim3(grid.x, 2 * p.key_tile / keys_each), 256, 0, st>>>(p, keys_each);
    });
}

// (a cap far above the scores is compiled apart: in one kernel with the others it took 20 to 45 registers more, and a wave a SIMD of dq)
inline bool far_cap(const AttentionArgs &g) { return g.cap > 256.0f; }
#define ALPA_BY_CAP(call, T, DB, g, ...) \
    (!extra(g) ? call<T, DB, false, false>(__VA_ARGS__) : far_cap(g) ? call<T, DB, true, sizeof(T) == 2>(__VA_ARGS__) : call<T, DB, true, false>(__VA_ARGS__))
#define ALPA_BY_DIM(call, T, g, ...)                                   \
    switch (dim_blocks((g).dim)) {                                     \
    case 2: return ALPA_BY_CAP(call, T, 2, g, __VA_ARGS__);            \
    case 3: return ALPA_BY_CAP(call, T, 3, g, __VA_ARGS__);            \
    case 4: return ALPA_BY_CAP(call, T, 4, g, __VA_ARGS__);            \
    default: return ALPA_BY_CAP(call, T, 8, g, __VA_ARGS__);           \
    }

}  // namespace alpa
