// C ABI of what a block has between its products: argument checks, work memory, choice of the kernels, launch order.
#include "../../include/alpa_blocks.h"
#include "blocks.hpp"

#include <cmath>

using namespace alpa;

extern "C" __attribute__((visibility("hidden"))) int alpa_dp_set_error_(int code, const char *msg);   // alpa_dp_abi.hip

namespace {

int fail(int code, const char *msg) { return alpa_dp_set_error_(code, msg); }

#define HIPCHK(expr)                                                            \
    do {                                                                        \
        const hipError_t e_ = (expr);                                           \
        if (e_ != hipSuccess) return fail(ALPA_DP_EHIP, hipGetErrorString(e_)); \
    } while (0)
#define TRY(expr)                          \
    do {                                   \
        const int rc_ = (expr);            \
        if (rc_ != ALPA_DP_OK) return rc_; \
    } while (0)

constexpr int64_t MAX_STRIDE = 1 << 22;                  // bytes, of matrices
constexpr int64_t FAR = (int64_t)1 << 40;                // bytes, of heads and their rows
constexpr int64_t NEAR_ROW = 1 << 22, NEAR_HEADS = 1 << 29;    // bytes: tensors that are further spread are copied, so that a tile's offsets stay in 31 bits

int64_t element(int dtype) { return dtype == ALPA_F32 ? 4 : 2; }
int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int64_t block(int64_t bytes) { return round_up(bytes, 256); }
bool by16(const void *p) { return ((uintptr_t)p & 15) == 0; }
bool type_ok(int dtype) { return dtype == ALPA_F32 || dtype == ALPA_F16 || dtype == ALPA_BF16; }

int check_work(const void *work, int64_t have, int64_t need)
{
    if (need > 0 && (!work || have < need)) return fail(ALPA_DP_EINVAL, "work memory is null or too small");
    if (need > 0 && ((uintptr_t)work & 255)) return fail(ALPA_DP_EINVAL, "work memory is not aligned to 256 bytes");
    return ALPA_DP_OK;
}
int check_vector(const void *p, int64_t es)
{
    return (uintptr_t)p % es ? fail(ALPA_DP_EINVAL, "a vector is not aligned to its elements") : ALPA_DP_OK;
}
int check_mat(const alpa_mat_t &m, int64_t rows, int64_t len, int dtype, bool optional, const char *what)
{
    if (rows == 0 || (optional && !m.p)) return ALPA_DP_OK;
    const int64_t es = element(dtype);
    if (!m.p) return fail(ALPA_DP_EINVAL, what);
    if ((uintptr_t)m.p % es) return fail(ALPA_DP_EINVAL, "a tensor is not aligned to its elements");
    if (m.ld < len || m.ld > MAX_STRIDE / es) return fail(ALPA_DP_EINVAL, "a stride is shorter than a row or above 2^22 bytes");
    return ALPA_DP_OK;
}
// `result`: heads of rows must not overlap
int check_heads(const alpa_heads_t &t, int64_t rows, int64_t heads, int64_t dim, int dtype, bool result, bool optional, const char *what)
{
    if (rows == 0 || (optional && !t.p)) return ALPA_DP_OK;
    const int64_t es = element(dtype);
    if (!t.p) return fail(ALPA_DP_EINVAL, what);
    if ((uintptr_t)t.p % es) return fail(ALPA_DP_EINVAL, "a tensor is not aligned to its elements");
    if (t.row < 0 || t.head < 0 || t.row > FAR / es || t.head > FAR / es) return fail(ALPA_DP_EINVAL, "a stride is negative or above 2^40 bytes");
    if (!result) return ALPA_DP_OK;
    const bool heads_in = (heads == 1 || t.head >= dim) && (rows == 1 || t.row >= (heads - 1) * t.head + dim);
    const bool rows_in = (rows == 1 || t.row >= dim) && (heads == 1 || t.head >= (rows - 1) * t.row + dim);
    return heads_in || rows_in ? ALPA_DP_OK : fail(ALPA_DP_EINVAL, "heads of a result overlap");
}
bool wide_heads(const alpa_heads_t &t, int dtype, int64_t bytes)
{
    const int64_t es = element(dtype);
    return !t.p || ((uintptr_t)t.p % bytes == 0 && t.row * es % bytes == 0 && t.head * es % bytes == 0);
}

// ---------------------------------------------------------------- attention

// NULL: fine
const char *wrong(const alpa_attention_t *a)
{
    if (!a) return "null pointer";
    if (!type_ok(a->dtype)) return "unknown type";
    if (a->rows < 0 || a->rows > ALPA_LAYER_MAX_ROWS || a->k_rows < 0 || a->k_rows > ALPA_LAYER_MAX_ROWS) return "rows out of range";
    if (a->seqs < 1 || a->seqs > ALPA_ATTENTION_MAX_SEQS) return "seqs out of range";
    if (a->heads < 1 || a->heads > ALPA_BLOCK_MAX_HEADS || a->kv_heads < 1 || a->heads % a->kv_heads) return "heads out of range or not a multiple of kv_heads";
    if (a->rows * a->heads > ALPA_ATTENTION_MAX_ITEMS || a->k_rows * a->kv_heads > ALPA_ATTENTION_MAX_ITEMS) return "rows x heads out of range";
    if (a->dim < 1 || a->dim > ALPA_ATTENTION_MAX_DIM) return "dim out of range";
    if (a->k_step != 1 && a->k_step != 2) return "k_step is neither 1 nor 2";
    if (!std::isfinite(a->scale) || !std::isfinite(a->cap) || a->cap < 0.0f) return "scale or cap is not finite, or cap is negative";
    if ((!a->offsets || !a->k_offsets) && a->seqs != 1) return "offsets are null with more than one sequence";
    if (((uintptr_t)a->offsets | (uintptr_t)a->k_offsets | (uintptr_t)a->prefix | (uintptr_t)a->slopes) % 4) return "a vector is not aligned to its elements";
    return nullptr;
}

bool needs_copy(const alpa_heads_t &t, const alpa_attention_t &a, bool queries)
{
    const int64_t es = element(a.dtype);
    return a.dim * es % 16 || !wide_heads(t, a.dtype, 16) || t.row * es > NEAR_ROW || (queries && a.heads / a.kv_heads * t.head * es > NEAR_HEADS);
}

// One call's work memory: copies, then sums.
struct Plan {
    const alpa_attention_t &a;
    AttentionArgs g{};
    HeadPack pack{};
    int64_t used = 0;
    char *work;

    Plan(const alpa_attention_t &how, void *memory) : a(how), work((char *)memory)
    {
        const int64_t es = element(a.dtype);
        g.rows = (int)a.rows;
        g.k_rows = (int)a.k_rows;
        g.seqs = a.seqs;
        g.heads = a.heads;
        g.kv_heads = a.kv_heads;
        g.group = a.heads / a.kv_heads;
        g.dim = a.dim;
        g.bytes = (int)round_up(a.dim * es, 16);
        g.offsets = a.offsets;
        g.k_offsets = a.k_offsets;
        g.prefix = a.prefix;
        g.slopes = a.slopes;
        g.k_step = a.k_step;
        g.causal = a.causal != 0;
        g.scale = a.scale;
        g.cap = a.cap;
        // (finite, so that a score of zero stays one)
        g.twice = a.cap > 0.0f ? (float)std::min(std::max(2.0 * a.scale * 1.4426950408889634 / a.cap, -3.4e38), 3.4e38) : 0.0f;
        g.splits = 1;
        pack.len = a.dim;
        pack.to_len = (int)(g.bytes / es);
    }
    template <class E>
    E *take(int64_t count)
    {
        char *p = work ? work + used : nullptr;
        used += block(count * (int64_t)sizeof(E));
        return (E *)p;
    }
    Heads operand(const alpa_heads_t &t, bool queries)
    {
        const int64_t es = element(a.dtype), rows = queries ? a.rows : a.k_rows, heads = queries ? a.heads : a.kv_heads;
        if (rows == 0 || !needs_copy(t, a, queries)) return Heads{(char *)t.p, t.row * es, t.head * es};
        auto &m = pack.t[pack.count++];
        m.from = (const char *)t.p;
        m.row = t.row;
        m.head = t.head;
        m.rows = rows;
        m.heads = (int)heads;
        m.to = take<char>(rows * heads * g.bytes);
        return Heads{m.to, heads * g.bytes, g.bytes};
    }
    Heads result(const alpa_heads_t &t) const
    {
        const int64_t es = element(a.dtype);
        return Heads{(char *)t.p, t.row * es, t.head * es};
    }
    // tiles that the sequences' packed rows can make at most, rows of none among them
    static int64_t tiles_of(int64_t packed, int64_t seqs, int tile) { return packed / tile + std::min(seqs + 2, packed); }
};

// What a call's rows are to the kernels.
struct Shape {
    int64_t packed, tiles;          // rows of a kv head; tiles of many rows, about
    bool few, direct;               // tiles of 32 rows whose keys the waves share; forward, a sequence a workgroup, without a search

    explicit Shape(const alpa_attention_t &a)
        : packed(a.rows * (a.heads / a.kv_heads)), tiles((packed / ATTENTION_TILE + std::min<int64_t>(a.seqs, packed)) * a.kv_heads)
    {
        // few rows of a sequence, so that the keys and not the products are what takes time; or few tiles, so that waves are short of work (777 rows, 6 heads of
        // 75 in 32 bits, 42 tiles: forward 73 and 33 us, dq 107 and 42)
        const bool short_rows = packed <= 64 * (int64_t)a.seqs;
        few = short_rows || tiles <= COMPUTE_UNITS;
        direct = packed <= 32 * (int64_t)a.seqs;
    }
};

// As many workgroups as are on the compute units at once.  With a causal mask a tile has half of all parts on average, and where one part each fills the units,
// two are better, as the tile with most work is what is waited for.
int64_t parts_for(int64_t tiles, int64_t slots, bool causal)
{
    return causal ? std::max<int64_t>(2 * slots / tiles - 1, tiles <= 2 * slots ? 2 : 1) : slots / tiles;
}

// Parts of the keys for y and dq (KeyParts in attention_kernel.hpp; causal, 4096 rows, 8 heads of 256: forward 280 us in one part, 164 in two, dq 308 and 222; parts
// of fewer than 2048 keys cost more than they save: 2048 rows, 16 heads on 1 kv head, 48 us in one, 60 in two).
int key_splits(const alpa_attention_t &a, const Shape &shape, bool backward)
{
    const int64_t keys = a.k_rows / a.seqs;
    if (!shape.few) {
        if (backward && a.dtype == ALPA_F32) return 1;           // (4096 rows, 16 heads: dq 879 us, 933 in two parts; forward 799 and 579)
        if (!backward && a.dtype != ALPA_F32 && 2 * shape.tiles > 3 * COMPUTE_UNITS && keys < 8192) return 1;       // (4096 rows, 16 heads: 101 us, 113 in two)
        return (int)std::max<int64_t>(1, std::min({(int64_t)64, parts_for(shape.tiles, 2 * COMPUTE_UNITS, a.causal), keys / 2048}));
    }
    // (one workgroup a unit where its tiles fill the LDS; rows that are few in front of their keys see nearly all of them)
    const int64_t slots = dim_blocks(a.dim) == 2 && a.dtype != ALPA_F32 ? 2 * COMPUTE_UNITS : COMPUTE_UNITS;
    const int64_t tiles = std::max<int64_t>(shape.packed / FEW_TILE, a.seqs) * a.kv_heads;
    return (int)std::max<int64_t>(1, std::min({(int64_t)64, parts_for(tiles, slots, a.causal && a.rows > a.k_rows / 4), keys / (a.dtype == ALPA_F32 ? 64 : 128)}));
}

// Keys of a workgroup for dk and dv: 256, one workgroup a compute unit, read queries and dy half as often as 128, two a unit, and have twice the time to
// bring a tile of rows; where tiles are few or sequences short, 128 fill the units better (causal, 8192 rows: 32 heads on 32 kv heads 1292 us with 128, 1155 with
// 256; 32 on 4 1439 and 1260; 2048 rows, 32 on 8 136 and 183; 4096 rows, 16 on 1 287 and 300).
int key_tile(const alpa_attention_t &a)
{
    const bool wide = a.dtype != ALPA_F32 && a.dim <= 128 && a.k_rows / a.seqs >= 512 && a.k_rows / 256 * a.kv_heads >= COMPUTE_UNITS / 2;
    return wide ? 256 : 128;
}

// Parts of the rows for dk and dv (RowParts in attention_kernel.hpp; tiles of 128 keys, causal, 8192 rows, 32 heads on 8 kv heads: 1963 us in one part, 1260 in two,
// 1435 in three; 2048 rows: 265 in two, 168 in four, 136 in six, 165 in eight; without the mask 8 heads of 8192 rows: 605, 634 in two; 32 on 8 of 2048: 294 in
// two, 182 in four, 227 in six).
int row_splits(const alpa_attention_t &a, int key_tile)
{
    const int64_t rows = a.rows * (a.heads / a.kv_heads) / a.seqs;
    const int64_t tiles = std::max<int64_t>((a.k_rows / key_tile + a.seqs / 2) * a.kv_heads, a.kv_heads);
    return (int)std::max<int64_t>(1, std::min({(int64_t)32, parts_for(tiles, (key_tile == 256 ? 1 : 2) * COMPUTE_UNITS, a.causal), rows / (a.dtype == ALPA_F32 ? 64 : 128)}));
}

void plan_forward(Plan &p, const alpa_heads_t &q, const alpa_heads_t &k, const alpa_heads_t &v)
{
    AttentionArgs &g = p.g;
    g.q = p.operand(q, true);
    g.k = p.operand(k, false);
    g.v = p.operand(v, false);
    const Shape shape(p.a);
    g.splits = key_splits(p.a, shape, false);
    g.tiles = shape.direct ? 0 : (int)Plan::tiles_of(shape.packed, p.a.seqs, shape.few ? FEW_TILE : ATTENTION_TILE);
    if (g.splits > 1) {
        const int64_t items = (int64_t)g.splits * p.a.rows * p.a.heads;
        g.part = p.take<float>(items * p.a.dim);
        g.stat = p.take<float2>(items);
    }
}

void plan_backward(Plan &p, const alpa_heads_t &dy, const alpa_heads_t &q, const alpa_heads_t &k, const alpa_heads_t &v, const alpa_heads_t &y)
{
    AttentionArgs &g = p.g;
    g.dy = p.operand(dy, true);
    g.q = p.operand(q, true);
    g.k = p.operand(k, false);
    g.v = p.operand(v, false);
    g.y = p.operand(y, true);
    g.delta = p.take<float>(p.a.rows * p.a.heads);
    g.key_tile = key_tile(p.a);
    const int rows = row_splits(p.a, g.key_tile), keys = key_splits(p.a, Shape(p.a), true);
    g.splits = rows;
    const int64_t items = rows > 1 ? (int64_t)rows * p.a.k_rows * p.a.kv_heads : 0, q_items = keys > 1 ? (int64_t)keys * p.a.rows * p.a.heads : 0;
    if (items || q_items) g.part = p.take<float>(std::max(items, q_items) * p.a.dim);          // (dq's are done with when dk's come)
    if (items) g.part2 = p.take<float>(items * p.a.dim);
}

hipError_t launch_rows_of(hipStream_t st, int dtype, int few, const AttentionArgs &g)
{
    return dtype == ALPA_F32 ? launch_attention_f32(st, few, g) : dtype == ALPA_F16 ? launch_attention_f16(st, few, g) : launch_attention_bf16(st, few, g);
}
hipError_t launch_dq_of(hipStream_t st, int dtype, int few, const AttentionArgs &g)
{
    return dtype == ALPA_F32 ? launch_attention_dq_f32(st, few, g) : dtype == ALPA_F16 ? launch_attention_dq_f16(st, few, g) : launch_attention_dq_bf16(st, few, g);
}
hipError_t launch_dkv_of(hipStream_t st, int dtype, const AttentionArgs &g)
{
    return dtype == ALPA_F32 ? launch_attention_dkv_f32(st, g) : dtype == ALPA_F16 ? launch_attention_dkv_f16(st, g) : launch_attention_dkv_bf16(st, g);
}

// ---------------------------------------------------------------- rotary positions, layer norm

int rotary(int dtype, int64_t rows, int heads, int dim, int rot, int interleaved, float scale, float sign, const int64_t *positions,
           const double *frequencies, const alpa_heads_t &x, const alpa_heads_t &y, hipStream_t st)
{
    if (!type_ok(dtype)) return fail(ALPA_DP_EINVAL, "unknown type");
    if (rows < 0 || rows > ALPA_LAYER_MAX_ROWS) return fail(ALPA_DP_EINVAL, "rows out of range");
    if (heads < 1 || heads > ALPA_BLOCK_MAX_HEADS || dim < 2 || dim > ALPA_BLOCK_MAX_DIM) return fail(ALPA_DP_EINVAL, "heads or dim out of range");
    if (rot < 2 || rot > dim || rot % 2) return fail(ALPA_DP_EINVAL, "rot is odd or not in 2 .. dim");
    if (!std::isfinite(scale)) return fail(ALPA_DP_EINVAL, "scale is not finite");
    if (rows == 0) return ALPA_DP_OK;
    if (!positions || !frequencies) return fail(ALPA_DP_EINVAL, "positions or frequencies are null");
    TRY(check_vector(positions, 8));
    TRY(check_vector(frequencies, 8));
    TRY(check_heads(x, rows, heads, dim, dtype, false, false, "x or dy is null"));
    TRY(check_heads(y, rows, heads, dim, dtype, true, false, "y or dx is null"));
    const bool in_place = x.p == y.p;
    if (in_place && (x.row != y.row || x.head != y.head)) return fail(ALPA_DP_EINVAL, "turned in place, x and y need the same strides");
    const int64_t es = element(dtype);
    RotaryArgs g{};
    g.x = Heads{(char *)x.p, x.row, x.head};
    g.y = Heads{(char *)y.p, y.row, y.head};
    g.rows = rows;
    g.heads = heads;
    g.dim = dim;
    g.rot = rot;
    g.interleaved = interleaved != 0;
    g.copy = !in_place && rot < dim;
    g.scale = scale;
    g.sign = sign;
    g.positions = positions;
    g.frequencies = frequencies;
    // bytes at once: of halves each starts and ends at a multiple of them, of interleaved pairs the whole does, and so does what is copied
    const auto fits = [&](int64_t b) {
        return wide_heads(x, dtype, b) && wide_heads(y, dtype, b) && (interleaved ? rot : rot / 2) * es % b == 0 && (!g.copy || dim * es % b == 0);
    };
    g.wide = fits(16) ? 16 : fits(8) ? 8 : 0;
    HIPCHK(launch_rotary(st, dtype, g));
    return ALPA_DP_OK;
}

int check_norm(int dtype, int64_t rows, int64_t n)
{
    if (!type_ok(dtype)) return fail(ALPA_DP_EINVAL, "unknown type");
    if (rows < 0 || rows > ALPA_LAYER_MAX_ROWS) return fail(ALPA_DP_EINVAL, "rows out of range");
    if (n < 1 || n > ALPA_LAYER_MAX_WIDTH) return fail(ALPA_DP_EINVAL, "n out of range");
    return ALPA_DP_OK;
}
bool wide_mat(const alpa_mat_t &m, int64_t es) { return !m.p || (by16(m.p) && m.ld * es % 16 == 0); }

}  // namespace

extern "C" {

int64_t alpa_attention_forward_work(const alpa_attention_t *how, alpa_heads_t q, alpa_heads_t k, alpa_heads_t v)
{
    if (wrong(how) || how->rows == 0) return 0;
    Plan p(*how, nullptr);
    plan_forward(p, q, k, v);
    return p.used;
}

int alpa_attention_forward(const alpa_attention_t *how, alpa_heads_t q, alpa_heads_t k, alpa_heads_t v, alpa_heads_t y,
                           float *lse, void *work, int64_t work_bytes, void *hip_stream)
{
    if (const char *w = wrong(how)) return fail(ALPA_DP_EINVAL, w);
    const alpa_attention_t &a = *how;
    TRY(check_heads(q, a.rows, a.heads, a.dim, a.dtype, false, false, "q is null"));
    TRY(check_heads(k, a.k_rows, a.kv_heads, a.dim, a.dtype, false, false, "k is null"));
    TRY(check_heads(v, a.k_rows, a.kv_heads, a.dim, a.dtype, false, false, "v is null"));
    TRY(check_heads(y, a.rows, a.heads, a.dim, a.dtype, true, false, "y is null"));
    TRY(check_vector(lse, 4));
    if (a.rows == 0) return ALPA_DP_OK;
    Plan p(a, work);
    plan_forward(p, q, k, v);
    TRY(check_work(work, work_bytes, p.used));
    hipStream_t st = (hipStream_t)hip_stream;
    AttentionArgs &g = p.g;
    g.out = p.result(y);
    g.wide = wide_heads(y, a.dtype, 4 * element(a.dtype));
    g.lse = lse;
    if (p.pack.count) HIPCHK(launch_head_pack(st, a.dtype, p.pack));
    HIPCHK(launch_rows_of(st, a.dtype, Shape(a).few, g));
    return ALPA_DP_OK;
}

int64_t alpa_attention_backward_work(const alpa_attention_t *how, alpa_heads_t dy, alpa_heads_t q, alpa_heads_t k,
                                     alpa_heads_t v, alpa_heads_t y)
{
    if (wrong(how) || how->k_step != 1) return 0;
    Plan p(*how, nullptr);
    plan_backward(p, dy, q, k, v, y);
    return p.used;
}

int alpa_attention_backward(const alpa_attention_t *how, alpa_heads_t dy, alpa_heads_t q, alpa_heads_t k, alpa_heads_t v,
                            alpa_heads_t y, const float *lse, alpa_heads_t dq, alpa_heads_t dk, alpa_heads_t dv, void *work,
                            int64_t work_bytes, void *hip_stream)
{
    if (const char *w = wrong(how)) return fail(ALPA_DP_EINVAL, w);
    const alpa_attention_t &a = *how;
    if (a.k_step != 1) return fail(ALPA_DP_EINVAL, "keys that are not packed have no gradients");
    TRY(check_heads(dy, a.rows, a.heads, a.dim, a.dtype, false, false, "dy is null"));
    TRY(check_heads(q, a.rows, a.heads, a.dim, a.dtype, false, false, "q is null"));
    TRY(check_heads(k, a.k_rows, a.kv_heads, a.dim, a.dtype, false, false, "k is null"));
    TRY(check_heads(v, a.k_rows, a.kv_heads, a.dim, a.dtype, false, false, "v is null"));
    TRY(check_heads(y, a.rows, a.heads, a.dim, a.dtype, false, false, "y is null"));
    if (a.rows > 0 && !lse) return fail(ALPA_DP_EINVAL, "lse is null");
    TRY(check_vector(lse, 4));
    TRY(check_heads(dq, a.rows, a.heads, a.dim, a.dtype, true, true, ""));
    TRY(check_heads(dk, a.k_rows, a.kv_heads, a.dim, a.dtype, true, true, ""));
    TRY(check_heads(dv, a.k_rows, a.kv_heads, a.dim, a.dtype, true, true, ""));
    Plan p(a, work);
    plan_backward(p, dy, q, k, v, y);
    TRY(check_work(work, work_bytes, p.used));
    hipStream_t st = (hipStream_t)hip_stream;
    AttentionArgs &g = p.g;
    g.lse = (float *)lse;
    const int splits = g.splits, bytes = 4 * (int)element(a.dtype);
    if (a.rows > 0 && (dq.p || dk.p || dv.p)) {
        if (p.pack.count) HIPCHK(launch_head_pack(st, a.dtype, p.pack));
        g.out = p.result(dq);
        g.wide = wide_heads(dq, a.dtype, bytes);
        const Shape shape(a);
        g.tiles = (int)Plan::tiles_of(shape.packed, a.seqs, shape.few ? FEW_TILE : ATTENTION_TILE);
        g.splits = key_splits(a, shape, true);
        HIPCHK(launch_dq_of(st, a.dtype, shape.few, g));
    }
    if (a.k_rows > 0 && (dk.p || dv.p)) {
        g.out = p.result(dk);
        g.out2 = p.result(dv);
        g.wide = wide_heads(dk, a.dtype, bytes) && wide_heads(dv, a.dtype, bytes);
        g.tiles = (int)Plan::tiles_of(a.k_rows, a.seqs, g.key_tile);
        g.splits = splits;
        HIPCHK(launch_dkv_of(st, a.dtype, g));
    }
    return ALPA_DP_OK;
}

int alpa_rotary_forward(int dtype, int64_t rows, int heads, int dim, int rot, int interleaved, float scale,
                        const int64_t *positions, const double *frequencies, alpa_heads_t x, alpa_heads_t y,
                        void *hip_stream)
{
    return rotary(dtype, rows, heads, dim, rot, interleaved, scale, 1.0f, positions, frequencies, x, y, (hipStream_t)hip_stream);
}

int alpa_rotary_backward(int dtype, int64_t rows, int heads, int dim, int rot, int interleaved, float scale,
                         const int64_t *positions, const double *frequencies, alpa_heads_t dy, alpa_heads_t dx,
                         void *hip_stream)
{
    return rotary(dtype, rows, heads, dim, rot, interleaved, scale, -1.0f, positions, frequencies, dy, dx, (hipStream_t)hip_stream);
}

int alpa_rotary_frequencies(int rot, double base, double factor, double context, double low, double high, double *frequencies)
{
    if (rot < 2 || rot > ALPA_BLOCK_MAX_DIM || rot % 2) return fail(ALPA_DP_EINVAL, "rot is odd or out of range");
    if (!(base > 0.0) || !(factor > 0.0) || !std::isfinite(base) || !std::isfinite(factor)) return fail(ALPA_DP_EINVAL, "base or factor is not positive");
    if (!(context >= 0.0) || !std::isfinite(context) || (context > 0.0 && !(low < high))) return fail(ALPA_DP_EINVAL, "context is negative, or low is not below high");
    if (!frequencies) return fail(ALPA_DP_EINVAL, "frequencies are null");
    for (int t = 0; t < rot / 2; ++t) {
        const double f = std::pow(base, -2.0 * t / rot), turns = context * f / 6.283185307179586477;
        const double kept = context > 0.0 ? std::min(std::max((turns - low) / (high - low), 0.0), 1.0) : 0.0;
        frequencies[t] = f * (kept + (1.0 - kept) / factor);
    }
    return ALPA_DP_OK;
}

int alpa_norm_forward(int dtype, int64_t rows, int64_t n, float eps, alpa_mat_t x, const void *weight, const void *bias,
                      alpa_mat_t y, float *mean, float *rstd, void *hip_stream)
{
    TRY(check_norm(dtype, rows, n));
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(ALPA_DP_EINVAL, "eps is negative or not finite");
    TRY(check_mat(x, rows, n, dtype, false, "x is null"));
    TRY(check_mat(y, rows, n, dtype, false, "y is null"));
    const int64_t es = element(dtype);
    TRY(check_vector(weight, es));
    TRY(check_vector(bias, es));
    if (!mean != !rstd) return fail(ALPA_DP_EINVAL, "of mean and rstd one is null");
    TRY(check_vector(mean, 4));
    TRY(check_vector(rstd, 4));
    if (rows == 0) return ALPA_DP_OK;
    NormArgs g{};
    g.x = (const char *)x.p;
    g.weight = (const char *)weight;
    g.bias = (const char *)bias;
    g.y = (char *)y.p;
    g.ldx = x.ld;
    g.ldy = y.ld;
    g.rows = (int)rows;
    g.n = (int)n;
    g.eps = eps;
    g.mean = mean;
    g.rstd = rstd;
    g.wide = wide_mat(x, es) && wide_mat(y, es) && by16(weight) && by16(bias) && n * es % 16 == 0;
    HIPCHK(launch_norm((hipStream_t)hip_stream, dtype, g));
    return ALPA_DP_OK;
}

int64_t alpa_norm_backward_work(int dtype, int64_t rows, int64_t n)
{
    if (!type_ok(dtype) || rows < 0 || rows > ALPA_LAYER_MAX_ROWS || n < 1 || n > ALPA_LAYER_MAX_WIDTH) return 0;
    return 2 * block(norm_groups(rows) * n * 4);
}

int alpa_norm_backward(int dtype, int64_t rows, int64_t n, alpa_mat_t dy, alpa_mat_t x, const float *mean,
                       const float *rstd, const void *weight, alpa_mat_t dx, void *dweight, void *dbias, void *work,
                       int64_t work_bytes, void *hip_stream)
{
    TRY(check_norm(dtype, rows, n));
    TRY(check_mat(dy, rows, n, dtype, false, "dy is null"));
    TRY(check_mat(x, rows, n, dtype, false, "x is null"));
    TRY(check_mat(dx, rows, n, dtype, true, ""));
    if (rows > 0 && (!mean || !rstd)) return fail(ALPA_DP_EINVAL, "mean or rstd is null");
    const int64_t es = element(dtype);
    TRY(check_vector(mean, 4));
    TRY(check_vector(rstd, 4));
    TRY(check_vector(weight, es));
    TRY(check_vector(dweight, es));
    TRY(check_vector(dbias, es));
    TRY(check_work(work, work_bytes, alpa_norm_backward_work(dtype, rows, n)));
    if (!(rows > 0 && dx.p) && !dweight && !dbias) return ALPA_DP_OK;
    NormArgs g{};
    g.x = (const char *)x.p;
    g.dy = (const char *)dy.p;
    g.weight = (const char *)weight;
    g.y = (char *)dx.p;
    g.ldx = x.ld;
    g.lddy = dy.ld;
    g.ldy = dx.ld;
    g.rows = (int)rows;
    g.n = (int)n;
    g.mean = (float *)mean;
    g.rstd = (float *)rstd;
    g.groups = norm_groups(rows);
    g.dweight = (char *)dweight;
    g.dbias = (char *)dbias;
    if (dweight) g.part_w = (float *)work;
    if (dbias) g.part_b = (float *)((char *)work + block((int64_t)g.groups * n * 4));
    g.wide = wide_mat(x, es) && wide_mat(dy, es) && wide_mat(dx, es) && by16(weight) && n * es % 16 == 0;
    HIPCHK(launch_norm_backward((hipStream_t)hip_stream, dtype, g));
    return ALPA_DP_OK;
}

}  // extern "C"
