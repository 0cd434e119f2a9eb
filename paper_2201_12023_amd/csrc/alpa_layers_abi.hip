// C ABI of the layer operators: argument checks, choice of the kernels, work memory, launch order.
#include "../../include/alpa_layers.h"
#include "layers.hpp"

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

constexpr int64_t MAX_STRIDE = 1 << 22;      // bytes: a tile's offsets stay in 32 bits

int64_t element(int dtype) { return dtype == ALPA_F32 ? 4 : 2; }
int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int64_t block(int64_t bytes) { return round_up(bytes, 256); }
bool by16(const void *p) { return ((uintptr_t)p & 15) == 0; }

bool type_ok(int dtype) { return dtype == ALPA_F32 || dtype == ALPA_F16 || dtype == ALPA_BF16; }
bool sizes_ok(int64_t rows, int64_t n_in, int64_t n_out, int64_t most_out)
{
    return rows >= 0 && rows <= ALPA_LAYER_MAX_ROWS && n_in >= 1 && n_in <= ALPA_LAYER_MAX_WIDTH && n_out >= 1 && n_out <= most_out;
}
int check_sizes(int dtype, int64_t rows, int64_t n_in, int64_t n_out, int64_t most_out)
{
    if (!type_ok(dtype)) return fail(ALPA_DP_EINVAL, "unknown type");
    if (rows < 0 || rows > ALPA_LAYER_MAX_ROWS) return fail(ALPA_DP_EINVAL, "rows out of range");
    if (n_in < 1 || n_in > ALPA_LAYER_MAX_WIDTH) return fail(ALPA_DP_EINVAL, "n_in out of range");
    if (n_out < 1 || n_out > most_out) return fail(ALPA_DP_EINVAL, "n_out or words out of range");
    return ALPA_DP_OK;
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
int check_vector(const void *p, int64_t es)
{
    return (uintptr_t)p % es ? fail(ALPA_DP_EINVAL, "a vector is not aligned to its elements") : ALPA_DP_OK;
}
int check_work(const void *work, int64_t have, int64_t need)
{
    if (need > 0 && (!work || have < need)) return fail(ALPA_DP_EINVAL, "work memory is null or too small");
    if (need > 0 && ((uintptr_t)work & 255)) return fail(ALPA_DP_EINVAL, "work memory is not aligned to 256 bytes");
    return ALPA_DP_OK;
}

// An activation as the product's epilogue takes it.
Epilogue epilogue_of(int act, ProductArgs &g)
{
    g.low = act == ALPA_ACT_RELU ? 0.0f : -INFINITY;
    g.c1 = act == ALPA_ACT_GELU_TANH ? 1.5957691216057308f : 1.0f;             // 2 sqrt(2 / pi), and 0.044715 of it
    g.c3 = act == ALPA_ACT_GELU_TANH ? 0.071354816272600257f : 0.0f;
    return act == ALPA_ACT_GELU ? EPI_ERF : act >= ALPA_ACT_GELU_TANH ? EPI_SIGMOID : EPI_LINE;
}

// An operand as the tiled product takes it: address, stride and row length are multiples of 16 bytes.
struct Source {
    const char *p;
    int64_t ld, len;        // elements; len with its padding, which holds zeros
};

// Work memory for the copy of a matrix that is not so (0: it is taken as it is).
int64_t pack_bytes(const alpa_mat_t &m, int64_t rows, int64_t len, int dtype)
{
    const int64_t es = element(dtype);
    if (!m.p || rows == 0 || (by16(m.p) && (m.ld * es) % 16 == 0 && (len * es) % 16 == 0)) return 0;
    return block(rows * round_up(len, 16 / es) * es);
}
// The copies that a call needs, all queued at once.
struct Packs {
    PackArgs g{};
    Source add(const alpa_mat_t &m, int64_t rows, int64_t len, int dtype, char *work)
    {
        if (pack_bytes(m, rows, len, dtype) == 0) return Source{(const char *)m.p, m.ld, len};
        const int64_t to = round_up(len, 16 / element(dtype));
        g.mats[g.count++] = {(const char *)m.p, work, m.ld, rows, (int)len, (int)to};
        return Source{work, to, to};
    }
    int queue(hipStream_t st, int dtype)
    {
        if (g.count) HIPCHK(launch_pack(st, dtype, g));
        return ALPA_DP_OK;
    }
};

// A product of `m` x `n` results over `k`; `groups`: matrices of results (GROUP_STEPS), or groups of rows.
struct Shape {
    int64_t m, n, k;
    Grouping grouping;
    int groups;
};

int64_t tiles_of(const Shape &s, int tile)
{
    const int64_t cols = (s.n + tile - 1) / tile;
    if (s.grouping == GROUP_ROWS) return slots_at_most(s.m, s.groups, tile) * cols;
    return (s.m + tile - 1) / tile * cols * (s.grouping == GROUP_STEPS ? s.groups : 1);
}

// How a product is cut: the tile, and into how many parts its contraction is split where the tiles alone leave compute units without work (the
// parts' sums go through memory in 32 bits and are joined in their order).
struct Cut {
    int tile, splits, split_steps;
};

// Of the three tiles and a few numbers of parts the ones with the least time by a model of it.  A compute unit holds one workgroup of the large tile or
// two of the others; a step of one takes `alone`, of two `both`, a workgroup's beginning and end `ends` microseconds, of the large
// tile's, which goes on to its next one, 4 for all but the first, and all of it no less than the
// operands take at 4.9 TB/s; a join adds a launch and its traffic.  The figures are measured (fifty products of 1 to 8192 rows and 296 to 16384 deep, all
// three forms, each with every tile and 1 to 32 parts): the choice was the best of them in most and within 8 % of it everywhere.  Ragged groups are taken to
// be of one size with half a tile left over; where they are contractions, one is taken to be twice as long.
Cut cut_of(const Shape &s, int dtype, bool may_split, bool may_be_big)
{
    struct Model { int tile; double alone, both, ends; };
    static const Model half[] = {{SMALL_TILE, 0.26, 0.40, 2.5}, {TILE, 0.65, 1.0, 4.0}, {BIG_TILE, 1.4, 0.0, 9.0}};
    static const Model full[] = {{SMALL_TILE, 0.60, 1.10, 2.5}, {TILE, 1.95, 3.8, 4.0}, {BIG_TILE, 7.2, 0.0, 9.0}};
    static const int parts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
    const double units = COMPUTE_UNITS;
    int64_t depth = s.k;
    if (s.grouping == GROUP_STEPS) depth = s.k / std::max(s.groups, 1) + 1;
    const int64_t steps = std::max<int64_t>((depth * element(dtype) + STEP_BYTES - 1) / STEP_BYTES, 1);
    const double weights = s.grouping == GROUP_ROWS ? (double)std::min<int64_t>(s.m, s.groups) : 1.0;
    const double memory = 3.0 + ((double)s.m + weights * (double)s.n) * (double)(s.k * element(dtype)) / 4.9e6;
    Cut best{TILE, 1, 0};
    double least = INFINITY;
    for (const Model &m : dtype == ALPA_F32 ? full : half) {
        if (m.tile == BIG_TILE && !may_be_big) break;
        double tiles = (double)tiles_of(s, m.tile);
        if (s.grouping == GROUP_ROWS)
            tiles = ((double)s.m / m.tile + 0.5 * (double)std::min<int64_t>(s.m, s.groups)) * (double)((s.n + m.tile - 1) / m.tile);
        for (int p : parts) {
            if (p > 1 && (!may_split || s.grouping != GROUP_NONE || steps / p < 4 || (double)s.m * (double)s.n * p > 1 << 26)) break;
            const int64_t share = (steps + p - 1) / p;
            const double each = std::ceil(tiles * p / units), pairs = m.both > 0.0 ? std::floor(each / 2.0) : 0.0, rest = each - 2.0 * pairs;
            double t = (double)share * (pairs * m.both + rest * m.alone) + (m.tile == BIG_TILE ? m.ends + 4.0 * (rest - 1.0) : (pairs + rest) * m.ends);
            if (s.grouping == GROUP_STEPS) t = std::max(t, 2.0 * (double)share * m.alone + m.ends);
            t = std::max(t, memory);
            if (p > 1) t += 6.0 + (double)(p + 1) * (double)s.m * (double)s.n * 4.0 / 3.5e6;
            if (t < least) {
                least = t;
                best = Cut{m.tile, (int)((steps + share - 1) / share), (int)share};
            }
        }
    }
    return best;
}
int64_t split_bytes(const Shape &s, int dtype)
{
    const int n = cut_of(s, dtype, true, s.n % 8 == 0).splits;
    return n > 1 ? block((int64_t)n * s.m * s.n * 4) : 0;
}

// Queues the product that `g` describes (operands, epilogue), and the join if it is split.
int run_product(hipStream_t st, int dtype, Forms forms, Epilogue epi, const Shape &s, ProductArgs g, void *split_work)
{
    if (s.m == 0 || (s.grouping == GROUP_STEPS && s.groups == 0)) return ALPA_DP_OK;
    const int64_t es = element(dtype);
    g.M = (int)s.m;
    g.N = (int)s.n;
    // the longer of the two operands' contractions: one may be padded with zeros
    g.K = s.grouping == GROUP_STEPS ? (int)s.k : std::max(g.a_k, g.b_k);
    g.grouping = s.grouping;
    g.experts = s.groups;
    g.wide = by16(g.out) && by16(g.z) && by16(g.residual) && by16(g.bias) && g.ldo * es % 16 == 0 && g.ldz * es % 16 == 0 &&
             g.ldr * es % 16 == 0 && (s.grouping == GROUP_NONE || s.n * es % 16 == 0) &&
             (s.grouping != GROUP_STEPS || g.b_expert * es % 16 == 0);
    const bool may_split = epi != EPI_LOSS && epi != EPI_GRAD && (epi != EPI_SUM || g.total);
    Cut cut = cut_of(s, dtype, may_split, s.n % 8 == 0 || epi == EPI_LOSS);
    // (parts of a split product and statistics go to work memory, where everything is aligned)
    if (cut.tile == BIG_TILE && cut.splits == 1 && epi != EPI_LOSS && !g.wide) cut = cut_of(s, dtype, false, false);
    const int64_t tiles = tiles_of(s, cut.tile);
    if (tiles > (1 << 30)) return fail(ALPA_DP_EINVAL, "result too large");
    g.row_tiles = (int)(s.grouping == GROUP_ROWS ? slots_at_most(s.m, s.groups, cut.tile) : (s.m + cut.tile - 1) / cut.tile);
    g.col_tiles = (int)((s.n + cut.tile - 1) / cut.tile);
    g.splits = cut.splits;
    g.split_steps = cut.splits > 1 ? cut.split_steps : (int)((g.K * es + STEP_BYTES - 1) / STEP_BYTES);
    if (g.splits > 1) {
        g.sum = (float *)split_work;
        ProductArgs part = g;
        part.first = 1;
        part.last = 0;
        part.scale = nullptr;
        part.bias = nullptr;
        HIPCHK(launch_product(st, dtype, forms, EPI_SUM, cut.tile, part));
        HIPCHK(launch_join(st, dtype, epi, g));
        return ALPA_DP_OK;
    }
    HIPCHK(launch_product(st, dtype, forms, epi, cut.tile, g));
    return ALPA_DP_OK;
}

// Operands of a product over `k`: an operand whose contraction is contiguous (its row) has it with its padding.
ProductArgs operands(Forms forms, const Source &a, const Source &b, int64_t k, int dtype)
{
    ProductArgs g{};
    g.a = a.p;
    g.b = b.p;
    g.lda = a.ld * element(dtype);
    g.ldb = b.ld * element(dtype);
    g.a_k = (int)(forms == FORM_CC ? k : a.len);
    g.b_k = (int)(forms == FORM_RR ? b.len : k);
    g.a_len = (int)a.len;
    g.b_len = (int)b.len;
    g.splits = 1;
    g.first = g.last = 1;
    g.low = -INFINITY;
    return g;
}
void result(ProductArgs &g, const alpa_mat_t &out)
{
    g.out = (char *)out.p;
    g.ldo = out.ld;
}

// ---------------------------------------------------------------- products of dense and expert layers

// Parts of the work memory, experts < 0: one weight for all rows.
struct ForwardWork {
    int64_t x, w, split, total;         // offsets
    ForwardWork(int dtype, int64_t rows, int experts, int64_t n_in, int64_t n_out, const alpa_mat_t &xm, const alpa_mat_t &wm)
    {
        x = 0;
        w = x + pack_bytes(xm, rows, n_in, dtype);
        split = w + (rows ? pack_bytes(wm, n_out * std::max(experts, 1), n_in, dtype) : 0);
        total = split + (experts < 0 ? split_bytes(Shape{rows, n_out, n_in, GROUP_NONE, 0}, dtype) : 0);
    }
};

int forward(int dtype, int act, int64_t rows, int experts, int64_t n_in, int64_t n_out, const int32_t *offsets, const alpa_mat_t &x,
            const alpa_mat_t &w, const void *bias, const alpa_mat_t &residual, const alpa_mat_t &y, const alpa_mat_t &z, char *work,
            int64_t work_bytes, hipStream_t st)
{
    TRY(check_sizes(dtype, rows, n_in, n_out, ALPA_LAYER_MAX_WIDTH));
    if (act < ALPA_ACT_NONE || act > ALPA_ACT_SILU) return fail(ALPA_DP_EINVAL, "unknown activation");
    if (rows == 0) return ALPA_DP_OK;
    TRY(check_mat(x, rows, n_in, dtype, false, "x is null"));
    TRY(check_mat(w, n_out, n_in, dtype, false, "w is null"));
    TRY(check_mat(y, rows, n_out, dtype, false, "y is null"));
    TRY(check_mat(z, rows, n_out, dtype, true, ""));
    TRY(check_mat(residual, rows, n_out, dtype, true, ""));
    TRY(check_vector(bias, element(dtype)));
    const ForwardWork at(dtype, rows, experts, n_in, n_out, x, w);
    TRY(check_work(work, work_bytes, at.total));
    Packs packs;
    const Source xs = packs.add(x, rows, n_in, dtype, work + at.x);
    const Source ws = packs.add(w, n_out * std::max(experts, 1), n_in, dtype, work + at.w);
    TRY(packs.queue(st, dtype));
    ProductArgs g = operands(FORM_RR, xs, ws, n_in, dtype);
    const Epilogue epi = epilogue_of(act, g);
    result(g, y);
    g.bias = (const char *)bias;
    g.residual = (const char *)residual.p;
    g.ldr = residual.p ? residual.ld : 0;
    g.z = (char *)z.p;
    g.ldz = z.p ? z.ld : 0;
    g.offsets = offsets;
    g.b_expert = n_out * g.ldb;
    return run_product(st, dtype, FORM_RR, epi, Shape{rows, n_out, n_in, experts < 0 ? GROUP_NONE : GROUP_ROWS, std::max(experts, 0)}, g,
                       work + at.split);
}

// Elements of dy below which a slot of the slope's kernel has 16 rows instead of 64, so that a wave has four and more of them run at once (backward pass to
// w and bias: 4096 x 4096 51 -> 42 us, 2000 x 4100 36 -> 33, 4096 x 8192 64 -> 65); the sums of the slots grow fourfold.
constexpr int SMALL_SLOPE = 1 << 25;

struct BackwardWork {
    int64_t dz, part, tops, x, w, split, total;     // offsets; tops: the scale of dz and what it is found from
    int64_t ldd;
    int slots, slot_rows;
    bool scaled;
    // (dym, xm and wm with p NULL if they are not read)
    BackwardWork(int dtype, int act, int64_t rows, int experts, int64_t n_in, int64_t n_out, const alpa_mat_t &dym, const alpa_mat_t &xm,
                 const alpa_mat_t &wm)
    {
        ldd = round_up(n_out, 16 / element(dtype));
        slot_rows = rows * n_out < SMALL_SLOPE ? 16 : 64;
        slots = (int)(experts < 0 ? (rows + slot_rows - 1) / slot_rows : slots_at_most(rows, experts, slot_rows));
        dz = 0;
        part = dz + (act == ALPA_ACT_NONE ? pack_bytes(dym, rows, n_out, dtype) : block(rows * ldd * element(dtype)));
        scaled = dtype == ALPA_F16 && act >= ALPA_ACT_GELU && rows > 0;
        tops = part + block((int64_t)slots * n_out * 4);
        x = tops + (scaled ? block((1 + TOP_PARTS) * 4) : 0);
        w = x + pack_bytes(xm, rows, n_in, dtype);
        split = w + (rows ? pack_bytes(wm, n_out * std::max(experts, 1), n_in, dtype) : 0);
        int64_t most = 0;
        if (experts < 0)
            most = std::max(split_bytes(Shape{rows, n_in, n_out, GROUP_NONE, 0}, dtype),
                            split_bytes(Shape{n_out, n_in, rows, GROUP_NONE, 0}, dtype));
        total = split + most;
    }
};

int backward(int dtype, int act, int64_t rows, int experts, int64_t n_in, int64_t n_out, const int32_t *offsets, const alpa_mat_t &dy,
             const alpa_mat_t &z, const alpa_mat_t &x, const alpa_mat_t &w, const alpa_mat_t &dx, const alpa_mat_t &dw, void *dbias,
             char *work, int64_t work_bytes, hipStream_t st)
{
    TRY(check_sizes(dtype, rows, n_in, n_out, ALPA_LAYER_MAX_WIDTH));
    if (act < ALPA_ACT_NONE || act > ALPA_ACT_SILU) return fail(ALPA_DP_EINVAL, "unknown activation");
    TRY(check_mat(dy, rows, n_out, dtype, false, "dy is null"));
    TRY(check_mat(z, rows, n_out, dtype, act == ALPA_ACT_NONE, "z is null, and the activation has a slope"));
    TRY(check_mat(x, rows, n_in, dtype, !dw.p, "x is null, and dw is wanted"));
    TRY(check_mat(w, rows ? n_out : 0, n_in, dtype, !dx.p, "w is null, and dx is wanted"));
    TRY(check_mat(dx, rows, n_in, dtype, true, ""));
    TRY(check_mat(dw, n_out, n_in, dtype, true, ""));
    TRY(check_vector(dbias, element(dtype)));
    const alpa_mat_t none{nullptr, 0};
    const BackwardWork at(dtype, act, rows, experts, n_in, n_out, dy, dw.p ? x : none, dx.p ? w : none);
    TRY(check_work(work, work_bytes, at.total));

    const bool grouped = experts >= 0, has_z = act != ALPA_ACT_NONE, products = dx.p || dw.p;
    Source dz{(const char *)dy.p, dy.ld, n_out}, xs{}, ws{};
    float *const scale = at.scaled ? (float *)(work + at.tops) : nullptr;
    if (rows > 0 && (dbias || (has_z && products))) {
        SlopeArgs s{};
        const int64_t es = element(dtype);
        s.dy = (const char *)dy.p;
        s.lddy = dy.ld;
        s.z = has_z ? (const char *)z.p : nullptr;
        s.ldz = has_z ? z.ld : 0;
        if (has_z && products) {
            s.dz = work + at.dz;
            s.ldd = at.ldd;
            dz = Source{s.dz, at.ldd, at.ldd};
            s.scale = scale;
            s.tops = scale ? scale + 1 : nullptr;
        }
        s.part = dbias ? (float *)(work + at.part) : nullptr;
        s.rows = (int)rows;
        s.N = (int)n_out;
        s.slots = at.slots;
        s.slot_rows = at.slot_rows;
        s.experts = grouped ? experts : 0;
        s.offsets = offsets;
        s.act = act;
        const uint64_t places = (uint64_t)s.dy | (uint64_t)s.z | (uint64_t)(s.lddy * es) | (uint64_t)(s.ldz * es);
        s.bytes = places % 16 == 0 ? 16 : places % 8 == 0 ? 8 : 0;
        HIPCHK(launch_slope(st, dtype, s));
    }
    Packs packs;
    if (rows > 0 && !has_z && products) dz = packs.add(dy, rows, n_out, dtype, work + at.dz);
    if (dx.p && rows > 0) ws = packs.add(w, n_out * std::max(experts, 1), n_in, dtype, work + at.w);
    if (dw.p) xs = packs.add(x, rows, n_in, dtype, work + at.x);
    TRY(packs.queue(st, dtype));
    if (dx.p && rows > 0) {
        ProductArgs g = operands(FORM_RC, dz, ws, n_out, dtype);
        result(g, dx);
        g.scale = scale;
        g.offsets = offsets;
        g.b_expert = n_out * g.ldb;
        TRY(run_product(st, dtype, FORM_RC, EPI_LINE, Shape{rows, n_in, n_out, grouped ? GROUP_ROWS : GROUP_NONE, std::max(experts, 0)}, g,
                        work + at.split));
    }
    if (dw.p) {
        ProductArgs g = operands(FORM_CC, dz, xs, rows, dtype);
        result(g, dw);
        g.scale = scale;
        g.offsets = offsets;
        g.b_expert = n_out * dw.ld;
        TRY(run_product(st, dtype, FORM_CC, EPI_LINE, Shape{n_out, n_in, rows, grouped ? GROUP_STEPS : GROUP_NONE, std::max(experts, 0)}, g,
                        work + at.split));
    }
    if (dbias)
        HIPCHK(launch_bias_sum(st, dtype, (const float *)(work + at.part), (char *)dbias, (int)rows, (int)n_out, rows ? at.slots : 0, at.slot_rows,
                               grouped ? experts : 0, offsets));
    return ALPA_DP_OK;
}

int check_experts(int experts, const int32_t *offsets)
{
    if (experts < 1 || experts > ALPA_LAYER_MAX_EXPERTS) return fail(ALPA_DP_EINVAL, "experts out of range");
    if (!offsets) return fail(ALPA_DP_EINVAL, "offsets is null");
    return check_vector(offsets, 4);
}

// ---------------------------------------------------------------- loss over a vocabulary

int64_t stripes_of(int64_t words) { return (words + STRIPE - 1) / STRIPE; }

// A piece's gradient of the logits is kept to 256 MiB, what the last-level cache holds, in pieces of one size: a multiple of the columns that
// give every compute unit the same number of the larger tiles.  A piece has 1024 words at least, as far as there are so many, so that its products
// have depth; rows that would then make it larger (131072 in 16 bits) go in blocks, whose shares of dw are summed in 32 bits.
struct LossWork {
    int64_t pieces, piece;              // number, words in each
    int64_t blocks, rows;               // number, rows in each
    int64_t coef, scale, x, w, grad, sum, sum_w, split, total;
    LossWork(int dtype, int64_t all_rows, int64_t n_in, int64_t words, const alpa_mat_t &xm, const alpa_mat_t &wm)
    {
        constexpr int64_t ROOM = 256ll << 20;
        const int64_t es = element(dtype), least = std::min<int64_t>(4 * BIG_TILE, round_up(words, BIG_TILE));
        const int64_t most_rows = ROOM / (least * es);
        blocks = std::max<int64_t>((all_rows + most_rows - 1) / most_rows, 1);
        rows = blocks > 1 ? round_up((all_rows + blocks - 1) / blocks, BIG_TILE) : all_rows;
        blocks = std::max<int64_t>(rows ? (all_rows + rows - 1) / rows : 1, 1);
        const int64_t r = std::max<int64_t>(rows, 1), row_tiles = (r + BIG_TILE - 1) / BIG_TILE;
        const int64_t most = std::min<int64_t>(std::max<int64_t>(ROOM / (r * es) / BIG_TILE * BIG_TILE, least), MAX_STRIDE / es);
        int64_t even = BIG_TILE;
        while (even * 2 <= most && even / BIG_TILE * row_tiles % 256 != 0) even *= 2;
        pieces = (words + most - 1) / most;
        piece = std::min(round_up((words + pieces - 1) / pieces, even), most);
        pieces = (words + piece - 1) / piece;
        piece = std::min(piece, round_up(words, BIG_TILE));
        coef = 0;
        scale = coef + block(std::max<int64_t>(all_rows, 1) * 4);
        x = scale + 256;
        w = x + pack_bytes(xm, all_rows, n_in, dtype);
        // (of the weights, a piece at a time; those behind the first piece lie as that does or not, so there may be room for nothing)
        grad = w + piece_bytes(wm, all_rows, n_in, dtype);
        sum = grad + block(r * piece * es);
        sum_w = sum + (pieces > 1 ? block(all_rows * n_in * 4) : 0);
        split = sum_w + (blocks > 1 ? block(piece * n_in * 4) : 0);
        int64_t parts = 0;
        for (const int64_t m : {rows, all_rows - (blocks - 1) * rows})
            for (const int64_t n : {piece, words - (pieces - 1) * piece})
                parts = std::max(parts, std::max(split_bytes(Shape{m, n_in, n, GROUP_NONE, 0}, dtype), split_bytes(Shape{n, n_in, m, GROUP_NONE, 0}, dtype)));
        total = split + parts;
    }
    int64_t piece_bytes(const alpa_mat_t &wm, int64_t rows, int64_t n_in, int dtype) const
    {
        return rows ? pack_bytes(wm, piece, n_in, dtype) : 0;
    }
};

// Forward: statistics of stripes, logits of the targets, copies of operands.
struct EvalWork {
    int64_t stat, at_target, x, w, total;
    EvalWork(int dtype, int64_t rows, int64_t n_in, int64_t words, const alpa_mat_t &xm, const alpa_mat_t &wm)
    {
        stat = 0;
        at_target = stat + block(stripes_of(words) * rows * 8);
        x = at_target + block(rows * 4);
        w = x + pack_bytes(xm, rows, n_in, dtype);
        total = w + (rows ? pack_bytes(wm, words, n_in, dtype) : 0);
    }
};

}  // namespace

extern "C" {

int64_t alpa_linear_forward_work(int dtype, int64_t rows, int64_t n_in, int64_t n_out, alpa_mat_t x, alpa_mat_t w)
{
    if (!type_ok(dtype) || !sizes_ok(rows, n_in, n_out, ALPA_LAYER_MAX_WIDTH)) return 0;
    return ForwardWork(dtype, rows, -1, n_in, n_out, x, w).total;
}

int alpa_linear_forward(int dtype, int act, int64_t rows, int64_t n_in, int64_t n_out, alpa_mat_t x, alpa_mat_t w, const void *bias,
                        alpa_mat_t residual, alpa_mat_t y, alpa_mat_t z, void *work, int64_t work_bytes, void *hip_stream)
{
    return forward(dtype, act, rows, -1, n_in, n_out, nullptr, x, w, bias, residual, y, z, (char *)work, work_bytes,
                   (hipStream_t)hip_stream);
}

int64_t alpa_linear_backward_work(int dtype, int act, int64_t rows, int64_t n_in, int64_t n_out, alpa_mat_t dy, alpa_mat_t x, alpa_mat_t w)
{
    if (!type_ok(dtype) || !sizes_ok(rows, n_in, n_out, ALPA_LAYER_MAX_WIDTH)) return 0;
    return BackwardWork(dtype, act, rows, -1, n_in, n_out, dy, x, w).total;
}

int alpa_linear_backward(int dtype, int act, int64_t rows, int64_t n_in, int64_t n_out, alpa_mat_t dy, alpa_mat_t z, alpa_mat_t x,
                         alpa_mat_t w, alpa_mat_t dx, alpa_mat_t dw, void *dbias, void *work, int64_t work_bytes, void *hip_stream)
{
    return backward(dtype, act, rows, -1, n_in, n_out, nullptr, dy, z, x, w, dx, dw, dbias, (char *)work, work_bytes,
                    (hipStream_t)hip_stream);
}

int64_t alpa_experts_forward_work(int dtype, int64_t rows, int experts, int64_t n_in, int64_t n_out, alpa_mat_t x, alpa_mat_t w)
{
    if (!type_ok(dtype) || !sizes_ok(rows, n_in, n_out, ALPA_LAYER_MAX_WIDTH) || experts < 1 || experts > ALPA_LAYER_MAX_EXPERTS) return 0;
    return ForwardWork(dtype, rows, experts, n_in, n_out, x, w).total;
}

int alpa_experts_forward(int dtype, int act, int64_t rows, int experts, int64_t n_in, int64_t n_out, const int32_t *offsets, alpa_mat_t x,
                         alpa_mat_t w, const void *bias, alpa_mat_t residual, alpa_mat_t y, alpa_mat_t z, void *work, int64_t work_bytes,
                         void *hip_stream)
{
    TRY(check_experts(experts, offsets));
    return forward(dtype, act, rows, experts, n_in, n_out, offsets, x, w, bias, residual, y, z, (char *)work, work_bytes,
                   (hipStream_t)hip_stream);
}

int64_t alpa_experts_backward_work(int dtype, int act, int64_t rows, int experts, int64_t n_in, int64_t n_out, alpa_mat_t dy, alpa_mat_t x,
                                   alpa_mat_t w)
{
    if (!type_ok(dtype) || !sizes_ok(rows, n_in, n_out, ALPA_LAYER_MAX_WIDTH) || experts < 1 || experts > ALPA_LAYER_MAX_EXPERTS) return 0;
    return BackwardWork(dtype, act, rows, experts, n_in, n_out, dy, x, w).total;
}

int alpa_experts_backward(int dtype, int act, int64_t rows, int experts, int64_t n_in, int64_t n_out, const int32_t *offsets,
                          alpa_mat_t dy, alpa_mat_t z, alpa_mat_t x, alpa_mat_t w, alpa_mat_t dx, alpa_mat_t dw, void *dbias, void *work,
                          int64_t work_bytes, void *hip_stream)
{
    TRY(check_experts(experts, offsets));
    return backward(dtype, act, rows, experts, n_in, n_out, offsets, dy, z, x, w, dx, dw, dbias, (char *)work, work_bytes,
                    (hipStream_t)hip_stream);
}

int64_t alpa_vocab_loss_forward_work(int dtype, int64_t rows, int64_t n_in, int64_t words, alpa_mat_t x, alpa_mat_t w)
{
    if (!type_ok(dtype) || !sizes_ok(rows, n_in, words, ALPA_LAYER_MAX_WORDS)) return 0;
    return EvalWork(dtype, rows, n_in, words, x, w).total;
}

int alpa_vocab_loss_forward(int dtype, int64_t rows, int64_t n_in, int64_t words, alpa_mat_t x, alpa_mat_t w, const int64_t *target,
                            float *loss, float *lse, void *work, int64_t work_bytes, void *hip_stream)
{
    TRY(check_sizes(dtype, rows, n_in, words, ALPA_LAYER_MAX_WORDS));
    if (rows == 0) return ALPA_DP_OK;
    TRY(check_mat(x, rows, n_in, dtype, false, "x is null"));
    TRY(check_mat(w, words, n_in, dtype, false, "w is null"));
    if (!target || !loss || !lse) return fail(ALPA_DP_EINVAL, "target, loss or lse is null");
    TRY(check_vector(target, 8));
    TRY(check_vector(loss, 4));
    TRY(check_vector(lse, 4));
    const EvalWork at(dtype, rows, n_in, words, x, w);
    TRY(check_work(work, work_bytes, at.total));
    const hipStream_t st = (hipStream_t)hip_stream;
    char *base = (char *)work;
    Packs packs;
    const Source xs = packs.add(x, rows, n_in, dtype, base + at.x), ws = packs.add(w, words, n_in, dtype, base + at.w);
    TRY(packs.queue(st, dtype));
    ProductArgs g = operands(FORM_RR, xs, ws, n_in, dtype);
    g.target = target;
    g.stat = (float2 *)(base + at.stat);
    g.at_target = (float *)(base + at.at_target);
    TRY(run_product(st, dtype, FORM_RR, EPI_LOSS, Shape{rows, words, n_in, GROUP_NONE, 0}, g, nullptr));
    HIPCHK(launch_loss(st, g.stat, (int)stripes_of(words), (int)rows, g.at_target, target, words, loss, lse));
    return ALPA_DP_OK;
}

int64_t alpa_vocab_loss_backward_work(int dtype, int64_t rows, int64_t n_in, int64_t words, alpa_mat_t x, alpa_mat_t w)
{
    if (!type_ok(dtype) || !sizes_ok(rows, n_in, words, ALPA_LAYER_MAX_WORDS)) return 0;
    return LossWork(dtype, rows, n_in, words, x, w).total;
}

int alpa_vocab_loss_backward(int dtype, int64_t rows, int64_t n_in, int64_t words, const float *dloss, alpa_mat_t x, alpa_mat_t w,
                             const int64_t *target, const float *lse, alpa_mat_t dx, alpa_mat_t dw, void *work, int64_t work_bytes,
                             void *hip_stream)
{
    TRY(check_sizes(dtype, rows, n_in, words, ALPA_LAYER_MAX_WORDS));
    TRY(check_mat(x, rows, n_in, dtype, false, "x is null"));
    TRY(check_mat(w, rows ? words : 0, n_in, dtype, false, "w is null"));
    TRY(check_mat(dx, rows, n_in, dtype, true, ""));
    TRY(check_mat(dw, words, n_in, dtype, true, ""));
    if (rows > 0 && (!target || !dloss || !lse)) return fail(ALPA_DP_EINVAL, "target, dloss or lse is null");
    TRY(check_vector(target, 8));
    TRY(check_vector(dloss, 4));
    TRY(check_vector(lse, 4));
    const LossWork at(dtype, rows, n_in, words, x, w);
    TRY(check_work(work, work_bytes, at.total));
    if (!dx.p && !dw.p) return ALPA_DP_OK;
    const hipStream_t st = (hipStream_t)hip_stream;
    char *base = (char *)work;
    float *coef = (float *)(base + at.coef), *scale = (float *)(base + at.scale);
    HIPCHK(launch_coef(st, dloss, target, words, (int)rows, coef, scale));
    const int64_t es = element(dtype);
    Source xs{}, ws{};
    for (int64_t p = 0; p < at.pieces; ++p) {
        const int64_t word0 = p * at.piece, n = std::min(at.piece, words - word0);
        const Source grad{base + at.grad, at.piece, round_up(n, 16 / es)};
        if (rows > 0) {
            // (pieces are multiples of 256 words, so a piece's rows are aligned as the first piece's are)
            Packs packs;
            if (p == 0) xs = packs.add(x, rows, n_in, dtype, base + at.x);
            ws = packs.add(alpa_mat_t{(char *)w.p + word0 * w.ld * es, w.ld}, n, n_in, dtype, base + at.w);
            TRY(packs.queue(st, dtype));
        }
        for (int64_t b = 0; b < at.blocks; ++b) {
            const int64_t row0 = b * at.rows, m = std::min(at.rows, rows - row0);
            const Source xb{xs.p + row0 * xs.ld * es, xs.ld, xs.len};
            if (rows > 0) {
                ProductArgs g = operands(FORM_RR, xb, ws, n_in, dtype);
                result(g, alpa_mat_t{base + at.grad, at.piece});
                g.target = target + row0;
                g.word0 = word0;
                g.lse = lse + row0;
                g.coef = coef + row0;
                TRY(run_product(st, dtype, FORM_RR, EPI_GRAD, Shape{m, n, n_in, GROUP_NONE, 0}, g, nullptr));
            }
            if (dx.p && rows > 0) {
                ProductArgs g = operands(FORM_RC, grad, ws, n, dtype);
                result(g, alpa_mat_t{(char *)dx.p + row0 * dx.ld * es, dx.ld});
                g.scale = scale;
                g.sum = (float *)(base + at.sum) + row0 * n_in;
                g.first = p == 0;
                g.last = p + 1 == at.pieces;
                TRY(run_product(st, dtype, FORM_RC, at.pieces > 1 ? EPI_SUM : EPI_LINE, Shape{m, n_in, n, GROUP_NONE, 0}, g, base + at.split));
            }
            if (dw.p) {
                ProductArgs g = operands(FORM_CC, grad, xb, m, dtype);
                result(g, alpa_mat_t{(char *)dw.p + word0 * dw.ld * es, dw.ld});
                g.scale = scale;
                if (at.blocks > 1) g.sum = g.total = (float *)(base + at.sum_w);
                g.first = b == 0;
                g.last = b + 1 == at.blocks;
                TRY(run_product(st, dtype, FORM_CC, at.blocks > 1 ? EPI_SUM : EPI_LINE, Shape{n, n_in, m, GROUP_NONE, 0}, g, base + at.split));
            }
        }
    }
    return ALPA_DP_OK;
}

}  // extern "C"

namespace alpa {

hipError_t launch_product(hipStream_t st, int dtype, Forms forms, Epilogue epi, int tile, const ProductArgs &g)
{
    return dtype == ALPA_F32   ? launch_product_f32(st, forms, epi, tile, g)
           : dtype == ALPA_F16 ? launch_product_f16(st, forms, epi, tile, g)
                               : launch_product_bf16(st, forms, epi, tile, g);
}

}  // namespace alpa
