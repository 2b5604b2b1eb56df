// C ABI of the refiner's attention and of its heads' norm (declared in
// include/mixrt.h): checks of their descriptors (pure host code), how a call is
// split, and the launches of the kernels in mixrt_attend_*.hip and
// mixrt_rotary_norm.hip on the context's stream.
#include "mixrt.h"

#include <cmath>

#include "mixrt_apart.hpp"
#include "mixrt_attend.hpp"
#include "mixrt_ctx.hpp"
#include "mixrt_refine.hpp"

namespace mixrt {
namespace {

constexpr int kCUs = 256;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Rows that one chain of 32-bit sums takes at most, a multiple of 64: the matrix
// instructions of float32 add two terms, those of the 16-bit types 16, and a chain is
// about 1024 or 2048 of them, so that its roundings stay below the result's.
int64_t longest(int dtype) { return attend_elem(dtype) == 4 ? 2048 : 32768; }

// Splits of a walk over n rows, none longer than most; per is a multiple of step.
void divide(int64_t n, int64_t s, int64_t most, int64_t step, int *splits, int *per)
{
    if (s < ceil_div(n, most)) s = ceil_div(n, most);
    if (s < 1) s = 1;
    int64_t p = ceil_div(ceil_div(n, s), step) * step;
    if (p < step) p = step;
    *per = (int)p;
    *splits = (int)(n > 0 ? ceil_div(n, p) : 1);
}

// Splits of a long walk in passes.  A chain's length bounds a split's, so their number
// grows with the walk, and with the rows the scratch would be their product (one entry,
// 16 heads of 128, 65,536 tokens among themselves, f32: 32 parts, 17 GB).  So a pass has
// at most four, or as many as the call runs at once, or a 64th of all, whose joins would
// else add up roundings.
void in_passes(AttendPlan *p, int64_t blocks, int64_t s)
{
    p->passes = 1;
    int64_t most = s > 4 ? s : 4;
    const int64_t fill = blocks > 0 ? ceil_div(8 * kCUs, blocks) : 1;
    if (most < fill) most = fill;
    if (most < ceil_div(p->splits, 64)) most = ceil_div(p->splits, 64);
    if (p->shared || p->splits <= most) return;
    p->passes = (int)ceil_div(p->splits, most);
    p->splits = (int)ceil_div(p->splits, p->passes);
}

// Blocks that run together, by the registers and LDS that the kernels take.
int64_t resident(int D, int dtype, int a_cu)
{
    return kCUs * (attend_dim(D) * attend_elem(dtype) <= 128 ? a_cu : 1);
}

// Splits of long walks: the blocks' rounds over the chip are whole, so s splits take
// ceil(blocks s / slots) / (blocks s / slots) of what they could, and each is a part to
// write and to join (about 1/25).  Two 720p views with two reference views each, 12 and
// 3 heads of 64, bf16: the keys' gradient has 342 blocks for 512 slots; all of a
// training step's calls take 1172 us with 1 split, 1122 with 2, 1139 with 3, 1029 with
// 4, 1077 with 6.
int64_t whole_rounds(int64_t n, int64_t blocks, int64_t slots, int64_t least)
{
    int64_t best = 1;
    double low = 1e30;
    for (int64_t s = 1; s <= 16 && blocks > 0 && (s == 1 || n / s >= least); ++s) {
        const double rounds = (double)(blocks * s) / slots;
        const double cost = std::ceil(rounds) / rounds + 0.04 * s;
        if (cost < low) {
            low = cost;
            best = s;
        }
    }
    return best;
}

// Splits where a block's waves share its columns: enough for two blocks a CU, of least
// rows.  (One token of 32 heads of 128 over 14,400 keys of 8, bf16: 28 splits 20.7 us,
// 57 19.4, 113 25.2.)
int64_t enough(int64_t n, int64_t blocks, int64_t least)
{
    const int64_t s = blocks > 0 ? 2 * kCUs / blocks : 1;
    return s < ceil_div(n, least) ? s : ceil_div(n, least);
}

// Whether blocks of 32 columns run, whose waves divide the rows, and not blocks of 128:
// where these would leave half of their waves without columns, or be few for the chip
// also when their walks of rows are split.  (8 queries of 32 heads of 128 over 32,768
// keys of 2, f32: the queries' gradient 262 us, with 128 columns 818.)
bool shares(int64_t heads, int64_t cols, int64_t rows)
{
    const int64_t splits = 1 + rows / 1024 < 16 ? 1 + rows / 1024 : 16;
    return cols <= 64 || heads * ceil_div(cols, 128) * splits < kCUs;
}

int blocks_of(int64_t n, int cols)
{
    const int64_t b = ceil_div(n, cols);
    return b < 1 ? 1 : (int)b;
}

}  // namespace

AttendPlan plan_attend(int B, int H, int Hk, int64_t Tq, int64_t Tk, int D, int dtype, int entries)
{
    AttendPlan p{};
    p.pack = 1;
    // few queries: the heads that share keys lie beside each other in the columns
    if (Tq <= 16)
        for (int n = 2; n <= 8; ++n)
            if (H / Hk % n == 0 && Tq * n <= 32) p.pack = n;
    const int64_t cols = Tq * p.pack, heads = (int64_t)B * (H / p.pack);
    p.shared = shares(heads, cols, Tk);
    p.cols = p.shared ? 32 : 128;
    if (attend_elem(dtype) == 2 && D <= 64 && entries == 0 && !p.shared && cols > 1024) p.cols = 256;
    p.blocks = blocks_of(cols, p.cols);
    const int64_t blocks = heads * p.blocks;
    const int64_t s = p.shared ? enough(Tk, blocks, 256)
                               : whole_rounds(Tk, blocks, resident(D, dtype, 2), 512);
    divide(Tk, s, longest(dtype), p.shared ? 128 : 64, &p.splits, &p.per);
    in_passes(&p, blocks, s);
    return p;
}

AttendPlan plan_attend_dq(int B, int H, int Hk, int64_t Tq, int64_t Tk, int D, int dtype,
                          int entries)
{
    AttendPlan p{};
    p.pack = 1;
    const int64_t heads = (int64_t)B * H;
    p.shared = shares(heads, Tq, Tk);
    // (a wave's own tiles beside the table's sums may be more than a CU's LDS; about
    // 16 KB are other things)
    const int tiles = 4 * 2 * 32 * (attend_dim(D) * attend_elem(dtype) + 16);
    if (entries && tiles + attend_hist_bytes(entries) + 16384 > 163840) p.shared = 0;
    p.cols = p.shared ? 32 : 128;
    p.blocks = blocks_of(Tq, p.cols);
    int64_t most = longest(dtype);
    if (entries && p.shared && most > 4096) most = 4096;   // (1024 keys of a lane's table sums)
    // (float32's products are so slow that a wave's second tile is worth a join)
    const int64_t blocks = heads * p.blocks, least = attend_elem(dtype) == 4 ? 128 : 256;
    const int64_t s = p.shared ? enough(Tk, blocks, least)
                               : whole_rounds(Tk, blocks, resident(D, dtype, entries ? 2 : 3), 512);
    divide(Tk, s, most, p.shared ? 128 : 32, &p.splits, &p.per);
    in_passes(&p, blocks, s);
    return p;
}

AttendPlan plan_attend_dkv(int B, int H, int Hk, int64_t Tq, int64_t Tk, int D, int dtype, int)
{
    AttendPlan p{};
    p.pack = 1;
    const int64_t heads = (int64_t)B * Hk;
    p.shared = shares(heads, Tk, H / Hk * Tq);
    p.cols = p.shared ? 32 : 128;
    p.blocks = blocks_of(Tk, p.cols);
    const int rows = attend_kv_rows(attend_dim(D), attend_elem(dtype), p.shared);
    const int64_t tiles = H / Hk * ceil_div(Tq, rows);
    const int64_t blocks = heads * p.blocks;
    const int64_t s = p.shared ? enough(tiles, blocks, 8)
                               : whole_rounds(tiles, blocks, resident(D, dtype, 2), 512 / rows);
    divide(tiles, s, longest(dtype) / rows, p.shared ? 4 : 1, &p.splits, &p.per);
    in_passes(&p, blocks, s);
    return p;
}

}  // namespace mixrt

namespace {

using mixrt::Arrays;
using mixrt::AttendPlan;
using mixrt::bind_device;
using mixrt::clear_err;
using mixrt::fail;
using mixrt::finish_launch;

constexpr int64_t kMaxElements = (int64_t)1 << 40;
constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr int64_t kMaxTokens = (int64_t)1 << 30;
constexpr int kMaxHeads = 65535;
constexpr int kMaxHeadDim = 1024;
constexpr float kLog2e = 1.4426950408889634f;

bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

int elem_size(int dtype)
{
    return dtype == MIXRT_F32 ? 4 : dtype == MIXRT_F16 || dtype == MIXRT_BF16 ? 2 : 0;
}

int check_workspace(mixrt_ctx *ctx, const void *ws, size_t have, size_t need)
{
    if (have < need)
        return fail(ctx, MIXRT_EINVAL, "workspace of %zu bytes, needs %zu", have, need);
    if (need && !ws) return fail(ctx, MIXRT_EINVAL, "workspace is NULL");
    if (!aligned(ws, 16)) return fail(ctx, MIXRT_EINVAL, "workspace not 16-byte aligned");
    return MIXRT_OK;
}

// --- attention --------------------------------------------------------------------

int check_bias(mixrt_ctx *ctx, const mixrt_relative_bias *b)
{
    if (!b) return MIXRT_OK;
    if (b->axes < 1 || b->axes > MIXRT_MAX_BIAS_AXES)
        return fail(ctx, MIXRT_EUNSUPPORTED, "bias.axes=%d outside 1..%d", b->axes,
                    MIXRT_MAX_BIAS_AXES);
    if (b->count < 1 || b->count > MIXRT_MAX_BIAS_BUCKETS)
        return fail(ctx, MIXRT_EUNSUPPORTED, "bias.count=%d outside 1..%d", b->count,
                    MIXRT_MAX_BIAS_BUCKETS);
    if (b->reach < 0 || b->reach > MIXRT_MAX_BIAS_REACH)
        return fail(ctx, MIXRT_EUNSUPPORTED, "bias.reach=%d outside 0..%d", b->reach,
                    MIXRT_MAX_BIAS_REACH);
    return MIXRT_OK;
}

int check_bias_data(mixrt_ctx *ctx, const mixrt_attention *a, const mixrt_relative_bias *b)
{
    if (!b) return MIXRT_OK;
    if (!b->table || !b->buckets) return fail(ctx, MIXRT_EINVAL, "bias.table or buckets is NULL");
    if ((a->queries && !b->q_pos) || (a->keys && !b->k_pos))
        return fail(ctx, MIXRT_EINVAL, "bias.q_pos or k_pos is NULL");
    if (!aligned(b->table, 4) || !aligned(b->q_pos, 4) || !aligned(b->k_pos, 4))
        return fail(ctx, MIXRT_EINVAL, "bias.table, q_pos or k_pos not 4-byte aligned");
    if (b->q_pos_stride < 0 || b->q_pos_stride >= kMaxStride || b->k_pos_stride < 0 ||
        b->k_pos_stride >= kMaxStride)
        return fail(ctx, MIXRT_EINVAL, "bias: position strides %lld, %lld",
                    (long long)b->q_pos_stride, (long long)b->k_pos_stride);
    return MIXRT_OK;
}

int check_attention(mixrt_ctx *ctx, const mixrt_attention *a, const mixrt_relative_bias *b)
{
    if (!a) return fail(ctx, MIXRT_EINVAL, "attention is NULL");
    if (a->batch < 0) return fail(ctx, MIXRT_EINVAL, "attention.batch=%d", a->batch);
    if (a->batch > 65535)
        return fail(ctx, MIXRT_EUNSUPPORTED, "attention.batch=%d above 65535", a->batch);
    if (a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads)
        return fail(ctx, MIXRT_EINVAL, "attention.heads=%d for kv_heads=%d", a->heads,
                    a->kv_heads);
    if (a->heads > kMaxHeads)
        return fail(ctx, MIXRT_EUNSUPPORTED, "attention.heads=%d above %d", a->heads, kMaxHeads);
    if (a->head_dim < 1) return fail(ctx, MIXRT_EINVAL, "attention.head_dim=%d", a->head_dim);
    if (a->head_dim > MIXRT_MAX_ATTENTION_DIM)
        return fail(ctx, MIXRT_EUNSUPPORTED, "attention.head_dim=%d above %d", a->head_dim,
                    MIXRT_MAX_ATTENTION_DIM);
    if (!elem_size(a->dtype))
        return fail(ctx, MIXRT_EUNSUPPORTED, "attention.dtype=%d (F32, F16 or BF16)", a->dtype);
    // (scores are in units of log2)
    if (!(a->scale > 0.0f) || !std::isfinite(a->scale * kLog2e))
        return fail(ctx, MIXRT_EINVAL, "attention.scale=%g", a->scale);
    if (a->queries < 0 || a->keys < 0)
        return fail(ctx, MIXRT_EINVAL, "attention.queries=%lld, keys=%lld", (long long)a->queries,
                    (long long)a->keys);
    if (a->queries >= kMaxTokens || a->keys >= kMaxTokens)
        return fail(ctx, MIXRT_EUNSUPPORTED, "attention: 2^30 queries or keys or more");
    const int64_t rows = (int64_t)a->batch * a->heads;
    if (rows > 0 && ((a->queries > a->keys ? a->queries : a->keys) + 1) > kMaxTokens / rows)
        return fail(ctx, MIXRT_EUNSUPPORTED, "attention: 2^30 rows of heads or more");
    if (!aligned(a->lens, 4)) return fail(ctx, MIXRT_EINVAL, "attention.lens not 4-byte aligned");
    if (!aligned(a->lse_rest, 4))
        return fail(ctx, MIXRT_EINVAL, "attention.lse_rest not 4-byte aligned");
    int stage = 0;
    for (auto plan : {mixrt::plan_attend, mixrt::plan_attend_dq, mixrt::plan_attend_dkv}) {
        const AttendPlan p = plan(a->batch, a->heads, a->kv_heads, a->queries, a->keys,
                                  a->head_dim, a->dtype, b ? b->axes * b->count : 0);
        if (mixrt::attend_blocks(p, a->batch, stage++ == 2 ? a->kv_heads : a->heads) >
            mixrt::kMostBlocks256)
            return fail(ctx, MIXRT_EUNSUPPORTED, "attention: %d entries of %d heads, %lld queries "
                        "and %lld keys are too many blocks", a->batch, a->heads,
                        (long long)a->queries, (long long)a->keys);
    }
    return MIXRT_OK;
}

// An array of heads that a call reads or, with out, writes: an output's elements lie
// apart, nested in some order of its three dimensions.
int check_sequence(mixrt_ctx *ctx, const mixrt_attention *a, const mixrt_sequence *s, bool queries,
                   const char *name, bool out)
{
    if (!s) return fail(ctx, MIXRT_EINVAL, "%s is NULL", name);
    const int64_t n[3] = {a->batch, queries ? a->queries : a->keys,
                          queries ? a->heads : a->kv_heads};
    if (n[0] == 0 || n[1] == 0) return MIXRT_OK;
    if (!s->data) return fail(ctx, MIXRT_EINVAL, "%s.data is NULL", name);
    if (!aligned(s->data, elem_size(a->dtype)))
        return fail(ctx, MIXRT_EINVAL, "%s.data not aligned to its element", name);
    const int64_t st[3] = {s->batch_stride, s->token_stride, s->head_stride};
    for (int i = 0; i < 3; ++i)
        if (st[i] < 0 || st[i] >= kMaxStride || (st[i] && n[i] > kMaxElements / st[i]))
            return fail(ctx, MIXRT_EINVAL, "%s: strides %lld, %lld, %lld", name, (long long)st[0],
                        (long long)st[1], (long long)st[2]);
    if (!out) return MIXRT_OK;
    static const int orders[6][3] = {{0, 1, 2}, {0, 2, 1}, {1, 0, 2},
                                     {1, 2, 0}, {2, 0, 1}, {2, 1, 0}};
    for (const auto &order : orders) {
        int64_t span = a->head_dim;
        bool apart = true;
        for (int i = 2; i >= 0; --i) {      // the innermost dimension first
            const int d = order[i];
            if (n[d] == 1) continue;
            apart = apart && st[d] >= span;
            span += (n[d] - 1) * st[d];
        }
        if (apart) return MIXRT_OK;
    }
    return fail(ctx, MIXRT_EINVAL, "%s: strides %lld, %lld, %lld make heads overlap", name,
                (long long)st[0], (long long)st[1], (long long)st[2]);
}

mixrt::Extent extent_of(const mixrt_attention *att, const mixrt_sequence *s, bool queries)
{
    const int64_t size = elem_size(att->dtype);
    return mixrt::Extent{(uint64_t)(uintptr_t)s->data, att->head_dim * size,
                         {att->batch, queries ? att->queries : att->keys,
                          queries ? att->heads : att->kv_heads},
                         {s->batch_stride * size, s->token_stride * size, s->head_stride * size}};
}

// The arrays that a forward and a backward call share.
void add_common(Arrays &m, const mixrt_attention *att, const mixrt_relative_bias *b,
                const mixrt_sequence *q, const mixrt_sequence *k, const mixrt_sequence *v)
{
    m.add(extent_of(att, q, true), "q");
    m.add(extent_of(att, k, false), "k");
    m.add(extent_of(att, v, false), "v");
    m.add(mixrt::flat_extent(att->lens, (int64_t)att->batch * 4), "lens");
    if (!b) return;
    const int64_t entries = att->batch > 0 ? att->batch - 1 : 0;
    m.add(mixrt::flat_extent(b->table, (int64_t)b->axes * b->count * att->heads * 4), "table");
    m.add(mixrt::flat_extent(b->buckets, (int64_t)b->axes * (2 * b->reach + 1)), "buckets");
    m.add(mixrt::Extent{(uint64_t)(uintptr_t)b->q_pos, att->queries * b->axes * 4,
                        {entries + 1, 1, 1}, {b->q_pos_stride * 4, 0, 0}}, "q_pos");
    m.add(mixrt::Extent{(uint64_t)(uintptr_t)b->k_pos, att->keys * b->axes * 4,
                        {entries + 1, 1, 1}, {b->k_pos_stride * 4, 0, 0}}, "k_pos");
}

// An output shares no memory with the other arrays.
int check_apart(mixrt_ctx *ctx, const Arrays &m)
{
    if (const Arrays::One *s = m.shared())
        return fail(ctx, MIXRT_EINVAL, "%s is also another array, or a part of one", s->name);
    return MIXRT_OK;
}

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

// Where a call's scratch lies in its workspace; total bytes.
struct Scratch {
    size_t part, part_lse, delta, table, table_sum, total;
};

Scratch scratch_of(const mixrt_attention *a, const mixrt_relative_bias *b, bool backward)
{
    const int axes = b ? b->axes : 0;
    const size_t rows = (size_t)a->batch * a->heads * a->queries;
    const size_t keys = (size_t)a->batch * a->kv_heads * a->keys;
    Scratch s{};
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t from = at;
        at += round16(bytes);
        return from;
    };
    auto plan = [&](auto fn) {
        return fn(a->batch, a->heads, a->kv_heads, a->queries, a->keys, a->head_dim, a->dtype,
                  axes ? axes * b->count : 0);
    };
    if (!backward) {
        const AttendPlan p = plan(mixrt::plan_attend);
        if (const int slots = mixrt::attend_slots(p)) {
            s.part = take((size_t)slots * rows * a->head_dim * 4);
            s.part_lse = take((size_t)(slots + 1) * rows * 8);
        }
    } else {
        const AttendPlan pq = plan(mixrt::plan_attend_dq), pk = plan(mixrt::plan_attend_dkv);
        const size_t part = (size_t)mixrt::attend_slots(pq) * rows * a->head_dim * 4;
        const size_t both = (size_t)mixrt::attend_slots(pk) * keys * a->head_dim * 8;
        s.part = take(part > both ? part : both);
        s.delta = take(rows * 4);
        if (axes) {
            const size_t entries = (size_t)axes * b->count;
            s.table = take((size_t)a->batch * a->heads * pq.splits * pq.blocks * entries * 4);
            if (pq.passes > 1) s.table_sum = take(entries * a->heads * 8);
        }
    }
    s.total = at;
    return s;
}

mixrt::SeqK seq_k(const mixrt_sequence *s)
{
    return mixrt::SeqK{s->data, s->batch_stride, s->token_stride, s->head_stride};
}

mixrt::AttendK attend_k(const mixrt_attention *a, const mixrt_relative_bias *b)
{
    mixrt::AttendK k{};
    k.B = a->batch;
    k.H = a->heads;
    k.Hk = a->kv_heads;
    k.D = a->head_dim;
    k.Tq = (int)a->queries;
    k.Tk = (int)a->keys;
    k.dtype = a->dtype;
    k.plain_scale = a->scale;
    k.scale = a->scale * kLog2e;
    k.lens = a->lens;
    k.lse_rest = a->lse_rest;
    if (b)
        k.bias = mixrt::BiasK{b->axes,  b->count, b->reach,        b->table,       b->buckets,
                              b->q_pos, b->k_pos, b->q_pos_stride, b->k_pos_stride};
    return k;
}

hipError_t launch_attend(const mixrt::AttendK &k, int stage, hipStream_t stream)
{
    if (k.dtype == mixrt::kF32) return mixrt::launch_attend_f32(k, stage, stream);
    if (k.dtype == mixrt::kF16) return mixrt::launch_attend_f16(k, stage, stream);
    return mixrt::launch_attend_bf16(k, stage, stream);
}

// --- heads normed and turned ----------------------------------------------------------

// Blocks read heads while others write theirs: an output is its own array's input
// (x forward, dy backward: each head is read before it is written, by the lanes that
// write it) or shares memory with no other array of the call.
int check_normed_apart(mixrt_ctx *ctx, const mixrt_rotary *r, const mixrt_normed_heads *heads,
                       int32_t n, bool backward)
{
    auto extent = [&](const mixrt_normed_heads &h, const void *p, int64_t token, int64_t head) {
        const int64_t size = elem_size(h.dtype);
        return mixrt::Extent{(uint64_t)(uintptr_t)p, h.head_dim * size, {r->tokens, h.heads, 1},
                             {token * size, head * size, 0}};
    };
    Arrays m;
    m.add(mixrt::flat_extent(r->pos, r->pairs ? r->tokens * r->axes * 4 : 0), "pos");
    m.add(mixrt::flat_extent(r->freq, (int64_t)r->pairs * 4), "freq");
    m.add(mixrt::flat_extent(r->axis, r->pairs), "axis");
    for (int i = 0; i < n; ++i) {
        const mixrt_normed_heads &h = heads[i];
        const bool in_place = h.out == (backward ? h.dy : h.x);
        m.add(mixrt::flat_extent(h.weight, (int64_t)h.head_dim * 4), "weight");
        if (backward || !in_place) m.add(extent(h, h.x, h.x_token_stride, h.x_head_stride), "x");
        if (backward && !in_place)
            m.add(extent(h, h.dy, h.dy_token_stride, h.dy_head_stride), "dy");
        m.add(extent(h, h.out, h.out_token_stride, h.out_head_stride), backward ? "dx" : "out",
              true);
        if (backward)
            m.add(mixrt::flat_extent(h.dweight, (int64_t)h.head_dim * 4), "dweight", true);
    }
    return check_apart(ctx, m);
}

int check_normed(mixrt_ctx *ctx, const mixrt_rotary *r, float eps, const mixrt_normed_heads *heads,
                 int32_t n, bool backward, bool data, mixrt::RotaryNormLaunch &L)
{
    if (!r) return fail(ctx, MIXRT_EINVAL, "rotary is NULL");
    if (r->tokens < 0) return fail(ctx, MIXRT_EINVAL, "rotary.tokens=%lld", (long long)r->tokens);
    if (r->tokens >= ((int64_t)1 << 31))
        return fail(ctx, MIXRT_EUNSUPPORTED, "rotary: 2^31 tokens or more");
    if (r->axes < 1 || r->axes > MIXRT_MAX_AXES)
        return fail(ctx, MIXRT_EUNSUPPORTED, "rotary.axes=%d outside 1..%d", r->axes,
                    MIXRT_MAX_AXES);
    if (r->layout != MIXRT_ROTARY_HALVES && r->layout != MIXRT_ROTARY_PAIRS)
        return fail(ctx, MIXRT_EUNSUPPORTED, "rotary.layout=%d", r->layout);
    if (r->pairs < 0) return fail(ctx, MIXRT_EINVAL, "rotary.pairs=%d", r->pairs);
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(ctx, MIXRT_EINVAL, "eps=%g", eps);
    if (n < 1 || n > MIXRT_MAX_HEADS_ARRAYS)
        return fail(ctx, MIXRT_EINVAL, "n=%d outside 1..%d", n, MIXRT_MAX_HEADS_ARRAYS);
    if (!heads) return fail(ctx, MIXRT_EINVAL, "heads is NULL");
    if (data && r->pairs > 0 && r->tokens > 0) {
        if (!r->pos || !r->freq || !r->axis)
            return fail(ctx, MIXRT_EINVAL, "rotary.pos, freq or axis is NULL");
        if (!aligned(r->pos, 4) || !aligned(r->freq, 4))
            return fail(ctx, MIXRT_EINVAL, "rotary.pos or freq not 4-byte aligned");
    }
    L.tokens = r->tokens;
    L.axes = r->axes;
    L.pairs = r->pairs;
    L.layout = r->layout;
    L.dtype = heads[0].dtype;
    L.eps = eps;
    L.pos = r->pos;
    L.freq = r->freq;
    L.axis = r->axis;
    L.n = n;
    if (!elem_size(L.dtype))
        return fail(ctx, MIXRT_EUNSUPPORTED, "heads[0].dtype=%d (F32, F16 or BF16)", L.dtype);
    for (int i = 0; i < n; ++i) {
        const mixrt_normed_heads &h = heads[i];
        if (h.dtype != L.dtype)
            return fail(ctx, MIXRT_EINVAL, "heads[%d].dtype=%d beside %d", i, h.dtype, L.dtype);
        if (h.heads < 0 || h.heads > kMaxHeads)
            return fail(ctx, MIXRT_EUNSUPPORTED, "heads[%d].heads=%d outside 0..%d", i, h.heads,
                        kMaxHeads);
        if (h.head_dim < 1 || h.head_dim > kMaxHeadDim)
            return fail(ctx, MIXRT_EUNSUPPORTED, "heads[%d].head_dim=%d outside 1..%d", i,
                        h.head_dim, kMaxHeadDim);
        if (2 * (int64_t)r->pairs > h.head_dim)
            return fail(ctx, MIXRT_EINVAL, "heads[%d].head_dim=%d for %d pairs", i, h.head_dim,
                        r->pairs);
        L.a[i] = mixrt::NormedHeadsK{h.heads,
                                     h.head_dim,
                                     h.x,
                                     h.dy,
                                     h.out,
                                     h.weight,
                                     h.dweight,
                                     h.x_token_stride,
                                     h.x_head_stride,
                                     h.dy_token_stride,
                                     h.dy_head_stride,
                                     h.out_token_stride,
                                     h.out_head_stride};
        if (!data) continue;
        if (!aligned(h.weight, 4) || !aligned(h.dweight, 4))
            return fail(ctx, MIXRT_EINVAL, "heads[%d].weight or dweight not 4-byte aligned", i);
        if (h.heads == 0 || r->tokens == 0) continue;   // none of its heads are touched
        const bool writes = !backward || h.out;
        if (!h.x || (backward && !h.dy) || (!backward && !h.out))
            return fail(ctx, MIXRT_EINVAL, "heads[%d].x, dy or out is NULL", i);
        const size_t size = elem_size(h.dtype);
        if (!aligned(h.x, size) || !aligned(h.out, size) || (backward && !aligned(h.dy, size)))
            return fail(ctx, MIXRT_EINVAL, "heads[%d].x, dy or out not aligned to its element", i);
        const int64_t D = h.head_dim, H = h.heads, T = r->tokens;
        const int64_t st[6] = {h.x_token_stride,   h.x_head_stride,   h.dy_token_stride,
                               h.dy_head_stride,   h.out_token_stride, h.out_head_stride};
        for (int s = 0; s < 6; ++s) {
            if ((s / 2 == 1 && !backward) || (s / 2 == 2 && !writes)) continue;
            const int64_t count = s % 2 ? H : T;
            if (st[s] < 0 || st[s] >= kMaxStride || (st[s] && count > kMaxElements / st[s]))
                return fail(ctx, MIXRT_EINVAL, "heads[%d]: stride %lld", i, (long long)st[s]);
        }
        if (!writes) continue;
        // the output's rows apart: heads inside a token, or tokens inside a head
        const int64_t ot = h.out_token_stride, oh = h.out_head_stride;
        const bool inner = (H == 1 || oh >= D) && (T == 1 || ot >= (H - 1) * oh + D);
        const bool outer = (T == 1 || ot >= D) && (H == 1 || oh >= (T - 1) * ot + D);
        if (!inner && !outer)
            return fail(ctx, MIXRT_EINVAL, "heads[%d]: out strides %lld, %lld make rows overlap",
                        i, (long long)ot, (long long)oh);
        const void *in = backward ? h.dy : h.x;
        const int64_t it = backward ? h.dy_token_stride : h.x_token_stride;
        const int64_t ih = backward ? h.dy_head_stride : h.x_head_stride;
        if (in == h.out && ((T > 1 && it != ot) || (H > 1 && ih != oh)))
            return fail(ctx, MIXRT_EINVAL, "heads[%d]: out is its input with other strides", i);
        if (backward && h.x == h.out)
            return fail(ctx, MIXRT_EINVAL, "heads[%d]: dx is x", i);
    }
    return data ? check_normed_apart(ctx, r, heads, n, backward) : MIXRT_OK;
}

}  // namespace

extern "C" {

int mixrt_rotary_norm_apply(mixrt_ctx *ctx, const mixrt_rotary *rotary, float eps,
                            const mixrt_normed_heads *heads, int32_t n)
{
    if (!ctx) return fail(nullptr, MIXRT_EINVAL, "ctx is NULL");
    clear_err(ctx);
    mixrt::RotaryNormLaunch L{};
    int rc;
    if ((rc = check_normed(ctx, rotary, eps, heads, n, false, true, L))) return rc;
    if ((rc = bind_device(ctx))) return rc;
    return finish_launch(ctx, mixrt::launch_rotary_norm(L, ctx->stream), "rotary_norm");
}

int mixrt_rotary_norm_workspace(const mixrt_rotary *rotary, const mixrt_normed_heads *heads,
                                int32_t n, size_t *bytes)
{
    clear_err(nullptr);
    if (!bytes) return fail(nullptr, MIXRT_EINVAL, "bytes is NULL");
    *bytes = 0;
    mixrt::RotaryNormLaunch L{};
    if (int rc = check_normed(nullptr, rotary, 0.0f, heads, n, true, false, L)) return rc;
    *bytes = mixrt::rotary_norm_workspace(L);
    return MIXRT_OK;
}

int mixrt_rotary_norm_backward(mixrt_ctx *ctx, const mixrt_rotary *rotary, float eps,
                               const mixrt_normed_heads *heads, int32_t n, void *workspace,
                               size_t workspace_bytes)
{
    if (!ctx) return fail(nullptr, MIXRT_EINVAL, "ctx is NULL");
    clear_err(ctx);
    mixrt::RotaryNormLaunch L{};
    int rc;
    if ((rc = check_normed(ctx, rotary, eps, heads, n, true, true, L))) return rc;
    if ((rc = check_workspace(ctx, workspace, workspace_bytes, mixrt::rotary_norm_workspace(L))))
        return rc;
    if ((rc = bind_device(ctx))) return rc;
    L.ws = (float *)workspace;
    return finish_launch(ctx, mixrt::launch_rotary_norm_back(L, ctx->stream),
                         "rotary_norm_backward");
}

int mixrt_attention_workspace(const mixrt_attention *att, const mixrt_relative_bias *bias,
                              int32_t backward, size_t *bytes)
{
    clear_err(nullptr);
    if (!bytes) return fail(nullptr, MIXRT_EINVAL, "bytes is NULL");
    *bytes = 0;
    int rc;
    if ((rc = check_bias(nullptr, bias)) || (rc = check_attention(nullptr, att, bias)))
        return rc;
    *bytes = scratch_of(att, bias, backward != 0).total;
    return MIXRT_OK;
}

int mixrt_attention_forward(mixrt_ctx *ctx, const mixrt_attention *att,
                            const mixrt_relative_bias *bias, const mixrt_sequence *q,
                            const mixrt_sequence *k, const mixrt_sequence *v,
                            const mixrt_sequence *out, float *lse, void *rest, void *workspace,
                            size_t workspace_bytes)
{
    if (!ctx) return fail(nullptr, MIXRT_EINVAL, "ctx is NULL");
    clear_err(ctx);
    int rc;
    if ((rc = check_bias(ctx, bias)) || (rc = check_attention(ctx, att, bias)) ||
        (rc = check_bias_data(ctx, att, bias)) ||
        (rc = check_sequence(ctx, att, q, true, "q", false)) ||
        (rc = check_sequence(ctx, att, k, false, "k", false)) ||
        (rc = check_sequence(ctx, att, v, false, "v", false)) ||
        (rc = check_sequence(ctx, att, out, true, "out", true)))
        return rc;
    const int64_t rows = (int64_t)att->batch * att->heads * att->queries;
    Arrays m;
    add_common(m, att, bias, q, k, v);
    m.add(extent_of(att, out, true), "out", true);
    m.add(mixrt::flat_extent(lse, rows * 4), "lse", true);
    m.add(mixrt::flat_extent(lse ? att->lse_rest : nullptr, rows * 4), "lse_rest", true);
    m.add(mixrt::flat_extent(rest, rows * att->head_dim * 2), "rest", true);
    if ((rc = check_apart(ctx, m))) return rc;
    if (!aligned(lse, 4)) return fail(ctx, MIXRT_EINVAL, "lse not 4-byte aligned");
    if (rest && att->dtype == MIXRT_F32) return fail(ctx, MIXRT_EINVAL, "rest for F32");
    if (!aligned(rest, 2)) return fail(ctx, MIXRT_EINVAL, "rest not aligned to its element");
    const Scratch s = scratch_of(att, bias, false);
    if ((rc = check_workspace(ctx, workspace, workspace_bytes, s.total))) return rc;
    if ((rc = bind_device(ctx))) return rc;
    if (att->batch == 0 || att->queries == 0) return MIXRT_OK;
    mixrt::AttendK a = attend_k(att, bias);
    a.q = seq_k(q);
    a.k = seq_k(k);
    a.v = seq_k(v);
    a.o = seq_k(out);
    a.lse = lse;
    a.rest = rest;
    a.part = (float *)((char *)workspace + s.part);
    a.part_lse = (float2 *)((char *)workspace + s.part_lse);
    return finish_launch(ctx, launch_attend(a, mixrt::kAttendForward, ctx->stream),
                         "attention_forward");
}

int mixrt_attention_backward(mixrt_ctx *ctx, const mixrt_attention *att,
                             const mixrt_relative_bias *bias, const mixrt_sequence *dout,
                             const mixrt_sequence *q, const mixrt_sequence *k,
                             const mixrt_sequence *v, const mixrt_sequence *out,
                             const float *lse, const void *rest, const mixrt_sequence *dq,
                             const mixrt_sequence *dk, const mixrt_sequence *dv, float *dtable,
                             void *workspace, size_t workspace_bytes)
{
    if (!ctx) return fail(nullptr, MIXRT_EINVAL, "ctx is NULL");
    clear_err(ctx);
    int rc;
    if ((rc = check_bias(ctx, bias)) || (rc = check_attention(ctx, att, bias)) ||
        (rc = check_bias_data(ctx, att, bias)) ||
        (rc = check_sequence(ctx, att, dout, true, "dout", false)) ||
        (rc = check_sequence(ctx, att, q, true, "q", false)) ||
        (rc = check_sequence(ctx, att, k, false, "k", false)) ||
        (rc = check_sequence(ctx, att, v, false, "v", false)) ||
        (rc = check_sequence(ctx, att, out, true, "out", false)) ||
        (rc = check_sequence(ctx, att, dq, true, "dq", true)) ||
        (rc = check_sequence(ctx, att, dk, false, "dk", true)) ||
        (rc = check_sequence(ctx, att, dv, false, "dv", true)))
        return rc;
    const int64_t all = (int64_t)att->batch * att->heads * att->queries;
    Arrays m;
    add_common(m, att, bias, q, k, v);
    m.add(extent_of(att, dout, true), "dout");
    m.add(extent_of(att, out, true), "out");
    m.add(mixrt::flat_extent(lse, all * 4), "lse");
    m.add(mixrt::flat_extent(att->lse_rest, all * 4), "lse_rest");
    m.add(mixrt::flat_extent(rest, all * att->head_dim * 2), "rest");
    m.add(extent_of(att, dq, true), "dq", true);
    m.add(extent_of(att, dk, false), "dk", true);
    m.add(extent_of(att, dv, false), "dv", true);
    if (bias)
        m.add(mixrt::flat_extent(dtable, (int64_t)bias->axes * bias->count * att->heads * 4),
              "dtable", true);
    if ((rc = check_apart(ctx, m))) return rc;
    if (dtable && !bias) return fail(ctx, MIXRT_EINVAL, "dtable without a bias");
    if (!aligned(lse, 4) || !aligned(dtable, 4))
        return fail(ctx, MIXRT_EINVAL, "lse or dtable not 4-byte aligned");
    if (!aligned(rest, 2)) return fail(ctx, MIXRT_EINVAL, "rest not aligned to its element");
    if (rest && att->dtype == MIXRT_F32) return fail(ctx, MIXRT_EINVAL, "rest for F32");
    const bool rows = att->batch > 0 && att->queries > 0;
    if (rows && (!lse || (!rest && att->dtype != MIXRT_F32)))
        return fail(ctx, MIXRT_EINVAL, "lse or rest is NULL");
    const Scratch s = scratch_of(att, bias, true);
    if ((rc = check_workspace(ctx, workspace, workspace_bytes, s.total))) return rc;
    if ((rc = bind_device(ctx))) return rc;
    mixrt::AttendK a = attend_k(att, bias);
    a.dout = seq_k(dout);
    a.q = seq_k(q);
    a.k = seq_k(k);
    a.v = seq_k(v);
    a.o = seq_k(out);
    a.lse = (float *)lse;
    a.rest = (void *)rest;
    a.dq = seq_k(dq);
    a.dk = seq_k(dk);
    a.dv = seq_k(dv);
    a.dtable = dtable;
    a.part = (float *)((char *)workspace + s.part);
    a.delta = (float *)((char *)workspace + s.delta);
    a.part_table = (float *)((char *)workspace + s.table);
    a.table_sum = (double *)((char *)workspace + s.table_sum);
    hipError_t e = launch_attend(a, mixrt::kAttendBackQ, ctx->stream);
    if (e == hipSuccess) e = launch_attend(a, mixrt::kAttendBackKV, ctx->stream);
    return finish_launch(ctx, e, "attention_backward");
}

}  // extern "C"
