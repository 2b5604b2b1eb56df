// Attention, forward: one pass over the keys with the running maximum and sum.
#pragma once

#include "mixrt_attend_tile.hpp"

namespace mixrt {
namespace {

// Where a block's work lies: its columns' first head, batch entry, keys.
struct ForwardWork {
    int rb, split, h0, b, kvh, len, first, last;
    __device__ __forceinline__ explicit ForwardWork(const AttendK &k)
    {
        int id = near_block();
        rb = id % k.blocks;
        id /= k.blocks;
        split = id % k.splits;
        id /= k.splits;
        const int packs = k.H / k.pack;
        h0 = id % packs * k.pack;
        b = id / packs;
        kvh = h0 / (k.H / k.Hk);
        len = valid_keys(k.lens, b, k.Tk);
        first = k.from + split * k.per;
        last = min(len, first + k.per);
    }
};

// A lane's columns, a token and a head each.
template <int NC>
struct Columns {
    int t[NC], head[NC];
    bool there[NC];
    __device__ __forceinline__ Columns(const AttendK &k, const ForwardWork &w, int first, int lane)
    {
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            const int col = first + 32 * n + (lane & 31);
            t[n] = col / k.pack;
            head[n] = w.h0 + col % k.pack;
            there[n] = t[n] < k.Tq;
        }
    }
    template <typename T, int DP>
    __device__ __forceinline__ void load(const AttendK &k, int b, int half,
                                         typename Matrix<T>::frag (&q)[NC][(kPairs<T, DP>)]) const
    {
#pragma unroll
        for (int n = 0; n < NC; ++n)
            load_column<T, DP>(q[n], (const T *)k.q.data + b * k.q.batch +
                                         (int64_t)t[n] * k.q.token + head[n] * k.q.head,
                               there[n], half, k.D);
    }
    __device__ __forceinline__ void places(const AttendK &k, int b,
                                           int (&pos)[NC][kMaxBiasAxes]) const
    {
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
            for (int a = 0; a < kMaxBiasAxes; ++a)
                pos[n][a] = there[n] && a < k.bias.axes
                                ? k.bias.qpos[b * k.bias.qbatch + (int64_t)t[n] * k.bias.axes + a]
                                : 0;
    }
};

// log2 of a row's sum of weights: their base and the logarithm of their sum, as a 32-bit
// number and what its rounding left.
struct RowSum {
    float lse, rest;
    __device__ __forceinline__ RowSum(float top, float l, float none)
    {
        const float add = __builtin_amdgcn_logf(l);     // (log2)
        lse = top + add;
        const float got = lse - top;
        rest = (top - (lse - got)) + (add - got);
        if (l == 0.0f) lse = none;
        // (no rest of what is not a finite number)
        if (!(fabsf(lse) < INFINITY)) rest = 0.0f;
    }
};

// The columns' results: sums of weighted values, of weights (the lane's own rows), and
// the base of the weights, in units of log2.
template <typename T, int DP, int NC>
__device__ __forceinline__ void finish(const AttendK &k, const ForwardWork &w,
                                       const Columns<NC> &c, int half,
                                       const f32x16 (&acc)[NC][DP / 32], const float (&sum)[NC],
                                       const float (&top)[NC])
{
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        const float l = half_sum(sum[n]);
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        if (!c.there[n]) continue;
        const int64_t row = ((int64_t)w.b * k.H + c.head[n]) * k.Tq + c.t[n];
        const RowSum sums(top[n], l, k.splits > 1 ? -INFINITY : INFINITY);
        if (k.splits > 1) {
            const int64_t rows = (int64_t)k.B * k.H * k.Tq;
            if (half == 0) k.part_lse[w.split * rows + row] = make_float2(sums.lse, sums.rest);
            float *o = k.part + (w.split * rows + row) * k.D;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    store_quad<float>(o, 32 * d + 8 * e + 4 * half, k.D, acc[n][d][4 * e] * inv,
                                      acc[n][d][4 * e + 1] * inv, acc[n][d][4 * e + 2] * inv,
                                      acc[n][d][4 * e + 3] * inv);
            continue;
        }
        if (k.lse && half == 0) {
            k.lse[row] = sums.lse;
            if (k.lse_rest) k.lse_rest[row] = sums.rest;
        }
        T *o = (T *)k.o.data + w.b * k.o.batch + (int64_t)c.t[n] * k.o.token +
               c.head[n] * k.o.head;
        T *rest = k.rest ? (T *)k.rest + (((int64_t)w.b * k.Tq + c.t[n]) * k.H + c.head[n]) * k.D
                         : nullptr;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float f[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] = acc[n][d][4 * e + i] * inv;
                const int at = 32 * d + 8 * e + 4 * half;
                store_quad<T>(o, at, k.D, f[0], f[1], f[2], f[3]);
                if (rest) store_rest<T>(rest, at, k.D, f);
            }
    }
}

// Weights are 2^(score - base), scores in units of log2.  float16 holds few powers of
// two: there the base lies below the largest score when it is chosen, by 7, or by 11
// where the output is trained on (EXACT), so that a weight counts down to 2^-32 or 2^-36
// of the largest one's.  (Below half of float16's least, 2^-24, it is 0 in the product
// with the values, and not in the weights' sum: on a base at the largest score 32,768
// keys of 2^-26 beside one large key took 0.05% off the row.)  A walk adds at most
// 32,768 keys, so what is lost is at most 2^-17 or 2^-21 of a row.  3600 queries over
// 14,400 keys, 8 heads of 64: the same time with 7 as with 0, with 11 156 to 172 us, as
// bases move more often.
template <typename T, bool EXACT>
inline constexpr float kLow = !std::is_same_v<T, f16> ? 0.0f : EXACT ? 11.0f : 7.0f;
// A new maximum moves the base only where weights on the old one would pass 2^8 (in
// float16 2^15): then the sums so far are brought to it.  That is the first tile and
// few others.
template <typename T> inline constexpr float kMost = std::is_same_v<T, f16> ? 15.0f : 8.0f;
// (float16 has no room for what base + kMost may round up by, beside a large base; the
// difference does not.  Where both are -inf it is no number.)
template <typename T>
__device__ __forceinline__ bool past_base(float m, float top)
{
    return std::is_same_v<T, f16> ? m - top > kMost<T> : m > top + kMost<T>;
}
template <typename T, bool EXACT, int ND>
__device__ __forceinline__ void rebase(float m, float &top, float &sum, f32x16 (&acc)[ND])
{
    if (past_base<T>(m, top)) {
        float to = m - kLow<T, EXACT>;
        if (past_base<T>(m, to)) to = m;        // (as a large m's difference is rounded)
        const float less = __builtin_amdgcn_exp2f(top - to);
        sum *= less;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] *= less;
        top = to;
    }
}

// Whether a wave's bases are so large that the product with unit, which a weight's
// exponent does not round, has to be rounded as the maximum's is: else a weight could
// pass its type's largest number by the maximum's rounding alone, from scores of 2^23 on
// in float16, of 2^31 in 32 bits.  The scores are then rounded, and their unit is 1.
__device__ __forceinline__ bool far_base(float top)
{
    return __builtin_amdgcn_ballot_w64(fabsf(top) >= 0x1p22f) != 0;
}
__device__ __forceinline__ void round_scores(f32x16 &s, float unit)
{
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] *= unit;
}

// The weights of a block of 32 rows, in place of the scores: 2^(s unit - base).
__device__ __forceinline__ void weigh(f32x16 &s, float unit, float top, float &sum)
{
    // (a column whose scores are all -inf so far keeps weights 0)
    const float base = top == -INFINITY ? 0.0f : top;
    float add = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], unit, -base));
        add += s[i];
    }
    sum += add;
}

__device__ __forceinline__ float most_of(const f32x16 &s)
{
    float m = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
    return half_max(m);
}

// Rows behind the last one have no weight.
__device__ __forceinline__ void cut_rows(f32x16 &s, int row0, int half, int last)
{
    rare();
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (row0 + tile_row(i, half) >= last) s[i] = -INFINITY;
}

// The same where four waves share the columns: their sums are brought to one base and
// joined in room.
template <typename T, int DP>
__device__ __forceinline__ void finish_shared(const AttendK &k, const ForwardWork &w,
                                              const Columns<1> &c, const Team<true> &team,
                                              const f32x16 (&acc)[DP / 32], float sum, float top,
                                              float *room, float (&tops)[2][4][32])
{
    const int column = team.lane & 31, half = team.half;
    sum = half_sum(sum);
    if (half == 0) {
        tops[0][team.wave][column] = top;
        tops[1][team.wave][column] = sum;
    }
    __syncthreads();
    float all = -INFINITY, l = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) all = fmaxf(all, tops[0][i][column]);
    const float base = all == -INFINITY ? 0.0f : all;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        l += tops[1][i][column] * __builtin_amdgcn_exp2f(tops[0][i][column] - base);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    float f[DP / 8];
    join_waves<DP>(room, team.lane, team.wave, acc, __builtin_amdgcn_exp2f(top - base), f);
    if (!c.there[0]) return;
    const int d = (2 * team.wave + half) * (DP / 8);
    const int64_t row = ((int64_t)w.b * k.H + c.head[0]) * k.Tq + c.t[0];
    const RowSum sums(base, l, k.splits > 1 ? -INFINITY : INFINITY);
    const bool first = team.wave == 0 && half == 0;
    if (k.splits > 1) {
        const int64_t rows = (int64_t)k.B * k.H * k.Tq;
        if (first) k.part_lse[w.split * rows + row] = make_float2(sums.lse, sums.rest);
        store_run<float>(k.part + (w.split * rows + row) * k.D, d, k.D, f, inv);
        return;
    }
    if (k.lse && first) {
        k.lse[row] = sums.lse;
        if (k.lse_rest) k.lse_rest[row] = sums.rest;
    }
    store_run<T>((T *)k.o.data + w.b * k.o.batch + (int64_t)c.t[0] * k.o.token +
                     c.head[0] * k.o.head, d, k.D, f, inv);
    if (k.rest) {
        T *rest = (T *)k.rest + (((int64_t)w.b * k.Tq + c.t[0]) * k.H + c.head[0]) * k.D;
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) f[i] *= inv;
#pragma unroll
        for (int i = 0; i < DP / 8; i += 4) store_rest<T>(rest, d + i, k.D, f + i);
    }
}

// Terms of a weight in the 16-bit types' second product (EXACT: see attend_flow_kernel).
// A served weight is rounded to its type, as the result is: the result's relative error
// is then 2.2e-3 in bfloat16 (one token over 14,400 keys; with a bias 2.3e-3) and 2.9e-4
// in float16, where its own rounding alone makes 1.7e-3 and 2.1e-4.  A second term takes
// that away, and 20.2 us for 19.4 there, 817 for 732 with a bias (8160 tokens among
// themselves, 16 heads of 64), 224 for 163 of 3600 queries over 14,400 keys.
template <typename T, bool BIAS, bool EXACT>
inline constexpr int kTerms = !EXACT ? 1 : BIAS && std::is_same_v<T, bf16> ? 3 : 2;

// 32 columns a wave, or a block (SHARED): float32, and calls with few columns.
// EXACT: see attend_flow_kernel.
//
// SHARED is bound by latency: a wave's walk is a few tiles, each read from HBM, put into
// LDS, multiplied, rebased.  One token of 32 heads of 128 over 14,400 keys of 8 in bf16
// (59 MB, 10 us at a large copy's rate): 19.5 us a call, 15.4 and 4.7 of join in a trace,
// vector units busy 30% of the time.  7 crops of 253 tokens over up to 391 keys, 6 heads
// of 40, f32: 23 us, matrix units busy 22%.  Not SHARED, f32 is bound by the matrix instructions, of 64
// cycles for two of a head's elements.
// Waves a SIMD: one token of 32 heads of 128 takes 19.5 us with two and 25 with one, which
// a few registers too many leave.
template <typename T, bool SHARED, bool BIAS>
inline constexpr int kSimpleWaves = SHARED && sizeof(T) == 2 && !BIAS ? 2 : 1;
template <typename T, int DP, bool SHARED, bool BIAS, bool EXACT>
__global__ __launch_bounds__(256, (kSimpleWaves<T, SHARED, BIAS>)) void attend_kernel(AttendK k)
{
    typedef typename Matrix<T>::frag frag;
    constexpr int ROWS = 32, NC = 1, WAVES = SHARED ? 4 : 1, BUFS = SHARED ? 1 : 2;
    constexpr int PK = BIAS && SHARED ? 8 : 1;      // heads that share the columns
    constexpr int TILE = ROWS * kStride<T, DP>;
    // (two tiles of each wave are more than the 128 DP floats that joining them takes)
    __shared__ __attribute__((aligned(16))) T tiles[WAVES][BUFS][2][TILE];
    __shared__ float dense[BIAS ? PK * kMaxBiasAxes * kReachRow : 1];
    __shared__ TilePos<BIAS ? ROWS : 1> kpos[WAVES][BUFS];
    __shared__ float tops[2][4][32];

    const Team<SHARED> team;
    const int lane = team.lane, half = team.half, me = team.mine(), stager = team.stager();
    constexpr int STEP = Team<SHARED>::kStep * ROWS;
    const ForwardWork w(k);
    const T *kp = (const T *)k.k.data + w.b * k.k.batch + w.kvh * k.k.head;
    const T *vp = (const T *)k.v.data + w.b * k.v.batch + w.kvh * k.v.head;
    const int32_t *pp = BIAS ? k.bias.kpos + w.b * k.bias.kbatch : nullptr;
    Stage<T, DP, ROWS, Team<SHARED>::kStagers> sk, sv;
    StagePos<BIAS ? ROWS : 1> sp;
    // (all fetched and then put, or one array after the other)
    constexpr bool AHEAD = !SHARED || kFetchAhead<T, DP>;
    auto fetch = [&](int row) {
        sk.fetch(stager, kp, k.k.token, row, w.last, k.D);
        if (!AHEAD) sk.put(stager, tiles[me][0][0]);
        sv.fetch(stager, vp, k.v.token, row, w.last, k.D);
        if (!AHEAD) sv.put(stager, tiles[me][0][1]);
        if (BIAS) sp.fetch(stager, pp, k.bias.axes, row, w.last);
    };
    auto put = [&](int to) {
        if (AHEAD) {
            sk.put(stager, tiles[me][to][0]);
            sv.put(stager, tiles[me][to][1]);
        }
        if (BIAS) sp.put(stager, kpos[me][to], k.bias.axes);
    };
    const int row1 = w.first + me * ROWS;
    if (row1 < w.last) fetch(row1);
    const Columns<NC> c(k, w, (SHARED ? w.rb : w.rb * 4 + team.wave) * 32, lane);
    frag q[NC][kPairs<T, DP>];
    c.template load<T, DP>(k, w.b, half, q);
    int qpos[NC][kMaxBiasAxes], hbase[NC];
    if (BIAS) {
        for (int p = 0; p < k.pack; ++p)
            load_bias(dense + p * kMaxBiasAxes * kReachRow, k.bias, w.h0 + p, k.H, threadIdx.x,
                      256, false);
        hbase[0] = (c.head[0] - w.h0) * kMaxBiasAxes * kReachRow;
        c.places(k, w.b, qpos);
    }
    f32x16 acc[NC][DP / 32];
    float top[NC] = {-INFINITY}, sum[NC] = {0.0f};
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[0][d][i] = 0.0f;
    if (row1 < w.last) put(0);
    if (SHARED && BIAS) __syncthreads();    // (the bias is the block's)
    team.meet();
    int cur = 0;
    bool far = false;       // (of the whole wave)
    for (int row0 = row1; row0 < w.last; row0 += STEP, cur ^= BUFS - 1) {
        const bool more = row0 + STEP < w.last;
        if (more && AHEAD) fetch(row0 + STEP);
        const T *kt = tiles[me][cur][0], *vt = tiles[me][cur][1];
        f32x16 s[NC] = {row_mul<T, DP>(kt, lane, q[0], k.D)};
        if constexpr (BIAS)
            add_bias<ROWS>(s[0], k.scale, kpos[me][cur], 0, half, dense, hbase[0], qpos[0],
                           k.bias.axes, k.bias.reach);
        if (row0 + ROWS > w.last) cut_rows(s[0], row0, half, w.last);
        const float unit = BIAS ? 1.0f : k.scale, m = most_of(s[0]) * unit;
        if (far || __builtin_amdgcn_ballot_w64(past_base<T>(m, top[0])) != 0) {
            rebase<T, EXACT>(m, top[0], sum[0], acc[0]);
            far = !BIAS && far_base(top[0]);
        }
        if (far) round_scores(s[0], unit);
        weigh(s[0], far ? 1.0f : unit, top[0], sum[0]);
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) col_mul<DP>(vt, lane, d, s[0], acc[0][d]);
        } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                frag p[kTerms<T, BIAS, EXACT>];
                split_rows<T>(s[0], e, p);
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) {
                    const frag a = col_frag<T, DP>(vt, lane, d, e);
#pragma unroll
                    for (const frag &term : p) acc[0][d] = Matrix<T>::mul(a, term, acc[0][d]);
                }
            }
        }
        if (more) {
            if (SHARED) team.meet();
            if (!AHEAD) fetch(row0 + STEP);
            put(cur ^ (BUFS - 1));
        }
        team.meet();
    }
    if constexpr (SHARED)
        finish_shared<T, DP>(k, w, c, team, acc[0], sum[0], top[0], (float *)&tiles[0][0][0][0],
                             tops);
    else
        finish<T, DP, NC>(k, w, c, half, acc, sum, top);
}

// Four waves a block, NC blocks of 32 columns a wave, for the 16-bit types.  There an
// exponential costs as much of a SIMD's time as the products of a score with heads of
// 64, so neither may wait for the other: a step forms the weights of 32 rows while the
// matrix unit works on the scores of the next 32 and on the values of the last 32.
// Keys lie in LDS one tile ahead, values stay one tile longer (rings of three).
//
// 3600 queries over 14,400 keys, 8 heads of 64 in f16: 155 to 163 us with its join, 650 to
// 680 TFLOP/s; vector units busy 61% of the time, matrix units 35%.  An exponential takes 8 cycles a wave, so the
// weights of 32 x 32 scores take 128 of a SIMD's cycles beside 256 of products, and their
// scaling, maxima, sums and roundings more than that.  With the bias (8160 tokens among
// themselves, 16 heads, bf16, two axes): 728 us, 53% and 15%; the bias is read from LDS
// between a score and its weight, at addresses formed there, and two waves a SIMD do not
// hide that chain (42% of a wave's time).  A block's 256
// columns halve the reads of the tiles (without a bias, from 1024 columns on); with a
// bias or EXACT a wave has one block of columns, as two do not fit its registers.
//
// EXACT (for training): the weights go into the second product as two terms, their
// rounded values and what that left.  The backward pass takes delta = sum_j P_ij dP_ij
// from the output, and dS = P (dP - delta) cancels where a row looks at few keys: an
// output from rounded weights would leave there the rounding itself, not a small part
// of it.
// With a bias in bfloat16 a third term, of 8 bits like the others: the table's gradient
// is in 32 bits, and sums what would be left of many rows that cancel (3600 queries over
// 7200 keys, 8 heads, three axes: a relative error of 1.7e-6 with two terms, 6e-7 to
// 8e-7 with three, and the training step took 873 and 890 us).
template <int DP> inline constexpr int kFlowWaves = DP <= 64 ? 2 : 1;   // a SIMD
template <typename T, int DP, int NC, bool BIAS, bool EXACT>
__global__ __launch_bounds__(256, kFlowWaves<DP>) void attend_flow_kernel(AttendK k)
{
    typedef typename Matrix<T>::frag frag;
    constexpr int ROWS = DP <= 64 ? 64 : 32, SUBS = ROWS / 32, THREADS = 256;
    constexpr int TILE = ROWS * kStride<T, DP>;
    __shared__ __attribute__((aligned(16))) T ktiles[3][TILE];
    __shared__ __attribute__((aligned(16))) T vtiles[3][TILE];
    __shared__ __attribute__((aligned(16))) T nothing[32 * kStride<T, DP>];     // zeros
    __shared__ float dense[BIAS ? kMaxBiasAxes * kReachRow : 1];
    __shared__ TilePos<BIAS ? ROWS : 1> kpos[3];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const ForwardWork w(k);
    const T *kp = (const T *)k.k.data + w.b * k.k.batch + w.kvh * k.k.head;
    const T *vp = (const T *)k.v.data + w.b * k.v.batch + w.kvh * k.v.head;
    const int32_t *pp = BIAS ? k.bias.kpos + w.b * k.bias.kbatch : nullptr;
    Stage<T, DP, ROWS, THREADS> sk, sv;
    StagePos<BIAS ? ROWS : 1> sp;
    auto put_keys = [&](int row, int slot) {
        sk.fetch(threadIdx.x, kp, k.k.token, row, w.last, k.D);
        sk.put(threadIdx.x, ktiles[slot]);
        if (BIAS) {
            sp.fetch(threadIdx.x, pp, k.bias.axes, row, w.last);
            sp.put(threadIdx.x, kpos[slot], k.bias.axes);
        }
    };
    const Columns<NC> c(k, w, (w.rb * 4 + wave) * NC * 32, lane);
    frag q[NC][kPairs<T, DP>];
    int qpos[NC][kMaxBiasAxes], hbase[NC];
    if (w.first < w.last) {
        put_keys(w.first, 0);
        put_keys(w.first + ROWS, 1);
        sv.fetch(threadIdx.x, vp, k.v.token, w.first, w.last, k.D);
        sv.put(threadIdx.x, vtiles[0]);
    }
    c.template load<T, DP>(k, w.b, half, q);
    if (BIAS) {
        load_bias(dense, k.bias, w.h0, k.H, threadIdx.x, THREADS, false);
        c.places(k, w.b, qpos);
#pragma unroll
        for (int n = 0; n < NC; ++n) hbase[n] = 0;
    }
    // (the small terms of three have sums of their own: in one they would round the
    // large one's three times as often)
    constexpr int ND = DP / 32, LOW = kTerms<T, BIAS, EXACT> > 2 ? ND : 0;
    f32x16 acc[NC][ND + LOW], s[NC];
    float top[NC], sum[NC];
    frag p[NC][2][kTerms<T, BIAS, EXACT>];      // weights of the last 32 rows
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        top[n] = -INFINITY;
        sum[n] = 0.0f;
#pragma unroll
        for (int d = 0; d < ND + LOW; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][d][i] = 0.0f;
    }
    for (int i = threadIdx.x; i < 32 * kStride<T, DP>; i += THREADS) nothing[i] = (T)0.0f;
    __syncthreads();
    if (w.first < w.last)
#pragma unroll
        for (int n = 0; n < NC; ++n) s[n] = row_mul<T, DP>(ktiles[0], lane, q[n], k.D);

    // acc += values of 32 rows, at weights p
    auto add_values = [&](const T *v) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) {
                const frag a = col_frag<T, DP>(v, lane, d, e);
#pragma unroll
                for (int n = 0; n < NC; ++n)
#pragma unroll
                    for (int i = 0; i < kTerms<T, BIAS, EXACT>; ++i) {
                        const int at = i == 0 ? d : d + LOW;
                        acc[n][at] = Matrix<T>::mul(a, p[n][e][i], acc[n][at]);
                    }
            }
    };
    const float unit = BIAS ? 1.0f : k.scale;
    bool far = false;       // (of the whole wave)
    // the values that p waits for: none yet
    const T *held = nothing;
#pragma unroll
    for (int n = 0; n < NC; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (frag &term : p[n][e]) term = frag{};
    int k0 = 0, k1 = 1, k2 = 2, v0 = 0, v1 = 1, v2 = 2;     // slots of this tile, the next ..
    for (int row0 = w.first; row0 < w.last; row0 += ROWS) {
        sk.fetch(threadIdx.x, kp, k.k.token, row0 + 2 * ROWS, w.last, k.D);
        sv.fetch(threadIdx.x, vp, k.v.token, row0 + ROWS, w.last, k.D);
        if (BIAS) sp.fetch(threadIdx.x, pp, k.bias.axes, row0 + 2 * ROWS, w.last);
#pragma unroll
        for (int u = 0; u < SUBS; ++u) {
            if constexpr (BIAS)
                add_bias<ROWS>(s[0], k.scale, kpos[k0], u, half, dense, 0, qpos[0], k.bias.axes,
                               k.bias.reach);
            if (row0 + 32 * u + 32 > w.last)
#pragma unroll
                for (int n = 0; n < NC; ++n) cut_rows(s[n], row0 + 32 * u, half, w.last);
            float m[NC];
            bool out = false;
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                m[n] = most_of(s[n]) * unit;
                out = out || past_base<T>(m[n], top[n]);
            }
            if (far || __builtin_amdgcn_ballot_w64(out) != 0) {
                // the values that wait have weights on the old base
                add_values(held);
                held = nothing;
                far = false;
#pragma unroll
                for (int n = 0; n < NC; ++n) {
                    rebase<T, EXACT>(m[n], top[n], sum[n], acc[n]);
                    far = far || (!BIAS && far_base(top[n]));
                }
                if (far)
#pragma unroll
                    for (int n = 0; n < NC; ++n) round_scores(s[n], unit);
            }
            const float by = far ? 1.0f : unit;
            const T *next = u + 1 < SUBS ? ktiles[k0] + 32 * (u + 1) * kStride<T, DP> : ktiles[k1];
            f32x16 s2[NC];
#pragma unroll
            for (int n = 0; n < NC; ++n) s2[n] = row_mul<T, DP>(next, lane, q[n], k.D);
            add_values(held);
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                weigh(s[n], by, top[n], sum[n]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    split_rows<T>(s[n], e, p[n][e]);
                    // (formed here, not where they are used)
#pragma unroll
                    for (const frag &term : p[n][e]) asm volatile("" ::"v"(term));
                }
            }
#pragma unroll
            for (int n = 0; n < NC; ++n) s[n] = s2[n];
            held = vtiles[v0] + 32 * u * kStride<T, DP>;
        }
        sk.put(threadIdx.x, ktiles[k2]);
        sv.put(threadIdx.x, vtiles[v1]);
        if (BIAS) sp.put(threadIdx.x, kpos[k2], k.bias.axes);
        __syncthreads();
        int x = k0;
        k0 = k1;
        k1 = k2;
        k2 = x;
        x = v0;
        v0 = v1;
        v1 = v2;
        v2 = x;
    }
    add_values(held);
    f32x16 whole[NC][ND];
#pragma unroll
    for (int n = 0; n < NC; ++n)
#pragma unroll
        for (int d = 0; d < ND; ++d) whole[n][d] = LOW ? acc[n][d] + acc[n][d + LOW] : acc[n][d];
    finish<T, DP, NC>(k, w, c, half, whole, sum, top);
}

// Joins the splits of a row: o = sum_s 2^(lse_s - top) o_s / sum_s 2^(lse_s - top).
// A block takes 256 / (8 G) rows and 32 elements of their heads: 8 lanes hold a row's
// quads, G groups of them share its splits.  (With the splits of a row one after
// another, the 113 of one token's 32 heads took 29 us.)  What the passes before left is
// one part more, and of a pass that is not the last the result is the next one's.
constexpr int kFewParts = 4;
template <typename T, int G, bool PASSES>
__device__ __forceinline__ void join_row(const AttendK &k, int64_t row, float (&part)[5][256])
{
    const int64_t rows = (int64_t)k.B * k.H * k.Tq;
    const int lane = threadIdx.x & 7, g = threadIdx.x / 8 % G;
    const bool there = row < rows;
    const int d = 32 * blockIdx.y + 4 * lane;
    // (blocks that share a row read what one of them writes for the next pass, so there
    // are two places for it)
    const auto lse_of = [&](int s) {
        return k.part_lse[(PASSES && s == k.splits ? s + ((k.pass + 1) & 1) : s) * rows + row];
    };
    const int parts = PASSES ? k.parts : k.splits;
    const auto value_of = [&](int s, float (&f)[4]) {
        const float *o = k.part + (s * rows + row) * k.D + d;
        if (d + 4 <= k.D) {
            load_vec<float, 4>(o, f);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = d + i < k.D ? o[i] : 0.0f;
        }
    };
    // the group's own maximum first: NaN stays
    float top = -INFINITY, base, a[4] = {0, 0, 0, 0}, w = 0.0f;
    const auto raise = [&](float x) { top = x > top || x != x ? x : top; };
    const auto add = [&](const float2 &lse, const float (&f)[4]) {
        const float e = __builtin_amdgcn_exp2f((lse.x - base) + lse.y);
        w += e;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = fmaf(f[i], e, a[i]);
    };
    if (G == 1) {
        // (few parts: all are on their way before the first is used)
        constexpr int MOST = kFewParts + PASSES;
        float2 lse[MOST];
        float f[MOST][4];
#pragma unroll
        for (int s = 0; s < MOST; ++s) {
            if (!there || s >= parts) continue;
            lse[s] = lse_of(s);
            value_of(s, f[s]);
        }
#pragma unroll
        for (int s = 0; s < MOST; ++s)
            if (there && s < parts) raise(lse[s].x);
        base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int s = 0; s < MOST; ++s)
            if (there && s < parts) add(lse[s], f[s]);
    } else {
        if (there)
#pragma unroll 4
            for (int s = g; s < parts; s += G) raise(lse_of(s).x);
        base = top == -INFINITY ? 0.0f : top;
        if (there)
#pragma unroll 4
            for (int s = g; s < parts; s += G) {
                float f[4];
                value_of(s, f);
                add(lse_of(s), f);
            }
    }
    if (G > 1) {
        // then the groups', in order, at their common maximum
        const bool none = top == -INFINITY;
        part[0][threadIdx.x] = top;
        __syncthreads();
        const int first = threadIdx.x - 8 * g;
        for (int j = 0; j < G; ++j) raise(part[0][first + 8 * j]);
        const float less = none ? 0.0f : __builtin_amdgcn_exp2f(base - top);
        base = top == -INFINITY ? 0.0f : top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) part[i][threadIdx.x] = a[i] * less;
        part[4][threadIdx.x] = w * less;
        __syncthreads();
        if (g == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = 0.0f;
            w = 0.0f;
#pragma unroll 8
            for (int j = 0; j < G; ++j) {
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] += part[i][first + 8 * j];
                w += part[4][first + 8 * j];
            }
        }
    }
    if (!there || g != 0) return;
    const float inv = w == 0.0f ? 0.0f : 1.0f / w;
    const int64_t bh = row / k.Tq;
    const int t = (int)(row - bh * k.Tq), b = (int)(bh / k.H), h = (int)(bh - (int64_t)b * k.H);
    const bool last = !PASSES || k.last;
    const RowSum sums(base, w, last ? INFINITY : -INFINITY);
    const bool first = lane == 0 && blockIdx.y == 0;
    if (!last) {
        if (first)
            k.part_lse[(k.splits + (k.pass & 1)) * rows + row] = make_float2(sums.lse, sums.rest);
        if (d < k.D)
            store_quad<float>(k.part + (k.splits * rows + row) * k.D, d, k.D, a[0] * inv,
                              a[1] * inv, a[2] * inv, a[3] * inv);
        return;
    }
    if (k.lse && first) {
        k.lse[row] = sums.lse;
        if (k.lse_rest) k.lse_rest[row] = sums.rest;
    }
    if (d >= k.D) return;
    T *o = (T *)k.o.data + b * k.o.batch + (int64_t)t * k.o.token + h * k.o.head;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] *= inv;
    store_quad<T>(o, d, k.D, a[0], a[1], a[2], a[3]);
    if (k.rest) {
        T *rest = (T *)k.rest + (((int64_t)b * k.Tq + t) * k.H + h) * k.D;
        store_rest<T>(rest, d, k.D, a);
    }
}

template <typename T, int G, bool PASSES>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendK k)
{
    constexpr int EACH = 32 / G;
    __shared__ float part[5][256];
    const int64_t rows = (int64_t)k.B * k.H * k.Tq;
    for (int64_t r0 = (int64_t)blockIdx.x * EACH; r0 < rows; r0 += (int64_t)gridDim.x * EACH) {
        join_row<T, G, PASSES>(k, r0 + threadIdx.x / (8 * G), part);
        if (G > 1) __syncthreads();     // (part is read to the end)
    }
}

template <typename T>
hipError_t launch_join(const AttendK &k, hipStream_t stream)
{
    const int64_t rows = (int64_t)k.B * k.H * k.Tq;
    auto go = [&](auto g, auto passes) {
        constexpr int G = decltype(g)::value, EACH = 32 / G;
        const dim3 grid((unsigned)join_blocks((rows + EACH - 1) / EACH), (unsigned)(k.D + 31) / 32);
        attend_join_kernel<T, G, decltype(passes)::value><<<grid, 256, 0, stream>>>(k);
    };
    auto groups = [&](auto passes) {
        if (k.splits > kFewParts)
            go(std::integral_constant<int, 32>(), passes);
        else
            go(std::integral_constant<int, 1>(), passes);
    };
    if (k.slots > k.splits)
        groups(std::true_type());
    else
        groups(std::false_type());
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch_forward(AttendK k, const AttendPlan &p, hipStream_t stream)
{
    const bool exact = sizeof(T) == 2 && k.rest;
    // (64 columns a wave leave no registers for more than the plain products)
    const bool twice = p.cols == 256 && !exact;
    if (p.cols == 256 && !twice) k.blocks = (k.Tq + 127) / 128;
    const unsigned grid = (unsigned)((int64_t)k.B * (k.H / k.pack) * k.splits * k.blocks);
    typedef std::true_type yes;
    typedef std::false_type no;
    auto variant = [&](auto go) {
        if constexpr (sizeof(T) == 2)
            if (exact) return k.bias.axes ? go(yes(), yes()) : go(no(), yes());
        return k.bias.axes ? go(yes(), no()) : go(no(), no());
    };
    auto simple = [&](auto shared) {
        variant([&](auto bias, auto ex) {
            attend_kernel<T, DP, decltype(shared)::value, decltype(bias)::value,
                          decltype(ex)::value><<<grid, 256, 0, stream>>>(k);
        });
    };
    if (p.shared) {
        simple(yes());
    } else if constexpr (sizeof(T) == 4) {
        simple(no());
    } else if (twice) {
        if constexpr (DP <= 64)
            attend_flow_kernel<T, DP, 2, false, false><<<grid, 256, 0, stream>>>(k);
    } else {
        variant([&](auto bias, auto ex) {
            attend_flow_kernel<T, DP, 1, decltype(bias)::value, decltype(ex)::value>
                <<<grid, 256, 0, stream>>>(k);
        });
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || k.splits == 1) return e;
    return launch_join<T>(k, stream);
}

}  // namespace
}  // namespace mixrt
