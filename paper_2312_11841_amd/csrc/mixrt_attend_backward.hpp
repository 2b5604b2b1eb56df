// Attention, backward: two walks that each form the weights and their gradients
// again, one with the queries in the lanes (their gradient, and the bias table's),
// one with the keys (the gradients of keys and values).  Nothing is added by
// several blocks to one place, so the sums' order is fixed.
#pragma once

#include "mixrt_attend_tile.hpp"

namespace mixrt {
namespace {

// float16 alone needs its dS and weights lifted; weights, at most 1, by 2^15.
template <typename T> inline constexpr bool kLifted = false;
template <> inline constexpr bool kLifted<f16> = true;
template <typename T> inline constexpr float kWeightLift = kLifted<T> ? 15.0f : 0.0f;

// Rows of a bias table's gradient that a walk over the keys sums in 32 bits before
// they move on to 64.
constexpr int kHistRows = 1024;

// acc[d][column] += sum over the tile's rows of tile[row][d] p[row][column].  The 16-bit
// types round dS, and the weights of dv, once: gradients have a relative error of 2.4e-3
// in bfloat16, where their own rounding alone makes 1.7e-3.  With a second term they have
// 1.7e-3, and two 720p views' training step takes 1229 us for 1024, one with a bias 966
// for 909.
template <typename T, int DP>
__device__ __forceinline__ void add_cols(const T *tile, int lane, const f32x16 &p,
                                         f32x16 (&acc)[DP / 32])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
            col_mul<DP>(tile, lane, d, p, acc[d]);
    } else {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const typename Matrix<T>::frag f = round_rows<T>(p, e);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) {
                const auto a = col_frag<T, DP>(tile, lane, d, e);
                acc[d] = Matrix<T>::mul(a, f, acc[d]);
            }
        }
    }
}

// s += a-tile's rows times b, g += e-tile's rows times f.  The operands of 16-bit heads
// of up to 64 elements are all read first: a wave is often alone on its SIMD, and would
// wait for LDS before each product.
template <typename T, int DP>
__device__ __forceinline__ void pair_mul(const T *a, const T *e, int lane,
                                         const typename Matrix<T>::frag (&b)[(kPairs<T, DP>)],
                                         const typename Matrix<T>::frag (&f)[(kPairs<T, DP>)],
                                         f32x16 &s, f32x16 &g, int D)
{
    constexpr bool FIRST = sizeof(T) == 2 && DP <= 64;
    typename Matrix<T>::frag x[kPairs<T, DP>], y[kPairs<T, DP>];
    if (FIRST) {
#pragma unroll
        for (int c = 0; c < kPairs<T, DP>; ++c) {
            x[c] = row_frag<T, DP>(a, lane, c);
            y[c] = row_frag<T, DP>(e, lane, c);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int c = 0; c < kPairs<T, DP>; ++c) {
        if (DP < 128 && past<T>(c, D)) continue;    // at 128 its branches cost registers
        if (!FIRST) {
            x[c] = row_frag<T, DP>(a, lane, c);
            y[c] = row_frag<T, DP>(e, lane, c);
        }
        s = Matrix<T>::mul(x[c], b[c], s);
        g = Matrix<T>::mul(y[c], f[c], g);
    }
}

template <int ND>
__device__ __forceinline__ void clear(f32x16 (&a)[ND])
{
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) a[d][i] = 0.0f;
}

// The exponent of a pair's weight, s unit - lse - rest, where lse is so large that its
// rounding counts (2^8 and more: 2^-16 of a weight): by three roundings, and from 2^22
// on of the score first, as the forward pass has it.  A weight is at most 2^lifted,
// whatever the roundings.  (In float32 what rounding took from lse counts always: it is
// most of a small step's error, and the matrix unit leaves the time.)
__device__ __forceinline__ bool large_sum(float lse)
{
    return fabsf(lse) >= 256.0f && fabsf(lse) < INFINITY;
}
// Whether it is so in any thread of the block; a barrier.
__device__ __forceinline__ bool block_any(bool x)
{
    return __builtin_amdgcn_readfirstlane(__syncthreads_or(x)) != 0;
}
__device__ __forceinline__ float exponent(float s, float unit, float lse, float rest, float lifted)
{
    const float whole = s * unit;
    const float near = fmaf(s, unit, -lse), far = whole - lse;
    const float x = (fabsf(lse) < 0x1p22f ? near : far) - rest;
    return x > lifted ? lifted : x;
}

// A walk whose lse are all small, whose lse count as large, or that asks for each tile:
// a block that meets a large one takes the walk written for it, without loads ahead, so
// that the other has no branch and no more registers (2048 queries over 2000 keys, 32
// heads of 128 on 8, bf16: the keys' gradient 265 us, with a branch a tile 300).  float32
// has one walk with a branch, which its products hide.
enum { kNoLarge, kAllLarge, kSomeLarge };
template <typename T> inline constexpr bool kTwoWalks = sizeof(T) == 2;

// float16 holds dS only inside a range: its gradients are small where a row looks at
// many keys, and large where a loss is scaled.  So each column's dS is multiplied by a
// power of two that brings the largest seen so far to 2^8..2^9 when it is chosen, and
// its sums with it; it is chosen anew where that one leaves 1..2^15.  (The first tile
// sets it, later ones seldom.)  The power is at most 2^100, and follows from the
// largest dS itself and not from a product with the last power, which may not be
// finite: a key may get weights of 2^-125 from the first queries and 1/2 from the next.
template <typename T, int ND>
struct Lift {
    float by, most;     // the power; the largest |dS| so far
    __device__ __forceinline__ void start()
    {
        by = 1.0f;
        most = 0.0f;
    }
    __device__ __forceinline__ void scale(f32x16 &g, f32x16 (&acc)[ND])
    {
        if (sizeof(T) != 2 || !kLifted<T>) return;
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(g[i]));
        m = fmaxf(most, half_max(m));
        most = m;
        // (a product that is not finite is out of range too; an m that is not has no
        // power)
        const float lifted = m * by;
        const bool out = (lifted > 0x1p15f || (lifted < 1.0f && m > 0.0f)) && m < INFINITY;
        if (__builtin_amdgcn_ballot_w64(out) != 0 && out) {
            const int now = (int)(__float_as_uint(by) >> 23);
            const int to = min(max(127 + 127 + 8 - (int)(__float_as_uint(m) >> 23), 27), 227);
            const float f = __uint_as_float((uint32_t)(127 + (to - now) / 2) << 23);
            const float e = __uint_as_float((uint32_t)(127 + (to - now) - (to - now) / 2) << 23);
            by = __uint_as_float((uint32_t)to << 23);
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] = acc[d][i] * f * e;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) g[i] *= by;
    }
    // the factor that takes a column's sums back
    __device__ __forceinline__ float back() const
    {
        return kLifted<T> ? 1.0f / by : 1.0f;
    }
};

// mine[e[i]] += v[i], for four places some of which may be the same: the sums of equal
// places go to the first (and the others to the spare place), so that the four reads and
// writes need not wait for each other.  (LDS has atomic adds in 32 bits, but they take 4
// cycles a lane: with them the gradient of 3600 queries over 7200 keys, 8 heads of 64 in
// bf16 and three axes, took 4.6 ms where it takes 0.45.)
__device__ __forceinline__ void join_places(int (&e)[4], float (&v)[4], int spare)
{
    const bool b0 = e[1] == e[0];
    const bool c0 = e[2] == e[0], c1 = !c0 && e[2] == e[1];
    const bool d0 = e[3] == e[0], d1 = !d0 && e[3] == e[1];
    const bool d2 = !d0 && !d1 && e[3] == e[2];
    v[0] += b0 ? v[1] : 0.0f;
    v[0] += c0 ? v[2] : 0.0f;
    v[0] += d0 ? v[3] : 0.0f;
    v[1] += c1 ? v[2] : 0.0f;
    v[1] += d1 ? v[3] : 0.0f;
    v[2] += d2 ? v[3] : 0.0f;
    e[1] = b0 ? spare : e[1];
    e[2] = c0 || c1 ? spare : e[2];
    e[3] = d0 || d1 || d2 ? spare : e[3];
}

__device__ __forceinline__ void put_places(float *mine, const int (&e)[4], const float (&v)[4])
{
    float a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = mine[e[i]];
#pragma unroll
    for (int i = 0; i < 4; ++i) mine[e[i]] = a[i] + v[i];
}

__device__ __forceinline__ void add_places(float *mine, int (&e)[4], float (&v)[4], int spare)
{
    join_places(e, v, spare);
    put_places(mine, e, v);
}

// Orders the LDS accesses of a wave's halves: those before come before those after, in
// every lane.  (A wave's accesses run in its order; this keeps the compiler's so.)
__device__ __forceinline__ void halves_meet()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Adds a column's dS to its places of the bias table's gradient.  The halves of a wave
// share the places; from one tile to the next its caller's Team::meet() orders them.
template <int ROWS>
__device__ __forceinline__ void add_table(const f32x16 &g, const TilePos<ROWS> &tile, int u,
                                          int half,
                                          const uint16_t *place,
                                          const int (&column)[kMaxBiasAxes], int axes, int reach,
                                          float *mine, int spare)
{
    float quad[4];      // of the octet's rows, those of the other half too
    int kind[kMaxBiasAxes], at[kMaxBiasAxes];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        quad[j] = half_sum((g[4 * j] + g[4 * j + 1]) + (g[4 * j + 2] + g[4 * j + 3]));
    // The two halves of a wave share a column's places: sums over both are added by one,
    // single rows by one half after the other.
    // the axes on which all rows have one place, together: their places lie apart (the
    // other axes, and the other half, add to the spare one)
#pragma unroll
    for (int a = 0; a < kMaxBiasAxes; ++a) {
        kind[a] = tile.kind_of(a, u);
        at[a] = place[a * kReachRow + bias_at(tile.at[a][32 * u], column[a], reach)];
    }
    float old[kMaxBiasAxes];
#pragma unroll
    for (int a = 0; a < kMaxBiasAxes; ++a) {
        at[a] = a < axes && kind[a] == kLevel && half == 0 ? at[a] : spare;
        old[a] = mine[at[a]];
    }
#pragma unroll
    for (int a = 0; a < kMaxBiasAxes; ++a)
        mine[at[a]] = old[a] + ((quad[0] + quad[1]) + (quad[2] + quad[3]));
#pragma unroll
    for (int a = 0; a < kMaxBiasAxes; ++a) {
        if (a >= axes) break;
        if (kind[a] == kLevel) continue;
        const uint16_t *row = place + a * kReachRow;
        const int32_t *p = &tile.at[a][32 * u + 4 * half];
        if (kind[a] == kLevel8) {
            int e[4];
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                e[j] = row[bias_at(p[8 * j], column[a], reach)];
                v[j] = quad[j];
            }
            if (half == 0) add_places(mine, e, v, spare);
            continue;
        }
        int e[4][4];
        if (kind[a] == kSteps) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint16_t *q = row + bias_at(p[8 * j], column[a], reach, kPad);
#pragma unroll
                for (int i = 0; i < 4; ++i) e[j][i] = q[i];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) e[j][i] = row[bias_at(p[8 * j + i], column[a], reach)];
        }
        // (all 16 places are read before the first is added to)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            asm volatile("" : "+v"(e[j][0]), "+v"(e[j][1]), "+v"(e[j][2]), "+v"(e[j][3]));
        float v[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[j][i] = g[4 * j + i];
            join_places(e[j], v[j], spare);
        }
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            if (half == h)
#pragma unroll
                for (int j = 0; j < 4; ++j) put_places(mine, e[j], v[j]);
            // (what one half has written is there for the other to read: else the two
            // turns are one to a compiler that looks at a single lane)
            halves_meet();
        }
    }
}

// A column's sums, times a factor, to its row of an output.
template <typename T, int DP>
__device__ __forceinline__ void store_column(T *row, int half, int D, const f32x16 (&a)[DP / 32],
                                             float by)
{
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            store_quad<T>(row, 32 * d + 8 * e + 4 * half, D, a[d][4 * e] * by, a[d][4 * e + 1] * by,
                          a[d][4 * e + 2] * by, a[d][4 * e + 3] * by);
}

// --- the queries' gradient -----------------------------------------------------------
//
// A column is a query: S = K q and dP = V dout tile by tile, P = 2^(S - lse), dS = P (dP -
// delta), dq += K^T dS; delta = dout (o + rest) is worked out first and kept for the
// keys' kernel.  The backward pass' five products run as seven in this kernel and the
// next, since both form S and dP: one kernel would add either gradient by several
// blocks to one place, in no fixed order.  Tiles of 32 rows leave three blocks a CU; of
// 64 rows two, and slower.
//
// Two entries of 3600 queries over 7200 keys, 12 heads of 64 on 3, bf16: 290 us, 820
// TFLOP/s.  While a CU is busy its matrix units work 46% of the time, its vector units
// 52%, its LDS 38%.  With a bias (one entry, 8 heads, three axes): 447 us, 8%, 41% and
// 31%: each pair of an axis that counts up is read from a place in LDS, added to and
// written back, by one half of the wave after the other, and the next pairs' reads wait
// for it (44% of a wave's time); the table's sums take LDS, so two blocks run on a CU.

template <typename T, int DP, bool BIAS, bool SHARED>
__global__ __launch_bounds__(256) void attend_dq_kernel(AttendK k)
{
    typedef typename Matrix<T>::frag frag;
    constexpr int ROWS = 32, THREADS = 256, WAVES = SHARED ? 4 : 1;
    constexpr int TILE = ROWS * kStride<T, DP>;
    // (two of the widest tiles and the table's sums are more than a CU's 160 KB)
    constexpr int BUFS = SHARED || (BIAS && sizeof(T) == 4 && DP == 128) ? 1 : 2;
    __shared__ __attribute__((aligned(16))) T tiles[WAVES][BUFS][2][TILE];
    __shared__ float dense[BIAS ? kMaxBiasAxes * kReachRow : 1];
    __shared__ uint16_t place[BIAS ? kMaxBiasAxes * kReachRow : 1];   // 32 entry
    __shared__ TilePos<BIAS ? ROWS : 1> kpos[WAVES][BUFS];
    extern __shared__ float hist[];     // [wave][entry, and a spare one][column]

    const Team<SHARED> team;
    const int lane = team.lane, wave = team.wave, half = team.half;
    const int me = team.mine(), stager = team.stager();
    constexpr int STEP = Team<SHARED>::kStep * ROWS;
    const int block = near_block();
    int id = block;
    const int rb = id % k.blocks;
    id /= k.blocks;
    const int split = id % k.splits;
    id /= k.splits;
    const int h = id % k.H, b = id / k.H;
    const int kvh = h / (k.H / k.Hk);
    const int len = valid_keys(k.lens, b, k.Tk);
    const int first = k.from + split * k.per, last = min(len, first + k.per);
    const int entries = BIAS ? k.bias.axes * k.bias.buckets : 0;

    const int t = (SHARED ? rb : rb * 4 + wave) * 32 + (lane & 31);
    const bool there = t < k.Tq;
    const int64_t tt = t;
    frag q[kPairs<T, DP>], dout[kPairs<T, DP>];
    load_column<T, DP>(q, (const T *)k.q.data + b * k.q.batch + tt * k.q.token + h * k.q.head,
                       there, half, k.D);
    load_column<T, DP>(dout, (const T *)k.dout.data + b * k.dout.batch + tt * k.dout.token +
                                 h * k.dout.head, there, half, k.D);
    // delta = sum_d dout o, with what rounding took from o
    float sum = 0.0f;
    {
        frag o[kPairs<T, DP>], rest[kPairs<T, DP>];
        load_column<T, DP>(o, (const T *)k.o.data + b * k.o.batch + tt * k.o.token + h * k.o.head,
                           there, half, k.D);
        if (sizeof(T) == 2)
            load_column<T, DP>(rest, (const T *)k.rest + ((b * (int64_t)k.Tq + tt) * k.H + h) * k.D,
                               there, half, k.D);
#pragma unroll
        for (int c = 0; c < kPairs<T, DP>; ++c)
#pragma unroll
            for (int i = 0; i < kChunk<T>; ++i) {
                float x = (float)o[c][i];
                if (sizeof(T) == 2) x = whole_of<T>(o[c][i], rest[c][i]);
                sum = fmaf((float)dout[c][i], x, sum);
            }
    }
    const float delta = half_sum(sum);
    const int64_t row = ((int64_t)b * k.H + h) * k.Tq + tt;
    const float lse = there ? k.lse[row] : INFINITY;
    const float lse_rest = there && k.lse_rest ? k.lse_rest[row] : 0.0f;
    int qpos[kMaxBiasAxes];
    if (there && half == 0 && split == 0 && me == 0) k.delta[row] = delta;
#pragma unroll
    for (int a = 0; a < kMaxBiasAxes; ++a)
        qpos[a] = BIAS && there && a < k.bias.axes
                      ? k.bias.qpos[b * k.bias.qbatch + tt * k.bias.axes + a]
                      : 0;
    const int held = entries + 1;
    if (BIAS) {
        load_bias(dense, k.bias, h, k.H, threadIdx.x, THREADS, false);
        const int n = 2 * k.bias.reach + 1 + 2 * kPad;
        for (int i = threadIdx.x; i < k.bias.axes * n; i += THREADS) {
            const int a = i / n, e = i - a * n;
            place[a * kReachRow + e] =
                (uint16_t)(32 * (a * k.bias.buckets + bucket_of(k.bias, a, e, false)));
        }
        for (int i = threadIdx.x; i < 4 * 32 * held; i += THREADS) hist[i] = 0.0f;
    }
    float *mine = hist + wave * 32 * held + (lane & 31);
    double table = 0.0;         // thread e: entry e's sum of the block

    f32x16 acc[DP / 32];
    clear(acc);
    Lift<T, DP / 32> lift;
    lift.start();
    const T *kp = (const T *)k.k.data + b * k.k.batch + kvh * k.k.head;
    const T *vp = (const T *)k.v.data + b * k.v.batch + kvh * k.v.head;
    const int32_t *pp = BIAS ? k.bias.kpos + b * k.bias.kbatch : nullptr;
    Stage<T, DP, ROWS, Team<SHARED>::kStagers> sk, sv;
    StagePos<BIAS ? ROWS : 1> sp;
    // (all fetched and then put, or one array after the other)
    constexpr bool AHEAD = !SHARED || kFetchAhead<T, DP>;
    auto fetch = [&](int row) __attribute__((always_inline)) {
        sk.fetch(stager, kp, k.k.token, row, last, k.D);
        if (!AHEAD) sk.put(stager, tiles[me][0][0]);
        sv.fetch(stager, vp, k.v.token, row, last, k.D);
        if (!AHEAD) sv.put(stager, tiles[me][0][1]);
        if (BIAS) sp.fetch(stager, pp, k.bias.axes, row, last);
    };
    auto put = [&](int to) __attribute__((always_inline)) {
        if (AHEAD) {
            sk.put(stager, tiles[me][to][0]);
            sv.put(stager, tiles[me][to][1]);
        }
        if (BIAS) sp.put(stager, kpos[me][to], k.bias.axes);
    };
    const int row1 = first + me * ROWS;
    if (row1 < last) {
        fetch(row1);
        put(0);
    }
    // (the bias and hist are the block's too)
    const bool large = block_any(large_sum(lse));
    // each entry's places of all columns; threads start at different columns, as the
    // same column of all entries lies in one bank
    auto collect = [&]() {
        if ((int)threadIdx.x >= entries) return;
        float sum = 0.0f;
#pragma unroll 1
        for (int w = 0; w < 4; ++w) {
            float *at = hist + (w * held + threadIdx.x) * 32;
#pragma unroll 4
            for (int i = 0; i < 32; ++i) {
                const int l = (i + threadIdx.x) & 31;
                sum += at[l];
                at[l] = 0.0f;
            }
        }
        table += sum;
    };
    auto walk = [&](auto kind) __attribute__((always_inline)) {
        constexpr int SUMS = decltype(kind)::value;
        constexpr bool EARLY = AHEAD && SUMS != kAllLarge;
        int cur = 0, counted = 0;
        for (int row0 = row1; row0 < last; row0 += STEP, cur ^= BUFS - 1) {
            const bool more = row0 + STEP < last;
            if (more && EARLY) fetch(row0 + STEP);
            const T *kt = tiles[me][cur][0], *vt = tiles[me][cur][1];
            f32x16 s, g;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = g[i] = 0.0f;
            pair_mul<T, DP>(kt, vt, lane, q, dout, s, g, k.D);
            if constexpr (BIAS) {
                add_bias<ROWS>(s, k.scale, kpos[me][cur], 0, half, dense, 0, qpos, k.bias.axes,
                                   k.bias.reach);
            }
            const float unit = BIAS ? 1.0f : k.scale;
            const bool one = SUMS == kAllLarge || (SUMS == kSomeLarge && large);
            if (one) {
                rare();
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = exponent(s[i], unit, lse, lse_rest, 0.0f);
            }
            const float by = one ? 1.0f : unit, less = one ? 0.0f : lse;
            const float left = one ? 0.0f : lse_rest;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float x = SUMS == kAllLarge ? s[i] : fmaf(s[i], by, -less);
                if (sizeof(T) == 4 && SUMS != kAllLarge) x -= left;
                g[i] = __builtin_amdgcn_exp2f(x) * (g[i] - delta);
            }
            if (row0 + ROWS > last) {
                rare();
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (row0 + tile_row(i, half) >= last)
                        g[i] = 0.0f;
            }
            if constexpr (BIAS) {
                add_table<ROWS>(g, kpos[me][cur], 0, half, place, qpos, k.bias.axes, k.bias.reach,
                                mine, 32 * entries);
            }
            lift.scale(g, acc);
            add_cols<T, DP>(kt, lane, g, acc);
            counted += ROWS;
            if (BUFS == 1) team.meet();
            if (more) {
                if (!EARLY) fetch(row0 + STEP);
                put(cur ^ (BUFS - 1));
            }
            team.meet();
            if (BIAS && !SHARED && counted == kHistRows) {
                collect();
                counted = 0;
                __syncthreads();
            }
        }
    };
    if constexpr (!kTwoWalks<T>)
        walk(std::integral_constant<int, kSomeLarge>());
    else if (large)
        walk(std::integral_constant<int, kAllLarge>());
    else
        walk(std::integral_constant<int, kNoLarge>());
    // the one key of a row has weight 1 whatever its score: no gradient
    const float some = len == 1 ? 0.0f : 1.0f;
    if (BIAS) {
        __syncthreads();
        collect();
        if ((int)threadIdx.x < entries)
            k.part_table[(int64_t)block * entries + threadIdx.x] = some * (float)table;
    }
    const int64_t rows = (int64_t)k.B * k.H * k.Tq;
    if constexpr (SHARED) {
        float f[DP / 8];
        join_waves<DP>((float *)&tiles[0][0][0][0], lane, wave, acc, lift.back(), f);
        if (!there) return;
        const int d = (2 * wave + half) * (DP / 8);
        if (k.splits > 1)
            store_run<float>(k.part + (split * rows + row) * k.D, d, k.D, f, some * k.plain_scale);
        else
            store_run<T>((T *)k.dq.data + b * k.dq.batch + tt * k.dq.token +
                             h * k.dq.head, d, k.D, f, some * k.plain_scale);
        return;
    }
    if (!there) return;
    const float by = some * lift.back() * k.plain_scale;
    if (k.splits > 1) {
        store_column<float, DP>(k.part + (split * rows + row) * k.D, half, k.D, acc, by);
    } else {
        store_column<T, DP>((T *)k.dq.data + b * k.dq.batch + tt * k.dq.token +
                                h * k.dq.head, half, k.D, acc, by);
    }
}

// --- the gradients of keys and values ---------------------------------------------------
//
// A column is a key, the rows are the queries of all heads that share it, one head after
// another: S and dP as above, dv += dout^T P, dk += q^T dS, so shared heads need no sums
// of their own.  The accumulators of dk and dv leave two waves a SIMD at heads of 64.
// The first example above: 413 us, 770 TFLOP/s; matrix units busy 41% of the time, vector
// units 42%, LDS 46%, a fifth of that conflicts of the transposing loads.  The second:
// 243 us, 20%, 40% and 34%.

// lse and delta of a tile's queries, and where it counts (wanted) what rounding took from
// lse.
template <int ROWS>
struct StageSums {
    float lse, delta, rest;
    __device__ __forceinline__ void fetch(int thread, const float *l, const float *d,
                                          const float *r, int first, int limit, float lifted,
                                          bool wanted)
    {
        const int row = first + thread;
        const bool there = thread < ROWS && row < limit;
        // (a row that is not there has weights 0)
        const float whole = there ? l[row] : INFINITY;
        lse = whole - lifted;
        delta = there ? d[row] : 0.0f;
        if (!wanted) return;
        rest = there && r ? r[row] : 0.0f;
        if (lifted != 0.0f && whole < INFINITY) rest += (whole - lse) - lifted;
    }
    __device__ __forceinline__ void put(int thread, float *at, bool wanted) const
    {
        if (thread < ROWS) {
            at[thread] = lse;
            at[ROWS + thread] = delta;
            if (wanted) at[2 * ROWS + thread] = rest;
        }
    }
};

template <typename T, int DP, bool BIAS, bool SHARED>
__global__ __launch_bounds__(256) void attend_dkv_kernel(AttendK k)
{
    typedef typename Matrix<T>::frag frag;
    constexpr int ROWS = attend_kv_rows(DP, sizeof(T), SHARED);
    constexpr int WAVES = SHARED ? 4 : 1, BUFS = SHARED ? 1 : 2;
    constexpr int TILE = ROWS * kStride<T, DP>, STEP = Team<SHARED>::kStep;
    __shared__ __attribute__((aligned(16))) T tiles[WAVES][BUFS][2][TILE];
    __shared__ float dense[WAVES][BIAS ? kMaxBiasAxes * kReachRow : 1];
    __shared__ TilePos<BIAS ? ROWS : 1> qpos[WAVES][BUFS];
    __shared__ __attribute__((aligned(16))) float sums[WAVES][BUFS][3 * ROWS];
    constexpr bool TWO = kTwoWalks<T>;
    __shared__ float zeros[TWO ? 1 : ROWS];

    const Team<SHARED> team;
    const int lane = team.lane, wave = team.wave, half = team.half;
    const int me = team.mine(), stager = team.stager();
    int id = near_block();
    const int rb = id % k.blocks;
    id /= k.blocks;
    const int split = id % k.splits;
    id /= k.splits;
    const int kvh = id % k.Hk, b = id / k.Hk;
    const int G = k.H / k.Hk;
    const int len = valid_keys(k.lens, b, k.Tk);
    // tiles of the group's heads, one head after another
    const int a_head = max((k.Tq + ROWS - 1) / ROWS, 1);
    const int first = k.from + split * k.per;
    int last = min(k.Tq > 0 ? G * a_head : 0, first + k.per);
    if (rb * (SHARED ? 32 : 128) >= len) last = first;

    const int t = (SHARED ? rb : rb * 4 + wave) * 32 + (lane & 31);
    const bool there = t < k.Tk, seen = t < len;
    const int64_t tt = t;
    frag key[kPairs<T, DP>], val[kPairs<T, DP>];
    load_column<T, DP>(key, (const T *)k.k.data + b * k.k.batch + tt * k.k.token + kvh * k.k.head,
                       seen, half, k.D);
    load_column<T, DP>(val, (const T *)k.v.data + b * k.v.batch + tt * k.v.token + kvh * k.v.head,
                       seen, half, k.D);
    int kpos[kMaxBiasAxes];
#pragma unroll
    for (int a = 0; a < kMaxBiasAxes; ++a)
        kpos[a] = BIAS && seen && a < k.bias.axes
                      ? k.bias.kpos[b * k.bias.kbatch + tt * k.bias.axes + a]
                      : 0;
    f32x16 dk[DP / 32], dv[DP / 32];
    clear(dk);
    clear(dv);
    Lift<T, DP / 32> lift;
    lift.start();

    const T *qp = (const T *)k.q.data + b * k.q.batch;
    const T *gp = (const T *)k.dout.data + b * k.dout.batch;
    const int64_t sums0 = (int64_t)b * k.H * k.Tq;
    const int32_t *pp = BIAS ? k.bias.qpos + b * k.bias.qbatch : nullptr;
    Stage<T, DP, ROWS, Team<SHARED>::kStagers> sq, sg;
    StagePos<BIAS ? ROWS : 1> sp;
    StageSums<ROWS> ss;
    // tile i: a head of the group, its rows; all fetched and then put, or one array
    // after the other
    constexpr bool AHEAD = !SHARED || kFetchAhead<T, DP>;
    auto fetch = [&](int i, bool rest) __attribute__((always_inline)) {
        const int g = i / a_head, row = (i - g * a_head) * ROWS;
        const int h = kvh * G + g;
        sq.fetch(stager, qp + h * k.q.head, k.q.token, row, k.Tq, k.D);
        if (!AHEAD) sq.put(stager, tiles[me][0][0]);
        sg.fetch(stager, gp + h * k.dout.head, k.dout.token, row, k.Tq, k.D);
        if (!AHEAD) sg.put(stager, tiles[me][0][1]);
        const int64_t at = sums0 + (int64_t)h * k.Tq;
        ss.fetch(stager, k.lse + at, k.delta + at, k.lse_rest ? k.lse_rest + at : nullptr, row,
                 k.Tq, kWeightLift<T>, rest);
        if (BIAS) sp.fetch(stager, pp, k.bias.axes, row, k.Tq);
    };
    auto put = [&](int to, bool rest) __attribute__((always_inline)) {
        if (AHEAD) {
            sq.put(stager, tiles[me][to][0]);
            sg.put(stager, tiles[me][to][1]);
        }
        ss.put(stager, sums[me][to], rest);
        if (BIAS) sp.put(stager, qpos[me][to], k.bias.axes);
    };
    int head = -1;              // whose bias is in LDS
    if (!TWO && lane < ROWS) zeros[lane] = 0.0f;    // (by each wave)
    const int first1 = first + me;
    if (first1 < last) {
        fetch(first1, true);
        put(0, true);
    }
    // whether the block meets a large lse
    bool some_large = false;
#pragma unroll 4
    for (int i = first + threadIdx.x / ROWS; i < last; i += 256 / ROWS) {
        const int g = i / a_head, row = (i - g * a_head) * ROWS + threadIdx.x % ROWS;
        if (row < k.Tq)
            some_large = some_large || large_sum(k.lse[sums0 + (int64_t)(kvh * G + g) * k.Tq + row]);
    }
    const bool large = block_any(some_large);
    auto walk = [&](auto kind) __attribute__((always_inline)) {
        constexpr int SUMS = decltype(kind)::value;
        constexpr bool EARLY = AHEAD && SUMS != kAllLarge;
        const bool one = SUMS == kAllLarge || (SUMS == kSomeLarge && large);
        const bool rest = one || sizeof(T) == 4;
        int cur = 0;
        for (int i0 = first1; i0 < last; i0 += STEP, cur ^= BUFS - 1) {
            const bool more = i0 + STEP < last;
            if (more && EARLY) fetch(i0 + STEP, rest);
            if (BIAS && head != i0 / a_head) {      // (the same for all that share it)
                head = i0 / a_head;
                // (mirrored: the rows are queries here)
                load_bias(dense[me], k.bias, kvh * G + head, k.H, stager, Team<SHARED>::kStagers,
                          true);
                team.meet();
            }
#pragma unroll
            for (int u = 0; u < ROWS / 32; ++u) {
                const T *qt = tiles[me][cur][0] + u * 32 * kStride<T, DP>;
                const T *gt = tiles[me][cur][1] + u * 32 * kStride<T, DP>;
                const float *sm = sums[me][cur] + 32 * u;
                f32x16 p, g;
#pragma unroll
                for (int i = 0; i < 16; ++i) p[i] = g[i] = 0.0f;
                pair_mul<T, DP>(qt, gt, lane, key, val, p, g, k.D);
                if constexpr (BIAS) {
                    add_bias<ROWS>(p, k.scale, qpos[me][cur], u, half, dense[me], 0, kpos, k.bias.axes,
                                   k.bias.reach);
                }
                const float unit = BIAS ? 1.0f : k.scale;
                if (one) {
                    rare();
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int at = tile_row(i, half);
                        p[i] = exponent(p[i], unit, sm[at], sm[2 * ROWS + at], kWeightLift<T>);
                    }
                }
                const float by = one ? 1.0f : unit;
                const float *less = SUMS == kSomeLarge && one ? zeros : sm;
                const float *left = SUMS == kSomeLarge && one ? zeros : sm + 2 * ROWS;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int at = tile_row(i, half);
                    float x = SUMS == kAllLarge ? p[i] : fmaf(p[i], by, -less[at]);
                    if (sizeof(T) == 4 && SUMS != kAllLarge) x -= left[at];
                    p[i] = __builtin_amdgcn_exp2f(x);
                    g[i] = p[i] * (g[i] - sm[ROWS + at]);
                }
                add_cols<T, DP>(gt, lane, p, dv);
                lift.scale(g, dk);
                add_cols<T, DP>(qt, lane, g, dk);
            }
            if (BUFS == 1) team.meet();
            if (more) {
                if (!EARLY) fetch(i0 + STEP, rest);
                put(cur ^ (BUFS - 1), rest);
            }
            team.meet();
        }
    };
    if constexpr (!kTwoWalks<T>)
        walk(std::integral_constant<int, kSomeLarge>());
    else if (large)
        walk(std::integral_constant<int, kAllLarge>());
    else
        walk(std::integral_constant<int, kNoLarge>());
    // (one key: as in the queries' gradient)
    const float plain = kLifted<T> ? 0x1p-15f : 1.0f;
    const float scale = len == 1 ? 0.0f : k.plain_scale * plain;
    const int64_t rows = (int64_t)k.B * k.Hk * k.Tk;
    const int64_t row = ((int64_t)b * k.Hk + kvh) * k.Tk + tt;
    if constexpr (SHARED) {
        float f[DP / 8], e[DP / 8];
        float *room = (float *)&tiles[0][0][0][0];
        join_waves<DP>(room, lane, wave, dk, lift.back(), f);
        join_waves<DP>(room, lane, wave, dv, 1.0f, e);
        if (!there) return;
        if (!seen)
#pragma unroll
            for (int i = 0; i < DP / 8; ++i) e[i] = f[i] = 0.0f;
        const int d = (2 * wave + half) * (DP / 8);
        if (k.splits > 1) {
            store_run<float>(k.part + (split * rows + row) * k.D, d, k.D, f, scale);
            store_run<float>(k.part + ((k.slots + split) * rows + row) * k.D, d, k.D, e, plain);
        } else {
            store_run<T>((T *)k.dk.data + b * k.dk.batch + tt * k.dk.token + kvh * k.dk.head, d,
                         k.D, f, scale);
            store_run<T>((T *)k.dv.data + b * k.dv.batch + tt * k.dv.token + kvh * k.dv.head, d,
                         k.D, e, plain);
        }
        return;
    }
    if (!there) return;
    if (!seen) {
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) dk[d][i] = dv[d][i] = 0.0f;
    }
    const float by = lift.back() * scale;
    if (k.splits > 1) {
        store_column<float, DP>(k.part + (split * rows + row) * k.D, half, k.D, dk, by);
        store_column<float, DP>(k.part + ((k.slots + split) * rows + row) * k.D, half, k.D, dv,
                                plain);
    } else {
        store_column<T, DP>((T *)k.dk.data + b * k.dk.batch + tt * k.dk.token + kvh * k.dk.head,
                            half, k.D, dk, by);
        store_column<T, DP>((T *)k.dv.data + b * k.dv.batch + tt * k.dv.token + kvh * k.dv.head,
                            half, k.D, dv, plain);
    }
}

// --- joins ----------------------------------------------------------------------------

// out[b][t][h][d] = sum of the splits' parts [split][b][h][t][d], a quad for G threads,
// which take every G-th split and join in order; with blockIdx.y = 1 the second array's
// parts, which follow.  A pass that is not the last leaves its sum as a part.  (256 splits
// of 40 rows of 128, twice: one thread a quad 71 us, 32 threads 6.7.)
template <typename T, int G>
__device__ __forceinline__ void sum_quad(const float *part, int parts, int64_t rows, int H,
                                         int Tn, int D, const SeqK &out, int64_t at,
                                         float4 (&sums)[G > 1 ? 256 : 1])
{
    const int quads = (D + 3) / 4;
    const int g = threadIdx.x / (256 / G);
    const bool there = at < rows * quads;
    const int64_t row = at / quads;
    const int d = (int)(at - row * quads) * 4;
    float a[4] = {0, 0, 0, 0};
    if (there) {
        const float *p = part + row * D + d;
#pragma unroll 4
        for (int s = g; s < parts; s += G) {
            const float *q = p + s * rows * D;
            if (d + 4 <= D) {
                float f[4];
                load_vec<float, 4>(q, f);
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] += f[i];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (d + i < D) a[i] += q[i];
            }
        }
    }
    if (G > 1) {
        sums[threadIdx.x] = make_float4(a[0], a[1], a[2], a[3]);
        __syncthreads();
        if (g == 0)
#pragma unroll 8
            for (int j = 1; j < G; ++j) {
                const float4 x = sums[threadIdx.x + j * (256 / G)];
                a[0] += x.x;
                a[1] += x.y;
                a[2] += x.z;
                a[3] += x.w;
            }
    }
    if (!there || g != 0) return;
    const int64_t bh = row / Tn;
    const int t = (int)(row - bh * Tn), b = (int)(bh / H), h = (int)(bh - (int64_t)b * H);
    store_quad<T>((T *)out.data + b * out.batch + (int64_t)t * out.token + h * out.head, d, D, a[0],
                  a[1], a[2], a[3]);
}

template <typename T, int G>
__global__ __launch_bounds__(256) void attend_sum_kernel(const float *part, int slots, int parts,
                                                         int B, int H, int Tn, int D, SeqK one,
                                                         SeqK two)
{
    constexpr int EACH = 256 / G;
    __shared__ float4 sums[G > 1 ? 256 : 1];
    const int64_t rows = (int64_t)B * H * Tn, all = rows * ((D + 3) / 4);
    for (int64_t first = (int64_t)blockIdx.x * EACH; first < all;
         first += (int64_t)gridDim.x * EACH) {
        sum_quad<T, G>(part + (int64_t)blockIdx.y * slots * rows * D, parts, rows, H, Tn, D,
                       blockIdx.y ? two : one, first + threadIdx.x % EACH, sums);
        if (G > 1) __syncthreads();     // (sums are read to the end)
    }
}

// dtable[axis][bucket][h] = sum over the parts of head h's blocks, in 64 bits: a block an
// axis and head, 32 lanes its buckets, 32 groups of them every 32nd part.  A row's dS sum
// to 0, and so do an axis' buckets; where all but one of them are 0 (one bucket, or one
// distance for all pairs), that one is 0 as well and not what roundings left of its sum
// (times 0, so that a NaN stays).  Passes add to held, the last one writes.
__global__ __launch_bounds__(1024) void attend_table_kernel(const float *part, int B, int H,
                                                            int each, int axes, int count,
                                                            double *held, bool more, bool last,
                                                            float *dtable)
{
    static_assert(kMaxBuckets == 32);
    __shared__ double sums[32][32];
    const int axis = blockIdx.x, h = blockIdx.y, e = threadIdx.x & 31, g = threadIdx.x >> 5;
    // block ((b H + h) each + i) of the queries' gradient
    double a = 0.0;
    if (e < count)
#pragma unroll 4
        for (int64_t i = g; i < (int64_t)B * each; i += 32) {
            const int64_t b = i / each;
            a += part[((b * H + h) * each + (i - b * each)) * (axes * count) + axis * count + e];
        }
    sums[g][e] = a;
    for (int n = 16; n > 0; n >>= 1) {
        __syncthreads();
        if (g < n) sums[g][e] += sums[g + n][e];
    }
    if (g != 0) return;
    a = sums[0][e];
    const int64_t at = ((int64_t)axis * count + e) * H + h;
    if (e < count && more) a += held[at];
    if (!last) {
        if (e < count) held[at] = a;
        return;
    }
    const uint32_t some = (uint32_t)__builtin_amdgcn_ballot_w64(a != 0.0);
    if ((some & (some - 1)) == 0) a = fabs(a * 0.0);
    if (e < count) dtable[at] = (float)a;
}

template <typename T>
hipError_t launch_sum(const AttendK &k, int H, int64_t Tn, const SeqK &one, const SeqK &two, int n,
                      hipStream_t stream)
{
    const int64_t quads = (int64_t)k.B * H * Tn * ((k.D + 3) / 4);
    if (quads == 0) return hipSuccess;
    auto go = [&](auto g) {
        constexpr int G = decltype(g)::value, each = 256 / G;
        const dim3 grid((unsigned)join_blocks((quads + each - 1) / each), n);
        if (k.last) {
            attend_sum_kernel<T, G><<<grid, 256, 0, stream>>>(k.part, k.slots, k.parts, k.B, H,
                                                              (int)Tn, k.D, one, two);
            return;
        }
        const int64_t rows = (int64_t)k.B * H * Tn;
        SeqK left{k.part + k.splits * rows * k.D, H * Tn * k.D, k.D, Tn * k.D}, more = left;
        more.data = (float *)left.data + k.slots * rows * k.D;
        attend_sum_kernel<float, G><<<grid, 256, 0, stream>>>(k.part, k.slots, k.parts, k.B, H,
                                                              (int)Tn, k.D, left, more);
    };
    if (k.splits > 8)
        go(std::integral_constant<int, 32>());
    else
        go(std::integral_constant<int, 1>());
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch_back_q(const AttendK &k, const AttendPlan &p, hipStream_t stream)
{
    const unsigned grid = (unsigned)((int64_t)k.B * k.H * k.splits * k.blocks);
    const int entries = k.bias.axes * k.bias.buckets;
    typedef std::true_type yes;
    typedef std::false_type no;
    auto go = [&](auto shared) {
        constexpr bool S = decltype(shared)::value;
        if (grid == 0) return;
        if (k.bias.axes)
            attend_dq_kernel<T, DP, true, S>
                <<<grid, 256, attend_hist_bytes(entries), stream>>>(k);
        else
            attend_dq_kernel<T, DP, false, S><<<grid, 256, 0, stream>>>(k);
    };
    if (p.shared)
        go(yes());
    else
        go(no());
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && k.splits > 1) e = launch_sum<T>(k, k.H, k.Tq, k.dq, k.dq, 1, stream);
    if (e == hipSuccess && entries && k.dtable) {
        attend_table_kernel<<<dim3(k.bias.axes, k.H), 1024, 0, stream>>>(
            k.part_table, k.B, k.H, k.splits * k.blocks, k.bias.axes, k.bias.buckets, k.table_sum,
            k.pass > 0, k.last, k.dtable);
        e = hipGetLastError();
    }
    return e;
}

template <typename T, int DP>
hipError_t launch_back_kv(const AttendK &k, const AttendPlan &p, hipStream_t stream)
{
    const unsigned grid = (unsigned)((int64_t)k.B * k.Hk * k.splits * k.blocks);
    if (grid == 0) return hipSuccess;
    auto go = [&](auto bias, auto shared) {
        attend_dkv_kernel<T, DP, decltype(bias)::value, decltype(shared)::value>
            <<<grid, 256, 0, stream>>>(k);
    };
    typedef std::true_type yes;
    typedef std::false_type no;
    if (k.bias.axes)
        p.shared ? go(yes(), yes()) : go(yes(), no());
    else
        p.shared ? go(no(), yes()) : go(no(), no());
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && k.splits > 1) e = launch_sum<T>(k, k.Hk, k.Tk, k.dk, k.dv, 2, stream);
    return e;
}

}  // namespace
}  // namespace mixrt
