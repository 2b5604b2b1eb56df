// Attention, forward: one pass over the keys with the running maximum and sum.
#pragma once

#include "mixrt_attend_tile.hpp"

namespace mixrt {
namespace {

// W waves a block, NC blocks of 32 columns a wave, PK heads' biases in LDS.
// EXACT (for training with the 16-bit types): the weights go into the second product
// as two terms, their rounded values and what that left.  The backward pass takes
// delta = sum_j P_ij dP_ij from the output, and dS = P (dP - delta) cancels where a
// row looks at few keys: an output from rounded weights would leave there the
// rounding itself, not a small part of it.
template <typename T, int DP, int W, int NC, bool BIAS, bool EXACT>
__global__ __launch_bounds__(64 * W) void attend_kernel(AttendK k)
{
    typedef typename Matrix<T>::frag frag;
    constexpr int ROWS = sizeof(T) == 2 && W > 1 ? 64 : 32;
    constexpr int THREADS = 64 * W;
    constexpr int PK = BIAS ? (W == 1 ? 8 : 1) : 1;
    constexpr int TILE = ROWS * kStride<T, DP>;
    __shared__ __attribute__((aligned(16))) T tiles[2][2][TILE];
    __shared__ float dense[BIAS ? PK * kMaxBiasAxes * kReachRow : 1];
    __shared__ TilePos<BIAS ? ROWS : 1> kpos[2];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    int id = near_block();
    const int rb = id % k.blocks;
    id /= k.blocks;
    const int split = id % k.splits;
    id /= k.splits;
    const int packs = k.H / k.pack;
    const int h0 = id % packs * k.pack, b = id / packs;
    const int kvh = h0 / (k.H / k.Hk);
    const int len = valid_keys(k.lens, b, k.Tk);
    const int first = split * k.per, last = min(len, first + k.per);

    // the lane's columns
    int t[NC], head[NC];
    bool there[NC];
    frag q[NC][kPairs<T, DP>];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        const int col = ((rb * W + wave) * NC + n) * 32 + (lane & 31);
        t[n] = col / k.pack;
        head[n] = h0 + col % k.pack;
        there[n] = t[n] < k.Tq;
        load_column<T, DP>(q[n], (const T *)k.q.data + b * k.q.batch + (int64_t)t[n] * k.q.token +
                                     head[n] * k.q.head,
                           there[n], half, k.D);
    }
    int qpos[NC][kMaxBiasAxes];
    int hbase[NC];
    if (BIAS) {
        for (int p = 0; p < k.pack; ++p)
            load_bias(dense + p * kMaxBiasAxes * kReachRow, k.bias, h0 + p, k.H, THREADS, false);
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            hbase[n] = (head[n] - h0) * kMaxBiasAxes * kReachRow;
#pragma unroll
            for (int a = 0; a < kMaxBiasAxes; ++a)
                qpos[n][a] = there[n] && a < k.bias.axes
                                 ? k.bias.qpos[b * k.bias.qbatch + (int64_t)t[n] * k.bias.axes + a]
                                 : 0;
        }
    }

    f32x16 acc[NC][DP / 32];
    float top[NC], sum[NC];     // in units of log2; sum: of the lane's own rows
#pragma unroll
    for (int n = 0; n < NC; ++n) {
        top[n] = -INFINITY;
        sum[n] = 0.0f;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][d][i] = 0.0f;
    }

    const T *kp = (const T *)k.k.data + b * k.k.batch + kvh * k.k.head;
    const T *vp = (const T *)k.v.data + b * k.v.batch + kvh * k.v.head;
    const int32_t *pp = BIAS ? k.bias.kpos + b * k.bias.kbatch : nullptr;
    Stage<T, DP, ROWS, THREADS> sk, sv;
    StagePos<BIAS ? ROWS : 1> sp;
    if (first < last) {
        sk.fetch(kp, k.k.token, first, last, k.D);
        sv.fetch(vp, k.v.token, first, last, k.D);
        if (BIAS) sp.fetch(pp, k.bias.axes, first, last);
        sk.put(tiles[0][0]);
        sv.put(tiles[0][1]);
        if (BIAS) sp.put(kpos[0], k.bias.axes);
    }
    __syncthreads();
    int cur = 0;
    for (int row0 = first; row0 < last; row0 += ROWS, cur ^= 1) {
        const bool more = row0 + ROWS < last;
        if (more) {
            sk.fetch(kp, k.k.token, row0 + ROWS, last, k.D);
            sv.fetch(vp, k.v.token, row0 + ROWS, last, k.D);
            if (BIAS) sp.fetch(pp, k.bias.axes, row0 + ROWS, last);
        }
        const T *kt = tiles[cur][0], *vt = tiles[cur][1];
        f32x16 s[ROWS / 32][NC];
#pragma unroll
        for (int u = 0; u < ROWS / 32; ++u) {
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[u][n][i] = 0.0f;
#pragma unroll
            for (int c = 0; c < kPairs<T, DP>; ++c) {
                const frag a = row_frag<T, DP>(kt + u * 32 * kStride<T, DP>, lane, c);
#pragma unroll
                for (int n = 0; n < NC; ++n) s[u][n] = Matrix<T>::mul(a, q[n][c], s[u][n]);
            }
        }
        if constexpr (BIAS) {
#pragma unroll
            for (int u = 0; u < ROWS / 32; ++u)
                add_bias<NC, ROWS>(s[u], k.scale, kpos[cur], u, half, dense, hbase, qpos,
                                   k.bias.axes, k.bias.reach);
        }
        if (!more && row0 + ROWS > last) {
#pragma unroll
            for (int u = 0; u < ROWS / 32; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (row0 + 32 * u + tile_row(i, half) >= last)
#pragma unroll
                        for (int n = 0; n < NC; ++n) s[u][n][i] = -INFINITY;
        }
        const float unit = BIAS ? 1.0f : k.scale;
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            float m = s[0][n][0];
#pragma unroll
            for (int u = 0; u < ROWS / 32; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) m = fmaxf(m, s[u][n][i]);
            m = fmaxf(half_max(m) * unit, top[n]);
            // (a row of -inf alone keeps weights 0)
            const float base = m == -INFINITY ? 0.0f : m;
            if (__builtin_amdgcn_ballot_w64(m != top[n]) != 0) {
                const float less = __builtin_amdgcn_exp2f(top[n] - base);
                sum[n] *= less;
#pragma unroll
                for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[n][d][i] *= less;
                top[n] = m;
            }
            float add = 0.0f;
#pragma unroll
            for (int u = 0; u < ROWS / 32; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[u][n][i], unit, -base));
                    s[u][n][i] = p;
                    add += p;
                }
            sum[n] += add;
        }
#pragma unroll
        for (int u = 0; u < ROWS / 32; ++u) {
            const T *v = vt + u * 32 * kStride<T, DP>;
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                    for (int n = 0; n < NC; ++n) col_mul<DP>(v, lane, d, s[u][n], acc[n][d]);
            } else {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    frag p[NC], less[NC];
#pragma unroll
                    for (int n = 0; n < NC; ++n) {
                        p[n] = round_rows<T>(s[u][n], e);
                        if (EXACT) less[n] = left_rows<T>(s[u][n], p[n], e);
                    }
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) {
                        const frag a = col_frag<T, DP>(v, lane, d, e);
#pragma unroll
                        for (int n = 0; n < NC; ++n) {
                            acc[n][d] = Matrix<T>::mul(a, p[n], acc[n][d]);
                            if (EXACT) acc[n][d] = Matrix<T>::mul(a, less[n], acc[n][d]);
                        }
                    }
                }
            }
        }
        if (more) {
            sk.put(tiles[cur ^ 1][0]);
            sv.put(tiles[cur ^ 1][1]);
            if (BIAS) sp.put(kpos[cur ^ 1], k.bias.axes);
        }
        __syncthreads();
    }

#pragma unroll
    for (int n = 0; n < NC; ++n) {
        const float l = half_sum(sum[n]);
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        if (!there[n]) continue;
        const int64_t row = ((int64_t)b * k.H + head[n]) * k.Tq + t[n];
        const float lse = top[n] + __builtin_amdgcn_logf(l);    // (log2)
        if (k.splits > 1) {
            const int64_t rows = (int64_t)k.B * k.H * k.Tq;
            if (half == 0) k.part_lse[split * rows + row] = l == 0.0f ? -INFINITY : lse;
            float *o = k.part + (split * rows + row) * k.D;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    store_quad<float>(o, 32 * d + 8 * e + 4 * half, k.D, acc[n][d][4 * e] * inv,
                                      acc[n][d][4 * e + 1] * inv, acc[n][d][4 * e + 2] * inv,
                                      acc[n][d][4 * e + 3] * inv);
            continue;
        }
        if (k.lse && half == 0) k.lse[row] = l == 0.0f ? INFINITY : lse;
        T *o = (T *)k.o.data + b * k.o.batch + (int64_t)t[n] * k.o.token + head[n] * k.o.head;
        T *rest = k.rest ? (T *)k.rest + (((int64_t)b * k.Tq + t[n]) * k.H + head[n]) * k.D
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
                if (rest) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) f[i] = rest_of<T>(f[i]);
                    store_quad<T>(rest, at, k.D, f[0], f[1], f[2], f[3]);
                }
            }
    }
}

// Joins the splits of a row: o = sum_s 2^(lse_s - top) o_s / sum_s 2^(lse_s - top).
// A block takes 256 / (8 G) rows and 32 elements of their heads: 8 lanes hold a row's
// quads, G groups of them share its splits.  (With the splits of a row one after
// another, the 113 of one token's 32 heads took 29 us.)
template <typename T, int G>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendK k)
{
    constexpr int EACH = 32 / G;
    __shared__ float part[5][256];
    const int64_t rows = (int64_t)k.B * k.H * k.Tq;
    const int lane = threadIdx.x & 7, g = threadIdx.x / 8 % G;
    const int64_t row = (int64_t)blockIdx.x * EACH + threadIdx.x / (8 * G);
    const bool there = row < rows;
    const int d = 32 * blockIdx.y + 4 * lane;
    // the group's own maximum first: NaN stays
    float top = -INFINITY;
    if (there)
#pragma unroll 4
        for (int s = g; s < k.splits; s += G) {
            const float x = k.part_lse[s * rows + row];
            top = x > top || x != x ? x : top;
        }
    float base = top == -INFINITY ? 0.0f : top;
    float a[4] = {0, 0, 0, 0}, w = 0.0f;
    if (there)
#pragma unroll 4
        for (int s = g; s < k.splits; s += G) {
            const float e = __builtin_amdgcn_exp2f(k.part_lse[s * rows + row] - base);
            w += e;
            const float *o = k.part + (s * rows + row) * k.D;
            if (d + 4 <= k.D) {
                float f[4];
                load_vec<float, 4>(o + d, f);
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = fmaf(f[i], e, a[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (d + i < k.D) a[i] = fmaf(o[d + i], e, a[i]);
            }
        }
    if (G > 1) {
        // then the groups', in order, at their common maximum
        const bool none = top == -INFINITY;
        part[0][threadIdx.x] = top;
        __syncthreads();
        const int first = threadIdx.x - 8 * g;
        for (int j = 0; j < G; ++j) {
            const float x = part[0][first + 8 * j];
            top = x > top || x != x ? x : top;
        }
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
    if (k.lse && lane == 0 && blockIdx.y == 0)
        k.lse[row] = w == 0.0f ? INFINITY : base + __builtin_amdgcn_logf(w);
    if (d >= k.D) return;
    T *o = (T *)k.o.data + b * k.o.batch + (int64_t)t * k.o.token + h * k.o.head;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] *= inv;
    store_quad<T>(o, d, k.D, a[0], a[1], a[2], a[3]);
    if (k.rest) {
        T *rest = (T *)k.rest + (((int64_t)b * k.Tq + t) * k.H + h) * k.D;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = rest_of<T>(a[i]);
        store_quad<T>(rest, d, k.D, a[0], a[1], a[2], a[3]);
    }
}

template <typename T>
hipError_t launch_join(const AttendK &k, hipStream_t stream)
{
    const int64_t rows = (int64_t)k.B * k.H * k.Tq;
    const unsigned by = (unsigned)(k.D + 31) / 32;
    if (k.splits > 4)
        attend_join_kernel<T, 32><<<dim3((unsigned)rows, by), 256, 0, stream>>>(k);
    else
        attend_join_kernel<T, 1><<<dim3((unsigned)((rows + 31) / 32), by), 256, 0, stream>>>(k);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t launch_forward(const AttendK &k, const AttendPlan &p, hipStream_t stream)
{
    const unsigned grid = (unsigned)((int64_t)k.B * (k.H / k.pack) * k.splits * k.blocks);
    auto go = [&](auto w, auto nc) {
        constexpr int W = decltype(w)::value, NC = decltype(nc)::value;
        if constexpr (sizeof(T) == 2)
            if (k.rest) {
                if (k.bias.axes)
                    attend_kernel<T, DP, W, NC, true, true><<<grid, 64 * W, 0, stream>>>(k);
                else
                    attend_kernel<T, DP, W, NC, false, true><<<grid, 64 * W, 0, stream>>>(k);
                return;
            }
        if (k.bias.axes)
            attend_kernel<T, DP, W, NC, true, false><<<grid, 64 * W, 0, stream>>>(k);
        else
            attend_kernel<T, DP, W, NC, false, false><<<grid, 64 * W, 0, stream>>>(k);
    };
    typedef std::integral_constant<int, 1> one;
    typedef std::integral_constant<int, 4> four;
    if (p.narrow)
        go(one(), one());
    else if constexpr (sizeof(T) == 2 && DP <= 64) {
        if (p.cols == 256)
            go(four(), std::integral_constant<int, 2>());
        else
            go(four(), one());
    } else
        go(four(), one());
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || k.splits == 1) return e;
    return launch_join<T>(k, stream);
}

}  // namespace
}  // namespace mixrt
