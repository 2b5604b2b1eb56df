// Group norm with an activation on channels-last feature maps: what the forward
// (mixrt_norm.hip) and the backward (mixrt_norm_back.hip) share.
//
// A row is a pixel's C channels.  Threads take vectors of V channels; a block's
// threads lie over `lanes` vectors of a row and over R rows, so that a thread
// keeps its channels (and their constants) while it walks down the image.
//
// Large images: sums over parts of the image, their join, then the normalised
// rows: three launches that read x twice.  Where an image has few parts, the
// blocks of the last launch join them themselves (two launches).  Small images,
// forward: one launch, whose blocks each sum up all rows of a few groups and
// then write a share of them.  A launch takes about 4 us beside its work.
// Joins add in a fixed order: the same inputs give the same bits.
#pragma once

#include "mixrt_refine.hpp"

#include <type_traits>

namespace mixrt {

inline constexpr int kThreads = 256;
inline constexpr int kSmallThreads = 1024;
inline constexpr int kJoinThreads = 1024;
// Rows a thread loads before it uses the first.  The backward's sums take one
// at a time: they gain more from more waves (8 x 360p x 64 in bf16: 97 us, with
// two 106, four 135; its writing 136 with one, 123 with two, 104 with four).
inline constexpr int kAhead = 4;
// Most rows that a thread of the backward's sums adds up in 32 bits: each addition
// rounds what is there, so equal terms are off by half as many units at most.
inline constexpr int kBackRows = 128;
inline constexpr int kFoldChannels = 512;   // most channels (and groups) of a join by the blocks

struct NormK {
    int N, C, G, Cg;
    int64_t P;
    int lanes, R;
    int S;              // parts of an image (of the sums that are joined)
    int slabs;
    float eps;
    const float *gamma, *beta;
    MapK x, y, dy, dx;
    float *stats;       // never null here: the caller's or the workspace's
    int8_t *codes;
    uint8_t *exps;
    float *dgamma, *dbeta;
    void *sums;         // forward: double2 [N][S * slabs][G]; backward: float2 [N][S][C]
    float *means;       // backward: [N][G][2]: the group means of gamma dz and gamma dz xh
    float2 *channels;   // backward: [N][C]: each image's sums of dz and dz xh
};

// exp(x) as 2^(x log2 e).  The product and its constant are rounded, so the result
// is off by up to about 2 |x| + 2 units of 2^-24 of itself.
__device__ __forceinline__ float fast_exp(float x)
{
    return __builtin_amdgcn_exp2f(x * 1.4426950408889634f);
}

// exp(-z^2 / 2)
__device__ __forceinline__ float density(float z)
{
    return __builtin_amdgcn_exp2f(z * z * -0.72134752f);
}

// erfc(|z| / sqrt 2) exp(z^2 / 2) / 2, the normal distribution's tail beyond |z|
// in units of exp(-z^2 / 2): t q(t), t = 1 / (1 + 0.26 |z|), where t q(t) is by linear
// programming the polynomial of its degree, one half at z = 0, whose largest
// relative error over 0 <= |z| <= 10 is least: 3.9e-7 with the coefficients in 32
// bits (and 1.0e-5 at 13).
// A form with a bounded absolute error leaves nothing of gelu's negative side:
// gelu(-4) then was off by a thousandth.
struct Tail {
    float q, t;
    __device__ __forceinline__ explicit Tail(float z)
    {
        t = __builtin_amdgcn_rcpf(fmaf(0.26f, fabsf(z), 1.0f));
        q = fmaf(-0.07529450207948685f, t, 0.2379440814256668f);
        q = fmaf(q, t, -0.12034948170185089f);
        q = fmaf(q, t, 0.17749814689159393f);
        q = fmaf(q, t, 0.06855196505784988f);
        q = fmaf(q, t, 0.1082243025302887f);
        q = fmaf(q, t, 0.10342548787593842f);
    }
};

template <int ACT>
__device__ __forceinline__ float act(float z)
{
    if (ACT == kActRelu) return z > 0.0f ? z : (z <= 0.0f ? 0.0f : z);   // keeps a NaN
    if (ACT == kActSilu) return z * __builtin_amdgcn_rcpf(1.0f + fast_exp(-z));
    // z and its tail apart: the positive side as z less a part, the negative one
    // the part alone.  (The bound: an infinity times a tail of 0 would be a NaN.)
    if (ACT == kActGelu) {
        const Tail tail(z);
        return fmaf(-fminf(fabsf(z), 1e38f), tail.q * tail.t * density(z), fmaxf(z, 0.0f));
    }
    return z;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float z)
{
    if (ACT == kActRelu) return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
    if (ACT == kActSilu) {
        const float s = __builtin_amdgcn_rcpf(1.0f + fast_exp(-z));
        return fmaf(fmaf(-z, s, z), s, s);   // s (1 + z (1 - s)); z (1 - s) stays finite
    }
    if (ACT == kActGelu) {
        // the tail less |z| times the density at its height, and 1 less that
        const Tail tail(z);
        const float d = fmaf(tail.q, tail.t, -0.39894228040143268f * fabsf(z)) * density(z);
        return z < 0.0f ? d : 1.0f - d;
    }
    return 1.0f;
}

// f(i, group) for the V channels from c0 on.
template <int V, typename F>
__device__ __forceinline__ void for_groups(const NormK &k, int c0, F f)
{
    int g = c0 / k.Cg, left = (g + 1) * k.Cg - c0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (i >= left) {
            ++g;
            left += k.Cg;
        }
        f(i, g);
    }
}

// A thread's constants, those of its V channels in one image, around
// t = x - mean: z = t scale + beta with scale = rstd gamma.
template <int V>
struct Channels {
    float mean[V], scale[V], be[V], rstd[V];
    // stats: (mean, rstd) of the image's groups; c0: the first channel
    __device__ __forceinline__ void set(const NormK &k, const float *stats, int c0)
    {
        float ga[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            ga[i] = 1.0f;
            be[i] = 0.0f;
        }
        if (k.gamma) load_vec<float, V>(k.gamma + c0, ga);
        if (k.beta) load_vec<float, V>(k.beta + c0, be);
        for_groups<V>(k, c0, [&](int i, int g) {
            const float2 st = ((const float2 *)stats)[g];
            mean[i] = st.x;
            rstd[i] = st.y;
        });
#pragma unroll
        for (int i = 0; i < V; ++i) scale[i] = rstd[i] * ga[i];
    }
};

// Walks a block's rows: runs of U * R rows, every `parts`th of them from run
// `at`, so that the blocks' runs of one time are neighbours in memory.  load(p)
// of a thread's U rows first, then use(p, what it gave).
template <typename D, int U, typename LOAD, typename USE>
__device__ __forceinline__ void walk(int64_t at, int64_t parts, int r, int R, int64_t P, LOAD load,
                                     USE use)
{
    const int64_t run = (int64_t)U * R;
    int64_t p = at * run + r;
    for (; p + (int64_t)(U - 1) * R < P; p += parts * run) {
        D d[U];
#pragma unroll
        for (int u = 0; u < U; ++u) d[u] = load(p + (int64_t)u * R);
        __builtin_amdgcn_sched_barrier(0);   // else the loads sink to their uses
#pragma unroll
        for (int u = 0; u < U; ++u) use(p + (int64_t)u * R, d[u]);
    }
    // the image's last run, where it is not whole: this block's if any
    if (U > 1)
        for (int u = 0; u < U && p < P; ++u, p += R) use(p, load(p));
}

// Adds the R rows' values of every lane; thread (0, j) ends with the sum.
// v: shared [K][kThreads].
template <int K, typename A>
__device__ __forceinline__ void join_rows(A (*v)[kThreads], int lanes, int R, int j, int r)
{
    for (int n = R; n > 1;) {
        const int half = (n + 1) / 2;
        __syncthreads();
        if (r < n - half)
#pragma unroll
            for (int k = 0; k < K; ++k) v[k][r * lanes + j] += v[k][(r + half) * lanes + j];
        n = half;
    }
    __syncthreads();
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// (mean, rstd) from a group's sums of x and x^2 over m elements.
__device__ __forceinline__ float2 group_stats(const NormK &k, double s, double q)
{
    const double m = (double)k.P * k.Cg, mean = k.P > 0 ? s / m : 0.0;
    double var = k.P > 0 ? q / m - mean * mean : 0.0;
    if (var < 0.0) var = 0.0;   // a NaN stays
    return make_float2((float)mean, (float)(1.0 / sqrt(var + (double)k.eps)));
}

// --- plans ------------------------------------------------------------------------

struct NormPlan {
    enum Way { kSmall, kFold, kLarge } way;
    int chunk;      // small: channels of a block
    int V;          // channels of a vector
    int lanes;      // vectors of a row in one slab or chunk (threads across a row)
    int slabs;      // slabs of a row
    int R;          // rows of one step of a block
    int S;          // parts an image is split into for the sums
    int share;      // blocks that share an image's rows when they are written
};

inline int64_t gcd(int64_t a, int64_t b) { return b ? gcd(b, a % b) : a; }

inline constexpr int64_t kSmallBytes = 192 << 10;
inline constexpr int64_t kSmallRow = 32;   // least bytes of a row that a block reads

// pad: x is kept in the same pass; a row takes whole kept groups of lanes, so
// that the lanes of a group are aligned neighbours.
inline NormPlan norm_plan(int N, int64_t P, int C, int G, int dtype, bool pad, bool back)
{
    NormPlan p{};
    const int size = dtype == kF32 ? 4 : 2, Cg = C / G;
    // (1 where there are no pixels: a grid has a block)
    const auto atmost = [](int64_t v, int64_t hi) {
        if (v > hi) v = hi;
        return v < 1 ? 1 : v;
    };
    if (!back) {
        p.V = 16 / size;
        while (Cg % p.V) p.V >>= 1;
        int64_t chunk = pad ? (int64_t)Cg / gcd(Cg, kKeptGroup) * kKeptGroup : Cg;
        while (chunk * size < kSmallRow && chunk < C) chunk += Cg;
        if (chunk > C) chunk = C;
        const int64_t vecs = pad ? (chunk + kKeptGroup - 1) / kKeptGroup * (kKeptGroup / p.V)
                                 : chunk / p.V;
        if (vecs <= kSmallThreads && P * chunk * size <= kSmallBytes) {
            p.way = NormPlan::kSmall;
            p.chunk = (int)chunk;
            p.lanes = (int)vecs;
            p.slabs = 1;
            p.R = kSmallThreads / p.lanes;
            p.S = 1;
            const int64_t blocks = (int64_t)N * ((C + chunk - 1) / chunk);
            p.share = (int)atmost(512 / (blocks > 0 ? blocks : 1), (P + p.R - 1) / p.R);
            return p;
        }
    }
    p.V = 16 / size;
    while (C % p.V) p.V >>= 1;
    const int wide = pad ? kept_groups(C) * (kKeptGroup / p.V) : C / p.V;
    p.lanes = wide < kThreads ? wide : kThreads;
    p.slabs = (wide + p.lanes - 1) / p.lanes;
    p.R = kThreads / p.lanes;
    const int64_t run = (int64_t)p.R * kAhead, runs = (P + run - 1) / run;
    // few runs: as many parts as runs, or half as many, joined by the blocks
    // that write (16 channels of 320 x 180 in f16, 57 parts: 12.2 us, joined by
    // a launch 13.6; backward, 32 channels of 160 x 90, 57 parts: 19.1 and 18.2,
    // but three crops of 24 channels, 12 parts: 32 and 35)
    const int64_t fold = runs <= 64 ? runs : (runs + 1) / 2;
    if (C <= kFoldChannels && fold <= (back ? 32 : 64) && (int64_t)N * fold <= 512 &&
        fold * (back ? C : G * p.slabs) <= 4096) {
        p.way = NormPlan::kFold;
        p.S = p.share = (int)atmost(fold, 1024);
        return p;
    }
    p.way = NormPlan::kLarge;
    // sums: 4 blocks a CU, at least one a CU for every image; writing: two
    // runs a block forward, 3 blocks a CU backward
    const int64_t images = N > 0 ? (int64_t)N * p.slabs : 1;
    int64_t S = 1024 / images;
    if (S < 256 && images < 64) S = 256;
    const int64_t least = (P + (int64_t)p.R * kBackRows - 1) / ((int64_t)p.R * kBackRows);
    if (back && S < least) S = least;
    p.S = (int)atmost(S, runs);
    p.share = back ? (int)atmost(768 / images, runs) : (int)atmost((runs + 1) / 2, 1 << 20);
    return p;
}

inline NormK norm_args(const NormLaunch &L, const NormPlan &p)
{
    NormK k{};
    k.N = L.N;
    k.C = L.C;
    k.G = L.G;
    k.Cg = L.C / L.G;
    k.P = L.P;
    k.lanes = p.lanes;
    k.R = p.R;
    k.S = p.S;
    k.slabs = p.slabs;
    k.eps = L.eps;
    k.gamma = L.gamma;
    k.beta = L.beta;
    k.x = L.x;
    k.y = L.y;
    k.dy = L.dy;
    k.dx = L.dx;
    k.stats = L.stats;
    k.codes = L.codes;
    k.exps = L.exps;
    k.dgamma = L.dgamma;
    k.dbeta = L.dbeta;
    return k;
}

inline size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

// Workspace: group values (float [N][G][2]), channel values (float2 [N][C],
// backward), then the parts' sums.
inline size_t group_bytes(int N, int G) { return up16((size_t)N * G * 8); }
inline size_t channel_bytes(int N, int C) { return up16((size_t)N * C * 8); }

// f(integral_constant<ACT>) for the activation.
template <typename F>
void with_act(int act, F f)
{
    switch (act) {
    case kActNone: f(std::integral_constant<int, kActNone>()); break;
    case kActRelu: f(std::integral_constant<int, kActRelu>()); break;
    case kActSilu: f(std::integral_constant<int, kActSilu>()); break;
    default: f(std::integral_constant<int, kActGelu>()); break;
    }
}

// f((T *)0, integral_constant<V>) for the element type and vector width.
template <typename F>
void with_type(int dtype, int V, F f)
{
    if (dtype == kF32) {
        if (V == 4) f((float *)0, std::integral_constant<int, 4>());
        else if (V == 2) f((float *)0, std::integral_constant<int, 2>());
        else f((float *)0, std::integral_constant<int, 1>());
    } else if (dtype == kF16) {
        if (V == 8) f((f16 *)0, std::integral_constant<int, 8>());
        else if (V == 4) f((f16 *)0, std::integral_constant<int, 4>());
        else if (V == 2) f((f16 *)0, std::integral_constant<int, 2>());
        else f((f16 *)0, std::integral_constant<int, 1>());
    } else {
        if (V == 8) f((bf16 *)0, std::integral_constant<int, 8>());
        else if (V == 4) f((bf16 *)0, std::integral_constant<int, 4>());
        else if (V == 2) f((bf16 *)0, std::integral_constant<int, 2>());
        else f((bf16 *)0, std::integral_constant<int, 1>());
    }
}

}  // namespace mixrt
