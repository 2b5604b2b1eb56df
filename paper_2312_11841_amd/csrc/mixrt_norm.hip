// Group norm with an activation on channels-last feature maps, forward and
// backward.
//
// A row is a pixel's C channels.  Threads take vectors of V channels; a block's
// threads lie over `lanes` vectors of a row and over R rows, so that a thread
// keeps its channels (and their constants) while it walks down the image.
// Forward: sums per group and part of the image, their join, then the
// normalised rows.  Backward the same with sums per channel.  Joins add the
// parts in a fixed order: the same inputs give the same bits.
#include "mixrt_refine.hpp"

#include <type_traits>

namespace mixrt {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kJoinBlocks = 1 << 16;   // most blocks of a join, 4 waves each

struct NormPlan {
    int V;          // channels of a vector
    int lanes;      // vectors of a row in one slab (threads across a row)
    int slabs;      // slabs of a row
    int R;          // rows of one step of a block
    int S;          // parts an image is split into
    int64_t part;   // rows of a part
};

// pad: a row takes whole kept groups of lanes, so that the lanes of a group
// are aligned neighbours.
NormPlan norm_plan(int N, int64_t P, int C, int dtype, bool pad)
{
    NormPlan p;
    p.V = dtype == kF32 ? 4 : 8;
    while (C % p.V) p.V >>= 1;
    const int vecs = pad ? kept_groups(C) * (kKeptGroup / p.V) : C / p.V;
    p.lanes = vecs < kThreads ? vecs : kThreads;
    p.slabs = (vecs + p.lanes - 1) / p.lanes;
    p.R = kThreads / p.lanes;
    const int64_t most = (P + (int64_t)p.R * 4 - 1) / ((int64_t)p.R * 4);
    int64_t S = 2048 / ((int64_t)N * p.slabs > 0 ? (int64_t)N * p.slabs : 1);
    if (S > most) S = most;
    if (S < 1) S = 1;
    p.part = (P + S - 1) / S;
    p.part = (p.part + p.R - 1) / p.R * p.R;
    if (p.part < 1) p.part = 1;
    p.S = P > 0 ? (int)((P + p.part - 1) / p.part) : 1;
    return p;
}

struct NormK {
    int N, C, G, Cg;
    int64_t P;
    int lanes, slabs, R, S;
    int64_t part;
    float eps;
    const float *gamma, *beta;
    MapK x, y, dy, dx;
    float *stats;       // never null here: the caller's or the workspace's
    int8_t *codes;
    uint8_t *exps;
    float *dgamma, *dbeta;
    void *sums;         // forward: double2 [N][S * slabs][G]; backward: float2 [N][S][C]
    float *means;       // backward: float2 [N][G]: the group means of gamma dz and gamma dz xh
};

template <int ACT>
__device__ __forceinline__ float act(float z)
{
    if (ACT == kActRelu) return z > 0.0f ? z : (z <= 0.0f ? 0.0f : z);   // keeps a NaN
    if (ACT == kActSilu) return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    if (ACT == kActGelu) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    return z;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float z)
{
    if (ACT == kActRelu) return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
    if (ACT == kActSilu) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    if (ACT == kActGelu)
        return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) +
               z * __expf(-0.5f * z * z) * 0.39894228040143268f;
    return 1.0f;
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

// Sums of x and x^2 per group over one part of an image, in 64 bits: the
// difference of squares then keeps 32-bit accuracy for |mean| up to 2^14
// deviations.  ONE: a vector lies in one group.  KEEP: x is also written in
// its 8-bit form.
template <typename T, int V, bool ONE, bool KEEP>
__global__ __launch_bounds__(kThreads) void norm_sums_kernel(NormK k)
{
    constexpr int A = ONE ? 1 : V;   // accumulator pairs of a thread
    __shared__ double sh[2 * A][kThreads];
    const int t = threadIdx.x, slab = blockIdx.y, n = blockIdx.z;
    const int r = t / k.lanes, j = t - r * k.lanes;
    const int vec = slab * k.lanes + j, c0 = vec * V;
    const bool in = r < k.R && c0 < k.C;
    double s[A], q[A];
#pragma unroll
    for (int a = 0; a < A; ++a) s[a] = q[a] = 0.0;
    if (r < k.R) {
        const T *x = (const T *)k.x.data + n * k.x.image + c0;
        const int64_t p1 = min(((int64_t)blockIdx.x + 1) * k.part, k.P);
        for (int64_t p = (int64_t)blockIdx.x * k.part + r; p < p1; p += k.R) {
            float f[V];
            if (in)
                load_vec<T, V>(x + p * k.x.pixel, f);
            else
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const double d = (double)f[i];
                s[ONE ? 0 : i] += d;
                q[ONE ? 0 : i] += d * d;
            }
            if (KEEP) {
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
#pragma unroll
                for (int d = 1; d < kKeptGroup / V; d <<= 1)
                    top = max(top, (uint32_t)__shfl_xor((int)top, d));
                const uint32_t byte = kept_byte<T>(top);
                const int64_t row = (int64_t)n * k.P + p;
                if (in) {
                    Pack<int8_t, V> out;
#pragma unroll
                    for (int i = 0; i < V; ++i) out.v[i] = (int8_t)kept_code<T>(f[i], byte);
                    *(Pack<int8_t, V> *)(k.codes + row * k.C + c0) = out;
                    if (c0 % kKeptGroup == 0)
                        k.exps[row * kept_groups(k.C) + c0 / kKeptGroup] = (uint8_t)byte;
                }
            }
        }
    }
#pragma unroll
    for (int a = 0; a < A; ++a) {
        sh[a][t] = s[a];
        sh[A + a][t] = q[a];
    }
    join_rows<2 * A>(sh, k.lanes, k.R, j, r);
    double2 *out = (double2 *)k.sums +
                   ((int64_t)n * gridDim.x * k.slabs + blockIdx.x * k.slabs + slab) * k.G;
    for (int g = t; g < k.G; g += kThreads) {
        // this slab's accumulators of group g
        int lo = g * k.Cg - slab * k.lanes * V, hi = lo + k.Cg;
        lo = max(lo, 0);
        hi = min(hi, k.lanes * V);
        double2 v = make_double2(0.0, 0.0);
        for (int c = lo; c < hi; c += ONE ? V : 1) {
            v.x += sh[ONE ? 0 : c % V][c / V];
            v.y += sh[A + (ONE ? 0 : c % V)][c / V];
        }
        out[g] = v;
    }
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// Joins the parts of every (image, group): one wave each.
__global__ __launch_bounds__(kThreads) void norm_stats_kernel(NormK k)
{
    const int lane = threadIdx.x & 63;
    for (int64_t w = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
         w < (int64_t)k.N * k.G; w += (int64_t)gridDim.x * (kThreads / 64)) {
    const int n = (int)(w / k.G), g = (int)(w - (int64_t)n * k.G);
    const int parts = k.S * k.slabs;
    const double2 *v = (const double2 *)k.sums + (int64_t)n * parts * k.G + g;
    double s = 0.0, q = 0.0;
    for (int i = lane; i < parts; i += 64) {
        const double2 d = v[(int64_t)i * k.G];
        s += d.x;
        q += d.y;
    }
    s = wave_sum(s);
    q = wave_sum(q);
    if (lane == 0) {
        const double m = (double)k.P * k.Cg, mean = k.P > 0 ? s / m : 0.0;
        double var = k.P > 0 ? q / m - mean * mean : 0.0;
        if (var < 0.0) var = 0.0;   // a NaN stays
        k.stats[2 * w] = (float)mean;
        k.stats[2 * w + 1] = (float)(1.0 / sqrt(var + (double)k.eps));
    }
    }
}

// The normalised and activated rows.
template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormK k)
{
    const int t = threadIdx.x, n = blockIdx.z;
    const int r = t / k.lanes, j = t - r * k.lanes;
    const int c0 = (blockIdx.y * k.lanes + j) * V;
    if (r >= k.R || c0 >= k.C) return;
    float mean[V], rstd[V], ga[V], be[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float *st = k.stats + 2 * ((int64_t)n * k.G + (c0 + i) / k.Cg);
        mean[i] = st[0];
        rstd[i] = st[1];
        ga[i] = k.gamma ? k.gamma[c0 + i] : 1.0f;
        be[i] = k.beta ? k.beta[c0 + i] : 0.0f;
    }
    const T *x = (const T *)k.x.data + n * k.x.image + c0;
    T *y = (T *)k.y.data + n * k.y.image + c0;
    const int64_t p1 = min(((int64_t)blockIdx.x + 1) * k.part, k.P);
    for (int64_t p = (int64_t)blockIdx.x * k.part + r; p < p1; p += k.R) {
        float f[V];
        load_vec<T, V>(x + p * k.x.pixel, f);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = act<ACT>((f[i] - mean[i]) * rstd[i] * ga[i] + be[i]);
        store_vec<T, V>(y + p * k.y.pixel, f);
    }
}

// A vector of the backward's x: read as it is, or from its 8-bit form.
template <typename T, int V, bool KEPT>
__device__ __forceinline__ void load_saved(const NormK &k, int n, int64_t p, int c0, float (&f)[V])
{
    if (KEPT) {
        const int64_t row = (int64_t)n * k.P + p;
        const Pack<int8_t, V> q = *(const Pack<int8_t, V> *)(k.codes + row * k.C + c0);
        const float s = kept_scale(k.exps[row * kept_groups(k.C) + c0 / kKeptGroup]);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = (float)q.v[i] * s;
    } else {
        load_vec<T, V>((const T *)k.x.data + n * k.x.image + p * k.x.pixel + c0, f);
    }
}

// Sums of dz and dz xh per channel over one part of an image.
template <typename T, int V, int ACT, bool KEPT>
__global__ __launch_bounds__(kThreads) void norm_back_sums_kernel(NormK k)
{
    __shared__ float sh[2 * V][kThreads];
    const int t = threadIdx.x, n = blockIdx.z;
    const int r = t / k.lanes, j = t - r * k.lanes;
    const int c0 = (blockIdx.y * k.lanes + j) * V;
    float a[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = b[i] = 0.0f;
    if (r < k.R && c0 < k.C) {
        float mean[V], rstd[V], ga[V], be[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float *st = k.stats + 2 * ((int64_t)n * k.G + (c0 + i) / k.Cg);
            mean[i] = st[0];
            rstd[i] = st[1];
            ga[i] = k.gamma ? k.gamma[c0 + i] : 1.0f;
            be[i] = k.beta ? k.beta[c0 + i] : 0.0f;
        }
        const T *dy = (const T *)k.dy.data + n * k.dy.image + c0;
        const int64_t p1 = min(((int64_t)blockIdx.x + 1) * k.part, k.P);
        for (int64_t p = (int64_t)blockIdx.x * k.part + r; p < p1; p += k.R) {
            float f[V], d[V];
            load_saved<T, V, KEPT>(k, n, p, c0, f);
            load_vec<T, V>(dy + p * k.dy.pixel, d);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (f[i] - mean[i]) * rstd[i];
                const float dz = d[i] * act_slope<ACT>(xh * ga[i] + be[i]);
                a[i] += dz;
                b[i] += dz * xh;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        sh[i][t] = a[i];
        sh[V + i][t] = b[i];
    }
    join_rows<2 * V>(sh, k.lanes, k.R, j, r);
    float2 *out = (float2 *)k.sums + ((int64_t)n * gridDim.x + blockIdx.x) * k.C;
    if (r == 0 && c0 < k.C)
#pragma unroll
        for (int i = 0; i < V; ++i) out[c0 + i] = make_float2(sh[i][t], sh[V + i][t]);
}

// Joins the backward's parts: one wave for every (image, group)'s means, then
// one for every channel's gradients.
__global__ __launch_bounds__(kThreads) void norm_back_join_kernel(NormK k)
{
    const int64_t ng = (int64_t)k.N * k.G;
    const int lane = threadIdx.x & 63;
    const float2 *v = (const float2 *)k.sums;
    for (int64_t w = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64; w < ng + k.C;
         w += (int64_t)gridDim.x * (kThreads / 64)) {
    double a = 0.0, b = 0.0;
    if (w < ng) {
        const int n = (int)(w / k.G), g = (int)(w - (int64_t)n * k.G);
        const int64_t count = (int64_t)k.S * k.Cg;
        for (int64_t i = lane; i < count; i += 64) {
            const int64_t s = i / k.Cg;
            const int c = g * k.Cg + (int)(i - s * k.Cg);
            const float2 d = v[((int64_t)n * k.S + s) * k.C + c];
            const double ga = k.gamma ? (double)k.gamma[c] : 1.0;
            a += ga * (double)d.x;
            b += ga * (double)d.y;
        }
        a = wave_sum(a);
        b = wave_sum(b);
        const double m = (double)k.P * k.Cg;
        if (lane == 0) {
            k.means[2 * w] = (float)(k.P > 0 ? a / m : 0.0);
            k.means[2 * w + 1] = (float)(k.P > 0 ? b / m : 0.0);
        }
    } else {
        const int c = (int)(w - ng);
        const int64_t count = (int64_t)k.N * k.S;
        for (int64_t i = lane; i < count; i += 64) {
            const float2 d = v[i * k.C + c];
            a += (double)d.x;
            b += (double)d.y;
        }
        a = wave_sum(a);
        b = wave_sum(b);
        if (lane == 0) {
            if (k.dbeta) k.dbeta[c] = (float)a;
            if (k.dgamma) k.dgamma[c] = (float)b;
        }
    }
    }
}

template <typename T, int V, int ACT, bool KEPT>
__global__ __launch_bounds__(kThreads) void norm_back_apply_kernel(NormK k)
{
    const int t = threadIdx.x, n = blockIdx.z;
    const int r = t / k.lanes, j = t - r * k.lanes;
    const int c0 = (blockIdx.y * k.lanes + j) * V;
    if (r >= k.R || c0 >= k.C) return;
    float mean[V], rstd[V], ga[V], be[V], ma[V], mb[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int64_t g = (int64_t)n * k.G + (c0 + i) / k.Cg;
        mean[i] = k.stats[2 * g];
        rstd[i] = k.stats[2 * g + 1];
        ma[i] = k.means[2 * g];
        mb[i] = k.means[2 * g + 1];
        ga[i] = k.gamma ? k.gamma[c0 + i] : 1.0f;
        be[i] = k.beta ? k.beta[c0 + i] : 0.0f;
    }
    const T *dy = (const T *)k.dy.data + n * k.dy.image + c0;
    T *dx = (T *)k.dx.data + n * k.dx.image + c0;
    const int64_t p1 = min(((int64_t)blockIdx.x + 1) * k.part, k.P);
    for (int64_t p = (int64_t)blockIdx.x * k.part + r; p < p1; p += k.R) {
        float f[V], d[V];
        load_saved<T, V, KEPT>(k, n, p, c0, f);
        load_vec<T, V>(dy + p * k.dy.pixel, d);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float xh = (f[i] - mean[i]) * rstd[i];
            const float dz = d[i] * act_slope<ACT>(xh * ga[i] + be[i]);
            f[i] = rstd[i] * (ga[i] * dz - ma[i] - xh * mb[i]);
        }
        store_vec<T, V>(dx + p * k.dx.pixel, f);
    }
}

NormK norm_args(const NormLaunch &L, const NormPlan &p)
{
    NormK k;
    k.N = L.N;
    k.C = L.C;
    k.G = L.G;
    k.Cg = L.C / L.G;
    k.P = L.P;
    k.lanes = p.lanes;
    k.slabs = p.slabs;
    k.R = p.R;
    k.S = p.S;
    k.part = p.part;
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
    k.sums = nullptr;
    k.means = nullptr;
    return k;
}

unsigned join_blocks(int64_t waves)
{
    const int64_t b = (waves + kThreads / 64 - 1) / (kThreads / 64);
    return (unsigned)(b < kJoinBlocks ? b : kJoinBlocks);
}

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

// Workspace: group values (float2 [N][G]), then the parts' sums.
size_t small_bytes(int N, int G) { return up16((size_t)N * G * 8); }

template <typename T, int V>
void forward_sums(const NormK &k, dim3 grid, hipStream_t s)
{
    const bool one = k.Cg % V == 0, keep = k.codes != nullptr;
    if (one && keep)
        norm_sums_kernel<T, V, true, true><<<grid, kThreads, 0, s>>>(k);
    else if (one)
        norm_sums_kernel<T, V, true, false><<<grid, kThreads, 0, s>>>(k);
    else if (keep)
        norm_sums_kernel<T, V, false, true><<<grid, kThreads, 0, s>>>(k);
    else
        norm_sums_kernel<T, V, false, false><<<grid, kThreads, 0, s>>>(k);
}

template <typename T, int V>
void forward_apply(const NormK &k, int act, dim3 grid, hipStream_t s)
{
    switch (act) {
    case kActNone: norm_apply_kernel<T, V, kActNone><<<grid, kThreads, 0, s>>>(k); break;
    case kActRelu: norm_apply_kernel<T, V, kActRelu><<<grid, kThreads, 0, s>>>(k); break;
    case kActSilu: norm_apply_kernel<T, V, kActSilu><<<grid, kThreads, 0, s>>>(k); break;
    default: norm_apply_kernel<T, V, kActGelu><<<grid, kThreads, 0, s>>>(k); break;
    }
}

template <typename T, int V, int ACT>
void backward_part(const NormK &k, bool sums, dim3 grid, hipStream_t s)
{
    if (k.codes) {
        if (sums)
            norm_back_sums_kernel<T, V, ACT, true><<<grid, kThreads, 0, s>>>(k);
        else
            norm_back_apply_kernel<T, V, ACT, true><<<grid, kThreads, 0, s>>>(k);
    } else {
        if (sums)
            norm_back_sums_kernel<T, V, ACT, false><<<grid, kThreads, 0, s>>>(k);
        else
            norm_back_apply_kernel<T, V, ACT, false><<<grid, kThreads, 0, s>>>(k);
    }
}

template <typename T, int V>
void backward_part(const NormK &k, int act, bool sums, dim3 grid, hipStream_t s)
{
    switch (act) {
    case kActNone: backward_part<T, V, kActNone>(k, sums, grid, s); break;
    case kActRelu: backward_part<T, V, kActRelu>(k, sums, grid, s); break;
    case kActSilu: backward_part<T, V, kActSilu>(k, sums, grid, s); break;
    default: backward_part<T, V, kActGelu>(k, sums, grid, s); break;
    }
}

// f(T(), std::integral_constant<V>) for the element type and vector width.
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

}  // namespace

size_t norm_workspace(int N, int64_t P, int C, int G, int dtype)
{
    size_t most = 0;
    for (int pad = 0; pad < 2; ++pad) {
        const NormPlan p = norm_plan(N, P, C, dtype, pad != 0);
        const size_t fwd = (size_t)N * p.S * p.slabs * G * sizeof(double2);
        const size_t bwd = (size_t)N * p.S * C * sizeof(float2);
        if (fwd > most) most = fwd;
        if (bwd > most) most = bwd;
    }
    return small_bytes(N, G) + up16(most);
}

hipError_t launch_norm_forward(const NormLaunch &L, hipStream_t stream)
{
    if (L.N == 0) return hipSuccess;
    const NormPlan ps = norm_plan(L.N, L.P, L.C, L.dtype, L.codes != nullptr);
    const NormPlan pa = norm_plan(L.N, L.P, L.C, L.dtype, false);
    NormK k = norm_args(L, ps);
    if (!k.stats) k.stats = (float *)L.ws;
    k.sums = (char *)L.ws + small_bytes(L.N, L.G);
    with_type(L.dtype, ps.V, [&](auto *t, auto v) {
        forward_sums<std::remove_pointer_t<decltype(t)>, decltype(v)::value>(
            k, dim3(ps.S, ps.slabs, L.N), stream);
    });
    const int64_t waves = (int64_t)L.N * L.G;
    norm_stats_kernel<<<join_blocks(waves), kThreads, 0, stream>>>(k);
    if (L.P > 0) {
        k.lanes = pa.lanes;
        k.slabs = pa.slabs;
        k.R = pa.R;
        k.S = pa.S;
        k.part = pa.part;
        with_type(L.dtype, pa.V, [&](auto *t, auto v) {
            forward_apply<std::remove_pointer_t<decltype(t)>, decltype(v)::value>(
                k, L.act, dim3(pa.S, pa.slabs, L.N), stream);
        });
    }
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormLaunch &L, hipStream_t stream)
{
    const NormPlan p = norm_plan(L.N, L.P, L.C, L.dtype, false);
    NormK k = norm_args(L, p);
    k.means = (float *)L.ws;
    k.sums = (char *)L.ws + small_bytes(L.N, L.G);
    auto part = [&](bool sums) {
        with_type(L.dtype, p.V, [&](auto *t, auto v) {
            backward_part<std::remove_pointer_t<decltype(t)>, decltype(v)::value>(
                k, L.act, sums, dim3(p.S, p.slabs, L.N), stream);
        });
    };
    if (L.N > 0) part(true);
    const int64_t waves = (int64_t)L.N * L.G + L.C;
    norm_back_join_kernel<<<join_blocks(waves), kThreads, 0, stream>>>(k);
    if (L.N > 0 && L.P > 0 && L.dx.data) part(false);
    return hipGetLastError();
}

}  // namespace mixrt
