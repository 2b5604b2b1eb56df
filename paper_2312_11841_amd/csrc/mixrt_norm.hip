// Group norm, forward (see mixrt_norm.hpp).
#include "mixrt_norm.hpp"

namespace mixrt {
namespace {

// Adds a row's vector to sums of x and x^2, in 64 bits: the difference of
// squares then keeps 32-bit accuracy for a mean up to 2^14 deviations away.
// Each of the A sums takes V / A channels, which lie in one group.
template <typename T, int V, int A>
__device__ __forceinline__ void add_squares(const Pack<T, V> &x, double (&s)[A], double (&q)[A])
{
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const double d = (double)(float)x.v[i];
        s[i / (V / A)] += d;
        q[i / (V / A)] = fma(d, d, q[i / (V / A)]);
    }
}

// Writes a vector's 8-bit form.  The 32 / V lanes of its kept group are
// neighbours and all here; in: the vector exists (else it counts as 0).
template <typename T, int V>
__device__ __forceinline__ void keep_row(const NormK &k, int64_t row, int c0, bool in,
                                         const Pack<T, V> &x)
{
    float f[V];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        f[i] = (float)x.v[i];
        top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
    }
    if (!in) top = 0;
#pragma unroll
    for (int d = 1; d < kKeptGroup / V; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    const uint32_t byte = kept_byte<T>(top);
    if (!in) return;
    *(Pack<int8_t, V> *)(k.codes + row * k.C + c0) = kept_codes<T, V>(f, byte);
    if (c0 % kKeptGroup == 0)
        k.exps[row * kept_groups(k.C) + c0 / kKeptGroup] = (uint8_t)byte;
}

template <typename T, int V, int ACT>
__device__ __forceinline__ void write_row(T *y, const Channels<V> &c, const Pack<T, V> &x)
{
    float f[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
        f[i] = act<ACT>(fmaf((float)x.v[i] - c.mean[i], c.scale[i], c.be[i]));
    store_vec<T, V>(y, f);
}

// Sums per group over one part of an image.  Bound by the stream of x: 8 x 1080p
// x 16 channels in f16, 531 MB in 123 us (4.3 TB/s); with 512 to 4096 blocks the
// call differs by 1%, and with two or eight rows ahead by 1 and 5%.  A: sums of x (and of x^2) that a
// thread holds.  KEEP: x is also written in its 8-bit form.
template <typename T, int V, int A, bool KEEP>
__global__ __launch_bounds__(kThreads) void norm_sums_kernel(NormK k)
{
    constexpr int W = V / A;   // channels of a sum
    __shared__ double sh[2 * A][kThreads];
    const int t = threadIdx.x, slab = blockIdx.y, n = blockIdx.z;
    const int r = t / k.lanes, j = t - r * k.lanes;
    const int c0 = (slab * k.lanes + j) * V;
    const bool in = c0 < k.C;
    double s[A], q[A];
#pragma unroll
    for (int a = 0; a < A; ++a) s[a] = q[a] = 0.0;
    if (r < k.R && (in || KEEP)) {
        // lanes of KEEP past the row's end read its start and use nothing of it
        const T *x = (const T *)k.x.data + n * k.x.image + (in ? c0 : 0);
        walk<Pack<T, V>, kAhead>(
            blockIdx.x, gridDim.x, r, k.R, k.P,
            [&](int64_t p) { return *(const Pack<T, V> *)(x + p * k.x.pixel); },
            [&](int64_t p, const Pack<T, V> &v) {
                if (in) add_squares<T, V, A>(v, s, q);
                if (KEEP) keep_row<T, V>(k, (int64_t)n * k.P + p, c0, in, v);
            });
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
        for (int c = lo; c < hi; c += W) {
            v.x += sh[c % V / W][c / V];
            v.y += sh[A + c % V / W][c / V];
        }
        out[g] = v;
    }
}

// Joins the parts of kJoinGroups groups of image n from g0 on, a block's
// threads over the groups and over the parts; out(g, mean and rstd) in one
// thread for each group.
constexpr int kJoinGroups = 8;

template <int THREADS, typename OUT>
__device__ __forceinline__ void join_groups(const NormK &k, int n, int g0, OUT out)
{
    __shared__ double2 sh[THREADS / 64][kJoinGroups];
    const int parts = k.S * k.slabs;
    const int gl = threadIdx.x % kJoinGroups, g = g0 + gl;
    const double2 *v = (const double2 *)k.sums + (int64_t)n * parts * k.G + g;
    double s = 0.0, q = 0.0;
    if (g < k.G)
#pragma unroll 4
        for (int i = threadIdx.x / kJoinGroups; i < parts; i += THREADS / kJoinGroups) {
            const double2 d = v[(int64_t)i * k.G];
            s += d.x;
            q += d.y;
        }
#pragma unroll
    for (int d = kJoinGroups; d < 64; d <<= 1) {
        s += __shfl_xor(s, d);
        q += __shfl_xor(q, d);
    }
    if ((threadIdx.x & 63) < kJoinGroups) sh[threadIdx.x / 64][gl] = make_double2(s, q);
    __syncthreads();
    if (threadIdx.x < kJoinGroups && g < k.G) {
        s = q = 0.0;
        for (int w = 0; w < THREADS / 64; ++w) {
            s += sh[w][gl].x;
            q += sh[w][gl].y;
        }
        out(g, group_stats(k, s, q));
    }
    __syncthreads();
}

__global__ __launch_bounds__(kJoinThreads) void norm_stats_kernel(NormK k)
{
    const int n = blockIdx.y;
    join_groups<kJoinThreads>(k, n, blockIdx.x * kJoinGroups, [&](int g, float2 st) {
        k.stats[2 * ((int64_t)n * k.G + g)] = st.x;
        k.stats[2 * ((int64_t)n * k.G + g) + 1] = st.y;
    });
}

// The normalised and activated rows, a stream of x and y (8 x 1080p x 16 in f16,
// 1062 MB in 166 us, 6.4 TB/s).  FOLD: the block joins the image's few
// parts itself (and the first one stores what it got).
template <typename T, int V, int ACT, bool FOLD>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormK k)
{
    __shared__ float2 folded[FOLD ? kFoldChannels : 1];
    const int t = threadIdx.x, n = blockIdx.z;
    const int r = t / k.lanes, j = t - r * k.lanes;
    const int c0 = (blockIdx.y * k.lanes + j) * V;
    const float *stats = k.stats + 2 * (int64_t)n * k.G;
    if (FOLD) {
        for (int g0 = 0; g0 < k.G; g0 += kJoinGroups)
            join_groups<kThreads>(k, n, g0, [&](int g, float2 st) {
                folded[g] = st;
                if (blockIdx.x == 0 && blockIdx.y == 0) {
                    k.stats[2 * ((int64_t)n * k.G + g)] = st.x;
                    k.stats[2 * ((int64_t)n * k.G + g) + 1] = st.y;
                }
            });
        stats = (const float *)folded;
    }
    if (r >= k.R || c0 >= k.C) return;
    Channels<V> c;
    c.set(k, stats, c0);
    const T *x = (const T *)k.x.data + n * k.x.image + c0;
    T *y = (T *)k.y.data + n * k.y.image + c0;
    walk<Pack<T, V>, kAhead>(
        blockIdx.x, gridDim.x, r, k.R, k.P,
        [&](int64_t p) { return *(const Pack<T, V> *)(x + p * k.x.pixel); },
        [&](int64_t p, const Pack<T, V> &v) { write_row<T, V, ACT>(y + p * k.y.pixel, c, v); });
}

// Small images: a block takes a run of `chunk` channels (whole groups, and
// whole kept groups where x is kept) of one image, lanes over its vectors, R
// rows at a time.  It sums up all rows, then writes (and keeps) every
// gridDim.z-th R rows.  A vector lies in one group.  In place (y is x) a block
// would sum up what another has written: then one block does it all.  Bound by
// the launch and one chain of loads, joins and stores (64 x 64 x 16 in f32, 6.2
// us of kernel; in two launches 9.3 a call against 7.1).
template <typename T, int V, int ACT, bool KEEP>
__global__ __launch_bounds__(kSmallThreads) void norm_small_kernel(NormK k, int chunk)
{
    __shared__ double sh[2][kSmallThreads];
    __shared__ float2 stats[kSmallThreads];
    const int t = threadIdx.x, n = blockIdx.y, base = blockIdx.x * chunk;
    const int r = t / k.lanes, j = t - r * k.lanes;
    const int c0 = base + j * V, c_end = min(base + chunk, k.C);
    const bool in = r < k.R && c0 < c_end;
    const T *x = (const T *)k.x.data + n * k.x.image + (in ? c0 : 0);
    const auto load = [&](int64_t p) { return *(const Pack<T, V> *)(x + p * k.x.pixel); };
    double s[1] = {0.0}, q[1] = {0.0};
    if (in)
        walk<Pack<T, V>, kAhead>(0, 1, r, k.R, k.P, load, [&](int64_t, const Pack<T, V> &v) {
            add_squares<T, V, 1>(v, s, q);
        });
    sh[0][t] = s[0];
    sh[1][t] = q[0];
    __syncthreads();
    // a wave for each group: its lanes' accumulators over the R rows
    const int per = k.Cg / V, first = base / k.Cg, groups = (c_end - base) / k.Cg;
    for (int g = t / 64; g < groups; g += kSmallThreads / 64) {
        double a = 0.0, b = 0.0;
        for (int i = t & 63; i < per * k.R; i += 64) {
            const int row = i / per, at = row * k.lanes + g * per + (i - row * per);
            a += sh[0][at];
            b += sh[1][at];
        }
        a = wave_sum(a);
        b = wave_sum(b);
        if ((t & 63) == 0) {
            const float2 st = group_stats(k, a, b);
            stats[g] = st;
            if (blockIdx.z == 0) {
                k.stats[2 * ((int64_t)n * k.G + first + g)] = st.x;
                k.stats[2 * ((int64_t)n * k.G + first + g) + 1] = st.y;
            }
        }
    }
    __syncthreads();
    if (!in && !(KEEP && r < k.R)) return;
    Channels<V> c;
    if (in) c.set(k, (const float *)(stats - first), c0);
    T *y = (T *)k.y.data + n * k.y.image + (in ? c0 : 0);
    walk<Pack<T, V>, 1>(blockIdx.z, gridDim.z, r, k.R, k.P, load,
                        [&](int64_t p, const Pack<T, V> &v) {
                            if (KEEP) keep_row<T, V>(k, (int64_t)n * k.P + p, c0, in, v);
                            if (in) write_row<T, V, ACT>(y + p * k.y.pixel, c, v);
                        });
}

// The sums with as few accumulators as the groups allow: one where a vector
// lies in a group, one a group where whole groups lie in a vector.
template <typename T, int V, int A>
void forward_sums(const NormK &k, dim3 grid, hipStream_t s)
{
    if constexpr (A < V)
        if (k.Cg % (V / A) != 0) return forward_sums<T, V, 2 * A>(k, grid, s);
    if (k.codes)
        norm_sums_kernel<T, V, A, true><<<grid, kThreads, 0, s>>>(k);
    else
        norm_sums_kernel<T, V, A, false><<<grid, kThreads, 0, s>>>(k);
}

}  // namespace

size_t norm_workspace(int N, int64_t P, int C, int G, int dtype)
{
    size_t most = 0;
    for (int i = 0; i < 3; ++i) {   // forward, forward with x kept, backward
        const NormPlan p = norm_plan(N, P, C, G, dtype, i == 1, i == 2);
        const size_t n = i == 2 ? (size_t)N * p.S * C * sizeof(float2)
                         : p.way == NormPlan::kSmall
                             ? 0
                             : (size_t)N * p.S * p.slabs * G * sizeof(double2);
        if (n > most) most = n;
    }
    return group_bytes(N, G) + channel_bytes(N, C) + up16(most);
}

hipError_t launch_norm_forward(const NormLaunch &L, hipStream_t stream)
{
    if (L.N == 0) return hipSuccess;
    const bool keep = L.codes != nullptr;
    const NormPlan p = norm_plan(L.N, L.P, L.C, L.G, L.dtype, keep, false);
    NormK k = norm_args(L, p);
    if (!k.stats) k.stats = (float *)L.ws;
    k.sums = (char *)L.ws + group_bytes(L.N, L.G) + channel_bytes(L.N, L.C);
    if (p.way == NormPlan::kSmall) {
        const dim3 grid((L.C + p.chunk - 1) / p.chunk, L.N, L.x.data == L.y.data ? 1 : p.share);
        with_type(L.dtype, p.V, [&](auto *t, auto v) {
            typedef std::remove_pointer_t<decltype(t)> T;
            constexpr int V = decltype(v)::value;
            with_act(L.act, [&](auto a) {
                constexpr int ACT = decltype(a)::value;
                if (keep)
                    norm_small_kernel<T, V, ACT, true>
                        <<<grid, kSmallThreads, 0, stream>>>(k, p.chunk);
                else
                    norm_small_kernel<T, V, ACT, false>
                        <<<grid, kSmallThreads, 0, stream>>>(k, p.chunk);
            });
        });
        return hipGetLastError();
    }
    with_type(L.dtype, p.V, [&](auto *t, auto v) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int V = decltype(v)::value;
        forward_sums<T, V, 1>(k, dim3(p.S, p.slabs, L.N), stream);
    });
    if (p.way == NormPlan::kLarge)
        norm_stats_kernel<<<dim3((L.G + kJoinGroups - 1) / kJoinGroups, L.N), kJoinThreads, 0,
                            stream>>>(k);
    const dim3 grid(p.share, p.slabs, L.N);
    with_type(L.dtype, p.V, [&](auto *t, auto v) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int V = decltype(v)::value;
        with_act(L.act, [&](auto a) {
            constexpr int ACT = decltype(a)::value;
            if (p.way == NormPlan::kFold)
                norm_apply_kernel<T, V, ACT, true><<<grid, kThreads, 0, stream>>>(k);
            else
                norm_apply_kernel<T, V, ACT, false><<<grid, kThreads, 0, stream>>>(k);
        });
    });
    return hipGetLastError();
}

}  // namespace mixrt
