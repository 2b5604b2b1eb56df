// Group norm, backward (see mixrt_norm.hpp).
#include "mixrt_norm.hpp"

namespace mixrt {
namespace {

// A row's vector of the backward: dy, and x as it is or in its 8-bit form.
template <typename T, int V, bool KEPT>
struct BackRow {
    typedef std::conditional_t<KEPT, int8_t, T> X;
    Pack<X, V> x;
    Pack<T, V> dy;
    uint8_t byte;
    // x - mean
    __device__ __forceinline__ float centred(int i, float scale, float mean) const
    {
        return KEPT ? fmaf((float)x.v[i], scale, -mean) : (float)x.v[i] - mean;
    }
};

template <typename T, int V, bool KEPT>
__device__ __forceinline__ BackRow<T, V, KEPT> load_back(const NormK &k, int n, int64_t p, int c0)
{
    BackRow<T, V, KEPT> d;
    typedef Pack<typename BackRow<T, V, KEPT>::X, V> PX;
    if (KEPT) {
        const int64_t row = (int64_t)n * k.P + p;
        d.x = *(const PX *)(k.codes + row * k.C + c0);
        d.byte = k.exps[row * kept_groups(k.C) + c0 / kKeptGroup];
    } else {
        d.x = *(const PX *)((const T *)k.x.data + n * k.x.image + p * k.x.pixel + c0);
        d.byte = 0;
    }
    d.dy = *(const Pack<T, V> *)((const T *)k.dy.data + n * k.dy.image + p * k.dy.pixel + c0);
    return d;
}

// Whether a deviation of the wave's groups lies beyond 2^40 either way.  Products
// of x - mean with dz, and rstd^2, could then leave the range of 32 bits where
// neither x nor the results do, so that (x - mean) rstd is formed first: a step an
// element, which costs up to 5%.
template <int V>
__device__ __forceinline__ bool far_deviation(const float (&rstd)[V])
{
    bool far = false;
#pragma unroll
    for (int i = 0; i < V; ++i) far |= rstd[i] > 0x1p40f || rstd[i] < 0x1p-40f;
    return __builtin_amdgcn_ballot_w64(far) != 0;
}

// Sums of dz and dz xh per channel over one part of an image: in 32 bits within
// a thread, whose rows are kBackRows at most, and in up to 8 steps over a block's
// rows; in 64 bits where the parts are joined.  Bound by the vector memory path
// (8 x 360p x 64 channels in bf16, silu: 361 MB in 97 us, 3.7 TB/s; data return
// busy 82% of the time, ALUs 53%, waves waiting for loads 74% of theirs).
template <typename T, int V, int ACT, bool KEPT>
__global__ __launch_bounds__(kThreads) void norm_back_sums_kernel(NormK k)
{
    __shared__ float sh[2 * V][kThreads];
    const int t = threadIdx.x, n = blockIdx.z;
    const int r = t / k.lanes, j = t - r * k.lanes;
    const int c0 = (blockIdx.y * k.lanes + j) * V;
    float a[V], b[V];   // of dz and of dz (x - mean)
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = b[i] = 0.0f;
    if (r < k.R && c0 < k.C) {
        Channels<V> c;
        c.set(k, k.stats + 2 * (int64_t)n * k.G, c0);
        const auto sum = [&](auto first) {
            walk<BackRow<T, V, KEPT>, 1>(
                blockIdx.x, gridDim.x, r, k.R, k.P,
                [&](int64_t p) { return load_back<T, V, KEPT>(k, n, p, c0); },
                [&](int64_t, const BackRow<T, V, KEPT> &d) {
                    const float ks = kept_scale(d.byte);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float u = d.centred(i, ks, c.mean[i]);
                        const float dz = (float)d.dy.v[i] *
                                         act_slope<ACT>(fmaf(u, c.scale[i], c.be[i]));
                        a[i] += dz;
                        b[i] = fmaf(dz, decltype(first)::value ? u * c.rstd[i] : u, b[i]);
                    }
                });
        };
        if (far_deviation<V>(c.rstd)) {
            sum(std::true_type());
        } else {
            sum(std::false_type());
#pragma unroll
            for (int i = 0; i < V; ++i) b[i] *= c.rstd[i];
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

// Joins an image's parts: every channel's sums, from them its groups' means.
// A block takes `groups` whole groups; its threads lie over kAcross channels
// at a time and over the parts.
template <int kAcross>
__global__ __launch_bounds__(kJoinThreads) void norm_back_join_kernel(NormK k, int groups)
{
    constexpr int kDown = kJoinThreads / kAcross;
    __shared__ double sh[2][kDown][kAcross + 1];
    const int n = blockIdx.y, g0 = blockIdx.x * groups;
    const int c_end = min((g0 + groups) * k.Cg, k.C);
    const int cl = threadIdx.x % kAcross, down = threadIdx.x / kAcross;
    const float2 *v = (const float2 *)k.sums + (int64_t)n * k.S * k.C;
    for (int cb = g0 * k.Cg; cb < c_end; cb += kAcross) {
        const int c = cb + cl;
        double a = 0.0, b = 0.0;
        if (c < c_end)
#pragma unroll 4
            for (int i = down; i < k.S; i += kDown) {
                const float2 d = v[(int64_t)i * k.C + c];
                a += (double)d.x;
                b += (double)d.y;
            }
        sh[0][down][cl] = a;
        sh[1][down][cl] = b;
        for (int half = kDown / 2; half > 0; half /= 2) {
            __syncthreads();
            if (down < half) {
                sh[0][down][cl] += sh[0][down + half][cl];
                sh[1][down][cl] += sh[1][down + half][cl];
            }
        }
        if (down == 0 && c < c_end) {
            const float2 d = make_float2((float)sh[0][0][cl], (float)sh[1][0][cl]);
            k.channels[(int64_t)n * k.C + c] = d;
            if (k.N == 1) {
                if (k.dbeta) k.dbeta[c] = d.x;
                if (k.dgamma) k.dgamma[c] = d.y;
            }
        }
        __syncthreads();
    }
    // the block's own writes, a wave for each group
    for (int g = g0 + (int)threadIdx.x / 64; g < min(g0 + groups, k.G); g += kJoinThreads / 64) {
        double a = 0.0, b = 0.0;
        for (int i = threadIdx.x & 63; i < k.Cg; i += 64) {
            const int c = g * k.Cg + i;
            const float2 d = k.channels[(int64_t)n * k.C + c];
            const double ga = k.gamma ? (double)k.gamma[c] : 1.0;
            a += ga * (double)d.x;
            b += ga * (double)d.y;
        }
        a = wave_sum(a);
        b = wave_sum(b);
        if ((threadIdx.x & 63) == 0) {
            const double m = (double)k.P * k.Cg;
            float *o = k.means + 2 * ((int64_t)n * k.G + g);
            o[0] = (float)(k.P > 0 ? a / m : 0.0);
            o[1] = (float)(k.P > 0 ? b / m : 0.0);
        }
    }
}

// Up to this many images, dx's first block adds up dgamma and dbeta as well (a
// launch less, 4 us); beyond, and without dx, a kernel of its own.
constexpr int kAffineImages = 64;

// dgamma and dbeta of several images (or of none): a wave for each channel.
__global__ __launch_bounds__(kThreads) void norm_affine_kernel(NormK k)
{
    const int c = blockIdx.x * (kThreads / 64) + threadIdx.x / 64, lane = threadIdx.x & 63;
    if (c >= k.C) return;
    double a = 0.0, b = 0.0;
    for (int n = lane; n < k.N; n += 64) {
        const float2 d = k.channels[(int64_t)n * k.C + c];
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

// dx; the first block also writes dgamma and dbeta, over all images.  FOLD:
// the block joins the image's few parts itself.  Bound by its stream (8 x 360p x
// 64 channels in bf16: 597 MB in 106 us, 5.6 TB/s).
template <typename T, int V, int ACT, bool KEPT, bool FOLD>
__global__ __launch_bounds__(kThreads) void norm_back_apply_kernel(NormK k)
{
    __shared__ double ca[FOLD ? kFoldChannels : 1], cx[FOLD ? kFoldChannels : 1];
    __shared__ float2 folded[FOLD ? kFoldChannels : 1];
    const int t = threadIdx.x, n = blockIdx.z;
    const int r = t / k.lanes, j = t - r * k.lanes;
    const int c0 = (blockIdx.y * k.lanes + j) * V;
    const float2 *means = (const float2 *)k.means + (int64_t)n * k.G;
    if (FOLD) {
        // threads over the channels and, where those are few, over the parts
        const float2 *v = (const float2 *)k.sums;
        __shared__ double2 across[kThreads];
        const int width = min(k.C, kThreads), down = kThreads / width;
        const int cl = t % width, dl = t / width;
        const auto add = [&](int c, int image, double2 &s) {
            if (c < k.C && dl < down)
#pragma unroll 8
                for (int i = dl; i < k.S; i += down) {
                    const float2 d = v[((int64_t)image * k.S + i) * k.C + c];
                    s.x += (double)d.x;
                    s.y += (double)d.y;
                }
        };
        const auto join = [&](double2 s) {   // in the first thread of a channel
            across[t] = s;
            __syncthreads();
            s = make_double2(0.0, 0.0);
            if (dl == 0)
                for (int i = 0; i < down; ++i) {
                    s.x += across[i * width + cl].x;
                    s.y += across[i * width + cl].y;
                }
            __syncthreads();
            return s;
        };
        const bool all = n == 0 && blockIdx.x == 0 && blockIdx.y == 0;
        for (int cb = 0; cb < k.C; cb += width) {
            const int c = cb + cl;
            double2 own = make_double2(0.0, 0.0);
            add(c, n, own);
            own = join(own);
            if (dl == 0 && c < k.C) {
                const double ga = k.gamma ? (double)k.gamma[c] : 1.0;
                ca[c] = ga * own.x;
                cx[c] = ga * own.y;
            }
            if (all) {
                double2 rest = make_double2(0.0, 0.0);
                for (int i = 1; i < k.N; ++i) add(c, i, rest);
                rest = join(rest);
                if (dl == 0 && c < k.C) {
                    if (k.dbeta) k.dbeta[c] = (float)(own.x + rest.x);
                    if (k.dgamma) k.dgamma[c] = (float)(own.y + rest.y);
                }
            }
        }
        __syncthreads();
        for (int g = t / 64; g < k.G; g += kThreads / 64) {
            double a = 0.0, b = 0.0;
            for (int i = t & 63; i < k.Cg; i += 64) {
                a += ca[g * k.Cg + i];
                b += cx[g * k.Cg + i];
            }
            a = wave_sum(a);
            b = wave_sum(b);
            const double m = (double)k.P * k.Cg;
            if ((t & 63) == 0)
                folded[g] = make_float2((float)(k.P > 0 ? a / m : 0.0),
                                        (float)(k.P > 0 ? b / m : 0.0));
        }
        __syncthreads();
        means = folded;
    }
    if (!FOLD && k.N > 1 && k.N <= kAffineImages && n == 0 && blockIdx.x == 0 && blockIdx.y == 0)
        for (int c = t; c < k.C; c += kThreads) {
            double a = 0.0, b = 0.0;
#pragma unroll 8
            for (int i = 0; i < k.N; ++i) {
                const float2 d = k.channels[(int64_t)i * k.C + c];
                a += (double)d.x;
                b += (double)d.y;
            }
            if (k.dbeta) k.dbeta[c] = (float)a;
            if (k.dgamma) k.dgamma[c] = (float)b;
        }
    if (r >= k.R || c0 >= k.C || !k.dx.data) return;
    Channels<V> c;
    c.set(k, k.stats + 2 * (int64_t)n * k.G, c0);
    // rstd (gamma dz - a - xh b) = scale dz - (rstd a + (x - mean) rstd^2 b)
    const bool far = far_deviation<V>(c.rstd);
    float ma[V], mb[V];
    for_groups<V>(k, c0, [&](int i, int g) {
        const float2 m = means[g];
        ma[i] = c.rstd[i] * m.x;
        mb[i] = c.rstd[i] * m.y;
        if (!far) mb[i] *= c.rstd[i];
    });
    T *dx = (T *)k.dx.data + n * k.dx.image + c0;
    const auto write = [&](auto first) {
        walk<BackRow<T, V, KEPT>, kAhead>(
            blockIdx.x, gridDim.x, r, k.R, k.P,
            [&](int64_t p) { return load_back<T, V, KEPT>(k, n, p, c0); },
            [&](int64_t p, const BackRow<T, V, KEPT> &d) {
                const float ks = kept_scale(d.byte);
                float f[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float u = d.centred(i, ks, c.mean[i]);
                    const float dz = (float)d.dy.v[i] *
                                     act_slope<ACT>(fmaf(u, c.scale[i], c.be[i]));
                    const float v = decltype(first)::value ? u * c.rstd[i] : u;
                    f[i] = fmaf(c.scale[i], dz, -fmaf(v, mb[i], ma[i]));
                }
                store_vec<T, V>(dx + p * k.dx.pixel, f);
            });
    };
    if (far) write(std::true_type());
    else write(std::false_type());
}

}  // namespace

hipError_t launch_norm_backward(const NormLaunch &L, hipStream_t stream)
{
    const NormPlan p = norm_plan(L.N, L.P, L.C, L.G, L.dtype, false, true);
    NormK k = norm_args(L, p);
    k.means = (float *)L.ws;
    k.channels = (float2 *)((char *)L.ws + group_bytes(L.N, L.G));
    k.sums = (char *)k.channels + channel_bytes(L.N, L.C);
    const bool fold = p.way == NormPlan::kFold;
    if (L.N > 0)
        with_type(L.dtype, p.V, [&](auto *t, auto v) {
            typedef std::remove_pointer_t<decltype(t)> T;
            constexpr int V = decltype(v)::value;
            with_act(L.act, [&](auto a) {
                constexpr int ACT = decltype(a)::value;
                const dim3 sums(p.S, p.slabs, L.N), grid(p.share, p.slabs, L.N);
                if (L.codes)
                    norm_back_sums_kernel<T, V, ACT, true><<<sums, kThreads, 0, stream>>>(k);
                else
                    norm_back_sums_kernel<T, V, ACT, false><<<sums, kThreads, 0, stream>>>(k);
                if (!fold) {
                    // narrow blocks, so that their chains of loads are short;
                    // wide ones where a group has many channels to go through
                    const int groups = k.Cg >= 8 ? 1 : 8 / k.Cg;
                    const dim3 joins((L.G + groups - 1) / groups, L.N);
                    if (k.Cg <= 32)
                        norm_back_join_kernel<8><<<joins, kJoinThreads, 0, stream>>>(k, groups);
                    else
                        norm_back_join_kernel<64><<<joins, kJoinThreads, 0, stream>>>(k, groups);
                    if (!L.dx.data) return;
                }
                if (L.codes && fold)
                    norm_back_apply_kernel<T, V, ACT, true, true>
                        <<<grid, kThreads, 0, stream>>>(k);
                else if (L.codes)
                    norm_back_apply_kernel<T, V, ACT, true, false>
                        <<<grid, kThreads, 0, stream>>>(k);
                else if (fold)
                    norm_back_apply_kernel<T, V, ACT, false, true>
                        <<<grid, kThreads, 0, stream>>>(k);
                else
                    norm_back_apply_kernel<T, V, ACT, false, false>
                        <<<grid, kThreads, 0, stream>>>(k);
            });
        });
    if (L.N == 0 || (!fold && (L.N > kAffineImages || (L.N > 1 && !L.dx.data))))
        if (L.dgamma || L.dbeta)
            norm_affine_kernel<<<(L.C + kThreads / 64 - 1) / (kThreads / 64), kThreads, 0,
                                 stream>>>(k);
    return hipGetLastError();
}

}  // namespace mixrt
