// Heads normed one by one (root mean square over the head's elements, a weight an
// element) and turned by their tokens' rotary positions in the same pass, and the
// gradients of both.
//
// A group of lanes holds a whole head in registers: a lane takes the same items of
// every head (an item is a vector of V pairs, or of 2 V elements past the pairs), so
// the weights and their gradient's sums stay in its registers from head to head.
// The group adds its squares by exchanges between lanes, and each element is read
// once and written once.  Sines and cosines of a block's tokens are worked out once
// in LDS for all heads of both arrays.  Large calls are bound by HBM: 65,280 tokens, 32
// heads of 64 in bf16, 100 us forward (5.4 TB/s); 28,800 of them backward 84 and 5 of
// join (4.2 TB/s; its waves wait 76% of their time).
// A few tokens take one launch's latency (5.7 us).
#include "mixrt_refine.hpp"

#include <type_traits>

namespace mixrt {
namespace {

constexpr int kThreads = 256;
constexpr int kTurns = 2048;     // most (token, pair) turns of a block
constexpr int64_t kMostBlocks = 1 << 20;
constexpr int kParts = 1024;     // blocks of the backward pass, while lanes' sums stay short

struct NormedK {
    int64_t tokens;
    int axes, pairs, n, run;
    int lanes_log2;          // lanes of a head: a power of two
    float eps;
    const float *pos, *freq;
    const uint8_t *axis;
    NormedHeadsK a[2];
    int per[2];              // heads of a block, per array
    float *part;             // backward: [block][array][D], each D padded to dmax
    int dmax;
};

// Where item number at of a head lies: first element, and for pairs the second
// half's; kind 0 pairs, 1 a vector, 2 an element, 3 nothing.
struct Item {
    int kind, one, two, turn;
};

template <int V, bool HALVES>
__device__ __forceinline__ Item item_of(int at, int pairs, int D)
{
    const int pv = pairs / V, rest = D - 2 * pairs, cv = rest / (2 * V), tail = rest - cv * 2 * V;
    Item it = {3, 0, 0, 0};
    if (at < pv) {
        it = HALVES ? Item{0, at * V, pairs + at * V, at * V}
                    : Item{0, 2 * at * V, 2 * at * V + V, at * V};
    } else if (at < pv + cv) {
        it = Item{1, 2 * pairs + (at - pv) * 2 * V, 0, 0};
    } else if (at < pv + cv + tail) {
        it = Item{2, D - tail + (at - pv - cv), 0, 0};
    }
    return it;
}

// Pairs as they lie in memory (x1, x2, x1, x2 ..) to halves (x1 .., x2 ..) or back.
template <int V, bool APART>
__device__ __forceinline__ void swap_order(const Item &it, float (&x)[2 * V])
{
    float y[2 * V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        y[APART ? i : 2 * i] = x[APART ? 2 * i : i];
        y[APART ? V + i : 2 * i + 1] = x[APART ? 2 * i + 1 : V + i];
    }
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) x[i] = it.kind == 0 ? y[i] : x[i];
}

// An item's elements: x[0..V) the first of the pairs, x[V..2V) the second, or 2 V in
// order; zeros where there is none.
template <typename T, int V, bool HALVES>
__device__ __forceinline__ void load_item(const T *p, const Item &it, float (&x)[2 * V])
{
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) x[i] = 0.0f;
    if (HALVES && it.kind == 0) {
        float f[V], g[V];
        load_vec<T, V>(p + it.one, f);
        load_vec<T, V>(p + it.two, g);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x[i] = f[i];
            x[V + i] = g[i];
        }
    } else if (it.kind <= 1) {
        load_vec<T, 2 * V>(p + it.one, x);
    } else if (it.kind == 2) {
        x[0] = (float)p[it.one];
    }
    if (!HALVES) swap_order<V, true>(it, x);
}

template <typename T, int V, bool HALVES>
__device__ __forceinline__ void store_item(T *p, const Item &it, float (&x)[2 * V])
{
    if (!HALVES) swap_order<V, false>(it, x);
    if (HALVES && it.kind == 0) {
        float f[V], g[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            f[i] = x[i];
            g[i] = x[V + i];
        }
        store_vec<T, V>(p + it.one, f);
        store_vec<T, V>(p + it.two, g);
    } else if (it.kind <= 1) {
        store_vec<T, 2 * V>(p + it.one, x);
    } else if (it.kind == 2) {
        p[it.one] = (T)x[0];
    }
}

// (x1, x2) -> (x1 cos - x2 sin, x2 cos + x1 sin), with sign -1 the other way.
template <int V>
__device__ __forceinline__ void turn_item(const Item &it, const float2 *turn, float sign,
                                          float (&x)[2 * V])
{
    if (it.kind != 0) return;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 cs = turn[it.turn + i];
        const float s = sign * cs.y, a = x[i], b = x[V + i];
        x[i] = a * cs.x - b * s;
        x[V + i] = b * cs.x + a * s;
    }
}

// Every lane's value of the lane that a data-parallel move pairs it with.
template <int CONTROL>
__device__ __forceinline__ float moved(float x)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(
        0, (int)__float_as_uint(x), CONTROL, 0xf, 0xf, true));
}

// The same over groups of 2^n lanes, in every lane of them: neighbours, pairs, then
// mirrored halves (which hold equal values by then), then swapped rows.
template <typename Join>
__device__ __forceinline__ float group_join(float x, int n, Join join)
{
    if (n >= 1) x = join(x, moved<0xb1>(x));
    if (n >= 2) x = join(x, moved<0x4e>(x));
    if (n >= 3) x = join(x, moved<0x141>(x));
    if (n >= 4) x = join(x, moved<0x140>(x));
    if (n >= 5) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x),
                                                        false, false);
        x = join(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if (n >= 6) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x),
                                                        false, false);
        x = join(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return x;
}

__device__ __forceinline__ float group_sum(float x, int n)
{
    return group_join(x, n, [](float a, float b) { return a + b; });
}

// 1 / sqrt(mean of squares + eps) of a head in the registers of its group, with
// squares that leave the range of 32 bits kept inside it: then the elements are
// first multiplied by a power of two, pre (1 else), which the caller's x holds too.
// It is about 1 over the larger of the largest element and sqrt(eps), so that neither
// the squares nor eps pre^2 leave the range (elements far below sqrt(eps) do not count
// beside it).
template <int M, int V>
__device__ __forceinline__ float rms(float (&x)[M][2 * V], int lanes_log2, int D, float eps, float &pre)
{
    float ss = 0.0f;
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) ss = fmaf(x[m][i], x[m][i], ss);
    ss = group_sum(ss, lanes_log2);
    pre = 1.0f;
    // (eps carries a head of small elements unless it is itself that small)
    const bool far = !(ss < 0x1p120f) || (ss < 0x1p-80f && eps < 0x1p-80f);
    if (__builtin_amdgcn_ballot_w64(far) != 0) {
        float most = 0.0f;
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) most = fmaxf(most, fabsf(x[m][i]));
        most = group_join(most, lanes_log2, [](float a, float b) { return fmaxf(a, b); });
        if (far) {
            const int e = (int)(__float_as_uint(fmaxf(most, sqrtf(eps))) >> 23);
            pre = __uint_as_float((uint32_t)min(max(254 - e, 1), 253) << 23);
            ss = 0.0f;
        }
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) {
                x[m][i] *= pre;
                if (far) ss = fmaf(x[m][i], x[m][i], ss);
            }
        const float all = group_sum(ss, lanes_log2);
        if (far) ss = all;
    }
    return rsqrtf(ss * (1.0f / (float)D) + eps * pre * pre);
}

// The sines of a run of tokens.
__device__ __forceinline__ void fill_turns(const NormedK &k, int64_t t0, int tokens, float2 *turn)
{
    const uint32_t turns = (uint32_t)(tokens * k.pairs);
    for (uint32_t i = threadIdx.x; i < turns; i += kThreads) {
        const uint32_t t = i / (uint32_t)k.pairs, j = i - t * k.pairs;
        const int a = min((int)k.axis[j], k.axes - 1);
        const float angle = k.pos[(t0 + t) * k.axes + a] * k.freq[j];
        float s, c;
        sincosf(angle, &s, &c);
        turn[i] = make_float2(c, s);
    }
}

template <int V, int M>
__device__ __forceinline__ void load_weights(const float *w, const Item (&it)[M], bool halves,
                                             float (&f)[M][2 * V])
{
#pragma unroll
    for (int m = 0; m < M; ++m) {
        if (!w) {
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) f[m][i] = 1.0f;
        } else if (halves) {
            load_item<float, V, true>(w, it[m], f[m]);
        } else {
            load_item<float, V, false>(w, it[m], f[m]);
        }
    }
}

// Heads of a group whose loads run together: two where they are narrow (the gradients
// of 3600 tokens, 15 heads of 80 in f32: 21.5 us a call, with four 24.5).
template <int V, int M> inline constexpr int kTogether = M > 1 || V == 8 ? 1 : 2;

template <typename T, int V, int M, bool HALVES>
__global__ __launch_bounds__(kThreads) void rotary_norm_kernel(NormedK k)
{
    constexpr int U = kTogether<V, M>;
    __shared__ float2 turn[kTurns];
    const int lanes = 1 << k.lanes_log2;
    const int lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> k.lanes_log2;
    const int groups = kThreads >> k.lanes_log2;
    for (int64_t t0 = (int64_t)blockIdx.x * k.run; t0 < k.tokens;
         t0 += (int64_t)gridDim.x * k.run) {
        const int tokens = (int)min((int64_t)k.run, k.tokens - t0);
        for (int n = 0; n < k.n; ++n) {
            const NormedHeadsK &h = k.a[n];
            const int h0 = blockIdx.y * k.per[n], heads = max(min(k.per[n], h.heads - h0), 0);
            Item it[M];
            float w[M][2 * V];
#pragma unroll
            for (int m = 0; m < M; ++m) it[m] = item_of<V, HALVES>(lane + m * lanes, k.pairs, h.D);
            load_weights<V, M>(h.w, it, HALVES, w);
            const uint32_t rows = (uint32_t)heads * tokens;
            float x[U][M][2 * V];
            uint32_t t[U], hd[U];
            auto load = [&](uint32_t r0) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const uint32_t r = r0 + u * groups + group;
                    t[u] = heads ? r / heads : 0;
                    hd[u] = r - t[u] * heads;
#pragma unroll
                    for (int m = 0; m < M; ++m) {
                        Item some = it[m];
                        if (r >= rows) some.kind = 3;
                        load_item<T, V, HALVES>(
                            (const T *)h.x + (t0 + t[u]) * h.xt + (h0 + hd[u]) * h.xh, some,
                            x[u][m]);
                    }
                }
            };
            load(0);
            if (n == 0) {       // (while the first heads are on their way)
                fill_turns(k, t0, tokens, turn);
                __syncthreads();
            }
            // (every lane of a wave goes through the exchanges)
            for (uint32_t r0 = 0; r0 < rows; r0 += U * groups) {
                if (r0) load(r0);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float pre;
                    const float rs = rms<M, V>(x[u], k.lanes_log2, h.D, k.eps, pre);
                    if (r0 + u * groups + group >= rows) continue;
                    T *o = (T *)h.out + (t0 + t[u]) * h.ot + (h0 + hd[u]) * h.oh;
#pragma unroll
                    for (int m = 0; m < M; ++m) {
#pragma unroll
                        for (int i = 0; i < 2 * V; ++i) x[u][m][i] = x[u][m][i] * rs * w[m][i];
                        turn_item<V>(it[m], turn + t[u] * k.pairs, 1.0f, x[u][m]);
                        store_item<T, V, HALVES>(o, it[m], x[u][m]);
                    }
                }
            }
        }
        __syncthreads();
    }
}

// With u = dy turned back, t = u w and xh = x r: dx = r (t - xh mean(t xh)), and the
// weights' gradient sums u xh.  A lane adds the rows of its items in 32 bits (at most
// about 1024 of them, by the grid's size), the block its groups in order, the join
// the blocks in 64 bits.
template <typename T, int V, int M, bool HALVES>
__global__ __launch_bounds__(kThreads) void rotary_norm_back_kernel(NormedK k)
{
    constexpr int U = kTogether<V, M>;
    __shared__ float2 turn[kTurns];
    __shared__ float sums[kThreads * 2 * V];
    const int lanes = 1 << k.lanes_log2;
    const int lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> k.lanes_log2;
    const int groups = kThreads >> k.lanes_log2;
    float *part = k.part + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * k.dmax;
    int64_t filled = -1;        // the tokens whose sines are in LDS
    for (int n = 0; n < k.n; ++n) {
        const NormedHeadsK &h = k.a[n];
        const int h0 = blockIdx.y * k.per[n], heads = min(k.per[n], h.heads - h0);
        Item it[M];
        float w[M][2 * V], dw[M][2 * V];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            it[m] = item_of<V, HALVES>(lane + m * lanes, k.pairs, h.D);
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) dw[m][i] = 0.0f;
        }
        load_weights<V, M>(h.w, it, HALVES, w);
        for (int64_t t0 = (int64_t)blockIdx.x * k.run; t0 < k.tokens && heads > 0;
             t0 += (int64_t)gridDim.x * k.run) {
            const int tokens = (int)min((int64_t)k.run, k.tokens - t0);
            if (t0 != filled) {
                __syncthreads();
                fill_turns(k, t0, tokens, turn);
                __syncthreads();
                filled = t0;
            }
            const uint32_t rows = (uint32_t)heads * tokens;
            for (uint32_t r0 = 0; r0 < rows; r0 += U * groups) {
                float x[U][M][2 * V], dy[U][M][2 * V];
                uint32_t t[U], hd[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const uint32_t r = r0 + u * groups + group;
                    t[u] = r / heads;
                    hd[u] = r - t[u] * heads;
                    const T *xp = (const T *)h.x + (t0 + t[u]) * h.xt + (h0 + hd[u]) * h.xh;
                    const T *dp = (const T *)h.dy + (t0 + t[u]) * h.dt + (h0 + hd[u]) * h.dh;
#pragma unroll
                    for (int m = 0; m < M; ++m) {
                        Item some = it[m];
                        if (r >= rows) some.kind = 3;
                        load_item<T, V, HALVES>(xp, some, x[u][m]);
                        load_item<T, V, HALVES>(dp, some, dy[u][m]);
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const bool there = r0 + u * groups + group < rows;
                    float pre;
                    const float rs = rms<M, V>(x[u], k.lanes_log2, h.D, k.eps, pre);
                    float along = 0.0f;
#pragma unroll
                    for (int m = 0; m < M; ++m) {
                        if (there) turn_item<V>(it[m], turn + t[u] * k.pairs, -1.0f, dy[u][m]);
#pragma unroll
                        for (int i = 0; i < 2 * V; ++i) {
                            x[u][m][i] *= rs;
                            if (there) dw[m][i] = fmaf(dy[u][m][i], x[u][m][i], dw[m][i]);
                            dy[u][m][i] *= w[m][i];
                            along = fmaf(dy[u][m][i], x[u][m][i], along);
                        }
                    }
                    along = group_sum(along, k.lanes_log2) * (1.0f / (float)h.D);
                    if (!there || !h.out) continue;
                    T *o = (T *)h.out + (t0 + t[u]) * h.ot + (h0 + hd[u]) * h.oh;
#pragma unroll
                    for (int m = 0; m < M; ++m) {
#pragma unroll
                        for (int i = 0; i < 2 * V; ++i)
                            x[u][m][i] = rs * fmaf(-x[u][m][i], along, dy[u][m][i]) * pre;
                        store_item<T, V, HALVES>(o, it[m], x[u][m]);
                    }
                }
            }
        }
        if (!h.dw) continue;
        // the groups' sums, item by item
#pragma unroll
        for (int m = 0; m < M; ++m) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) sums[i * kThreads + threadIdx.x] = dw[m][i];
            __syncthreads();
            for (int at = threadIdx.x; at < lanes * 2 * V; at += kThreads) {
                const int l = at & (lanes - 1), i = at >> k.lanes_log2;
                float s = 0.0f;
                for (int g = 0; g < groups; ++g) s += sums[i * kThreads + g * lanes + l];
                const Item e = item_of<V, HALVES>(l + m * lanes, k.pairs, h.D);
                int d = -1;
                if (e.kind == 0)
                    d = HALVES ? (i < V ? e.one + i : e.two + i - V)
                               : e.one + 2 * (i < V ? i : i - V) + (i < V ? 0 : 1);
                else if (e.kind == 1)
                    d = e.one + i;
                else if (e.kind == 2 && i == 0)
                    d = e.one;
                if (d >= 0) part[n * k.dmax + d] = s;
            }
        }
    }
}

// dw[array][d] = sum over the blocks' parts, in 64 bits: 4 elements a block, 64 threads
// an element (16 elements a block took 13 to 20 us for 1024 parts of 64 elements).
__global__ __launch_bounds__(kThreads) void rotary_norm_join_kernel(NormedK k, int blocks)
{
    __shared__ double sums[kThreads];
    const NormedHeadsK &h = k.a[blockIdx.y];
    const int d = blockIdx.x * 4 + (threadIdx.x & 3), g = threadIdx.x >> 2;
    if (!h.dw) return;
    double a = 0.0;
    if (d < h.D)
#pragma unroll 8
        for (int b = g; b < blocks; b += 64)
            a += k.part[((int64_t)b * 2 + blockIdx.y) * k.dmax + d];
    sums[threadIdx.x] = a;
    for (int n = 32; n > 0; n >>= 1) {
        __syncthreads();
        if (g < n) sums[threadIdx.x] += sums[threadIdx.x + 4 * n];
    }
    if (g == 0 && d < h.D) h.dw[d] = (float)sums[threadIdx.x];
}

// How a call is dealt: vector width, items a lane, lanes a head, tokens a block.
struct NormedPlan {
    int V, M, lanes_log2, run;
    unsigned bx, by;
};

int items_of(int V, int pairs, int D)
{
    const int rest = D - 2 * pairs;
    return pairs / V + rest / (2 * V) + rest % (2 * V);
}

NormedPlan plan_normed(const RotaryNormLaunch &L, bool back)
{
    NormedPlan p{};
    int D = 1, heads = 0;
    int64_t elements = 0;
    for (int i = 0; i < L.n; ++i) {
        D = D > L.a[i].D ? D : L.a[i].D;
        heads = heads > L.a[i].heads ? heads : L.a[i].heads;
        elements += (int64_t)L.a[i].heads * L.a[i].D;
    }
    p.V = L.dtype == kF32 ? 4 : 8;
    if (L.layout) p.V /= 2;
    while (L.pairs % p.V) p.V /= 2;
    // a head wider than a wave's items: several a lane, of fewer elements so that
    // they stay in registers
    auto items = [&](int V) {
        int most = 1;
        for (int i = 0; i < L.n; ++i) {
            const int n = items_of(V, L.pairs, L.a[i].D);
            most = most > n ? most : n;
        }
        return most;
    };
    if (items(p.V) > 64 && p.V > 4) p.V = 4;
    if (items(p.V) > 256) p.V = 1;
    const int most = items(p.V);
    p.M = most <= 64 ? 1 : most <= 256 ? 4 : 8;   // (512 items at most)
    while ((1 << p.lanes_log2) * p.M < most) ++p.lanes_log2;
    const int64_t turns = L.pairs > 0 ? kTurns / L.pairs : 64;
    // tokens of a block: forward about 24 elements a thread; backward all tokens in
    // kParts blocks if their sines fit, since each block's sums are a part to join.
    // Then more, so that the heads divide among the block's groups (65,280 tokens, 16
    // heads of 64 and as many keys, forward: 3 tokens leave a quarter of each pass idle,
    // 122 us, 4 take 106, 8 the same, 12 109; with the first heads fetched beside the
    // sines 4 take 100)
    int64_t run = back ? (L.tokens + kParts - 1) / kParts
                       : elements > 0 ? 24 * kThreads / elements : 1;
    const int groups = kThreads >> p.lanes_log2;
    int64_t step = groups;
    while (heads > 0 && step > 1 && heads * (step / 2) % groups == 0) step /= 2;
    if (step <= 2 * run) run = (run + step - 1) / step * step;
    if (run > turns) run = turns;
    if (run < 1) run = 1;
    p.run = (int)run;
    int64_t bx = (L.tokens + run - 1) / run;
    if (back) {
        // (sums of about 1024 rows a lane at most)
        const int64_t rows = L.tokens * heads;
        int64_t parts = rows / (groups * 1024);
        if (parts < kParts) parts = kParts;
        if (bx > parts) bx = parts;
    }
    if (bx > kMostBlocks) bx = kMostBlocks;
    if (bx < 1) bx = 1;
    int64_t by = 512 / bx;
    if (by > heads) by = heads;
    if (by < 1) by = 1;
    p.bx = (unsigned)bx;
    p.by = (unsigned)by;
    return p;
}

NormedK normed_k(const RotaryNormLaunch &L, const NormedPlan &p)
{
    NormedK k{};
    k.tokens = L.tokens;
    k.axes = L.axes;
    k.pairs = L.pairs;
    k.n = L.n;
    k.run = p.run;
    k.lanes_log2 = p.lanes_log2;
    k.eps = L.eps;
    k.pos = L.pos;
    k.freq = L.freq;
    k.axis = L.axis;
    k.part = L.ws;
    for (int i = 0; i < L.n; ++i) {
        k.a[i] = L.a[i];
        k.per[i] = (L.a[i].heads + (int)p.by - 1) / (int)p.by;
        k.dmax = k.dmax > L.a[i].D ? k.dmax : L.a[i].D;
    }
    return k;
}

template <typename Go>
void by_variant(const RotaryNormLaunch &L, const NormedPlan &p, Go go)
{
    auto layout = [&](auto t, auto v, auto m) {
        if (L.layout)
            go(t, v, m, std::false_type());
        else
            go(t, v, m, std::true_type());
    };
    auto width = [&](auto t) {
        typedef std::integral_constant<int, 1> i1;
        typedef std::integral_constant<int, 2> i2;
        typedef std::integral_constant<int, 4> i4;
        typedef std::integral_constant<int, 8> i8;
        if (p.M == 8) return layout(t, i1(), i8());
        if (p.M == 4) {
            if (p.V == 4) return layout(t, i4(), i4());
            if (p.V == 2) return layout(t, i2(), i4());
            return layout(t, i1(), i4());
        }
        if constexpr (sizeof(*t) == 2)
            if (p.V == 8) return layout(t, i8(), i1());
        if (p.V == 4) return layout(t, i4(), i1());
        if (p.V == 2) return layout(t, i2(), i1());
        return layout(t, i1(), i1());
    };
    if (L.dtype == kF32) width((float *)0);
    else if (L.dtype == kF16) width((f16 *)0);
    else width((bf16 *)0);
}

}  // namespace

size_t rotary_norm_workspace(const RotaryNormLaunch &L)
{
    const NormedPlan p = plan_normed(L, true);
    int D = 0;
    for (int i = 0; i < L.n; ++i) D = D > L.a[i].D ? D : L.a[i].D;
    return ((size_t)p.bx * p.by * 2 * D * 4 + 15) / 16 * 16;
}

hipError_t launch_rotary_norm(const RotaryNormLaunch &L, hipStream_t stream)
{
    int heads = 0;
    for (int i = 0; i < L.n; ++i) heads += L.a[i].heads;
    if (L.tokens == 0 || heads == 0) return hipSuccess;
    const NormedPlan p = plan_normed(L, false);
    const NormedK k = normed_k(L, p);
    by_variant(L, p, [&](auto t, auto v, auto m, auto halves) {
        typedef std::remove_pointer_t<decltype(t)> T;
        rotary_norm_kernel<T, decltype(v)::value, decltype(m)::value, decltype(halves)::value>
            <<<dim3(p.bx, p.by), kThreads, 0, stream>>>(k);
    });
    return hipGetLastError();
}

hipError_t launch_rotary_norm_back(const RotaryNormLaunch &L, hipStream_t stream)
{
    if (L.n == 0) return hipSuccess;
    const NormedPlan p = plan_normed(L, true);
    const NormedK k = normed_k(L, p);
    by_variant(L, p, [&](auto t, auto v, auto m, auto halves) {
        typedef std::remove_pointer_t<decltype(t)> T;
        rotary_norm_back_kernel<T, decltype(v)::value, decltype(m)::value,
                                decltype(halves)::value>
            <<<dim3(p.bx, p.by), kThreads, 0, stream>>>(k);
    });
    hipError_t e = hipGetLastError();
    bool any = false;
    for (int i = 0; i < L.n; ++i) any = any || L.a[i].dw;
    if (e != hipSuccess || !any) return e;
    rotary_norm_join_kernel<<<dim3((k.dmax + 3) / 4, L.n), kThreads, 0, stream>>>(
        k, (int)(p.bx * p.by));
    return hipGetLastError();
}

}  // namespace mixrt
