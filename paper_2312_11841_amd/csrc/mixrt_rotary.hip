// Rotary positions with several axes, on up to two arrays of heads in one launch.
//
// A block takes a run of tokens (and, where there are few, a run of heads):
// first its threads work out the cosines and sines of its tokens' pairs into
// LDS, once for all heads and both arrays, then they walk over the heads'
// elements in memory order.  The sines are sincosf's, of the angle as rounded to
// 32 bits; the turn is in 32 bits and rounded once.
//
// What bounds it: the stream of the heads (65,280 tokens, 16 heads of 64 and as
// many keys, bf16: 535 MB in 93 us, 5.7 TB/s); with few tokens the launch (one
// token, 4 us of kernel).
#include "mixrt_refine.hpp"

#include <type_traits>

namespace mixrt {
namespace {

constexpr int kThreads = 256;
constexpr int kTurns = 2048;     // most (token, pair) turns of a block
constexpr int64_t kMostBlocks = 1 << 20;

struct RotaryK {
    int64_t tokens;
    int axes, pairs, n;
    int run;                 // tokens of a block
    float sign;
    const float *pos, *freq;
    const uint8_t *axis;
    HeadsK a[2];
    int per[2];              // heads of a block, per array
};

// One array's heads of the block's tokens.  An item is a vector of V pairs
// (or, past the pairs, V elements to copy).
template <typename T, int V, bool HALVES>
__device__ __forceinline__ void turn_heads(const HeadsK &h, int per, const RotaryK &k, int64_t t0,
                                           int tokens, const float2 *turn)
{
    const int h0 = blockIdx.y * per;
    const int heads = min(per, h.heads - h0);
    if (heads <= 0) return;
    const uint32_t pv = (uint32_t)k.pairs / V, rest = (uint32_t)(h.D - 2 * k.pairs);
    const uint32_t cv = rest / V, tail = rest - cv * V;
    const uint32_t items = pv + cv + tail;      // items of a head
    const uint32_t total = items * heads * tokens;
    for (uint32_t i = threadIdx.x; i < total; i += kThreads) {
        const uint32_t th = i / items, at = i - th * items;
        const uint32_t t = th / heads, hd = th - t * heads;
        const T *x = (const T *)h.x + (t0 + t) * h.xt + (h0 + hd) * h.xh;
        T *o = (T *)h.out + (t0 + t) * h.ot + (h0 + hd) * h.oh;
        if (at < pv) {
            const uint32_t j = at * V;
            const float2 *cs = turn + t * k.pairs + j;
            if (HALVES) {
                float f[V], g[V];
                load_vec<T, V>(x + j, f);
                load_vec<T, V>(x + k.pairs + j, g);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float c = cs[e].x, s = cs[e].y, a = f[e], b = g[e];
                    f[e] = a * c - b * s;
                    g[e] = b * c + a * s;
                }
                store_vec<T, V>(o + j, f);
                store_vec<T, V>(o + k.pairs + j, g);
            } else {
                float f[2 * V];
                load_vec<T, 2 * V>(x + 2 * j, f);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float c = cs[e].x, s = cs[e].y, a = f[2 * e], b = f[2 * e + 1];
                    f[2 * e] = a * c - b * s;
                    f[2 * e + 1] = b * c + a * s;
                }
                store_vec<T, 2 * V>(o + 2 * j, f);
            }
        } else if (at < pv + cv) {
            const uint32_t d = 2 * k.pairs + (at - pv) * V;
            *(Pack<T, V> *)(o + d) = *(const Pack<T, V> *)(x + d);
        } else {
            const uint32_t d = h.D - tail + (at - pv - cv);
            o[d] = x[d];
        }
    }
}

template <typename T, int V, bool HALVES>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryK k)
{
    __shared__ float2 turn[kTurns];
    for (int64_t t0 = (int64_t)blockIdx.x * k.run; t0 < k.tokens;
         t0 += (int64_t)gridDim.x * k.run) {
    const int tokens = (int)min((int64_t)k.run, k.tokens - t0);
    const uint32_t turns = (uint32_t)(tokens * k.pairs);
    for (uint32_t i = threadIdx.x; i < turns; i += kThreads) {
        const uint32_t t = i / (uint32_t)k.pairs, j = i - t * k.pairs;
        const int a = min((int)k.axis[j], k.axes - 1);
        const float angle = k.pos[(t0 + t) * k.axes + a] * k.freq[j];
        float s, c;
        sincosf(angle, &s, &c);
        turn[i] = make_float2(c, k.sign * s);
    }
    __syncthreads();
    for (int n = 0; n < k.n; ++n)
        turn_heads<T, V, HALVES>(k.a[n], k.per[n], k, t0, tokens, turn);
    __syncthreads();
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryLaunch &L, hipStream_t stream)
{
    RotaryK k;
    k.tokens = L.tokens;
    k.axes = L.axes;
    k.pairs = L.pairs;
    k.sign = L.inverse ? -1.0f : 1.0f;
    k.pos = L.pos;
    k.freq = L.freq;
    k.axis = L.axis;
    k.n = L.n;
    int64_t heads = 0, elements = 0;
    for (int i = 0; i < L.n; ++i) {
        k.a[i] = L.a[i];
        if (L.a[i].heads > heads) heads = L.a[i].heads;
        elements += (int64_t)L.a[i].heads * L.a[i].D;
    }
    if (L.tokens == 0 || heads == 0) return hipSuccess;
    // tokens of a block: about 24 elements a thread, within the LDS.  Fewer
    // repeat the start of a block too often (16 heads of 64 and as many keys,
    // 65,000 tokens: 157 us at 8, 101 at 16, 93 at 24 and 32, 99 at 48), more
    // leave short calls with few blocks (15 heads of 80 in f32, 3600 tokens:
    // 11.8 us at 24, 16.4 at 48)
    const int most = L.pairs > 0 ? kTurns / L.pairs : 64;
    int64_t run = 24 * kThreads / elements;
    if (run > most) run = most;
    if (run < 1) run = 1;
    k.run = (int)run;
    int64_t bx = (L.tokens + run - 1) / run;
    if (bx > kMostBlocks) bx = kMostBlocks;
    // few tokens: the heads are split too
    int64_t by = 512 / bx;
    if (by > heads) by = heads;
    if (by < 1) by = 1;
    for (int i = 0; i < L.n; ++i) k.per[i] = (int)((L.a[i].heads + by - 1) / by);
    const dim3 grid((unsigned)bx, (unsigned)by);
    auto launch = [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int W = sizeof(T) == 4 ? 4 : 8;
        int V = L.layout ? W / 2 : W;
        while (L.pairs % V) V >>= 1;
        auto go = [&](auto v) {
            constexpr int VV = decltype(v)::value;
            if (L.layout)
                rotary_kernel<T, VV, false><<<grid, kThreads, 0, stream>>>(k);
            else
                rotary_kernel<T, VV, true><<<grid, kThreads, 0, stream>>>(k);
        };
        if (V == 8) go(std::integral_constant<int, 8>());
        else if (V == 4) go(std::integral_constant<int, 4>());
        else if (V == 2) go(std::integral_constant<int, 2>());
        else go(std::integral_constant<int, 1>());
    };
    if (L.dtype == kF32) launch((float *)0);
    else if (L.dtype == kF16) launch((f16 *)0);
    else launch((bf16 *)0);
    return hipGetLastError();
}

}  // namespace mixrt
