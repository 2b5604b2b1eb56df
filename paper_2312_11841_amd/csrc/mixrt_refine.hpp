// The view refiner's operators: launch interface between the C ABI
// (mixrt_refine_api.cpp) and the kernels (mixrt_norm.hip, mixrt_kept.hip,
// mixrt_rotary.hip), and the element access the kernels share.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mixrt {

enum { kF32 = 0, kF16 = 1, kBF16 = 3 };                        // mixrt_dtype
enum { kActNone = 0, kActRelu = 1, kActSilu = 2, kActGelu = 3 };  // mixrt_act
inline constexpr int kKeptGroup = 32;

// One array of a norm call: strides in elements.
struct MapK {
    void *data;
    int64_t image, pixel;
};

struct NormLaunch {
    int N, C, G, dtype, act;
    int64_t P;
    float eps;
    const float *gamma, *beta;
    MapK x, y, dy, dx;        // forward: x, y; backward: dy, dx and (codes null) x
    float *stats;             // [N][G][2] or null (forward only)
    int8_t *codes;            // kept form of x, or null
    uint8_t *exps;
    float *dgamma, *dbeta;
    void *ws;
};

// Workspace bytes of both directions.
size_t norm_workspace(int N, int64_t P, int C, int G, int dtype);
hipError_t launch_norm_forward(const NormLaunch &L, hipStream_t stream);
hipError_t launch_norm_backward(const NormLaunch &L, hipStream_t stream);

hipError_t launch_kept_pack(int dtype, int64_t rows, int C, const void *x, int64_t stride,
                            int8_t *codes, uint8_t *exps, hipStream_t stream);
hipError_t launch_kept_unpack(int out_dtype, int64_t rows, int C, const int8_t *codes,
                              const uint8_t *exps, void *out, int64_t stride, hipStream_t stream);
size_t linear_grad_workspace(int64_t rows, int C, int outs, int dtype);
hipError_t launch_linear_grad(int dtype, int64_t rows, int C, int outs, const int8_t *codes,
                              const uint8_t *exps, const void *dy, int64_t dy_stride, float *dw,
                              float *db, void *ws, hipStream_t stream);

struct HeadsK {
    int heads, D;
    const void *x;
    void *out;
    int64_t xt, xh, ot, oh;   // token and head strides, in elements
};

struct RotaryLaunch {
    int64_t tokens;
    int axes, pairs, layout, dtype, n;
    bool inverse;
    const float *pos, *freq;
    const uint8_t *axis;
    HeadsK a[2];
};

hipError_t launch_rotary(const RotaryLaunch &L, hipStream_t stream);

// --- element access -----------------------------------------------------------

typedef __bf16 bf16;
typedef _Float16 f16;

// V elements of T moved as one access; the array may start at any element
// (the hardware takes unaligned vector accesses; aligned ones are faster).
template <typename T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
    T v[V];
};

template <typename T, int V>
__device__ __forceinline__ void load_vec(const T *p, float (&f)[V])
{
    const Pack<T, V> t = *(const Pack<T, V> *)p;
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = (float)t.v[i];
}

template <typename T, int V>
__device__ __forceinline__ void store_vec(T *p, const float (&f)[V])
{
    Pack<T, V> t;
#pragma unroll
    for (int i = 0; i < V; ++i) t.v[i] = (T)f[i];
    *(Pack<T, V> *)p = t;
}

// --- the 8-bit form -------------------------------------------------------------

// Scale bytes of one row.
__host__ __device__ inline int kept_groups(int C) { return (C + kKeptGroup - 1) / kKeptGroup; }

// 2^e of a scale byte; 255 gives an infinity, which turns the group's codes
// (all 0) into NaN.
__device__ __forceinline__ float kept_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// The scale byte of a group whose largest |x| has these bits: e = exponent - 6,
// one more where the largest code would round to 128, that is from 127.5 / 64
// in the mantissa up; 255 where |x| is not finite.  T gives the least e.
template <typename T> struct KeptRange { static constexpr int kLow = -126, kTop = 122; };
template <> struct KeptRange<f16> { static constexpr int kLow = -24, kTop = 10; };

template <typename T>
__device__ __forceinline__ uint32_t kept_byte(uint32_t bits)
{
    int e = (int)(bits >> 23) - 127 - 6 + ((bits & 0x7fffffu) >= 0x7f0000u ? 1 : 0);
    if (e < KeptRange<T>::kLow) e = KeptRange<T>::kLow;
    return bits >= 0x7f800000u ? 255u : (uint32_t)(e + 127);
}

// The codes of V values at their group's scale byte.  x 2^-e is exact; added to
// 1.5 * 2^23 it leaves its nearest integer (halves to even) in the sum's low
// bits, and by the choice of e that is at most 127 in magnitude.  From kTop on,
// where 64 * 2^e is not finite in T, the codes stop at 63; at byte 255 they are
// 0, whatever the sum made of an infinity or of a NaN and its payload.
template <typename T, int V>
__device__ __forceinline__ Pack<int8_t, V> kept_codes(const float (&x)[V], uint32_t byte)
{
    const float inv = __uint_as_float((254u - byte) << 23);   // 2^-e
    Pack<int8_t, V> q;
#pragma unroll
    for (int i = 0; i < V; ++i)
        q.v[i] = (int8_t)(__float_as_uint(fmaf(x[i], inv, 12582912.0f)) & 255u);
    // (a branch for the wave: as a choice for each lane it costs two steps a value)
    if (__builtin_amdgcn_ballot_w64(byte >= (uint32_t)(KeptRange<T>::kTop + 127)) != 0 &&
        byte >= (uint32_t)(KeptRange<T>::kTop + 127)) {
        const int most = byte == 255u ? 0 : 63;
#pragma unroll
        for (int i = 0; i < V; ++i) q.v[i] = (int8_t)max(min((int)q.v[i], most), -most);
    }
    return q;
}

}  // namespace mixrt
