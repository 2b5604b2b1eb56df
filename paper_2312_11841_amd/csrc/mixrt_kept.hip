// Activations kept in 8 bits: packing, reading back, and the weight gradient
// of a linear layer computed from the codes.
#include "mixrt_refine.hpp"

#include <type_traits>

namespace mixrt {
namespace {

constexpr int kThreads = 256;

// One kept group (32 channels of a row) per 32/V neighbouring lanes, groups in
// the order of the scale bytes; a block takes kPackSteps steps of its threads
// at a time, and further such runs where the grid is at its most.
constexpr int kPackSteps = 8;
constexpr int64_t kMostBlocks = 1 << 20;

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void kept_pack_kernel(const T *x, int64_t stride,
                                                             int64_t groups, int C, int per_row,
                                                             int8_t *codes, uint8_t *exps)
{
    constexpr int L = kKeptGroup / V;            // lanes of a group
    constexpr int kStep = kThreads / L;          // groups of a step
    const uint32_t slot = threadIdx.x / L, lane = threadIdx.x % L;
    for (int64_t first = (int64_t)blockIdx.x * (kStep * kPackSteps); first < groups;
         first += (int64_t)gridDim.x * (kStep * kPackSteps)) {
    const int64_t row0 = first / per_row;
    const uint32_t at0 = (uint32_t)(first - row0 * per_row);
#pragma unroll
    for (int s = 0; s < kPackSteps; ++s) {
        const uint32_t g = at0 + s * kStep + slot;   // counted from row0's first group
        if (row0 * per_row + g >= groups) return;     // the whole group's lanes
        const uint32_t dr = g / (uint32_t)per_row;
        const int64_t row = row0 + dr;
        const int c0 = (int)(g - dr * per_row) * kKeptGroup + (int)lane * V;
        const bool in = c0 < C;
        float f[V];
        if (in)
            load_vec<T, V>(x + row * stride + c0, f);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = 0.0f;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
#pragma unroll
        for (int d = 1; d < L; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
        const uint32_t byte = kept_byte<T>(top);
        if (in) {
            Pack<int8_t, V> out;
#pragma unroll
            for (int i = 0; i < V; ++i) out.v[i] = (int8_t)kept_code<T>(f[i], byte);
            *(Pack<int8_t, V> *)(codes + row * C + c0) = out;
        }
        if (lane == 0) exps[row0 * per_row + g] = (uint8_t)byte;
    }
    }
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void kept_unpack_kernel(const int8_t *codes,
                                                               const uint8_t *exps, int64_t rows,
                                                               int C, int per_row, T *out,
                                                               int64_t stride)
{
    const uint32_t vecs = (uint32_t)C / V;
    for (int64_t first = (int64_t)blockIdx.x * (kThreads * kPackSteps); first < rows * vecs;
         first += (int64_t)gridDim.x * (kThreads * kPackSteps)) {
    const int64_t row0 = first / vecs;
    const uint32_t at0 = (uint32_t)(first - row0 * vecs);
#pragma unroll
    for (int s = 0; s < kPackSteps; ++s) {
        const uint32_t v = at0 + s * kThreads + threadIdx.x;
        const uint32_t dr = v / vecs;
        const int64_t row = row0 + dr;
        if (row >= rows) return;
        const int c0 = (int)(v - dr * vecs) * V;
        const Pack<int8_t, V> q = *(const Pack<int8_t, V> *)(codes + row * C + c0);
        const float sc = kept_scale(exps[row * per_row + c0 / kKeptGroup]);
        float f[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = (float)q.v[i] * sc;
        store_vec<T, V>(out + row * stride + c0, f);
    }
    }
}

// --- the weight gradient of a linear layer -----------------------------------------
//
// dw = x^T dy is a matrix product whose long axis is the rows, so both operands
// have their contracted index outermost in memory.  A lane loads 4
// neighbouring channels of 8 rows; element i of its 8 loads is then the lane's
// part (8 rows, one channel) of an MFMA operand over the channels 4 m + i, so
// the transposition costs byte permutations in registers and no LDS.  A wave
// holds a 64 x 64 block of dw (16 tiles); the rows are split over blocks and
// over the 4 waves of a block, which add theirs in LDS; a second kernel adds
// the blocks' sums in a fixed order.

constexpr int kTile = 64;     // channels of a wave's block of dw, each way
constexpr int kRows = 32;     // rows of a step

typedef float f4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f8 __attribute__((ext_vector_type(8)));

template <typename T> struct Frag;
template <> struct Frag<f16> { typedef h8 type; };
template <> struct Frag<bf16> { typedef b8 type; };
template <> struct Frag<float> { typedef f8 type; };

__device__ __forceinline__ f4 mac(h8 a, h8 b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f4 mac(b8 a, b8 b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// rows 8 q + i for the lanes' quarters q, one i at a time
__device__ __forceinline__ f4 mac(f8 a, f8 b, f4 c)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

struct LinearK {
    const int8_t *codes;
    const uint8_t *exps;
    const void *dy;
    int64_t rows, dy_stride, part;   // part: rows of one block
    int C, outs, per_row;
    float *sums;      // [parts][C * outs + outs]
};

// 4 channels of a row; what lies past the array's end is 0.
template <bool WHOLE>
__device__ __forceinline__ uint32_t load_codes(const int8_t *p, int left)
{
    if (WHOLE) return left > 0 ? *(const uint32_t *)p : 0u;
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) v |= (uint32_t)(uint8_t)p[i] << (8 * i);
    return v;
}

template <typename T, bool WHOLE>
__device__ __forceinline__ Pack<T, 4> load_dy(const T *p, int left)
{
    Pack<T, 4> v;
    if (WHOLE) {
        if (left > 0) return *(const Pack<T, 4> *)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) v.v[i] = (T)0.0f;
        return v;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v.v[i] = i < left ? p[i] : (T)0.0f;
    return v;
}

// WC, WO: the channels and outs are multiples of 4.
template <typename T, bool WC, bool WO>
__global__ __launch_bounds__(kThreads) void linear_grad_kernel(LinearK k)
{
    typedef typename Frag<T>::type F;
    __shared__ float sh[kTile * kTile + kTile];
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const int q = lane >> 4, c = lane & 15;
    const int ci = blockIdx.y * kTile + 4 * c, co = blockIdx.z * kTile + 4 * c;
    const int lc = k.C - ci, lo = k.outs - co;   // channels left from here
    f4 acc[4][4], bias[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        bias[m] = (f4)0.0f;
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[m][n] = (f4)0.0f;
    }
    F ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (T)1.0f;
    const int64_t r1 = min(((int64_t)blockIdx.x + 1) * k.part, k.rows);
    for (int64_t r0 = (int64_t)blockIdx.x * k.part + wave * kRows; r0 < r1; r0 += 4 * kRows) {
        uint32_t code[8], byte[8];
        Pack<T, 4> dy[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t row = r0 + 8 * q + i;
            const bool in = row < r1;
            code[i] = in ? load_codes<WC>(k.codes + row * k.C + ci, lc) : 0u;
            byte[i] = in && lc > 0 ? k.exps[row * k.per_row + ci / kKeptGroup] : 0u;
            dy[i] = load_dy<T, WO>((const T *)k.dy + row * k.dy_stride + co, in ? lo : 0);
        }
        F a[4], b[4];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // code * 2^e from the code plus 128: u s - 128 s is exact
            const float s = kept_scale(byte[i]), off = -128.0f * s;
            const uint32_t u = code[i] ^ 0x80808080u;
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                a[m][i] = (T)fmaf((float)((u >> (8 * m)) & 255u), s, off);
                b[m][i] = dy[i].v[m];
            }
        }
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int n = 0; n < 4; ++n) acc[m][n] = mac(a[m], b[n], acc[m][n]);
        if (blockIdx.y == 0)
#pragma unroll
            for (int n = 0; n < 4; ++n) bias[n] = mac(ones, b[n], bias[n]);
    }
    // the waves add in turn: a tile's row m (channel 4 m + i) is in quarter
    // m / 4, register m % 4, its column n (out 4 n + j) in lane n
    for (int w = 0; w < 4; ++w) {
        if (wave == w) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float *p = &sh[(4 * (4 * q + e) + i) * kTile + 4 * c + j];
                        *p = w == 0 ? acc[i][j][e] : *p + acc[i][j][e];
                    }
            if (q == 0)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float *p = &sh[kTile * kTile + 4 * c + j];
                    *p = w == 0 ? bias[j][0] : *p + bias[j][0];
                }
        }
        __syncthreads();
    }
    float *out = k.sums + (int64_t)blockIdx.x * ((int64_t)k.C * k.outs + k.outs);
    const int o = threadIdx.x & 63, og = blockIdx.z * kTile + o;
    if (og < k.outs) {
        for (int i = threadIdx.x >> 6; i < kTile; i += 4) {
            const int cg = blockIdx.y * kTile + i;
            if (cg < k.C) out[(int64_t)cg * k.outs + og] = sh[i * kTile + o];
        }
        if (blockIdx.y == 0 && threadIdx.x < 64)
            out[(int64_t)k.C * k.outs + og] = sh[kTile * kTile + o];
    }
}

// Adds the parts, in order.  n: values of one part; the last outs are db.
__global__ __launch_bounds__(kThreads) void linear_join_kernel(const float *sums, int64_t n,
                                                               int64_t weights, int parts,
                                                               float *dw, float *db)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= n) return;
    double v = 0.0;
    for (int p = 0; p < parts; ++p) v += (double)sums[(int64_t)p * n + i];
    if (i < weights)
        dw[i] = (float)v;
    else if (db)
        db[i - weights] = (float)v;
}

struct LinearPlan {
    int parts, ty, tz;
    int64_t part;
};

LinearPlan linear_plan(int64_t rows, int C, int outs)
{
    LinearPlan p;
    p.ty = (C + kTile - 1) / kTile;
    p.tz = (outs + kTile - 1) / kTile;
    const int64_t most = (rows + 4 * kRows - 1) / (4 * kRows);   // a step for every wave
    int64_t parts = 768 / ((int64_t)p.ty * p.tz);
    if (parts > most) parts = most;
    if (parts < 1) parts = 1;
    p.part = ((rows + parts - 1) / parts + kRows - 1) / kRows * kRows;
    if (p.part < 1) p.part = kRows;
    p.parts = rows > 0 ? (int)((rows + p.part - 1) / p.part) : 1;
    return p;
}

template <typename F>
void with_vector(int C, int widest, F f)
{
    int V = widest;
    while (C % V) V >>= 1;
    if (V == 8) f(std::integral_constant<int, 8>());
    else if (V == 4) f(std::integral_constant<int, 4>());
    else if (V == 2) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 1>());
}

template <typename F>
void with_type(int dtype, F f)
{
    if (dtype == kF32) f((float *)0);
    else if (dtype == kF16) f((f16 *)0);
    else f((bf16 *)0);
}

unsigned blocks(int64_t n, int64_t per)
{
    const int64_t b = (n + per - 1) / per;
    return (unsigned)(b < kMostBlocks ? b : kMostBlocks);
}

}  // namespace

hipError_t launch_kept_pack(int dtype, int64_t rows, int C, const void *x, int64_t stride,
                            int8_t *codes, uint8_t *exps, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    const int per_row = kept_groups(C);
    const int64_t groups = rows * per_row;
    with_type(dtype, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        with_vector(C, sizeof(T) == 4 ? 4 : 8, [&](auto v) {
            constexpr int V = decltype(v)::value;
            const int64_t per = (int64_t)kThreads * V / kKeptGroup * kPackSteps;
            kept_pack_kernel<T, V><<<blocks(groups, per), kThreads, 0, stream>>>(
                (const T *)x, stride, groups, C, per_row, codes, exps);
        });
    });
    return hipGetLastError();
}

hipError_t launch_kept_unpack(int out_dtype, int64_t rows, int C, const int8_t *codes,
                              const uint8_t *exps, void *out, int64_t stride, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    with_type(out_dtype, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        with_vector(C, sizeof(T) == 4 ? 4 : 8, [&](auto v) {
            constexpr int V = decltype(v)::value;
            kept_unpack_kernel<T, V>
                <<<blocks(rows * (C / V), (int64_t)kThreads * kPackSteps), kThreads, 0, stream>>>(
                    codes, exps, rows, C, kept_groups(C), (T *)out, stride);
        });
    });
    return hipGetLastError();
}

size_t linear_grad_workspace(int64_t rows, int C, int outs, int)
{
    const LinearPlan p = linear_plan(rows, C, outs);
    return (size_t)p.parts * ((size_t)C * outs + outs) * sizeof(float);
}

hipError_t launch_linear_grad(int dtype, int64_t rows, int C, int outs, const int8_t *codes,
                              const uint8_t *exps, const void *dy, int64_t dy_stride, float *dw,
                              float *db, void *ws, hipStream_t stream)
{
    const LinearPlan p = linear_plan(rows, C, outs);
    LinearK k{codes, exps, dy, rows, dy_stride, p.part, C, outs, kept_groups(C), (float *)ws};
    const dim3 grid(p.parts, p.ty, p.tz);
    // whole 4-byte loads of codes need rows that start at a multiple of 4
    const bool wc = C % 4 == 0 && ((uintptr_t)codes & 3u) == 0, wo = outs % 4 == 0;
    with_type(dtype, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        if (wc && wo) linear_grad_kernel<T, true, true><<<grid, kThreads, 0, stream>>>(k);
        else if (wc) linear_grad_kernel<T, true, false><<<grid, kThreads, 0, stream>>>(k);
        else if (wo) linear_grad_kernel<T, false, true><<<grid, kThreads, 0, stream>>>(k);
        else linear_grad_kernel<T, false, false><<<grid, kThreads, 0, stream>>>(k);
    });
    const int64_t weights = (int64_t)C * outs, n = weights + outs;
    linear_join_kernel<<<blocks(n, kThreads), kThreads, 0, stream>>>(k.sums, n, weights, p.parts,
                                                                     dw, db);
    return hipGetLastError();
}

}  // namespace mixrt
