// What the attention kernels share: 32 x 32 matrix products on tiles in LDS.
//
// Every kernel keeps "columns" in lanes (queries in the forward pass and in
// their own gradient, keys in theirs) and walks over tiles of "rows" that the
// block's waves share through LDS.  A product S[row][column] = sum_d A[row][d]
// B[d][column] has its operand B in registers for the whole walk; its result
// leaves each lane with 16 rows of one column,
//   row(i) = 8 (i / 4) + 4 (lane / 32) + i % 4,
// so a softmax along the rows is a sum over a lane's own registers and one
// exchange with the lane 32 further, and factors of a column are a lane's.
// The same registers are operand B of the next product, O[d][column] = sum_row
// V[row][d] P[row][column], when its operand A lists the rows in that order:
// no value moves between lanes.
#pragma once

#include "mixrt_attend.hpp"
#include "mixrt_refine.hpp"

namespace mixrt {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Elements of a 16-byte chunk, and the row stride in LDS for heads padded to DP:
// 16 bytes more than a row, so that the same chunk of 8 rows lies in different banks.
template <typename T> inline constexpr int kChunk = 16 / (int)sizeof(T);
template <typename T, int DP> inline constexpr int kStride = DP + kChunk<T>;

__device__ __forceinline__ int tile_row(int i, int half) { return 8 * (i >> 2) + 4 * half + (i & 3); }

// The value of the lane 32 further beside the lane's own, combined.
__device__ __forceinline__ float half_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                    false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <typename T> struct Matrix;

template <> struct Matrix<f16> {
    typedef _Float16 frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x16 mul(frag a, frag b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};
template <> struct Matrix<bf16> {
    typedef __bf16 frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x16 mul(frag a, frag b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Matrix<float> {
    typedef float frag __attribute__((ext_vector_type(4)));
    // four steps of two terms: element i of both halves is one step's pair
    static __device__ __forceinline__ f32x16 mul(frag a, frag b, f32x16 c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

// Chunk pairs of a padded head: operands of one mul each.
template <typename T, int DP> inline constexpr int kPairs = DP / (2 * kChunk<T>);

// Operand A of S: chunk pair c of tile row (lane % 32).
template <typename T, int DP>
__device__ __forceinline__ typename Matrix<T>::frag row_frag(const T *tile, int lane, int c)
{
    return *(const typename Matrix<T>::frag *)(tile + (lane & 31) * kStride<T, DP> +
                                               (2 * c + (lane >> 5)) * kChunk<T>);
}

// acc[d][column] += sum over 32 rows of tile[row][32 block + d] p[row][column].
template <int DP>
__device__ __forceinline__ void col_mul(const float *tile, int lane, int block, const f32x16 &p,
                                        f32x16 &acc)
{
    const float *at = tile + 4 * (lane >> 5) * kStride<float, DP> + 32 * block + (lane & 31);
#pragma unroll
    for (int i = 0; i < 16; ++i)
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(at[tile_row(i, 0) * kStride<float, DP>], p[i],
                                                   acc, 0, 0, 0);
}

// The 16-bit types' operand A of the same: rows 16 s + {0..3, 8..11} + 4 half of
// column d = 32 block + lane % 32, read with two transposing loads.  In each, 16
// lanes address four rows of 16 columns, four columns a lane, and get a column each.
template <typename T, int DP>
__device__ __forceinline__ typename Matrix<T>::frag col_frag(const T *tile, int lane, int block,
                                                             int s)
{
    typedef __attribute__((address_space(3))) s16x4 *lds4;
    const int n = lane & 15;
    const T *at = tile + (16 * s + 4 * (lane >> 5) + (n >> 2)) * kStride<T, DP> + 32 * block +
                  16 * ((lane >> 4) & 1) + 4 * (n & 3);
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)at);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 8 * kStride<T, DP>));
    const s16x8 both = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(typename Matrix<T>::frag, both);
}

// Rows 8 s .. 8 s + 7 of a lane's 16, rounded to T: operand B of step s.
template <typename T>
__device__ __forceinline__ typename Matrix<T>::frag round_rows(const f32x16 &p, int s)
{
    typename Matrix<T>::frag f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (T)p[8 * s + i];
    return f;
}

// What that rounding left of them, rounded in turn.
template <typename T>
__device__ __forceinline__ typename Matrix<T>::frag left_rows(const f32x16 &p,
                                                              typename Matrix<T>::frag f, int s)
{
    typename Matrix<T>::frag g;
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = (T)(p[8 * s + i] - (float)f[i]);
    return g;
}

// A row's chunk in registers: elements [at, at + chunk) of a head of D, zeros behind.
template <typename T>
__device__ __forceinline__ u32x4 load_chunk(const T *row, int at, int D)
{
    constexpr int V = kChunk<T>;
    Pack<T, V> t;
    if (at + V <= D) {
        t = *(const Pack<T, V> *)(row + at);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) t.v[i] = at + i < D ? row[at + i] : (T)0.0f;
    }
    return __builtin_bit_cast(u32x4, t);
}

// A tile of ROWS rows of a block of THREADS: fetched into registers, put into LDS
// when the tile before is used up.
template <typename T, int DP, int ROWS, int THREADS>
struct Stage {
    static constexpr int kChunks = DP / kChunk<T>;
    static constexpr int kAll = ROWS * kChunks;
    static constexpr int kEach = (kAll + THREADS - 1) / THREADS;
    static constexpr bool kEven = kEach * THREADS == kAll;
    u32x4 r[kEach];

    // rows [first, limit) of the array at base, as far as the tile reaches
    __device__ __forceinline__ void fetch(const T *base, int64_t stride, int first, int limit,
                                          int D)
    {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int at = threadIdx.x + j * THREADS;
            const int row = at / kChunks, c = at % kChunks;
            r[j] = u32x4{0, 0, 0, 0};
            if ((kEven || at < kAll) && first + row < limit && c * kChunk<T> < D)
                r[j] = load_chunk<T>(base + (int64_t)(first + row) * stride, c * kChunk<T>, D);
        }
    }
    __device__ __forceinline__ void put(T *tile) const
    {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int at = threadIdx.x + j * THREADS;
            if (kEven || at < kAll)
                *(u32x4 *)(tile + at / kChunks * kStride<T, DP> + at % kChunks * kChunk<T>) = r[j];
        }
    }
};

// Operand B of a column's head, from memory (zeros for a column that is not there).
template <typename T, int DP>
__device__ __forceinline__ void load_column(typename Matrix<T>::frag (&f)[(kPairs<T, DP>)],
                                            const T *row, bool there, int half, int D)
{
#pragma unroll
    for (int c = 0; c < kPairs<T, DP>; ++c) {
        const int at = (2 * c + half) * kChunk<T>;
        u32x4 x = {0, 0, 0, 0};
        if (there && at < D) x = load_chunk<T>(row, at, D);
        f[c] = __builtin_bit_cast(typename Matrix<T>::frag, x);
    }
}

// d = 32 block + 8 quad + 4 half + 0..3 of a column's result.
template <typename T>
__device__ __forceinline__ void store_quad(T *row, int d, int D, float a, float b, float c, float e)
{
    const float f[4] = {a, b, c, e};
    if (d + 4 <= D) {
        store_vec<T, 4>(row + d, f);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (d + i < D) row[d + i] = (T)f[i];
    }
}

// Blocks of one head next to each other on one XCD: the hardware deals blocks to
// the 8 XCDs in turn, and their L2s are their own.
__device__ __forceinline__ int near_block()
{
    const int n = gridDim.x >> 3, id = blockIdx.x;
    return id < 8 * n ? (id & 7) * n + (id >> 3) : id;
}

__device__ __forceinline__ int valid_keys(const int32_t *lens, int b, int Tk)
{
    return lens ? min(max(lens[b], 0), Tk) : Tk;
}

constexpr float kLog2e = 1.4426950408889634f;
// (4096 for float16, whose remainders would be subnormal)
template <typename T> inline constexpr float kRestScale = 1.0f;
template <> inline constexpr float kRestScale<f16> = 4096.0f;

// What is left of o when it is rounded to T, for the backward pass (nothing of an
// o that is not finite).
template <typename T>
__device__ __forceinline__ float rest_of(float o)
{
    const float x = (float)(T)o;
    return __builtin_isfinite(x) ? (o - x) * kRestScale<T> : 0.0f;
}

// --- the bias ---------------------------------------------------------------------

constexpr int kReachRow = 2 * kMaxReach + 2;    // entries of an axis and head in LDS

// bias[distance] of head's axes, times log2(e), for distances -reach .. reach.
__device__ __forceinline__ void load_bias(float *dense, const BiasK &b, int head, int H,
                                          int threads)
{
    const int n = 2 * b.reach + 1;
    for (int i = threadIdx.x; i < b.axes * n; i += threads) {
        const int a = i / n, d = i - a * n;
        const int m = min((int)b.map[i], b.buckets - 1);
        dense[a * kReachRow + d] = b.table[((int64_t)a * b.buckets + m) * H + head] * kLog2e;
    }
}

// Entry of the distance from a query to a key.
__device__ __forceinline__ int bias_at(int kpos, int qpos, int reach)
{
    return min(max(__builtin_elementwise_sub_sat(kpos, qpos), -reach), reach) + reach;
}

}  // namespace mixrt
