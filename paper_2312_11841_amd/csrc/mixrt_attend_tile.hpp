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

// At the start of a branch that a wave takes seldom: keeps the compiler from working
// out both sides for every tile (its selects made up a third of the forward kernel's
// instructions).
__device__ __forceinline__ void rare() { asm volatile(""); }

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

// Whether chunk pair c is padding alone: float32's products, four of 64 cycles a pair,
// leave it out (the 16-bit types' take 32 cycles, less than a branch gives).
template <typename T>
__device__ __forceinline__ bool past(int c, int D)
{
    return sizeof(T) == 4 && 2 * c * kChunk<T> >= D;
}

// Operand A of S: chunk pair c of tile row (lane % 32).
template <typename T, int DP>
__device__ __forceinline__ typename Matrix<T>::frag row_frag(const T *tile, int lane, int c)
{
    return *(const typename Matrix<T>::frag *)(tile + (lane & 31) * kStride<T, DP> +
                                               (2 * c + (lane >> 5)) * kChunk<T>);
}

// S of 32 rows: operand A from LDS, B a lane's column.
template <typename T, int DP>
__device__ __forceinline__ f32x16 row_mul(const T *tile, int lane,
                                          const typename Matrix<T>::frag (&b)[kPairs<T, DP>], int D)
{
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
    for (int c = 0; c < kPairs<T, DP>; ++c)
        if (!past<T>(c, D)) s = Matrix<T>::mul(row_frag<T, DP>(tile, lane, c), b[c], s);
    return s;
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

// The same as a sum of TERMS: their rounded values, what that left, rounded in turn, ..
template <typename T, int TERMS>
__device__ __forceinline__ void split_rows(const f32x16 &p, int s,
                                           typename Matrix<T>::frag (&f)[TERMS])
{
    f[0] = round_rows<T>(p, s);
    float left[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) left[i] = p[8 * s + i];
#pragma unroll
    for (int n = 1; n < TERMS; ++n) {
        // (taken from the pairs, not rounded once more one by one)
        asm("" : "+v"(f[n - 1]));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            left[i] -= (float)f[n - 1][i];
            f[n][i] = (T)left[i];
        }
    }
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

// A tile of ROWS rows, fetched by THREADS threads into registers and put into LDS when
// the tile before is used up.
template <typename T, int DP, int ROWS, int THREADS>
struct Stage {
    static constexpr int kChunks = DP / kChunk<T>;
    static constexpr int kAll = ROWS * kChunks;
    static constexpr int kEach = (kAll + THREADS - 1) / THREADS;
    static constexpr bool kEven = kEach * THREADS == kAll;
    u32x4 r[kEach];

    // rows [first, limit) of the array at base, as far as the tile reaches
    __device__ __forceinline__ void fetch(int thread, const T *base, int64_t stride, int first,
                                          int limit, int D)
    {
        if (kEven && D == DP && first + ROWS <= limit) {    // nothing to leave out
            // (the tile's place is the same for all threads, a thread's place in it for
            // all tiles)
            const char *tile = (const char *)(base + (int64_t)first * stride);
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const int at = thread + j * THREADS;
                const int64_t off = (int64_t)(at / kChunks) * stride + at % kChunks * kChunk<T>;
                r[j] = __builtin_bit_cast(
                    u32x4, *(const Pack<T, kChunk<T>> *)(tile + off * (int64_t)sizeof(T)));
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int at = thread + j * THREADS;
            const int row = at / kChunks, c = at % kChunks;
            r[j] = u32x4{0, 0, 0, 0};
            if ((kEven || at < kAll) && first + row < limit && c * kChunk<T> < D)
                r[j] = load_chunk<T>(base + (int64_t)(first + row) * stride, c * kChunk<T>, D);
        }
    }
    __device__ __forceinline__ void put(int thread, T *tile) const
    {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int at = thread + j * THREADS;
            if (kEven || at < kAll)
                *(u32x4 *)(tile + at / kChunks * kStride<T, DP> + at % kChunks * kChunk<T>) = r[j];
        }
    }
};

// How a block's four waves divide its work.  Alone: a wave has columns of its own and
// the tiles are the block's.  Shared, where a call has few columns: all waves have the
// same 32 and every fourth tile each, staged by itself, and their sums are joined in
// LDS at the end.
template <bool SHARED>
struct Team {
    static constexpr int kStagers = SHARED ? 64 : 256;
    static constexpr int kStep = SHARED ? 4 : 1;        // tiles from one to the next
    int lane, wave, half;
    __device__ __forceinline__ Team()
        : lane(threadIdx.x & 63), wave(threadIdx.x >> 6), half(threadIdx.x >> 5 & 1)
    {
    }
    __device__ __forceinline__ int stager() const { return SHARED ? lane : (int)threadIdx.x; }
    __device__ __forceinline__ int mine() const { return SHARED ? wave : 0; }
    // tiles written are there to be read, tiles read may be written
    __device__ __forceinline__ void meet() const
    {
        if (SHARED) {
            // (a wave's accesses to LDS take place in its order)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
            __syncthreads();
        }
    }
};

// Whether a wave that stages alone has registers to fetch a tile ahead.
template <typename T, int DP> inline constexpr bool kFetchAhead = DP * sizeof(T) <= 256;

// Joins the sums of four waves that share their columns: a lane gets DP / 8 of its
// column's, from d = (2 wave + half) DP / 8 on.  room: 128 DP floats.
template <int DP>
__device__ __forceinline__ void join_waves(float *room, int lane, int wave,
                                           const f32x16 (&acc)[DP / 32], float by,
                                           float (&out)[DP / 8])
{
    const int half = lane >> 5, column = lane & 31;
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            room[(wave * DP + 32 * d + tile_row(i, half)) * 32 + column] = acc[d][i] * by;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) {
        const int d = (2 * wave + half) * (DP / 8) + i;
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) s += room[(w * DP + d) * 32 + column];
        out[i] = s;
    }
}

template <typename T, int N>
__device__ __forceinline__ void store_run(T *row, int d, int D, const float (&f)[N], float by)
{
#pragma unroll
    for (int i = 0; i < N; i += 4)
        store_quad<T>(row, d + i, D, f[i] * by, f[i + 1] * by, f[i + 2] * by, f[i + 3] * by);
}

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
// What is left of o when it is rounded to T, for the backward pass (nothing of an o
// that is not finite), in T's bits: of float16's 13 lost bits 11, times 2048: it is then
// subnormal only where o is below 2^-14, and at most 2^15 (half a step of an o below
// 65520 is 16; times 4096 that would not be finite); of bfloat16's 16, whose exponent is o's own, all of them, as the
// difference of the bits.  (Rounded to bfloat16, which keeps 8, it was most of the
// error of a bias table's gradient.)
template <typename T>
__device__ __forceinline__ T rest_of(float o)
{
    const T x = (T)o;
    if (!__builtin_isfinite((float)x)) return (T)0.0f;
    if constexpr (std::is_same_v<T, bf16>) {
        const uint32_t n = __float_as_uint(o) - __float_as_uint((float)x);
        return __builtin_bit_cast(bf16, (int16_t)min(max((int)n, -32768), 32767));
    } else {
        return (T)((o - (float)x) * 2048.0f);
    }
}

// o again.
template <typename T>
__device__ __forceinline__ float whole_of(T x, T rest)
{
    if constexpr (std::is_same_v<T, bf16>)
        return __uint_as_float(__float_as_uint((float)x) +
                               (uint32_t)(int)__builtin_bit_cast(int16_t, rest));
    else
        return (float)x + (float)rest * (1.0f / 2048.0f);
}

// What is left of four elements of a column's result to a dense row of D.
template <typename T>
__device__ __forceinline__ void store_rest(T *row, int d, int D, const float *o)
{
    Pack<T, 4> x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = rest_of<T>(o[i]);
    if (d + 4 <= D) {
        *(Pack<T, 4> *)(row + d) = x;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (d + i < D) row[d + i] = x.v[i];
    }
}

// --- the bias ---------------------------------------------------------------------
//
// A lane's column and a tile's row have a distance on each axis.  Tokens of views come
// row by row, so of 32 rows that follow each other mostly all have the same place on an
// axis, or every 8 of them have places that count up by one, or one place.  A tile
// carries for each axis which of these holds: then one place in the table serves 32
// rows, four neighbours of one place a lane's four rows of an octet, or one place an
// octet, and only blocks that mix them work out each row's own.  Each kind is one
// stretch of code without branches, so that its reads of LDS run together.  (With a
// branch an octet they waited for each other: 8160 tokens among themselves, 16 heads of
// 64 in bf16 and two axes took 897 us a call, without 750.)
//
// So the time depends on the width of the views' rows.  An octet that crosses the end of
// one makes its 32 rows mixed on every axis: about as many pairs take 729 us in rows of
// 120, 713 of 64, 763 of 40, 789 of 24, 774 of 107, 865 of 119 and 939 of 12 or 7; a
// training step of 3600 queries over 7200 keys with three axes 907 in rows of 80, 881 of
// 64, 977 of 24, 1041 of 67, 1022 of 79 and 1219 of 12.

constexpr int kPad = 4;                                     // entries beyond either end
constexpr int kReachRow = 2 * kMaxReach + 2 + 2 * kPad;     // of an axis and head in LDS

// Entry of the distance row - column, cut to -reach - beyond .. reach.
__device__ __forceinline__ int bias_at(int row, int column, int reach, int beyond = 0)
{
    return min(max(__builtin_elementwise_sub_sat(row, column), -reach - beyond), reach) + reach +
           kPad;
}

// The bucket of an entry (mirrored: of the distance column - row).
__device__ __forceinline__ int bucket_of(const BiasK &b, int axis, int entry, bool mirrored)
{
    const int d = min(max(entry - kPad, 0), 2 * b.reach);
    return min((int)b.map[axis * (2 * b.reach + 1) + (mirrored ? 2 * b.reach - d : d)],
               b.buckets - 1);
}

// bias[entry] of head's axes, times log2(e), a finite one at most 2^125: a mask of the
// lowest float has to stay finite there, and where the axes' are added.
constexpr float kMostBias = 0x1p125f;
__device__ __forceinline__ void load_bias(float *dense, const BiasK &b, int head, int H,
                                          int thread, int threads, bool mirrored)
{
    const int n = 2 * b.reach + 1 + 2 * kPad;
    for (int i = thread; i < b.axes * n; i += threads) {
        const int a = i / n, e = i - a * n;
        const float entry =
            b.table[((int64_t)a * b.buckets + bucket_of(b, a, e, mirrored)) * H + head];
        float x = entry * kLog2e;
        if (fabsf(x) > kMostBias && fabsf(entry) < INFINITY) x = copysignf(kMostBias, x);
        dense[a * kReachRow + e] = x;
    }
}

enum { kMixed, kLevel, kSteps, kLevel8 };

// Places of a tile's rows on each axis, and the kind of each block of 32 rows.
template <int ROWS>
struct TilePos {
    __attribute__((aligned(16))) int32_t at[kMaxBiasAxes][ROWS];
    uint32_t kind[kMaxBiasAxes];    // 2 bits a block
    __device__ __forceinline__ int kind_of(int axis, int u) const
    {
        return __builtin_amdgcn_readfirstlane((int)kind[axis]) >> (2 * u) & 3;
    }
};

template <int ROWS>
struct StagePos {
    int32_t r[kMaxBiasAxes];
    bool there;
    __device__ __forceinline__ void fetch(int thread, const int32_t *pos, int axes, int first,
                                          int limit)
    {
        const int row = first + thread;
        there = thread < ROWS && row < limit;
#pragma unroll
        for (int a = 0; a < kMaxBiasAxes; ++a)
            r[a] = there && a < axes ? pos[(int64_t)row * axes + a] : 0;
    }
    __device__ __forceinline__ void put(int thread, TilePos<ROWS> &tile, int axes) const
    {
        if (thread >= 64) return;           // the first wave holds the rows
        const int lane = thread;
#pragma unroll
        for (int a = 0; a < kMaxBiasAxes; ++a) {
            if (a >= axes) break;
            // (rows that are not there fit in anywhere)
            const int one = __shfl(r[a], lane & ~7), all = __shfl(r[a], lane & ~31);
            const bool level = !there || r[a] == one;
            const bool steps = !there || (one < 0x7fffffff - 8 && r[a] == one + (lane & 7));
            const bool alike = !there || r[a] == all;
            const uint64_t l = __builtin_amdgcn_ballot_w64(level);
            const uint64_t s = __builtin_amdgcn_ballot_w64(steps);
            const uint64_t w = __builtin_amdgcn_ballot_w64(alike);
            uint32_t kind = 0;
#pragma unroll
            for (int u = 0; u < ROWS / 32; ++u) {
                const auto all_of = [&](uint64_t m) { return (uint32_t)(m >> (32 * u)) == ~0u; };
                const uint32_t is = all_of(w) ? kLevel : all_of(s) ? kSteps : all_of(l) ? kLevel8
                                                                                         : kMixed;
                kind |= is << (2 * u);
            }
            if (lane < ROWS) tile.at[a][lane] = r[a];
            if (lane == 0) tile.kind[a] = kind;
        }
    }
};

// s[i] = s[i] scale + the bias of row i of the tile's block u and the lane's column.
template <int ROWS>
__device__ __forceinline__ void add_bias(f32x16 &s, float scale, const TilePos<ROWS> &tile,
                                         int u, int half, const float *dense, int base,
                                         const int (&column)[kMaxBiasAxes], int axes, int reach)
{
    // (an axis that is not there reads places in LDS too, and adds nothing)
    float level = 0.0f, b[kMaxBiasAxes];
    int kind[kMaxBiasAxes];
#pragma unroll
    for (int a = 0; a < kMaxBiasAxes; ++a) kind[a] = tile.kind_of(a, u);
#pragma unroll
    for (int a = 0; a < kMaxBiasAxes; ++a)
        b[a] = dense[base + a * kReachRow + bias_at(tile.at[a][32 * u], column[a], reach)];
#pragma unroll
    for (int a = 0; a < kMaxBiasAxes; ++a) level += a < axes && kind[a] == kLevel ? b[a] : 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], scale, level);
#pragma unroll
    for (int a = 0; a < kMaxBiasAxes; ++a) {
        if (a >= axes) break;
        const int32_t *p = &tile.at[a][32 * u + 4 * half];
        const float *row = dense + base + a * kReachRow;
        if (kind[a] == kSteps) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float *four = row + bias_at(p[8 * j], column[a], reach, kPad);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * j + i] += four[i];
            }
        } else if (kind[a] == kLevel8) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float one = row[bias_at(p[8 * j], column[a], reach)];
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * j + i] += one;
            }
        } else if (kind[a] == kMixed) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[i] += row[bias_at(p[tile_row(i, 0)], column[a], reach)];
        }
    }
}

}  // namespace mixrt
