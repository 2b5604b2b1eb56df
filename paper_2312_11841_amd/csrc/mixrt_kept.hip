// Activations kept in 8 bits: packing, reading back, and the weight gradient
// of a linear layer computed from the codes.
#include "mixrt_refine.hpp"

#include <type_traits>

namespace mixrt {
namespace {

constexpr int kThreads = 256;

// Packing and reading back are streams: L neighbouring lanes of V channels
// take a kept group (rows narrower than a group only as many lanes as they
// need), groups in the order of the scale bytes.  A block takes kPackSteps
// steps of its threads and ends; larger runs and loads ahead were slower (64
// channels of a 720p frame in bf16, both ways: 65 us at 4 steps, 66 at 8, 73 at
// 16, 81 with 8 loads ahead; the copy's rate for its 358 MB makes 62).  Now 60:
// packing 33 us of kernel (5.4 TB/s), reading back 27 (6.5).
constexpr int kPackSteps = 4;
constexpr int64_t kMostBlocks = 1 << 20;   // then blocks take further runs

// Where a lane is: its group, counted from the block's first row, and channels.
struct KeptLane {
    int64_t row, group;   // group: the scale byte's index
    int c0, left;         // left: channels from c0 to the row's end, 0 past the last group
    __device__ __forceinline__ KeptLane(int64_t row0, uint32_t g, int64_t groups, int C,
                                        int per_row, int at)
    {
        const uint32_t dr = per_row == 1 ? g : g / (uint32_t)per_row;
        row = row0 + dr;
        group = row0 * per_row + g;
        c0 = (int)(g - dr * per_row) * kKeptGroup + at;
        left = group < groups ? C - c0 : 0;
    }
};

// Calls f(lane) for the steps of the runs that are this block's.
template <int V, int L, typename F>
__device__ __forceinline__ void walk_groups(int64_t groups, int C, int per_row, F f)
{
    constexpr int kStep = kThreads / L;   // groups of a step
    constexpr int64_t kRun = (int64_t)kStep * kPackSteps;
    for (int64_t first = (int64_t)blockIdx.x * kRun; first < groups;
         first += (int64_t)gridDim.x * kRun) {
        const int64_t row0 = first / per_row;
        const uint32_t at0 = (uint32_t)(first - row0 * per_row) + threadIdx.x / L;
#pragma unroll 1
        for (int s = 0; s < kPackSteps; ++s)
            f(KeptLane(row0, at0 + s * kStep, groups, C, per_row, (int)(threadIdx.x % L) * V));
    }
}

// A vector may start at any element; where the row ends inside it (never with
// WHOLE), its elements are moved one by one.
template <typename T, int V, int L, bool WHOLE>
__global__ __launch_bounds__(kThreads) void kept_pack_kernel(const T *x, int64_t stride,
                                                             int64_t groups, int C, int per_row,
                                                             int8_t *codes, uint8_t *exps)
{
    walk_groups<V, L>(groups, C, per_row, [&](const KeptLane &l) {
        const T *p = x + l.row * stride + l.c0;
        float f[V];
        if (l.left >= V)
            load_vec<T, V>(p, f);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = !WHOLE && i < l.left ? (float)p[i] : 0.0f;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
#pragma unroll
        for (int e = 1; e < L; e <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, e));
        const uint32_t byte = kept_byte<T>(top);
        const Pack<int8_t, V> out = kept_codes<T, V>(f, byte);
        int8_t *q = codes + l.row * C + l.c0;
        if (l.left >= V)
            *(Pack<int8_t, V> *)q = out;
        else if (!WHOLE)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < l.left) q[i] = out.v[i];
        if (threadIdx.x % L == 0 && l.left > 0) exps[l.group] = (uint8_t)byte;
    });
}

template <typename T, int V, int L, bool WHOLE>
__global__ __launch_bounds__(kThreads) void kept_unpack_kernel(const int8_t *codes,
                                                               const uint8_t *exps, int64_t groups,
                                                               int C, int per_row, T *out,
                                                               int64_t stride)
{
    walk_groups<V, L>(groups, C, per_row, [&](const KeptLane &l) {
        if (l.left <= 0) return;
        const int8_t *q = codes + l.row * C + l.c0;
        const float scale = kept_scale(exps[l.group]);
        T *p = out + l.row * stride + l.c0;
        if (l.left >= V) {
            const Pack<int8_t, V> v = *(const Pack<int8_t, V> *)q;
            float f[V];
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = (float)v.v[i] * scale;
            store_vec<T, V>(p, f);
        } else if (!WHOLE) {
            for (int i = 0; i < l.left; ++i) p[i] = (T)((float)q[i] * scale);
        }
    });
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
//
// What bounds it: few weights, the stream of codes and dy (720p rows, 64 x 64,
// bf16: 179 MB in 35 us of kernel, 5.1 TB/s); many weights, the vector memory
// path through which every tile's rows go again, busy 80% of the time (100,000
// rows, 512 x 512, bf16: 121 us, 433 TFLOP/s; 3600 rows, 512 x 1536, f16: 21
// us).  Wide loads turned by way of LDS instead took 110 us of the first, no
// less of the second, and 250 us where f32 takes 183 (100,000 rows, 320 x 320; 112
// TFLOP/s).

constexpr int kTile = 64;     // channels of a wave's block of dw, each way
constexpr int kRows = 32;     // rows of a step
// Steps of a wave whose sums stay in registers, where a part is one chain of them
// (kOneChain at most) and where it is several, which move on to LDS in turn.  32
// steps are 1024 rows added one after another in 32 bits in f32 (a matrix
// instruction adds its 4 rows so), 128 are as many matrix instructions of 32 rows
// in 16 bits.  Without it a wide layer of many rows, which is one part, lost its
// lower bits (921,600 equal rows, 2048 x 2048 in f32: off by 2.3e-3).
template <typename T> constexpr int kOneChain = sizeof(T) == 4 ? 32 : 128;
template <typename T> constexpr int kChainSteps = sizeof(T) == 4 ? 27 : 120;   // 3 n

typedef float f4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

// 8 rows of one channel: an MFMA operand of a lane.
template <typename T> struct Frag;
template <> struct Frag<f16> { typedef h8 type; };
template <> struct Frag<bf16> { typedef b8 type; };

__device__ __forceinline__ f4 mac(h8 a, h8 b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f4 mac(b8 a, b8 b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
struct LinearK {
    const int8_t *codes;
    const uint8_t *exps;
    const void *dy;
    int64_t rows, dy_stride;
    int64_t part;     // rows of one block
    int64_t whole;    // rows whose vectors stay inside the arrays
    int C, outs, per_row;
    int ty, tz;       // tiles of dw along its channels and its outs
    // where a part's sums go: parts of C * outs weights and outs column sums,
    // or, of one part, dw and db (which may be null)
    float *sums, *bias;
    int64_t stride;
};

// A lane's share of a step as it is in memory: 4 channels (a word) and 4 outs
// (kWords words) of 8 rows.
template <typename T>
struct LinearStep {
    static constexpr int kWords = sizeof(T);
    uint32_t code[8], byte[8], dy[8][kWords];
};

template <int N>
struct __attribute__((packed, aligned(1))) Words {   // loads may start at any byte
    uint32_t v[N];
};

// Where a lane's channels and outs lie in its quarter's rows.  Lanes past the
// channels or the outs take the row's start: what they compute is not stored.
struct LinearOffsets {
    uint32_t code, byte, dy;
};

// row (the step's first) is the same for the wave, so the addresses are scalar
// ones with a 32-bit offset of the lane's own, in bytes.
template <typename T>
__device__ __forceinline__ void load_step(LinearStep<T> &s, int64_t row, const LinearOffsets &o,
                                          const LinearK &k)
{
    constexpr int W = LinearStep<T>::kWords;
    const int8_t *codes = k.codes + row * k.C;
    const uint8_t *exps = k.exps + row * k.per_row;
    const char *dy = (const char *)k.dy + row * k.dy_stride * sizeof(T);
    // the offsets are made new to the compiler here, so that it sees 32-bit
    // ones beside the loads and uses the scalar address form (else it keeps
    // them as 64 bits and adds each address in vector registers)
    uint32_t oc = o.code, ob = o.byte, od = o.dy;
    asm("" : "+v"(oc), "+v"(ob), "+v"(od));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        s.code[i] = ((const Words<1> *)(codes + oc))->v[0];
        s.byte[i] = exps[ob];
        const Words<W> d = *(const Words<W> *)(dy + od);
#pragma unroll
        for (int w = 0; w < W; ++w) s.dy[i][w] = d.v[w];
        codes += k.C;
        exps += k.per_row;
        dy += k.dy_stride * sizeof(T);
    }
}

// The same near the arrays' end.  row: the lane's first.  Rows from r1 on
// read the last row and count as 0 (2^e of byte 0 is 0); a vector that would
// pass the end of its array starts earlier and is shifted down.
template <typename T>
__device__ __forceinline__ void load_last(LinearStep<T> &s, int64_t row, int64_t r1, int ci,
                                          int co, const LinearK &k)
{
    constexpr int W = LinearStep<T>::kWords;
    const int64_t n_code = k.rows * k.C, n_dy = (k.rows - 1) * k.dy_stride + k.outs;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool in = row + i < r1;
        const int64_t r = in ? row + i : r1 - 1;
        const int64_t ac = r * k.C + ci, ad = r * k.dy_stride + co;
        const int over_c = (int)max(ac + 4 - n_code, (int64_t)0);
        const int over_d = (int)max(ad + 4 - n_dy, (int64_t)0);
        s.code[i] = ((const Words<1> *)(k.codes + ac - over_c))->v[0] >> (8 * over_c);
        const uint32_t byte = k.exps[r * k.per_row + ci / kKeptGroup];
        s.byte[i] = in ? byte : 0u;
        const Words<W> d = *(const Words<W> *)((const T *)k.dy + ad - over_d);
        uint32_t v[W];
#pragma unroll
        for (int w = 0; w < W; ++w) v[w] = d.v[w];
        if (W == 2) {
            const uint64_t both = (((uint64_t)v[W - 1] << 32) | v[0]) >> (16 * over_d);
            v[0] = (uint32_t)both;
            v[W - 1] = (uint32_t)(both >> 32);
        } else {
#pragma unroll
            for (int t = 0; t < 3; ++t)
                if (over_d > t)
#pragma unroll
                    for (int w = 0; w + 1 < W; ++w) v[w] = v[w + 1];
        }
#pragma unroll
        for (int w = 0; w < W; ++w) s.dy[i][w] = in ? v[w] : 0u;
    }
}

// The scales of 8 rows, as the conversion below takes them.
template <typename T> struct Scales {
    float v[8];
    __device__ __forceinline__ explicit Scales(const uint32_t (&byte)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = kept_scale(byte[i]);
    }
};
template <> struct Scales<f16> {
    h2 v[4];
    __device__ __forceinline__ explicit Scales(const uint32_t (&byte)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = (h2){(f16)kept_scale(byte[2 * i]), (f16)kept_scale(byte[2 * i + 1])};
    }
};

// Element m of 8 rows' codes as an operand.  bf16: the product with 2^e in 32
// bits, without rounding; its upper half is the bf16.
__device__ __forceinline__ float code_value(uint32_t code, int m, float scale)
{
    return (float)(int8_t)(code >> (8 * m)) * scale;
}
__device__ __forceinline__ b8 code_frag(const uint32_t (&code)[8], const Scales<bf16> &s, int m)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = __builtin_amdgcn_perm(
            __float_as_uint(code_value(code[2 * i + 1], m, s.v[2 * i + 1])),
            __float_as_uint(code_value(code[2 * i], m, s.v[2 * i])), 0x07060302u);
    return __builtin_bit_cast(b8, w);
}
// f16: two rows at once.  The byte of code + 128 (its top bit turned) below
// 0x64 is the f16 1024 + 128 + code; less 1152 it is the code, and its product
// with 2^e is exact.
__device__ __forceinline__ h8 code_frag(const uint32_t (&code)[8], const Scales<f16> &s, int m)
{
    h2 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t pair = __builtin_amdgcn_perm(code[2 * i + 1], code[2 * i],
                                                    0x0c040c00u + 0x00010001u * m) ^
                              0x64806480u;
        w[i] = (__builtin_bit_cast(h2, pair) - (f16)1152.0f) * s.v[i];
    }
    return __builtin_bit_cast(h8, w);
}

// Element n of 8 rows of dy as an operand.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type dy_frag(const LinearStep<T> &s, int n)
{
    typedef typename Frag<T>::type F;
    const uint32_t sel = n & 1 ? 0x07060302u : 0x05040100u;
    uint4 w;
    w.x = __builtin_amdgcn_perm(s.dy[1][n >> 1], s.dy[0][n >> 1], sel);
    w.y = __builtin_amdgcn_perm(s.dy[3][n >> 1], s.dy[2][n >> 1], sel);
    w.z = __builtin_amdgcn_perm(s.dy[5][n >> 1], s.dy[4][n >> 1], sel);
    w.w = __builtin_amdgcn_perm(s.dy[7][n >> 1], s.dy[6][n >> 1], sel);
    return __builtin_bit_cast(F, w);
}

template <typename T>
__device__ __forceinline__ void multiply_step(const LinearStep<T> &s, bool biased, f4 (&acc)[4][4],
                                              f4 (&bias)[4])
{
    typedef typename Frag<T>::type F;
    const Scales<T> sc(s.byte);
    F b[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) b[n] = dy_frag(s, n);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const F a = code_frag(s.code, sc, m);
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[m][n] = mac(a, b[n], acc[m][n]);
    }
    if (biased) {
        F ones;
#pragma unroll
        for (int i = 0; i < 8; ++i) ones[i] = (T)1.0f;
#pragma unroll
        for (int n = 0; n < 4; ++n) bias[n] = mac(ones, b[n], bias[n]);
    }
}

// f32: a step's rows 8 q + i of the lanes' quarters q, one i at a time.  bias:
// the lane's own sums, in element 0, added beside the matrix unit (by it they
// are a fifth of its work: 921,600 rows, 64 x 64, 102 us a call and 83).
template <>
__device__ __forceinline__ void multiply_step(const LinearStep<float> &s, bool biased,
                                              f4 (&acc)[4][4], f4 (&bias)[4])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float sc = kept_scale(s.byte[i]);
        float b[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) b[n] = __uint_as_float(s.dy[i][n]);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const float a = code_value(s.code[i], m, sc);
#pragma unroll
            for (int n = 0; n < 4; ++n)
                acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, b[n], acc[m][n], 0, 0, 0);
        }
        if (biased)
#pragma unroll
            for (int n = 0; n < 4; ++n) bias[n][0] += b[n];
    }
}

// CHAINS: a part has more steps than one chain.
template <typename T, bool CHAINS>
__global__ __launch_bounds__(kThreads) void linear_grad_kernel(LinearK k)
{
    __shared__ __align__(16) float sh[CHAINS ? 4 : 2][kTile * kTile + kTile];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
    const int q = lane >> 4, c = lane & 15;
    // Blocks are dealt to the 8 XCDs in turn.  Each XCD takes a run of a part's
    // tiles, which read the same rows at the same time and find them in its L2
    // (100,000 rows, 512 x 512, bf16: codes read by every XCD take 134 us)
    const int nb = gridDim.x, x = blockIdx.x & 7;
    int at = x * (nb >> 3) + min(x, nb & 7) + (blockIdx.x >> 3);
    const int ty = at % k.ty;
    at /= k.ty;
    const int tz = at % k.tz, part = at / k.tz;
    int ci = ty * kTile + 4 * c, co = tz * kTile + 4 * c;
    if (ci >= k.C) ci = 0;
    if (co >= k.outs) co = 0;
    f4 acc[4][4], bias[4];
    const auto clear = [&] {
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            bias[m] = (f4)0.0f;
#pragma unroll
            for (int n = 0; n < 4; ++n) acc[m][n] = (f4)0.0f;
        }
    };
    clear();
    // Puts this wave's sums into its place in LDS or adds them there.  A tile's
    // row m (channel 4 m + i) is in quarter m / 4, register m % 4, its column n
    // (outs 4 n + j) in lane n: a lane's four neighbours go at once (one at a
    // time, and the waves one after another, 0.5 to 0.8 us more a call).
    const auto move = [&](float *mine, bool store) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f4 *const p = (f4 *)&mine[(4 * (4 * q + e) + i) * kTile + 4 * c];
                const f4 v = {acc[i][0][e], acc[i][1][e], acc[i][2][e], acc[i][3][e]};
                *p = store ? v : *p + v;
            }
        if (sizeof(T) == 4)   // the quarters' column sums
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bias[j][0] += __shfl_xor(bias[j][0], 16);
                bias[j][0] += __shfl_xor(bias[j][0], 32);
            }
        if (q == 0) {
            f4 *const p = (f4 *)&mine[kTile * kTile + 4 * c];
            const f4 v = {bias[0][0], bias[1][0], bias[2][0], bias[3][0]};
            *p = store ? v : *p + v;
        }
    };
    const bool biased = ty == 0;
    const int64_t first = part * k.part, r1 = min(first + k.part, k.rows);
    const int64_t whole = min(r1, k.whole);
    int64_t r0 = first + wave * kRows;
    const int n = r0 + kRows <= whole ? (int)((whole - r0 - kRows) / (4 * kRows)) + 1 : 0;
    const LinearOffsets off{(uint32_t)(8 * q * k.C + ci),
                            (uint32_t)(8 * q * k.per_row + ci / kKeptGroup),
                            (uint32_t)(8 * q * (uint32_t)k.dy_stride + co) * (uint32_t)sizeof(T)};
    bool moved = false;   // this wave has sums in LDS
    if (n > 0) {
        // Two steps are on their way while one is multiplied.  The loads past
        // the last step repeat it: a condition around them would end the
        // overlap, since waits are counted.
        const auto load = [&](LinearStep<T> &s, int i) {
            load_step(s, r0 + (int64_t)min(i, n - 1) * (4 * kRows), off, k);
            __builtin_amdgcn_sched_barrier(0);   // else loads may sink to their uses
        };
        LinearStep<T> s0, s1, s2;
        load(s0, 0);
        load(s1, 1);
        // (two forms of one loop: the first takes 10% less where a part is one
        // chain in 16 bits, the second where it is several in f32)
        if (!CHAINS)
            for (int i = 0;; i += 3) {
                load(s2, i + 2);
                multiply_step(s0, biased, acc, bias);
                if (i + 1 >= n) break;
                load(s0, i + 3);
                multiply_step(s1, biased, acc, bias);
                if (i + 2 >= n) break;
                load(s1, i + 4);
                multiply_step(s2, biased, acc, bias);
                if (i + 3 >= n) break;
            }
        else {
            int i = 0;
            while (i + 3 <= n) {
                const int end = min(i + kChainSteps<T>, n);
                for (; i + 3 <= end; i += 3) {
                    load(s2, i + 2);
                    multiply_step(s0, biased, acc, bias);
                    load(s0, i + 3);
                    multiply_step(s1, biased, acc, bias);
                    load(s1, i + 4);
                    multiply_step(s2, biased, acc, bias);
                }
                move(sh[wave], !moved);
                clear();
                moved = true;
            }
            if (i < n) multiply_step(s0, biased, acc, bias);
            if (i + 1 < n) multiply_step(s1, biased, acc, bias);
        }
    }
    // (rows near the arrays' end, or all where vectors cannot be used)
    int tail = 0;
    for (r0 += (int64_t)n * (4 * kRows); r0 < r1; r0 += 4 * kRows) {
        if (CHAINS && ++tail % kChainSteps<T> == 0) {
            move(sh[wave], !moved);
            clear();
            moved = true;
        }
        LinearStep<T> s;
        load_last(s, r0 + 8 * q, r1, ci, co, k);
        multiply_step(s, biased, acc, bias);
    }
    if (CHAINS) {
        move(sh[wave], !moved);
        __syncthreads();
    } else {
        // two waves store their sums, the other two add theirs, and the halves
        // are added on the way out
        for (int w = 0; w < 4; w += 2) {
            if ((wave & 2) == w) move(sh[wave & 1], w == 0);
            __syncthreads();
        }
    }
    const auto sum = [&](int at) {
        const float v = sh[0][at] + sh[1][at];
        return CHAINS ? v + (sh[CHAINS ? 2 : 0][at] + sh[CHAINS ? 3 : 0][at]) : v;
    };
    float *const out = k.sums + (int64_t)part * k.stride;
    const int o = threadIdx.x & 63, og = tz * kTile + o;
    if (og < k.outs) {
        for (int i = threadIdx.x >> 6; i < kTile; i += 4) {
            const int cg = ty * kTile + i;
            if (cg < k.C)
                out[(int64_t)cg * k.outs + og] = sum(i * kTile + o);
        }
        if (biased && k.bias && threadIdx.x < 64)
            k.bias[(int64_t)part * k.stride + og] = sum(kTile * kTile + o);
    }
}

// Few channels and outs on one side (a frame has 4) and not many on the other:
// a tile of 64 would be mostly empty.  L neighbouring lanes take a row, each CT
// of its channels and OT of its outs, and keep the CT * OT = 64 sums themselves
// (921,600 rows in 16 bits, us a call, by tiles and so: 16 channels, 4 outs 24.4,
// 13.3; 32 and 4 23.9, 16.4; 15 and 3 29.6, 14.7; 4 and 32 23.3, 20.4).  Bound by
// the vector memory path, as a lane's rows lie apart; rows in flight hide the
// rest.
constexpr int kFew = 4, kMany = 16;   // a lane's channels and outs, either way
constexpr int kNarrowLanes = 4;       // most lanes of a row
constexpr int kNarrowAhead = 4;       // rows a lane loads before it uses the first

template <int CT, int OT, typename T>
struct NarrowRow {
    Pack<int8_t, CT> code;
    uint8_t byte;
    Pack<T, OT> dy;
};

template <typename T, int CT, int OT, int L>
__global__ __launch_bounds__(kThreads) void linear_narrow_kernel(LinearK k)
{
    static_assert(CT * OT == 64 && kKeptGroup % CT == 0, "a sum for each lane, one kept group");
    constexpr int kDown = kThreads / L;   // rows of a step
    __shared__ float sh[kThreads / 64][L][64 + OT];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, l = lane % L;
    // lanes past the channels or the outs take the row's start: what they
    // compute is not stored
    const bool in = CT > OT ? l * CT < k.C : l * OT < k.outs;
    const int c0 = in && CT > OT ? l * CT : 0, o0 = in && OT > CT ? l * OT : 0;
    float acc[64], bias[OT];
#pragma unroll
    for (int i = 0; i < 64; ++i) acc[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < OT; ++j) bias[j] = 0.0f;
    const int64_t first = blockIdx.x * k.part, r1 = min(first + k.part, k.rows);
    // vectors that pass a row's end take elements of the next rows, which only
    // meet sums that are not stored; near the arrays' end, element by element
    const auto load = [&](int64_t r, bool vectors) {
        NarrowRow<CT, OT, T> d;
        const int8_t *x = k.codes + r * k.C + c0;
        const T *dy = (const T *)k.dy + r * k.dy_stride + o0;
        d.byte = k.exps[r * k.per_row + c0 / kKeptGroup];
        if (vectors) {
            d.code = *(const Pack<int8_t, CT> *)x;
            d.dy = *(const Pack<T, OT> *)dy;
        } else {
#pragma unroll
            for (int i = 0; i < CT; ++i) d.code.v[i] = c0 + i < k.C ? x[i] : (int8_t)0;
#pragma unroll
            for (int j = 0; j < OT; ++j) d.dy.v[j] = o0 + j < k.outs ? dy[j] : (T)0.0f;
        }
        return d;
    };
    const auto add = [&](const NarrowRow<CT, OT, T> &d) {
        const float scale = kept_scale(d.byte);
        float y[OT];
#pragma unroll
        for (int j = 0; j < OT; ++j) {
            y[j] = (float)d.dy.v[j];
            bias[j] += y[j];
        }
#pragma unroll
        for (int i = 0; i < CT; ++i) {
            const float x = (float)d.code.v[i] * scale;
#pragma unroll
            for (int j = 0; j < OT; ++j) acc[i * OT + j] = fmaf(x, y[j], acc[i * OT + j]);
        }
    };
    int64_t r = first + threadIdx.x / L;
    const int64_t whole = min(r1, k.whole);
    for (; r + (kNarrowAhead - 1) * kDown < whole; r += kNarrowAhead * kDown) {
        NarrowRow<CT, OT, T> d[kNarrowAhead];
#pragma unroll
        for (int u = 0; u < kNarrowAhead; ++u) d[u] = load(r + u * kDown, true);
        __builtin_amdgcn_sched_barrier(0);   // else the loads sink to their uses
#pragma unroll
        for (int u = 0; u < kNarrowAhead; ++u) add(d[u]);
    }
    for (; r < r1; r += kDown) add(load(r, r < whole));
    // the sums over a wave's lanes: each step halves the sums that a lane still
    // holds; it ends with L of them, from (lane rounded down to L) on
#pragma unroll
    for (int d = 32; d >= L; d >>= 1)
#pragma unroll
        for (int i = 0; i < d; ++i) {
            const bool up = (lane & d) != 0;
            const float keep = up ? acc[i + d] : acc[i], send = up ? acc[i] : acc[i + d];
            acc[i] = keep + __shfl_xor(send, d);
        }
#pragma unroll
    for (int a = 0; a < L; ++a) sh[wave][l][lane - l + a] = acc[a];
#pragma unroll
    for (int j = 0; j < OT; ++j) {
#pragma unroll
        for (int d = 32; d >= L; d >>= 1) bias[j] += __shfl_xor(bias[j], d);
        if (lane < L) sh[wave][l][64 + j] = bias[j];
    }
    __syncthreads();
    float *const out = k.sums + (int64_t)blockIdx.x * k.stride;
    for (int t = threadIdx.x; t < L * (64 + OT); t += kThreads) {
        const int at = t / (64 + OT), e = t - at * (64 + OT);
        float v = 0.0f;
        for (int w = 0; w < kThreads / 64; ++w) v += sh[w][at][e];
        const int o = (OT > CT ? at * OT : 0) + (e < 64 ? e % OT : e - 64);
        const int c = (CT > OT ? at * CT : 0) + e / OT;
        if (o >= k.outs) continue;
        if (e < 64) {
            if (c < k.C) out[(int64_t)c * k.outs + o] = v;
        } else if (k.bias && (OT > CT || at == 0)) {
            k.bias[(int64_t)blockIdx.x * k.stride + o] = v;
        }
    }
}

// Arrays shorter than a vector (few elements, or one short row of dy that all
// rows share): a thread's sum for each weight of a part.
template <typename T>
__global__ __launch_bounds__(kThreads) void linear_tiny_kernel(LinearK k)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t c = i / k.outs, part = blockIdx.y;
    if (c > k.C) return;
    const int o = (int)(i - c * k.outs);
    const int64_t first = part * k.part, r1 = min(first + k.part, k.rows);
    double v = 0.0;   // a part may have many rows
    for (int64_t r = first; r < r1; ++r) {
        const float d = (float)((const T *)k.dy)[r * k.dy_stride + o];
        const float x = c < k.C ? (float)k.codes[r * k.C + c] *
                                      kept_scale(k.exps[r * k.per_row + c / kKeptGroup])
                                : 1.0f;
        v = fma((double)x, (double)d, v);
    }
    if (c < k.C)
        k.sums[part * k.stride + i] = (float)v;
    else if (k.bias)
        k.bias[part * k.stride + o] = (float)v;
}

// Adds the parts.  n: values of one part; the last outs are db.  ACROSS
// threads take every ACROSSth part of a value each, then their sums are added
// in order.
template <int ACROSS, int THREADS>
__global__ __launch_bounds__(THREADS) void linear_join_kernel(const float *sums, int64_t n,
                                                              int64_t weights, int parts,
                                                              float *dw, float *db)
{
    constexpr int kValues = THREADS / ACROSS;
    __shared__ float sh[ACROSS][kValues + 1];
    const int o = threadIdx.x % kValues, a = threadIdx.x / kValues;
    const int64_t i = (int64_t)blockIdx.x * kValues + o;
    float v = 0.0f;
    if (i < n)
#pragma unroll 8
        for (int p = a; p < parts; p += ACROSS) v += sums[(int64_t)p * n + i];
    if (ACROSS > 1) {
        sh[a][o] = v;
        for (int half = ACROSS / 2; half > 0; half /= 2) {
            __syncthreads();
            if (a < half) sh[a][o] += sh[a + half][o];
        }
        v = sh[0][o];
    }
    if (a == 0 && i < n) {
        if (i < weights)
            dw[i] = v;
        else if (db)
            db[i - weights] = v;
    }
}

constexpr int kCus = 256;

constexpr int kNarrowBlocks = 512;
constexpr int kNarrowRows = 1024;   // about as many rows a lane adds up in 32 bits

struct LinearPlan {
    int parts, ty, tz;
    int64_t part;
    int narrow;   // lanes of a row, 0: tiles of 64
};

// How many parts the rows are split into.  The time is estimated in steps of a
// block, about 1.2 us while a CU holds two blocks (as many as their registers
// allow) and 0.6 of that while it holds one; a block takes about 3 more for its
// start and its end, a join about 5, and writing and reading n sums n / 500,000.
// One part needs no join.  (720p rows, 64 x 64: 256 parts 40.6 us, 512 41.2, 128
// 50.8; 3600 rows, 512 x 1536, f16: one part 21.6, two with their join 24.2,
// five 29.6; 100,000 rows, 512 x 512: 8 parts 121, 4 143, 16 140.)  Narrow layers:
// two runs of loads a lane at least, and 2 blocks a CU (2,000,000 rows of one by
// one: 9 us more a call with 1, 4 with 3) or as many parts as leave a lane about
// kNarrowRows rows.
LinearPlan linear_plan(int64_t rows, int C, int outs, int dtype)
{
    LinearPlan p;
    p.narrow = 0;
    // (64 channels, 4 outs: 27.8 us in f16 where tiles take 24.6; in f32 tiles of
    // 4 x 48 take 92 and this 40)
    const int few = C < outs ? C : outs, many = C < outs ? outs : C;
    if (few <= kFew && many <= kMany * kNarrowLanes && (C <= 3 * kMany || dtype == kF32)) {
        p.narrow = many <= kMany ? 1 : many <= 2 * kMany ? 2 : 4;
        p.ty = p.tz = 1;
        const int64_t run = (int64_t)kThreads / p.narrow * 2 * kNarrowAhead;
        int64_t parts = (rows + run - 1) / run;
        const int64_t least = rows / ((int64_t)kThreads / p.narrow * kNarrowRows);
        if (parts > kNarrowBlocks) parts = least > kNarrowBlocks ? least : kNarrowBlocks;
        if (parts < 1) parts = 1;
        p.part = (rows + parts - 1) / parts;
        p.parts = (int)parts;
        return p;
    }
    p.ty = (C + kTile - 1) / kTile;
    p.tz = (outs + kTile - 1) / kTile;
    const int tiles = p.ty * p.tz;
    const int64_t steps = (rows + 4 * kRows - 1) / (4 * kRows);
    const double sums = ((double)C * outs + outs) / 500000.0;
    int64_t best = 1;
    double least = 0.0;
    for (int filled = 0; filled <= 16; ++filled) {   // blocks a CU; 0: one part
        int64_t parts = (int64_t)filled * kCus / tiles;
        if (parts > steps) parts = steps;
        if (parts < 1) parts = 1;
        const int64_t each = (steps + parts - 1) / parts;
        const int64_t turns = (parts * tiles + 2 * kCus - 1) / (2 * kCus);
        const double load = parts * tiles <= kCus ? 0.6 : (double)turns;
        const double join = parts > 1 ? 5.0 + sums * (double)parts : 0.0;
        const double cost = load * (double)(each + 3) + join;
        if (filled == 0 || cost < least) {
            least = cost;
            best = parts;
        }
    }
    p.part = ((rows + best - 1) / best + kRows - 1) / kRows * kRows;
    if (p.part < 1) p.part = kRows;
    p.parts = rows > 0 ? (int)((rows + p.part - 1) / p.part) : 1;
    return p;
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

namespace {

// f(lanes of a group, whether vectors end with the row) for rows of C channels
// in vectors of V.
template <int V, typename F>
void with_lanes(int C, F f)
{
    auto go = [&](auto l) {
        if (C % V == 0) f(l, std::true_type());
        else f(l, std::false_type());
    };
    if (C <= V) go(std::integral_constant<int, 1>());
    else if (C <= 2 * V) go(std::integral_constant<int, 2>());
    else if constexpr (V == 8) go(std::integral_constant<int, 4>());
    else if (C <= 4 * V) go(std::integral_constant<int, 4>());
    else go(std::integral_constant<int, 8>());
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
        constexpr int V = sizeof(T) == 4 ? 4 : 8;
        with_lanes<V>(C, [&](auto l, auto whole) {
            constexpr int L = decltype(l)::value;
            kept_pack_kernel<T, V, L, decltype(whole)::value>
                <<<blocks(groups, (int64_t)kThreads / L * kPackSteps), kThreads, 0, stream>>>(
                    (const T *)x, stride, groups, C, per_row, codes, exps);
        });
    });
    return hipGetLastError();
}

hipError_t launch_kept_unpack(int out_dtype, int64_t rows, int C, const int8_t *codes,
                              const uint8_t *exps, void *out, int64_t stride, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    const int per_row = kept_groups(C);
    const int64_t groups = rows * per_row;
    with_type(out_dtype, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        constexpr int V = sizeof(T) == 4 ? 4 : 8;
        with_lanes<V>(C, [&](auto l, auto whole) {
            constexpr int L = decltype(l)::value;
            kept_unpack_kernel<T, V, L, decltype(whole)::value>
                <<<blocks(groups, (int64_t)kThreads / L * kPackSteps), kThreads, 0, stream>>>(
                    codes, exps, groups, C, per_row, (T *)out, stride);
        });
    });
    return hipGetLastError();
}

size_t linear_grad_workspace(int64_t rows, int C, int outs, int dtype)
{
    const LinearPlan p = linear_plan(rows, C, outs, dtype);
    return p.parts > 1 ? (size_t)p.parts * ((size_t)C * outs + outs) * sizeof(float) : 0;
}

hipError_t launch_linear_grad(int dtype, int64_t rows, int C, int outs, const int8_t *codes,
                              const uint8_t *exps, const void *dy, int64_t dy_stride, float *dw,
                              float *db, void *ws, hipStream_t stream)
{
    const LinearPlan p = linear_plan(rows, C, outs, dtype);
    // A vector of 4 (16 where a lane takes whole rows) that is not whole in its
    // row goes on into the next rows: at most 3 (15) of them, rows of one
    // element, and none where rows of dy repeat.
    const int vc = p.narrow && outs <= C ? kMany : 4, vo = p.narrow && outs > C ? kMany : 4;
    int64_t whole = rows;
    if (C % vc || outs % vo) whole = rows - (p.narrow ? kMany - 1 : 3);
    if (outs % vo && dy_stride < outs) whole = 0;
    if (!p.narrow && dy_stride >= (1 << 24)) whole = 0;   // the lanes' offsets are 32 bits
    const int64_t weights = (int64_t)C * outs, n = weights + outs;
    float *const sums = (float *)ws;
    const bool one = p.parts == 1;
    const LinearK k{codes, exps, dy, rows, dy_stride, p.part, whole, C, outs, kept_groups(C),
                    p.ty,  p.tz, one ? dw : sums, one ? db : sums + weights, n};
    const int grid = p.parts * p.ty * p.tz;
    const bool tiny = rows * C < 4 || (rows - 1) * dy_stride + outs < 4;
    with_type(dtype, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        auto narrow = [&](auto ct, auto ot, auto l) {
            constexpr int CT = decltype(ct)::value, OT = decltype(ot)::value;
            constexpr int L = decltype(l)::value;
            linear_narrow_kernel<T, CT, OT, L><<<grid, kThreads, 0, stream>>>(k);
        };
        auto with_side = [&](auto l) {
            const std::integral_constant<int, kFew> few;
            const std::integral_constant<int, kMany> many;
            if (outs <= C) narrow(many, few, l);
            else narrow(few, many, l);
        };
        if (p.narrow == 1)
            with_side(std::integral_constant<int, 1>());
        else if (p.narrow == 2)
            with_side(std::integral_constant<int, 2>());
        else if (p.narrow == 4)
            with_side(std::integral_constant<int, 4>());
        else if (tiny)
            linear_tiny_kernel<T>
                <<<dim3(blocks(n, kThreads), p.parts), kThreads, 0, stream>>>(k);
        else if (p.part > (int64_t)kOneChain<T> * 4 * kRows)
            linear_grad_kernel<T, true><<<grid, kThreads, 0, stream>>>(k);
        else
            linear_grad_kernel<T, false><<<grid, kThreads, 0, stream>>>(k);
    });
    // many parts of few weights: 32 threads a value (4160 values of 506 parts
    // 4.7 us, against 120 with one); few parts: one (788,000 values of 2 parts
    // 53 us with 32)
    if (one) return hipGetLastError();
    if (p.parts > 8)
        linear_join_kernel<32, 1024><<<blocks(n, 32), 1024, 0, stream>>>(sums, n, weights,
                                                                         p.parts, dw, db);
    else
        linear_join_kernel<1, 256><<<blocks(n, 256), 256, 0, stream>>>(sums, n, weights, p.parts,
                                                                       dw, db);
    return hipGetLastError();
}

}  // namespace mixrt
