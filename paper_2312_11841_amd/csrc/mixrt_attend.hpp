// The refiner's attention: launch interface between the C ABI
// (mixrt_attend_api.cpp) and the kernels (mixrt_attend_forward.hpp and
// mixrt_attend_backward.hpp, built for one element type each).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mixrt {

inline constexpr int kMaxBiasAxes = 3;
inline constexpr int kMaxBuckets = 32;
inline constexpr int kMaxReach = 127;
inline constexpr int kMaxAttendDim = 128;

// An array of heads [batch][token][head][d]: strides in elements.
struct SeqK {
    void *data;
    int64_t batch, token, head;
};

struct BiasK {
    int axes;                 // 0: none
    int buckets, reach;
    const float *table;       // [axes][buckets][heads]
    const uint8_t *map;       // [axes][2 reach + 1]
    const int32_t *qpos, *kpos;   // [tokens][axes]
    int64_t qbatch, kbatch;   // elements from one batch entry's to the next's
};

struct AttendK {
    int B, H, Hk, D, Tq, Tk;
    int dtype;
    float scale;              // of q k, times log2(e)
    float plain_scale;
    const int32_t *lens;      // [B] or null
    BiasK bias;
    SeqK q, k, v, o;
    void *rest;               // [B][Tq][H][D], dense, or null
    float *lse;               // [B][H][Tq] or null
    float *lse_rest;          // the same, or null: what rounding took from lse
    // backward
    SeqK dout, dq, dk, dv;
    float *dtable;
    // how the work is dealt (see AttendPlan), and a pass of it: the row (tile) it starts
    // from, parts of an array in scratch, the parts that its join reads (with what the
    // passes before left, in the part behind its own), and whether it is the last
    int pack, blocks, splits, per;
    int from, slots, parts, pass;
    bool last;
    float *part, *delta, *part_table;
    float2 *part_lse;         // (lse and its rest; what passes leave in two by turns)
    double *table_sum;        // of the passes
};

// How a call is dealt.  Forward: a block takes cols columns (a column is a token and
// one of pack heads that share their keys) and per keys; queries' gradient: likewise,
// pack 1; keys' gradient: a block takes cols keys and per tiles of attend_kv_rows
// (the heads of a group one after another).  A long walk runs in passes, one after
// another, each of so many splits, whose join adds what the passes before left: the
// scratch is then a few arrays' size, however long the walk.
struct AttendPlan {
    int shared;               // a block's waves share 32 columns and divide the rows
    int pack;
    int cols, blocks;         // columns of a block, blocks of one head
    int splits, per, passes;
};

// Parts of an array in scratch.
inline int attend_slots(const AttendPlan &p)
{
    return p.passes > 1 ? p.splits + 1 : p.splits > 1 ? p.splits : 0;
}

// A launch holds fewer than 2^32 threads in x: blocks of 256 that a kernel whose grid is
// its work may have; the kernels that join splits walk over theirs in fewer.
inline constexpr int64_t kMostBlocks256 = ((int64_t)1 << 24) - 1;
inline constexpr int64_t kMostJoinBlocks = 1 << 16;
inline int64_t join_blocks(int64_t blocks)
{
    return blocks < kMostJoinBlocks ? blocks : kMostJoinBlocks;
}

// Blocks of a stage's launch (a training forward call has 128 columns a block where
// others have 256).
inline int64_t attend_blocks(const AttendPlan &p, int B, int heads)
{
    return (int64_t)B * (heads / p.pack) * p.splits * p.blocks * (p.cols == 256 ? 2 : 1);
}

// LDS of the queries' gradient for the bias table's: a place an entry, and one more,
// of each of its 128 columns (or four waves' 32).
inline int attend_hist_bytes(int entries) { return 512 * (entries + 1); }

// entries: of the bias' table, 0 without one (the keys' gradient keeps none of them).
AttendPlan plan_attend(int B, int H, int Hk, int64_t Tq, int64_t Tk, int D, int dtype, int entries);
AttendPlan plan_attend_dq(int B, int H, int Hk, int64_t Tq, int64_t Tk, int D, int dtype,
                          int entries);
AttendPlan plan_attend_dkv(int B, int H, int Hk, int64_t Tq, int64_t Tk, int D, int dtype,
                           int entries);

// Launches of one element type.
hipError_t launch_attend_f32(const AttendK &k, int stage, hipStream_t stream);
hipError_t launch_attend_f16(const AttendK &k, int stage, hipStream_t stream);
hipError_t launch_attend_bf16(const AttendK &k, int stage, hipStream_t stream);
enum { kAttendForward, kAttendBackQ, kAttendBackKV };

inline int attend_elem(int dtype) { return dtype == 0 ? 4 : 2; }
// Head widths the kernels are built for: multiples of 32.
inline int attend_dim(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : D <= 96 ? 96 : 128; }

// Rows of a tile of the keys' gradient: 64 where two blocks of them still fit a CU's
// registers (two 720p views with two reference views each, 12 and 3 heads of 64, bf16:
// 399 us, with 32 rows 424; the queries' gradient, whose blocks are smaller, takes 303
// with 32 and 330 with 64).
constexpr int attend_kv_rows(int dim, int elem, bool shared)
{
    return !shared && elem == 2 && dim <= 64 ? 64 : 32;
}

}  // namespace mixrt
