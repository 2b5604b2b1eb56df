// One element type's attention launches by the heads' padded width.
#pragma once

#include <type_traits>

#include "mixrt_attend_forward.hpp"

#include "mixrt_attend_backward.hpp"

namespace mixrt {
namespace {

template <typename T>
hipError_t launch_attend(AttendK k, int stage, hipStream_t stream)
{
    auto plan = stage == kAttendForward ? plan_attend
                : stage == kAttendBackQ ? plan_attend_dq
                                        : plan_attend_dkv;
    const AttendPlan p = plan(k.B, k.H, k.Hk, k.Tq, k.Tk, k.D, k.dtype,
                              k.bias.axes * k.bias.buckets);
    k.pack = p.pack;
    k.blocks = p.blocks;
    k.splits = p.splits;
    k.per = p.per;
    k.slots = attend_slots(p);
    auto go = [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        hipError_t e = hipSuccess;
        for (k.pass = 0; k.pass < p.passes && e == hipSuccess; ++k.pass) {
            k.from = k.pass * p.splits * p.per;
            k.parts = p.splits + (k.pass > 0);
            k.last = k.pass + 1 == p.passes;
            e = stage == kAttendForward ? launch_forward<T, DP>(k, p, stream)
                : stage == kAttendBackQ ? launch_back_q<T, DP>(k, p, stream)
                                        : launch_back_kv<T, DP>(k, p, stream);
        }
        return e;
    };
    switch (attend_dim(k.D)) {
    case 32: return go(std::integral_constant<int, 32>());
    case 64: return go(std::integral_constant<int, 64>());
    case 96: return go(std::integral_constant<int, 96>());
    default: return go(std::integral_constant<int, 128>());
    }
}

}  // namespace
}  // namespace mixrt
