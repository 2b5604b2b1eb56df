// The attention kernels for bf16 heads.
#include "mixrt_attend_launch.hpp"

namespace mixrt {

hipError_t launch_attend_bf16(const AttendK &k, int stage, hipStream_t stream)
{
    return launch_attend<bf16>(k, stage, stream);
}

}  // namespace mixrt
