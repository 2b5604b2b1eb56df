// The attention kernels for f16 heads.
#include "mixrt_attend_launch.hpp"

namespace mixrt {

hipError_t launch_attend_f16(const AttendK &k, int stage, hipStream_t stream)
{
    return launch_attend<f16>(k, stage, stream);
}

}  // namespace mixrt
