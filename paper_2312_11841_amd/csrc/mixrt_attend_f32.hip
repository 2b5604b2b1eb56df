// The attention kernels for float heads.
#include "mixrt_attend_launch.hpp"

namespace mixrt {

hipError_t launch_attend_f32(const AttendK &k, int stage, hipStream_t stream)
{
    return launch_attend<float>(k, stage, stream);
}

}  // namespace mixrt
