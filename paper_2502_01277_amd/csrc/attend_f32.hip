// The attention kernels of one storage type.
#include "attend.h"

namespace octo {
hipError_t launch_attend_direct_f32(int format, int how, const AttendArgs& a, hipStream_t s) { return launch_attend_direct<float>(format, how, a, s); }
}  // namespace octo
