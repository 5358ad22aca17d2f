// The attention kernels of one storage type.
#include "attend.h"

namespace octo {
hipError_t launch_attend_direct_bf16(int format, int how, const AttendArgs& a, hipStream_t s) { return launch_attend_direct<__bf16>(format, how, a, s); }
}  // namespace octo
