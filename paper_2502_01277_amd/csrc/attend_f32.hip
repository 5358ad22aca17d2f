// The attention kernels of one storage type.
#include "attend.h"

namespace octo {
hipError_t launch_attend_direct_f32(int format, int share, const AttendArgs& a, int row_blocks, hipStream_t s) { return launch_attend_direct<float>(format, share, a, row_blocks, s); }
}  // namespace octo
