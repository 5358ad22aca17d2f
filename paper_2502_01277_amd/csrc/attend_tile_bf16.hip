// The attention kernel for many rows, one storage type.
#include "attend_tile.h"

namespace octo {
hipError_t launch_attend_tile_bf16(int format, const AttendArgs& a, hipStream_t s) { return launch_attend_tile<__bf16>(format, a, s); }
}  // namespace octo
