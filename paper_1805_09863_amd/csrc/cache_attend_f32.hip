#include "cache_attend.hpp"

namespace kb {
hipError_t launch_cache_attend_f32(const AttendArgs& a, hipStream_t st) { return launch_attend_dim<float>(a, st); }
}  // namespace kb
