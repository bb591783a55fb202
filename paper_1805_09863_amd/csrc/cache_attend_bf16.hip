#include "cache_attend.hpp"

namespace kb {
hipError_t launch_cache_attend_bf16(const AttendArgs& a, hipStream_t st) { return launch_attend_dim<__bf16>(a, st); }
}  // namespace kb
