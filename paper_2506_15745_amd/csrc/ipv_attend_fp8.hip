// Attention over fp8 pages.
#include "ipv_attend_launch.hpp"

template hipError_t ipv::launch_attend<ipv::kFmtFp8>(int, ipv::AttendKind, uint32_t, const ipv::AttendArgs&, hipStream_t);
