// Attention over lists of blocks of fp32 pages.
#include "ipv_blocks_launch.hpp"

template hipError_t ipv::launch_attend_blocks<ipv::kFmtF32>(int, bool, bool, const ipv::BlocksArgs&, hipStream_t);
