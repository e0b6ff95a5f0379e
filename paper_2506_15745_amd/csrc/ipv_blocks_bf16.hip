// Attention over lists of blocks of bf16 pages.
#include "ipv_blocks_launch.hpp"

template hipError_t ipv::launch_attend_blocks<ipv::kFmtBf16>(int, bool, bool, const ipv::BlocksArgs&, hipStream_t);
