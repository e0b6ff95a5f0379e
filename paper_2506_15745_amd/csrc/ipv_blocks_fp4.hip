// Attention over lists of blocks of e2m1 pages.
#include "ipv_blocks_launch.hpp"

template hipError_t ipv::launch_attend_blocks<ipv::kFmtFp4>(int, bool, bool, const ipv::BlocksArgs&, hipStream_t);
