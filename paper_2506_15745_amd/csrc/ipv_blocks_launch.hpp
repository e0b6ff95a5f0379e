// The attention kernels over lists of one page format (included by one source file a format).
#pragma once

#include "ipv_blocks.hpp"

namespace ipv {

template <int F, int D>
hipError_t launch_attend_blocks_d(bool wide, uint32_t grid, const BlocksArgs& a, hipStream_t st) {
  if constexpr (F == kFmtF32) k_attend_blocks_f32<D><<<dim3(grid), dim3(64 * kFewWaves), 0, st>>>(a);
  else if (wide) k_attend_blocks<F, D, 2><<<dim3(grid), dim3(64 * kFewWaves), 0, st>>>(a);
  else k_attend_blocks<F, D, 1><<<dim3(grid), dim3(64 * kFewWaves), 0, st>>>(a);
  return hipGetLastError();
}

template <int F>
hipError_t launch_attend_blocks(int D, bool wide, uint32_t grid, const BlocksArgs& a, hipStream_t st) {
  switch (D) {
    case 32: return launch_attend_blocks_d<F, 32>(wide, grid, a, st);
    case 64: return launch_attend_blocks_d<F, 64>(wide, grid, a, st);
    case 128: return launch_attend_blocks_d<F, 128>(wide, grid, a, st);
    default: return launch_attend_blocks_d<F, 256>(wide, grid, a, st);
  }
}

}  // namespace ipv
