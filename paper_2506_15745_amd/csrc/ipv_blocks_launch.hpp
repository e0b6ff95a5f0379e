// The attention kernels over lists of one page format (included by one source file a format).
#pragma once

#include "ipv_blocks.hpp"

namespace ipv {

template <int F, int D>
hipError_t launch_attend_blocks_d(bool wide, bool solo, const BlocksArgs& a, hipStream_t st) {
  const uint32_t each = solo ? 8u * kFewWaves : 8u;
  const dim3 grid(((uint32_t)a.slots + each - 1u) / each * 8u), block(64 * kFewWaves);
  if constexpr (F == kFmtF32) {
    if (solo) k_attend_blocks_f32<D, true><<<grid, block, 0, st>>>(a);
    else k_attend_blocks_f32<D, false><<<grid, block, 0, st>>>(a);
  } else if (wide && solo) k_attend_blocks<F, D, 2, true><<<grid, block, 0, st>>>(a);
  else if (wide) k_attend_blocks<F, D, 2, false><<<grid, block, 0, st>>>(a);
  else if (solo) k_attend_blocks<F, D, 1, true><<<grid, block, 0, st>>>(a);
  else k_attend_blocks<F, D, 1, false><<<grid, block, 0, st>>>(a);
  return hipGetLastError();
}

template <int F>
hipError_t launch_attend_blocks(int D, bool wide, bool solo, const BlocksArgs& a, hipStream_t st) {
  switch (D) {
    case 32: return launch_attend_blocks_d<F, 32>(wide, solo, a, st);
    case 64: return launch_attend_blocks_d<F, 64>(wide, solo, a, st);
    case 128: return launch_attend_blocks_d<F, 128>(wide, solo, a, st);
    default: return launch_attend_blocks_d<F, 256>(wide, solo, a, st);
  }
}

}  // namespace ipv
