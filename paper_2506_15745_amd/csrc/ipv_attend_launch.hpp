// The attention kernels of one page format (included by one source file a format).
#pragma once

#include "ipv_attend.hpp"

namespace ipv {

template <int F, int D, bool WHOLE>
void launch_attend_w(AttendKind kind, uint32_t grid, const AttendArgs& a, hipStream_t st) {
  if constexpr (F == kFmtF32) k_attend_f32<D, WHOLE><<<dim3(grid), dim3(64 * kFewWaves), 0, st>>>(a);
  else if (kind == kFew1) k_attend_few<F, D, 1, WHOLE><<<dim3(grid), dim3(64 * kFewWaves), 0, st>>>(a);
  else if (kind == kFew2) k_attend_few<F, D, 2, WHOLE><<<dim3(grid), dim3(64 * kFewWaves), 0, st>>>(a);
  else k_attend_tile<F, D, WHOLE><<<dim3(grid), dim3(64 * tile_waves(D)), 0, st>>>(a);
}

template <int F, int D>
hipError_t launch_attend_d(AttendKind kind, uint32_t grid, const AttendArgs& a, hipStream_t st) {
  if (a.pool.T.d % (uint32_t)attend_keys(kind) == 0) launch_attend_w<F, D, true>(kind, grid, a, st);
  else launch_attend_w<F, D, false>(kind, grid, a, st);
  return hipGetLastError();
}

template <int F>
hipError_t launch_attend(int D, AttendKind kind, uint32_t grid, const AttendArgs& a, hipStream_t st) {
  switch (D) {
    case 32: return launch_attend_d<F, 32>(kind, grid, a, st);
    case 64: return launch_attend_d<F, 64>(kind, grid, a, st);
    case 128: return launch_attend_d<F, 128>(kind, grid, a, st);
    default: return launch_attend_d<F, 256>(kind, grid, a, st);
  }
}

}  // namespace ipv
