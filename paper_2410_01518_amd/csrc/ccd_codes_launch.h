// Attention over codes: what its sources share.
#pragma once
#include "ccd_attend_launch.h"

namespace ccd {

void launch_attend_int8(const Paged& P, int dtype, const AttendCuts& c, const AttendArgs& even, const AttendArgs& grid, hipStream_t s);
void launch_attend_e4m3(const Paged& P, int dtype, const AttendCuts& c, const AttendArgs& even, const AttendArgs& grid, hipStream_t s);

template <int CODE>
static void launch_attend_of(const Paged& P, int dtype, const AttendCuts& c, const AttendArgs& even, const AttendArgs& grid, hipStream_t s) {
  if (dtype == 0 && P.d == 64) attend_launch<Coded<float, CODE>, 64>(P, c, even, grid, s);
  else if (dtype == 0)         attend_launch<Coded<float, CODE>, 128>(P, c, even, grid, s);
  else if (P.d == 64)          attend_launch<Coded<uint16_t, CODE>, 64>(P, c, even, grid, s);
  else                         attend_launch<Coded<uint16_t, CODE>, 128>(P, c, even, grid, s);
}

}  // namespace ccd
