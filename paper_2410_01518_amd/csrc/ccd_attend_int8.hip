// Attention over int8 codes: kernels of few rows per unit and of fp32 queries.
#include "ccd_codes_launch.h"

namespace ccd {

void launch_attend_int8(const Paged& P, int dtype, const AttendCuts& c, const AttendArgs& even, const AttendArgs& grid, hipStream_t s) {
  launch_attend_of<kInt8>(P, dtype, c, even, grid, s);
}

}  // namespace ccd
