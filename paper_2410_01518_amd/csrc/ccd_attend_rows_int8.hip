// Attention of many rows per unit over caches of int8 codes (ccd_attend_rows.h).
#include "ccd_attend_rows.h"

namespace ccd {

template <>
void launch_attend_rows<Coded<uint16_t, kInt8>>(const Paged& P, const AttendPlan& pl, const AttendArgs& A, const AttendPlan& even, const Partials& even_part, hipStream_t s) {
  launch_rows<Coded<uint16_t, kInt8>>(P, pl, A, even, even_part, s);
}

}  // namespace ccd
