// Attention of many rows per unit over bf16 caches (ccd_attend_rows.h).
#include "ccd_attend_rows.h"

namespace ccd {

template <>
void launch_attend_rows<uint16_t>(const Paged& P, const AttendPlan& pl, const AttendArgs& A, const AttendPlan& even, const Partials& even_part, hipStream_t s) {
  launch_rows<uint16_t>(P, pl, A, even, even_part, s);
}

}  // namespace ccd
