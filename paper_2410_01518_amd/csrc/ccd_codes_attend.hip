// ccd_paged_attend_codes: host side.  The kernels are compiled by kind of code (ccd_attend_int8.hip, ccd_attend_e4m3.hip).
#include "ccd_codes_launch.h"

namespace ccd {

size_t attend_codes_workspace_bytes(const Paged& P, const Codes&, int dtype, int max_new, int max_len) {
  return lay_out(P, plan_attend(P, dtype, true, max_new, max_len)).total;
}

void launch_attend_codes(const Paged& P, const Codes& C, int code, int dtype, int max_new, int max_len, const void* Q, const void* K, const void* V,
                         const float* K_scales, const float* V_scales, const int32_t* table, const int32_t* q_start, const int32_t* kv_len, void* out, float* lse,
                         void* workspace, hipStream_t s) {
  const AttendCuts c = plan_attend(P, dtype, true, max_new, max_len);
  const AttendSpace w = lay_out(P, c);
  char* ws = static_cast<char*>(workspace);
  AttendArgs even{Q, K, V, table, q_start, kv_len, out, lse,
                  {reinterpret_cast<float*>(ws + w.even_o), reinterpret_cast<float2*>(ws + w.even_ml), reinterpret_cast<int2*>(ws + w.meta)}, C, K_scales, V_scales};
  AttendArgs grid = even;
  grid.part = {reinterpret_cast<float*>(ws + w.grid_o), reinterpret_cast<float2*>(ws + w.grid_ml), nullptr};
  if (code == kInt8) launch_attend_int8(P, dtype, c, even, grid, s);
  else               launch_attend_e4m3(P, dtype, c, even, grid, s);
}

}  // namespace ccd
