// Paged caches: what the host hands to the kernels of ccd_paged_plan, ccd_rope, ccd_paged_append and ccd_paged_attend.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ccd {

// t / page for 0 <= t < 2^31 as one 64-bit product and a shift: mul = ceil(2^(31 + l) / page) with 2^(l-1) < page <= 2^l; the
// product exceeds t * 2^(31+l) / page by less than t / 2^31 < 1 of 2^(31+l) / page, so the quotient is exact.
struct PageDiv {
  uint32_t mul;
  int32_t shift, page;
};
inline PageDiv make_page_div(int32_t page) {
  int l = 0;
  while (((int64_t)1 << l) < page) ++l;
  const uint64_t one = (uint64_t)1 << (31 + l);
  return {(uint32_t)((one + (uint64_t)page - 1) / (uint64_t)page), 31 + l, page};
}
__device__ __forceinline__ int page_of(const PageDiv& p, int t) { return (int)(((uint64_t)(uint32_t)t * p.mul) >> p.shift); }

struct Paged {
  int32_t B, tokens, Hq, Hkv, G, d, n_pages, table_width;
  int32_t window, behind, max_len;        // max_len: tokens a row of the table can hold
  PageDiv div;
  float scale_log2;
  int64_t page_stride, head_stride, row_stride, new_t, new_h;
  int64_t q_b, q_t, q_h, o_b, o_t, o_h, l_b, l_t, l_h;
};

// the part of a rotary descriptor that the kernels read
struct Rotary {
  int32_t tokens, heads, d, rot, half, inverse;      // half: pairs (i, i + rot/2)
  float amplitude;
  int64_t x_t, x_h, y_t, y_h;
};

constexpr int kPlanMaxSequences = 4096;

void launch_paged_plan(const Paged& P, const int32_t* before, const int32_t* after, const int32_t* table, int32_t* table_next,
                       int32_t* ring, int32_t* cursor, int32_t* cursor_next, int32_t* q_start, int32_t* slots, int32_t* positions,
                       hipStream_t s);
void launch_rotary(const Rotary& R, int dtype, const void* X, const int32_t* positions, const uint64_t* turns, void* Y, hipStream_t s);
// rope: null, or rot, half, inverse and amplitude of the keys' embedding
void launch_paged_append(const Paged& P, int dtype, const Rotary* rope, const void* K_new, const void* V_new, const int32_t* slots,
                         const int32_t* positions, const uint64_t* turns, void* K, void* V, hipStream_t s);
size_t attend_workspace_bytes(const Paged& P, int dtype, int max_new, int max_len);
void launch_attend(const Paged& P, int dtype, int max_new, int max_len, const void* Q, const void* K, const void* V, const int32_t* table,
                   const int32_t* q_start, const int32_t* kv_len, void* out, float* lse, void* workspace, hipStream_t s);

}  // namespace ccd
