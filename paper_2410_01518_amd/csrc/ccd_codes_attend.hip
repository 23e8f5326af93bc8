// ccd_paged_attend_codes.
#include "ccd_attend.h"
#include "ccd_codes.h"

namespace ccd {

// A wave per row, 64 tokens at a time: a lane has the logit of one of them, and then d / 64 elements of the sums.
template <class T, int CODE, int D>
__global__ __launch_bounds__(256) void attend_codes_kernel(Paged P, Codes C, AttendArgs A, const float* __restrict__ K_scales, const float* __restrict__ V_scales) {
  constexpr int kPer = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t at0 = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int row = (int)(at0 / P.Hq), head = (int)(at0 % P.Hq), hkv = head / P.G;
  if (row >= P.tokens) return;
  int b = 0;                                                          // sequences that end at or before the row: counted, no chain of loads
  for (int b0 = 1; b0 <= P.B; b0 += 64) b += __popcll(__ballot(b0 + lane <= P.B && A.q_start[b0 + lane <= P.B ? b0 + lane : P.B] <= row));
  if (b >= P.B || row < A.q_start[0]) return;
  const Sequence sq = load_sequence(P, b, A.q_start, A.kv_len);
  const int i = row - sq.first, pos = sq.base + i, low = first_seen(P, pos);
  if (i < 0 || i >= sq.m) return;
  const int32_t* pages = A.table + (int64_t)b * P.table_width;
  const uint8_t* K = static_cast<const uint8_t*>(A.K) + hkv * P.head_stride;
  const uint8_t* V = static_cast<const uint8_t*>(A.V) + hkv * P.head_stride;
  const T* from = static_cast<const T*>(A.Q) + b * P.q_b + row * P.q_t + head * P.q_h;
  auto of_lane = [](float x, int u) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), u)); };
  float q[kPer], m = -INFINITY, l = 0.f, o[kPer] = {};
#pragma unroll
  for (int j = 0; j < kPer; ++j) q[j] = load_elem(from + j * 64 + lane);
  const int end = pos + 1 < sq.n ? pos + 1 : sq.n;
  for (int t0 = low; t0 < end; t0 += 64) {
    int64_t off = -1;                                                 // of token t0 + lane
    float ks = 0.f, vs = 0.f, x = 0.f;
    if (t0 + lane < end) {
      const int t = t0 + lane, c = page_of(P.div, t), id = pages[c], r = t - c * P.div.page;
      if (id >= 0 && id < P.n_pages) {
        off = id * P.page_stride + r * P.row_stride;
        const int64_t s = id * C.page + hkv * C.head + (r >> C.shift);
        ks = K_scales[s];
        vs = V_scales[s];
      }
    }
    const uint8_t* k = off >= 0 ? K + off : reinterpret_cast<const uint8_t*>(g_zero_row);
#pragma unroll
    for (int j = 0; j < kPer; ++j)
#pragma unroll 4
      for (int p = 0; p < 64; p += 4) {
        float y[4];
        numbers<CODE>(*reinterpret_cast<const uint32_t*>(k + j * 64 + p), y);
#pragma unroll
        for (int e = 0; e < 4; ++e) x = fmaf(of_lane(q[j], p + e), y[e], x);
      }
    x = off >= 0 ? x * (ks * P.scale_log2) : -INFINITY;
    float next = fmaxf(m, x);
#pragma unroll
    for (int s = 32; s; s >>= 1) next = fmaxf(next, __shfl_xor(next, s));
    const float keep = next == -INFINITY ? 1.f : fast_exp2(m - next), w = fast_exp2(x - (next == -INFINITY ? 0.f : next));
    m = next;
    l = l * keep + w;
    const float weight = off >= 0 ? w * vs : 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) o[j] *= keep;
    for (int u = 0; u < 64 && t0 + u < end; ++u) {
      const int64_t at = (int64_t)__builtin_amdgcn_readlane((int)(off >> 32), u) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)off, u);
      const uint8_t* v = at >= 0 ? V + at : reinterpret_cast<const uint8_t*>(g_zero_row);
#pragma unroll
      for (int j = 0; j < kPer; ++j) o[j] = fmaf(of_lane(weight, u), number<CODE>(v[j * 64 + lane]), o[j]);
    }
  }
#pragma unroll
  for (int s = 32; s; s >>= 1) l += __shfl_xor(l, s);
  const float inv = inverse_sum(l);
#pragma unroll
  for (int j = 0; j < kPer; ++j) store_elem(static_cast<T*>(A.out) + b * P.o_b + row * P.o_t + head * P.o_h + j * 64 + lane, o[j] * inv);
  if (A.lse != nullptr && lane == 0) A.lse[b * P.l_b + row * P.l_t + head * P.l_h] = to_natural_lse(m, l);
}

size_t attend_codes_workspace_bytes(const Paged&, const Codes&, int, int, int) { return 256; }

template <class T, int CODE>
static void attend_of(const Paged& P, const Codes& C, const AttendArgs& A, const float* K_scales, const float* V_scales, hipStream_t s) {
  const dim3 wgs((unsigned)(((int64_t)P.tokens * P.Hq + 3) / 4));
  if (P.d == 64) launch(attend_codes_kernel<T, CODE, 64>, wgs, dim3(256), s, P, C, A, K_scales, V_scales);
  else           launch(attend_codes_kernel<T, CODE, 128>, wgs, dim3(256), s, P, C, A, K_scales, V_scales);
}

void launch_attend_codes(const Paged& P, const Codes& C, int code, int dtype, int, int, const void* Q, const void* K, const void* V, const float* K_scales,
                         const float* V_scales, const int32_t* table, const int32_t* q_start, const int32_t* kv_len, void* out, float* lse, void*, hipStream_t s) {
  const AttendArgs A{Q, K, V, table, q_start, kv_len, out, lse, {}};
  auto of = dtype == 0 ? (code == kInt8 ? attend_of<float, kInt8> : attend_of<float, kE4m3>) : (code == kInt8 ? attend_of<uint16_t, kInt8> : attend_of<uint16_t, kE4m3>);
  of(P, C, A, K_scales, V_scales, s);
}

}  // namespace ccd
