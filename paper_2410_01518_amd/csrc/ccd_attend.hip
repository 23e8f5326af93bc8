// ccd_paged_attend: attention of a step's new tokens over the pages of their sequences.
//
//   out = sum_t w_t v_t / sum_t w_t,   w_t = 2^(scale log2(e) <q, k_t> - m)
// in one pass over the tokens: m is a running reference, and when it rises the sums so far are scaled down by 2^(old - new).
#include "ccd_common.h"
#include "ccd_paged.h"
#include "ccd_rotary.h"

namespace ccd {

// one wave per (new token, query head)
template <class T, int D>
__global__ __launch_bounds__(64) void attend_row_kernel(Paged P, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
                                                        const int32_t* __restrict__ table, const int32_t* __restrict__ q_start,
                                                        const int32_t* __restrict__ kv_len, T* __restrict__ out, float* __restrict__ lse) {
  const int r = blockIdx.x / P.Hq, hq = blockIdx.x % P.Hq, lane = threadIdx.x;
  int lo = 0, hi = P.B;
  if (r < q_start[0] || r >= q_start[P.B]) return;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (q_start[mid] <= r) lo = mid; else hi = mid;
  }
  const int b = lo, i = r - q_start[b], m = q_start[b + 1] - q_start[b];
  int n = kv_len[b];
  n = n < 0 ? 0 : n < P.max_len ? n : P.max_len;
  const int pos = (P.behind ? n : n - m) + i;
  const int end = pos + 1 < n ? pos + 1 : n;
  const int begin = P.window > 0 && pos - P.window + 1 > 0 ? pos - P.window + 1 : 0;
  const int64_t head = (int64_t)(hq / P.G) * P.head_stride;
  const T* q = Q + b * P.q_b + r * P.q_t + hq * P.q_h;
  float top = -INFINITY, sum = 0.f, acc[D / 64] = {};
  for (int t0 = begin; t0 < end; t0 += 64) {
    const int t = t0 + lane;
    int64_t row = -1;
    if (t < end) {
      const int c = page_of(P.div, t), id = table[(int64_t)b * P.table_width + c];
      if (id >= 0 && id < P.n_pages) row = id * P.page_stride + head + (int64_t)(t - c * P.div.page) * P.row_stride;
    }
    float x = -INFINITY;
    if (row >= 0) {
      float s = 0.f;
      for (int e = 0; e < D; e += 4) {
        const float4 a = load4(q + e), k = load4(K + row + e);
        s = fmaf(a.x, k.x, fmaf(a.y, k.y, fmaf(a.z, k.z, fmaf(a.w, k.w, s))));
      }
      x = s * P.scale_log2;
    }
    float mx = x;
    for (int o = 32; o; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o));
    if (mx == -INFINITY) continue;
    const float next = fmaxf(top, mx), w = row >= 0 ? exp2f(x - next) : 0.f, keep = exp2f(top - next);
    top = next;
    sum = sum * keep + w;
    for (int j = 0; j < D / 64; ++j) acc[j] *= keep;
    for (int l = 0; l < 64; ++l) {
      const int64_t vrow = __shfl(row, l);
      const float wl = __shfl(w, l);
      if (vrow < 0) continue;
      for (int j = 0; j < D / 64; ++j) acc[j] = fmaf(wl, load_elem(V + vrow + j * 64 + lane), acc[j]);
    }
  }
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
  const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
  T* o = out + b * P.o_b + r * P.o_t + hq * P.o_h;
  for (int j = 0; j < D / 64; ++j) store_elem(o + j * 64 + lane, acc[j] * inv);
  if (lse != nullptr && lane == 0)
    lse[b * P.l_b + r * P.l_t + hq * P.l_h] = sum > 0.f ? (top + log2f(sum)) * 0.6931471805599453f : sum == sum ? -INFINITY : sum;
}

size_t attend_workspace_bytes(const Paged&, int, int, int) { return 256; }

void launch_attend(const Paged& P, int dtype, int max_new, int max_len, const void* Q, const void* K, const void* V, const int32_t* table,
                   const int32_t* q_start, const int32_t* kv_len, void* out, float* lse, void* workspace, hipStream_t s) {
  const dim3 grid((unsigned)(P.tokens * P.Hq)), block(64);
  if (dtype == 0) {
    const float *q = static_cast<const float*>(Q), *k = static_cast<const float*>(K), *v = static_cast<const float*>(V);
    float* o = static_cast<float*>(out);
    if (P.d == 64) launch(attend_row_kernel<float, 64>, grid, block, s, P, q, k, v, table, q_start, kv_len, o, lse);
    else           launch(attend_row_kernel<float, 128>, grid, block, s, P, q, k, v, table, q_start, kv_len, o, lse);
  } else {
    const uint16_t *q = static_cast<const uint16_t*>(Q), *k = static_cast<const uint16_t*>(K), *v = static_cast<const uint16_t*>(V);
    uint16_t* o = static_cast<uint16_t*>(out);
    if (P.d == 64) launch(attend_row_kernel<uint16_t, 64>, grid, block, s, P, q, k, v, table, q_start, kv_len, o, lse);
    else           launch(attend_row_kernel<uint16_t, 128>, grid, block, s, P, q, k, v, table, q_start, kv_len, o, lse);
  }
}

}  // namespace ccd
