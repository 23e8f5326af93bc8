// Rows of a cache in 8 bits: ccd_paged_append_codes, ccd_paged_read_codes, ccd_paged_compact_codes.
#include "ccd_codes.h"

namespace ccd {

// A row (one token and head) is D / 8 lanes wide, eight elements a lane.
constexpr int kPer = 8;

__device__ __forceinline__ void load_eight(const float* p, float (&x)[kPer]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load_eight(const uint16_t* p, float (&x)[kPer]) { load_f32(*reinterpret_cast<const v4u*>(p), x, p); }
__device__ __forceinline__ void store_eight(float* p, const float (&x)[kPer]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store_eight(uint16_t* p, const float (&x)[kPer]) { *reinterpret_cast<v4u*>(p) = store_bits(x, p); }

template <int CODE>
__device__ __forceinline__ uint2 eight_codes(const float (&x)[kPer], float scale, float inverse) {
  const float a[4] = {x[0], x[1], x[2], x[3]}, b[4] = {x[4], x[5], x[6], x[7]};
  return make_uint2(four_codes<CODE>(a, scale, inverse), four_codes<CODE>(b, scale, inverse));
}
template <int CODE>
__device__ __forceinline__ void eight_numbers(uint2 w, float scale, float (&x)[kPer]) {
  float a[4], b[4];
  numbers<CODE>(w.x, a);
  numbers<CODE>(w.y, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i] * scale; x[4 + i] = b[i] * scale; }
}

// The rotation of a lane's eight elements of a token: y = c x + s z, z being each one's partner in its pair.
template <class T>
struct TurnEight {
  float c[kPer], s[kPer];
  __device__ __forceinline__ void angles(const Rotary& R, int e0, int position, const uint64_t* __restrict__ turns) {
    const int pairs = R.rot / 2;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int e = e0 + j;
      c[j] = 1.f;
      s[j] = 0.f;
      if (e >= R.rot) continue;
      const bool first = R.half ? e < pairs : (e & 1) == 0;
      cos_sin_of_phase((uint64_t)(uint32_t)position * turns[R.half ? (first ? e : e - pairs) : e >> 1], c[j], s[j]);
      c[j] *= R.amplitude;
      s[j] *= first == (R.inverse == 0) ? -R.amplitude : R.amplitude;
    }
  }
  // row: the head's first element
  __device__ __forceinline__ void turn(const Rotary& R, const T* row, int e0, float (&x)[kPer]) const {
    if (e0 >= R.rot) return;
    float z[kPer];
    const int pairs = R.rot / 2;
    if (!R.half) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) z[j] = x[j ^ 1];
    } else if (pairs % kPer == 0) {
      load_eight(row + (e0 < pairs ? e0 + pairs : e0 - pairs), z);
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j) z[j] = e0 + j < R.rot ? load_elem(row + (e0 + j < pairs ? e0 + j + pairs : e0 + j - pairs)) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) x[j] = fmaf(z[j], s[j], x[j] * c[j]);
  }
};

// the largest finite |x|, and whether all are finite
__device__ __forceinline__ void measure(const float (&x)[kPer], float& top, bool& fine) {
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const float a = fabsf(x[j]);
    const bool ok = a < INFINITY;
    top = fmaxf(top, ok ? a : 0.f);
    fine = fine && ok;
  }
}

// A wave per token that begins a block's new rows (scale_rows = 1: per token), keys or values: for four or eight heads at a time the largest element of the
// rows, then their codes.
template <class T, int CODE, int D>
__global__ __launch_bounds__(256) void append_codes_kernel(Paged P, Codes C, Rotary R, bool rope, const T* __restrict__ K_new, const T* __restrict__ V_new,
                                                           const int32_t* __restrict__ slots, const int32_t* __restrict__ positions,
                                                           const uint64_t* __restrict__ turns, uint8_t* K, uint8_t* V, float* K_scales, float* V_scales) {
  constexpr int kLanes = D / kPer, kHeads = 64 / kLanes;
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, e0 = lane % kLanes * kPer;
  if (t >= P.tokens) return;
  const bool keys = blockIdx.y == 0, turned = keys && rope;
  const int rows = 1 << C.shift;
  const int64_t slots_all = (int64_t)P.div.page * P.n_pages;
  auto slot_of = [&](int i) { return i < 0 || i >= P.tokens || (rope && positions[i] < 0) || slots[i] >= slots_all ? -1 : slots[i]; };
  const int slot = slot_of(t);
  if (slot < 0) return;
  const int block = slot >> C.shift;
  int last = t + 1, first = slot;                     // the block's new tokens t .. last - 1, and the lowest of their rows
  if (rows > 1) {
    const int before = slot_of(t - 1);
    if (before >= 0 && before >> C.shift == block) return;
    for (int next = slot_of(last); next >= 0 && next >> C.shift == block; next = slot_of(++last)) first = next < first ? next : first;
  }
  const int page = page_of(P.div, slot), at0 = (block << C.shift) - page * P.div.page;       // the block's first row in the page
  const bool anew = first == block << C.shift;
  const T* from = keys ? K_new : V_new;
  uint8_t* to = (keys ? K : V) + page * P.page_stride;
  float* scales = (keys ? K_scales : V_scales) + page * C.page + (at0 >> C.shift);
  auto row_of = [&](int i, int h) {
    const int64_t b = C.new_rows > 0 ? i / C.new_rows : 0, r = C.new_rows > 0 ? i - b * C.new_rows : i;
    return from + b * C.new_b + r * P.new_t + h * P.new_h;
  };
  for (int h0 = 0; h0 < P.Hkv; h0 += kHeads) {
    const int h = h0 + lane / kLanes;
    const bool there = h < P.Hkv;
    float top = 0.f, x[kPer];
    bool fine = true;
    TurnEight<T> turn;
    auto load = [&](int i) {
      if (!there) return;
      if (turned) turn.angles(R, e0, positions[i], turns);
      load_eight(row_of(i, h) + e0, x);
      if (turned) turn.turn(R, row_of(i, h), e0, x);
    };
    for (int i = t; i < last; ++i) {
      load(i);
      if (there) measure(x, top, fine);
    }
#pragma unroll
    for (int s = 1; s < kLanes; s <<= 1) {
      top = fmaxf(top, __shfl_xor(top, s));
      if (CODE == kInt8) fine = __shfl_xor((int)fine, s) && fine;
    }
    if (!there) continue;
    float scale = scale_for<CODE>(top);
    const float old = anew ? 0.f : scales[h * C.head];
    if (!anew) scale = fmaxf(old, scale);
    const float inverse = 1.f / scale;
    uint8_t* head = to + h * P.head_stride + e0;
    if (!anew && scale > old)
      for (int r = block << C.shift; r < first; ++r) {
        uint2* p = reinterpret_cast<uint2*>(head + (int64_t)(r - page * P.div.page) * P.row_stride);
        float y[kPer];
        eight_numbers<CODE>(*p, old, y);
        *p = eight_codes<CODE>(y, scale, inverse);
      }
    for (int i = t; i < last; ++i) {
      if (rows > 1) load(i);
      *reinterpret_cast<uint2*>(head + (int64_t)(slots[i] - page * P.div.page) * P.row_stride) = eight_codes<CODE>(x, scale, inverse);
    }
    if (e0 == 0) scales[h * C.head] = CODE == kInt8 && !fine ? __uint_as_float(0x7FC00000u) : scale;
  }
}

// a wave per row of K_out and V_out
template <class T, int CODE, int D>
__global__ __launch_bounds__(256) void read_codes_kernel(Paged P, Codes C, const uint8_t* __restrict__ K, const uint8_t* __restrict__ V, const float* __restrict__ K_scales,
                                                         const float* __restrict__ V_scales, const int32_t* __restrict__ table, const int32_t* __restrict__ q_start,
                                                         const int32_t* __restrict__ kv_len, T* K_out, T* V_out) {
  constexpr int kLanes = D / kPer, kHeads = 64 / kLanes;
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, e0 = lane % kLanes * kPer;
  if (row >= P.tokens) return;
  int b = 0;                                                                // sequences that end at or before the row: counted, no chain of loads
  for (int b0 = 1; b0 <= P.B; b0 += 64) b += __popcll(__ballot(b0 + lane <= P.B && q_start[b0 + lane <= P.B ? b0 + lane : P.B] <= row));
  if (b >= P.B || row < q_start[0]) return;
  int n = kv_len[b];
  n = n < 0 ? 0 : n < P.max_len ? n : P.max_len;
  const int64_t t = (int64_t)n - q_start[b + 1] + row;                      // the token's position
  int page = -1, at = 0;
  if (t >= 0 && t < n) {
    const int c = page_of(P.div, (int)t), id = table[(int64_t)b * P.table_width + c];
    at = (int)t - c * P.div.page;
    page = id >= 0 && id < P.n_pages ? id : -1;
  }
  auto side = [&](const uint8_t* X, const float* scales, T* out) {
    for (int h = lane / kLanes; h < P.Hkv; h += kHeads) {
      float x[kPer] = {};
      if (page >= 0) {
        const uint2 w = *reinterpret_cast<const uint2*>(X + page * P.page_stride + h * P.head_stride + at * P.row_stride + e0);
        eight_numbers<CODE>(w, scales[page * C.page + h * C.head + (at >> C.shift)], x);
      }
      store_eight(out + b * P.o_b + row * P.o_t + h * P.o_h + e0, x);
    }
  };
  if (K_out != nullptr) side(K, K_scales, K_out);
  if (V_out != nullptr) side(V, V_scales, V_out);
}

// A workgroup per (page, head).  Rows move towards the front: row j comes from keep[j] >= j, so a piece of rows may be written once it has been read, and what later pieces
// read lies behind it.
template <int D>
__global__ __launch_bounds__(256) void compact_codes_kernel(Paged P, Codes C, uint8_t* K, uint8_t* V, float* K_scales, float* V_scales, const int32_t* __restrict__ keep_all,
                                                            int k, float* novelty) {
  constexpr int kLanes = D / 16, kRows = 256 / kLanes;
  const int page = blockIdx.x / P.Hkv, h = blockIdx.x % P.Hkv;
  const int32_t* keep = keep_all + (int64_t)blockIdx.x * k;
  uint8_t* Kh = K + page * P.page_stride + h * P.head_stride;
  uint8_t* Vh = V + page * P.page_stride + h * P.head_stride;
  float* ks = K_scales + page * C.page + h * C.head;
  float* vs = V_scales + page * C.page + h * C.head;
  float* nov = novelty != nullptr ? novelty + (int64_t)blockIdx.x * P.div.page : nullptr;
  const int tid = threadIdx.x, e0 = tid % kLanes * 16;
  for (int j0 = 0; j0 < k; j0 += kRows) {
    const int j = j0 + tid / kLanes, i = j < k ? keep[j] : -1;
    const bool moves = i >= 0 && i < P.div.page && i != j;
    v4u a = {}, b = {};
    float x = 0.f, y = 0.f, z = 0.f;
    if (moves) {
      a = *reinterpret_cast<const v4u*>(Kh + i * P.row_stride + e0);
      b = *reinterpret_cast<const v4u*>(Vh + i * P.row_stride + e0);
      if (e0 == 0) { x = ks[i]; y = vs[i]; z = nov != nullptr ? nov[i] : 0.f; }
    }
    asm volatile("" ::"v"(a), "v"(b), "v"(x), "v"(y), "v"(z));          // (read, not just asked for)
    __syncthreads();
    if (moves) {
      *reinterpret_cast<v4u*>(Kh + j * P.row_stride + e0) = a;
      *reinterpret_cast<v4u*>(Vh + j * P.row_stride + e0) = b;
      if (e0 == 0) {
        ks[j] = x;
        vs[j] = y;
        if (nov != nullptr) nov[j] = z;
      }
    }
  }
}

template <class T, int CODE>
static void append_of(const Paged& P, const Codes& C, const Rotary* rope, const void* K_new, const void* V_new, const int32_t* slots, const int32_t* positions,
                      const uint64_t* turns, void* K, void* V, float* K_scales, float* V_scales, hipStream_t s) {
  const dim3 wgs((P.tokens + 3) / 4, 2);
  launch(P.d == 64 ? append_codes_kernel<T, CODE, 64> : append_codes_kernel<T, CODE, 128>, wgs, dim3(256), s, P, C, rope ? *rope : Rotary{}, rope != nullptr,
         static_cast<const T*>(K_new), static_cast<const T*>(V_new), slots, positions, turns, static_cast<uint8_t*>(K), static_cast<uint8_t*>(V), K_scales, V_scales);
}

void launch_append_codes(const Paged& P, const Codes& C, int code, int dtype, const Rotary* rope, const void* K_new, const void* V_new, const int32_t* slots,
                         const int32_t* positions, const uint64_t* turns, void* K, void* V, float* K_scales, float* V_scales, hipStream_t s) {
  auto of = dtype == 0 ? (code == kInt8 ? append_of<float, kInt8> : append_of<float, kE4m3>) : (code == kInt8 ? append_of<uint16_t, kInt8> : append_of<uint16_t, kE4m3>);
  of(P, C, rope, K_new, V_new, slots, positions, turns, K, V, K_scales, V_scales, s);
}

template <class T, int CODE>
static void read_of(const Paged& P, const Codes& C, const void* K, const void* V, const float* K_scales, const float* V_scales, const int32_t* table,
                    const int32_t* q_start, const int32_t* kv_len, void* K_out, void* V_out, hipStream_t s) {
  launch(P.d == 64 ? read_codes_kernel<T, CODE, 64> : read_codes_kernel<T, CODE, 128>, dim3((P.tokens + 3) / 4), dim3(256), s, P, C, static_cast<const uint8_t*>(K),
         static_cast<const uint8_t*>(V), K_scales, V_scales, table, q_start, kv_len, static_cast<T*>(K_out), static_cast<T*>(V_out));
}

void launch_read_codes(const Paged& P, const Codes& C, int code, int dtype, const void* K, const void* V, const float* K_scales, const float* V_scales,
                       const int32_t* table, const int32_t* q_start, const int32_t* kv_len, void* K_out, void* V_out, hipStream_t s) {
  auto of = dtype == 0 ? (code == kInt8 ? read_of<float, kInt8> : read_of<float, kE4m3>) : (code == kInt8 ? read_of<uint16_t, kInt8> : read_of<uint16_t, kE4m3>);
  of(P, C, K, V, K_scales, V_scales, table, q_start, kv_len, K_out, V_out, s);
}

void launch_compact_codes(const Paged& P, const Codes& C, void* K, void* V, float* K_scales, float* V_scales, const int32_t* keep, int32_t k, float* novelty,
                          hipStream_t s) {
  launch(P.d == 64 ? compact_codes_kernel<64> : compact_codes_kernel<128>, dim3((unsigned)(P.n_pages * P.Hkv)), dim3(256), s, P, C, static_cast<uint8_t*>(K),
         static_cast<uint8_t*>(V), K_scales, V_scales, keep, k, novelty);
}

}  // namespace ccd
