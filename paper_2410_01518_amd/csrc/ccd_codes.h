// Caches in 8 bits: what the host hands to the kernels of ccd_paged_*_codes, and what a code stands for.
//
// int8: c * scale, a scale per token and head.  e4m3: c * scale, c a float of four bits of exponent and three of mantissa, the scale a
// power of two for every 2^shift tokens and head.  Both kinds of code are bf16 numbers exactly (8 bits of significand hold -127 .. 127; e4m3 has 4,
// down to 2^-9), so products of codes on the matrix cores are as exact as those of a bf16 cache.
#pragma once
#include "ccd_common.h"
#include "ccd_paged.h"
#include "ccd_rotary.h"

namespace ccd {

enum { kInt8 = 0, kE4m3 = 1 };
constexpr float kLeastScale = 7.52316384526264e-37f;        // 2^-120

struct Codes {
  int32_t shift;                                  // log2 of the tokens that share a scale
  int64_t page, head;                             // strides of the scales
  int64_t new_rows, new_b;                        // 0, or new tokens per batch of K_new and V_new and the batches' distance
};

// four codes of a word as floats
template <int CODE>
__device__ __forceinline__ void numbers(uint32_t w, float (&x)[4]) {
  if constexpr (CODE == kInt8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  } else {
    typedef float v2f __attribute__((ext_vector_type(2)));
    const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
  }
}
// one code as a float
template <int CODE>
__device__ __forceinline__ float number(uint8_t c) {
  if constexpr (CODE == kInt8) return (float)(int8_t)c;
  return __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
}

// The scale that rows of a largest finite |x| of `top` need.  int8: top / 127 rounded; e4m3: with top = m 2^e, 1 <= m < 2, and 448 = 1.75 * 2^8 the
// smallest power of two is 2^(e - 8) up to m = 1.75, else 2^(e - 7): worked out on the bits, exact.
template <int CODE>
__device__ __forceinline__ float scale_for(float top) {
  if constexpr (CODE == kInt8) {
    // (a product by the rounded 1 / 127 and one correction: the rounded quotient, for every fp32 number that is not clamped)
    const float q = top * (1.f / 127.f);
    return fmaxf(fmaf(fmaf(-q, 127.f, top), 1.f / 127.f, q), kLeastScale);
  }
  const uint32_t bits = __float_as_uint(top);
  const int e = (int)(bits >> 23) - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);          // biased
  return __uint_as_float((uint32_t)(e < 7 ? 7 : e) << 23);                                  // (7: 2^-120)
}
// The scale of a block that a call finds, as one that e4m3 codes are rounded to: the smallest power of two that is not below it, 2^120 at most (no fp32 number needs more; a scale
// from elsewhere may be any number), 0 where it is negative or none, as no row then reads as what a scale could keep.
__device__ __forceinline__ float power_of_two_scale(float scale) {
  const uint32_t bits = __float_as_uint(scale);
  return bits >= 0x7F800000u ? 0.f : fminf(__uint_as_float((bits + 0x7FFFFFu) & 0x7F800000u), 1.329227995784916e36f);
}
// 1 / scale: exact for a power of two, 2^-22 of it off at most otherwise (int8; e4m3 takes powers of two alone)
template <int CODE>
__device__ __forceinline__ float inverse_scale(float scale) {
  if constexpr (CODE == kInt8) return __builtin_amdgcn_rcpf(scale);
  return __uint_as_float(0x7F000000u - __float_as_uint(scale));
}

// x / scale as a code; inverse: of inverse_scale.  int8: the quotient by the inverse is within 2^-14 of the exact one, so the nearest whole number is
// found or missed by one, close to a half.  What is left over, x - c scale, is exact in fp32 (an integer below 2^24 of scale's last
// bit), and says which: less than half a scale is right.  Otherwise (eight_codes) the quotients are taken in 64 bits: 2^-43 off, rounded to 2^-40, so that a half is exactly one,
// where quotients that are no half are 2^-26 from one (x and scale have 24 bits).  e4m3: the quotient by a power of two is exact, and the conversion rounds to
// nearest even; no number lies above 448.
__device__ __forceinline__ uint32_t four_bytes(int a, int b, int c, int d) {
  return __builtin_amdgcn_perm((uint32_t)__builtin_amdgcn_perm((uint32_t)d, (uint32_t)c, 0x0c0c0400), (uint32_t)__builtin_amdgcn_perm((uint32_t)b, (uint32_t)a, 0x0c0c0400), 0x05040100);
}
// eight numbers as codes; fine: all are finite
template <int CODE>
__device__ __forceinline__ uint2 eight_codes(const float (&x)[8], float scale, float inverse, bool fine) {
  if constexpr (CODE == kInt8) {
    // (added to 3 2^22 a quotient is rounded to a whole number, whose byte is the sum's last one)
    float c[8], left = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      c[i] = fmaf(x[i], inverse, 12582912.f);
      left = fmaxf(left, fabsf(fmaf(12582912.f - c[i], scale, x[i])));
    }
    if (__builtin_expect(fine && left < 0.5f * scale, 1)) {
      auto byte = [&](int i) { return (int)__float_as_uint(c[i]); };
      return make_uint2(four_bytes(byte(0), byte(1), byte(2), byte(3)), four_bytes(byte(4), byte(5), byte(6), byte(7)));
    }
    // (infinite values and NaN end as 0: their row's scale says that they are no numbers)
    const double wide = (double)scale;
    double by = __builtin_amdgcn_rcp(wide);
    by = fma(fma(-wide, by, 1.0), by, by);
    by = fma(fma(-wide, by, 1.0), by, by);
    int k[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double q = fma((double)x[i], by, 6144.0) - 6144.0;                        // (1.5 2^12, 1.5 2^52: the sum's last bits)
      k[i] = (int)(uint32_t)__builtin_bit_cast(uint64_t, q + 6755399441055744.0);
    }
    return make_uint2(four_bytes(k[0], k[1], k[2], k[3]), four_bytes(k[4], k[5], k[6], k[7]));
  } else {
    int w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inverse, x[4 * i + 1] * inverse, 0, false);
      w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inverse, x[4 * i + 3] * inverse, w[i], true);
    }
    if (!fine) {                                             // (an infinite quotient has no e4m3 number: NaN, as for a NaN)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (!(fabsf(x[i]) < INFINITY)) w[i >> 2] = (w[i >> 2] & ~(0xFF << (8 * (i & 3)))) | (0x7F << (8 * (i & 3)));
    }
    return make_uint2((uint32_t)w[0], (uint32_t)w[1]);
  }
}

void launch_append_codes(const Paged& P, const Codes& C, int code, int dtype, const Rotary* rope, const void* K_new, const void* V_new, const int32_t* slots,
                         const int32_t* positions, const uint64_t* turns, void* K, void* V, float* K_scales, float* V_scales, hipStream_t s);
void launch_read_codes(const Paged& P, const Codes& C, int code, int dtype, const void* K, const void* V, const float* K_scales, const float* V_scales,
                       const int32_t* table, const int32_t* q_start, const int32_t* kv_len, void* K_out, void* V_out, hipStream_t s);
void launch_compact_codes(const Paged& P, const Codes& C, void* K, void* V, float* K_scales, float* V_scales, const int32_t* keep, int32_t k, float* novelty,
                          hipStream_t s);
size_t attend_codes_workspace_bytes(const Paged& P, const Codes& C, int dtype, int max_new, int max_len);
void launch_attend_codes(const Paged& P, const Codes& C, int code, int dtype, int max_new, int max_len, const void* Q, const void* K, const void* V,
                         const float* K_scales, const float* V_scales, const int32_t* table, const int32_t* q_start, const int32_t* kv_len, void* out, float* lse,
                         void* workspace, hipStream_t s);

}  // namespace ccd
