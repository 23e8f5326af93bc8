// Rotary positions, device side: the angle of a position as a 64-bit fraction of a turn, its cosine and sine, and the
// rotation of 16 bytes of a head.
//
// turns = frequency / 2 pi in units of 2^-64 turn.  position * turns modulo 2^64 is the angle with the whole turns gone: the
// product of two integers loses nothing, at position 10^9 no more than at 1.  (As a product of floats the angle of a fast
// pair at position 10^6 is off by 0.06 radian in fp32.)
#pragma once
#include "ccd_common.h"
#include "ccd_rope.h"

namespace ccd {

// cosine and sine of a phase: the nearest quarter turn is taken off (exact, the phase is an integer), the rest lies within
// an eighth of a turn, |x| <= pi/4, where the Taylor sums up to x^10 (cosine) and x^11 (sine) stop 1.2e-10 and 7e-12 short
__device__ __forceinline__ void cos_sin_of_phase(uint64_t phase, float& c, float& s) {
  const uint32_t ph = (uint32_t)(phase >> 32);
  const uint32_t q = (ph + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(ph - (q << 30)) * 1.4629180792671596e-9f;        // 2 pi / 2^32
  const float z = x * x;
  float sn = fmaf(z, -2.5052108e-8f, 2.7557319e-6f);
  sn = fmaf(z, sn, -1.9841270e-4f);
  sn = fmaf(z, sn, 8.3333333e-3f);
  sn = fmaf(z, sn, -1.6666667e-1f);
  sn = fmaf(x * z, sn, x);
  float cs = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  cs = fmaf(z, cs, -1.3888889e-3f);
  cs = fmaf(z, cs, 4.1666667e-2f);
  cs = fmaf(z, cs, -0.5f);
  cs = fmaf(z, cs, 1.0f);
  const float a = (q & 1u) ? sn : cs, b = (q & 1u) ? cs : sn;
  c = ((q + 1u) & 2u) ? -a : a;                    // quarters 1 and 2
  s = (q & 2u) ? -b : b;                           // quarters 2 and 3
}

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// rounded to nearest even (v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  const v2bf r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}

__device__ __forceinline__ void load_f32(const v4u& w, float (&x)[4], const float*) {
  x[0] = __uint_as_float(w[0]); x[1] = __uint_as_float(w[1]); x[2] = __uint_as_float(w[2]); x[3] = __uint_as_float(w[3]);
}
__device__ __forceinline__ void load_f32(const v4u& w, float (&x)[8], const uint16_t*) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ v4u store_bits(const float (&y)[4], const float*) {
  return {__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])};
}
__device__ __forceinline__ v4u store_bits(const float (&y)[8], const uint16_t*) {
  v4u u;
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = pack_bf16(y[2 * i], y[2 * i + 1]);
  return u;
}
__device__ __forceinline__ void store_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_elem(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16_bits(v); }

// One lane's share of the rows of a token, by pieces of 16 bytes.  With pairs (i, i + rot/2) a lane has the piece of the first
// and of the second half (EPL pairs), with neighbouring pairs one piece (EPL/2 pairs).  Cosines and sines are worked out once and
// serve all heads of the token.
template <class T, bool HALF>
struct RotaryLane {
  static constexpr int kEPL = 16 / sizeof(T), kPairs = HALF ? kEPL : kEPL / 2;
  float c[kPairs], s[kPairs];
  // piece: 0 .. rot / (HALF ? 2 : 1) / EPL - 1
  __device__ __forceinline__ void angles(const Rotary& R, int piece, int position, const uint64_t* __restrict__ turns) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      cos_sin_of_phase((uint64_t)(uint32_t)position * turns[piece * kPairs + i], c[i], s[i]);
      c[i] *= R.amplitude;
      s[i] *= R.inverse ? -R.amplitude : R.amplitude;
    }
  }
  __device__ __forceinline__ void rotate(v4u& lo, v4u& hi) const {      // HALF: both pieces; else `hi` is not used
    const T* tag = nullptr;
    float x[kEPL];
    load_f32(lo, x, tag);
    if constexpr (HALF) {
      float z[kEPL], y[kEPL];
      load_f32(hi, z, tag);
#pragma unroll
      for (int i = 0; i < kEPL; ++i) y[i] = fmaf(-z[i], s[i], x[i] * c[i]);
      lo = store_bits(y, tag);
#pragma unroll
      for (int i = 0; i < kEPL; ++i) y[i] = fmaf(x[i], s[i], z[i] * c[i]);
      hi = store_bits(y, tag);
    } else {
      float y[kEPL];
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        y[2 * i] = fmaf(-x[2 * i + 1], s[i], x[2 * i] * c[i]);
        y[2 * i + 1] = fmaf(x[2 * i], s[i], x[2 * i + 1] * c[i]);
      }
      lo = store_bits(y, tag);
    }
  }
};

// can the rotated part be cut into whole pieces?  (else pair by pair)
inline bool rotary_by_pieces(int rot, int half, int elem_bytes) { return rot % ((half ? 32 : 16) / elem_bytes) == 0; }

}  // namespace ccd
