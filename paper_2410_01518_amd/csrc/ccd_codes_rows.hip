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
__device__ __forceinline__ void eight_numbers(uint2 w, float scale, float (&x)[kPer]) {
  float a[4], b[4];
  numbers<CODE>(w.x, a);
  numbers<CODE>(w.y, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i] * scale; x[4 + i] = b[i] * scale; }
}

// Rotation: y = c x + t z, z being an element's partner in its pair.  Cosines and sines of a token's pairs are worked out once, a pair to a lane, and lie in LDS for all its
// heads; a lane takes those of its eight elements.
struct Angle { float c, s; };
__device__ __forceinline__ Angle angle_of(const Rotary& R, int pair, int position, const uint64_t* __restrict__ turns) {
  Angle a;
  cos_sin_of_phase((uint64_t)(uint32_t)position * turns[pair], a.c, a.s);
  a.c *= R.amplitude;
  a.s *= R.inverse ? -R.amplitude : R.amplitude;
  return a;
}
enum Turned { kNot, kPieces, kAnyhow };
static Turned turned_how(const Rotary& R, bool rope) { return !rope ? kNot : R.half && R.rot / 2 % kPer == 0 ? kPieces : kAnyhow; }
struct TurnEight {
  float c[kPer], t[kPer];
  // kPieces: the pairs are whole pieces of eight, so that all of a lane's elements are first ones, second ones, or not turned, and their angles lie side by side
  template <Turned MODE>
  __device__ __forceinline__ void take(const Rotary& R, const Angle* lds, int e0) {
    const int pairs = R.rot / 2;
    if constexpr (MODE == kPieces) {
      const bool turned = e0 < R.rot, first = e0 < pairs;
      const float4* from = reinterpret_cast<const float4*>(lds + (!turned ? 0 : first ? e0 : e0 - pairs));
      const float other = first ? -1.f : 1.f;
#pragma unroll
      for (int j = 0; j < kPer / 2; ++j) {
        const float4 a = from[j];
        c[2 * j] = a.x; c[2 * j + 1] = a.z;
        t[2 * j] = other * a.y; t[2 * j + 1] = other * a.w;
      }
      if (!turned) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) { c[j] = 1.f; t[j] = 0.f; }
      }
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const int e = e0 + j;
        const bool turned = e < R.rot, first = R.half ? e < pairs : (e & 1) == 0;
        const Angle a = lds[!turned ? 0 : R.half ? (first ? e : e - pairs) : e >> 1];
        c[j] = turned ? a.c : 1.f;
        t[j] = turned ? (first ? -a.s : a.s) : 0.f;
      }
    }
  }
};
// where the partners of a lane's eight elements begin (kPieces)
__device__ __forceinline__ int partners_at(const Rotary& R, int e0) { return e0 >= R.rot ? e0 : e0 < R.rot / 2 ? e0 + R.rot / 2 : e0 - R.rot / 2; }
// ... and otherwise, one by one: x's neighbours, or from the row.  An element that is not turned is its own partner in any layout: taken 0 times, another's that is no number
// would make it none.
template <class T>
__device__ __forceinline__ void load_partners(const Rotary& R, const T* row, int e0, const float (&x)[kPer], float (&z)[kPer]) {
  const int pairs = R.rot / 2;
#pragma unroll
  for (int j = 0; j < kPer; ++j)
    z[j] = R.half ? load_elem(row + (e0 + j >= R.rot ? e0 + j : e0 + j < pairs ? e0 + j + pairs : e0 + j - pairs)) : e0 + j >= R.rot ? x[j] : x[j ^ 1];
}

// the largest |x|, as bits: an infinite value or a NaN is larger than all numbers
__device__ __forceinline__ uint32_t largest_bits(const float (&x)[kPer], uint32_t top) {
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const uint32_t b = __float_as_uint(x[j]) & 0x7FFFFFFFu;
    top = top > b ? top : b;
  }
  return top;
}
constexpr uint32_t kInfiniteBits = 0x7F800000u;
// ... of those that are finite
__device__ __forceinline__ uint32_t largest_finite_bits(const float (&x)[kPer], uint32_t top) {
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const uint32_t b = __float_as_uint(x[j]) & 0x7FFFFFFFu;
    top = b < kInfiniteBits && b > top ? b : top;
  }
  return top;
}
// over the lanes of a row, which are eight or sixteen side by side
template <int LANES>
__device__ __forceinline__ uint32_t row_largest(uint32_t x) {
  auto with = [&](uint32_t y) { x = x > y ? x : y; };
  with((uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));                   // quad_perm 1 0 3 2, 2 3 0 1, row_half_mirror, row_mirror
  with((uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));
  with((uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xF, 0xF, true));
  if constexpr (LANES == 16) with((uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xF, 0xF, true));
  return x;
}

// the new rows, and where they go
template <class T>
struct Append {
  const T *K_new, *V_new;
  const int32_t *slots, *positions;
  const uint64_t* turns;
  uint8_t *K, *V;
  float *K_scales, *V_scales;
};
template <class T>
__device__ __forceinline__ int slot_of(const Paged& P, const Append<T>& N, bool rope, int t) {
  if (t < 0 || t >= P.tokens) return -1;
  const int s = N.slots[t];
  return (rope && N.positions[t] < 0) || s >= (int64_t)P.div.page * P.n_pages ? -1 : s;
}
template <class T>
__device__ __forceinline__ const T* new_row(const Paged& P, const Codes& C, const T* X, int t, int h) {
  const int rows = (int)C.new_rows, b = rows > 0 ? t / rows : 0, r = t - b * rows;
  return X + b * C.new_b + r * P.new_t + h * P.new_h;
}

// A scale per token: a wave per token, four or eight heads at once, and those of the next time are asked for before these are worked on.  Keys and values come as they are
// and become floats one row after the other: what is alive at once decides how many waves there are to wait for memory (80 registers; with two sets of rows worked on at once,
// and both ways of finding partners in one kernel, 128).  Measured, 16384 tokens of 8 heads of 128, bf16 to int8: embedded 22.7 us, 20.1 without (4.5 and 5.0 TB/s of the 101 MB
// read and written, as much as a copy; 30 and 27 before).
template <class T>
struct Raw { v4u w[sizeof(T) / 2]; };
template <class T>
__device__ __forceinline__ void ask_eight(Raw<T>& r, const T* p) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = reinterpret_cast<const v4u*>(p)[i];
}
__device__ __forceinline__ void eight_of(const Raw<uint16_t>& r, float (&x)[kPer]) { load_f32(r.w[0], x, static_cast<const uint16_t*>(nullptr)); }
__device__ __forceinline__ void eight_of(const Raw<float>& r, float (&x)[kPer]) {
#pragma unroll
  for (int j = 0; j < kPer; ++j) x[j] = __uint_as_float(r.w[j >> 2][j & 3]);
}

template <class T, int CODE, int D, Turned MODE>
__global__ __launch_bounds__(256, 4) void append_tokens_kernel(Paged P, Codes C, Rotary R, Append<T> N) {
  constexpr int kLanes = D / kPer, kHeads = 64 / kLanes;
  __shared__ __align__(16) Angle angles[4][64];
  // (uniform: all that belongs to the token is worked out once a wave)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = blockIdx.x * 4 + wave, lane = threadIdx.x & 63, e0 = lane % kLanes * kPer, own = lane / kLanes;
  if (t >= P.tokens) return;
  const T *K_row = new_row(P, C, N.K_new, t, 0), *V_row = new_row(P, C, N.V_new, t, 0);
  struct Set { Raw<T> k, z, v; };
  auto ask = [&](Set& s, int h0) __attribute__((always_inline)) {
    const int64_t h = (h0 + own < P.Hkv ? h0 + own : 0) * P.new_h;
    ask_eight(s.k, K_row + h + e0);
    if (MODE == kPieces) ask_eight(s.z, K_row + h + partners_at(R, e0));
    ask_eight(s.v, V_row + h + e0);
  };
  Set a, b;
  ask(a, 0);
  if (kHeads < P.Hkv) ask(b, kHeads);
  const int slot = slot_of(P, N, MODE != kNot, t);
  if (slot < 0) return;
  const int page = page_of(P.div, slot), at = slot - page * P.div.page;
  const int64_t to = page * P.page_stride + at * P.row_stride, scale_to = page * C.page + at;
  TurnEight turn;
  if (MODE != kNot) {
    if (lane < R.rot / 2) angles[wave][lane] = angle_of(R, lane, N.positions[t], N.turns);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    turn.take<MODE>(R, angles[wave], e0);
  }
  auto put = [&](const float (&x)[kPer], uint8_t* row, float* to_scale) __attribute__((always_inline)) {
    uint32_t top = row_largest<kLanes>(largest_bits(x, 0));
    const bool fine = top < kInfiniteBits;
    if (!fine) top = row_largest<kLanes>(largest_finite_bits(x, 0));
    const float scale = scale_for<CODE>(__uint_as_float(top));
    *reinterpret_cast<uint2*>(row) = eight_codes<CODE>(x, scale, inverse_scale<CODE>(scale), fine);
    if (e0 == 0) *to_scale = CODE == kInt8 && !fine ? __uint_as_float(0x7FC00000u) : scale;
  };
  auto work = [&](const Set& s, int h0) __attribute__((always_inline)) {
    const int h = h0 + own;
    if (h >= P.Hkv) return;
    float x[kPer];
    eight_of(s.k, x);
    if (MODE != kNot) {
      float z[kPer];
      if (MODE == kPieces) eight_of(s.z, z);
      else load_partners(R, K_row + h * P.new_h, e0, x, z);
#pragma unroll
      for (int j = 0; j < kPer; ++j) x[j] = fmaf(z[j], turn.t[j], x[j] * turn.c[j]);
    }
    put(x, N.K + to + h * P.head_stride + e0, N.K_scales + scale_to + h * C.head);
    __builtin_amdgcn_sched_barrier(0);
    eight_of(s.v, x);
    put(x, N.V + to + h * P.head_stride + e0, N.V_scales + scale_to + h * C.head);
    __builtin_amdgcn_sched_barrier(0);
  };
  for (int h0 = 0;;) {
    work(a, h0);
    if (h0 + kHeads >= P.Hkv) break;
    if (h0 + 2 * kHeads < P.Hkv) ask(a, h0 + 2 * kHeads);
    work(b, h0 + kHeads);
    h0 += 2 * kHeads;
    if (h0 >= P.Hkv) break;
    if (h0 + kHeads < P.Hkv) ask(b, h0 + kHeads);
  }
}

// A scale per block of 2^shift tokens: a workgroup per `each` tokens, at most 64, takes those that begin a run, tokens of one block side by side, and the run with them.  A
// wave per head; lanes side by side have a token's row, kKeep times four or eight tokens at a time.  First the run's largest element, then the codes; a run of that many tokens
// stays in registers in between, longer ones are read twice.  Measured, 16384 tokens of 8 heads of 128, bf16: blocks of 16 25 us (4.0 TB/s), embedded 35; of 64, read twice, 36.
// A block has one scale, so a run is one workgroup's (of keys, and one of values): 4096 tokens in blocks of 16, 64, 256, 4096: 13, 42, 117, 698 us.
template <class T, int D, Turned MODE>
__global__ __launch_bounds__(512, 4) void append_blocks_kernel(Paged P, Codes C, Rotary R, Append<T> N, int each) {
  constexpr int kLanes = D / kPer, kTokens = 64 / kLanes, kKeep = 4, kPart = kKeep * kTokens;
  __shared__ __align__(16) Angle angles[kPart][D / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, e0 = lane % kLanes * kPer, own = lane / kLanes;
  const bool keys = blockIdx.y == 0, turned = MODE != kNot && keys;
  const T* from = keys ? N.K_new : N.V_new;
  const int t0 = blockIdx.x * each;
  uint64_t begins;
  {
    const int s = lane < each ? slot_of(P, N, MODE != kNot, t0 + lane) : -1, before = lane < each ? slot_of(P, N, MODE != kNot, t0 + lane - 1) : -1;
    begins = __ballot(s >= 0 && (before < 0 || before >> C.shift != s >> C.shift));
  }
  for (; begins != 0; begins &= begins - 1) {
    const int t = t0 + __builtin_ctzll(begins);
    // the run: tokens t .. t + n - 1, and the lowest of their rows
    const int slot = N.slots[t], block = slot >> C.shift;
    int n = 0, first = slot;
    for (bool more = true; more;) {
      const int s = slot_of(P, N, MODE != kNot, t + n + lane);
      const uint64_t others = ~__ballot(s >= 0 && s >> C.shift == block);
      const int here = others == 0 ? 64 : __builtin_ctzll(others);
      int low = lane < here ? s : first;
#pragma unroll
      for (int k = 32; k; k >>= 1) { const int y = __shfl_xor(low, k); low = y < low ? y : low; }
      first = low < first ? low : first;
      n += here;
      more = here == 64;
    }
    const int page = page_of(P.div, slot), page0 = page * P.div.page, rounds = (P.Hkv + waves - 1) / waves;
    const bool anew = first == block << C.shift;
    for (int h0 = 0; h0 < rounds; ++h0) {
      const bool there = h0 * waves + wave < P.Hkv;
      const int h = there ? h0 * waves + wave : 0;
      uint8_t* to = (keys ? N.K : N.V) + page * P.page_stride + h * P.head_stride + e0;
      float* to_scale = (keys ? N.K_scales : N.V_scales) + page * C.page + h * C.head + (((block << C.shift) - page0) >> C.shift);
      const float old = anew ? 0.f : *to_scale;
      float x[kKeep][kPer];
      int at[kKeep];                                        // row in the page, negative where there is no token
      // tokens t + part .. of the run
      auto load = [&](int part) __attribute__((always_inline)) {
        float z[kKeep][kPer];
#pragma unroll
        for (int g = 0; g < kKeep; ++g) {
          // (all are read, the last token's row in the place of those behind it: how many loads are under way is known then)
          const int i = part + g * kTokens + own, ti = t + (i < n ? i : n - 1);
          const T* row = new_row(P, C, from, ti, h);
          at[g] = N.slots[ti] - page0;
          if (i >= n) at[g] = -1;
          load_eight(row + e0, x[g]);
          if (turned && MODE == kPieces) load_eight(row + partners_at(R, e0), z[g]);
          else if (turned) load_partners(R, row, e0, x[g], z[g]);
        }
        if (turned) {
          const int tokens = n - part < kPart ? n - part : kPart;
          __syncthreads();
          for (int i = wave; i < tokens; i += waves)
            if (lane < R.rot / 2) angles[i][lane] = angle_of(R, lane, N.positions[t + part + i], N.turns);
          __syncthreads();
        }
#pragma unroll
        for (int g = 0; g < kKeep; ++g) {
          if (turned && at[g] >= 0) {
            TurnEight turn;
            turn.take<MODE>(R, angles[g * kTokens + own], e0);
#pragma unroll
            for (int j = 0; j < kPer; ++j) x[g][j] = fmaf(z[g][j], turn.t[j], x[g][j] * turn.c[j]);
          }
        }
      };
      uint32_t top = 0;
      bool fine = true;
      for (int part = 0; part < n; part += kPart) {
        load(part);
#pragma unroll
        for (int g = 0; g < kKeep; ++g) {
          if (at[g] < 0) continue;
          const uint32_t all = largest_bits(x[g], 0);
          fine = fine && all < kInfiniteBits;
          top = all < kInfiniteBits ? (all > top ? all : top) : largest_finite_bits(x[g], top);
        }
      }
#pragma unroll
      for (int k = 32; k; k >>= 1) { const uint32_t y = __shfl_xor(top, k); top = y > top ? y : top; }
      const float scale = fmaxf(power_of_two_scale(old), scale_for<kE4m3>(__uint_as_float(top))), inverse = inverse_scale<kE4m3>(scale);
      // (what stands before is rounded again wherever its scale becomes another one, NaN among them)
      if (there && !anew && scale != old)
        for (int r0 = block << C.shift; r0 < first; r0 += kPart) {
          uint2 w[kKeep];
#pragma unroll
          for (int g = 0; g < kKeep; ++g) {
            const int r = r0 + g * kTokens + own;
            w[g] = *reinterpret_cast<const uint2*>(to + (int64_t)((r < first ? r : r0) - page0) * P.row_stride);
          }
#pragma unroll
          for (int g = 0; g < kKeep; ++g) {
            const int r = r0 + g * kTokens + own;
            float y[kPer];
            eight_numbers<kE4m3>(w[g], old, y);
            if (r < first) *reinterpret_cast<uint2*>(to + (int64_t)(r - page0) * P.row_stride) = eight_codes<kE4m3>(y, scale, inverse, false);
          }
        }
      for (int part = 0; part < n; part += kPart) {
        if (n > kPart) load(part);
#pragma unroll
        for (int g = 0; g < kKeep; ++g) {
          if (there && at[g] >= 0) *reinterpret_cast<uint2*>(to + at[g] * P.row_stride) = eight_codes<kE4m3>(x[g], scale, inverse, fine);
        }
      }
      if (there && lane == 0) *to_scale = scale;
    }
  }
}

// A wave per row of K_out and V_out.  The row's sequence, page and place are uniform: scalar loads, one chain a wave.  Bound by memory: 131072 tokens of 8 heads of 128 to bf16, keys alone, 76 us
// (406 MB, 5.3 TB/s; 83 with the chain in vector registers).
template <class T, int CODE, int D>
__global__ __launch_bounds__(256) void read_codes_kernel(Paged P, Codes C, const uint8_t* __restrict__ K, const uint8_t* __restrict__ V, const float* __restrict__ K_scales,
                                                         const float* __restrict__ V_scales, const int32_t* __restrict__ table, const int32_t* __restrict__ q_start,
                                                         const int32_t* __restrict__ kv_len, T* K_out, T* V_out) {
  constexpr int kLanes = D / kPer, kHeads = 64 / kLanes;
  const int row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, e0 = lane % kLanes * kPer;
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

// A workgroup per (page, head), keys or values, and all of a row or 64 bytes of it.  Rows move towards the front: row j comes from keep[j] >= j, so a piece of rows may be
// written once all of it has been read, and what later pieces read lies behind it: a piece is read while the one before is written, its indices a piece earlier.
// Bound by memory: 32 pots of 8 heads, 4096 -> 2048 rows of 128 and novelty, 57 - 61 us for 283 MB, 4.6 - 5.0 TB/s (107 with a piece at a time); one such pot 5.
constexpr int kCompactThreads = 512;
template <int BYTES>
__global__ __launch_bounds__(kCompactThreads) void compact_codes_kernel(Paged P, Codes C, uint8_t* K, uint8_t* V, float* K_scales, float* V_scales,
                                                                        const int32_t* __restrict__ keep_all, int k, float* novelty) {
  constexpr int kLanes = BYTES / 16, kRows = kCompactThreads / kLanes, kSide = 2, kPiece = kSide * kRows;
  const int page = blockIdx.x / P.Hkv, h = blockIdx.x % P.Hkv, tid = threadIdx.x, lane = tid % kLanes, row = tid / kLanes, column = blockIdx.y >> 1;
  const bool keys = (blockIdx.y & 1) == 0, scaled = column == 0 && lane == 0;
  const int32_t* keep = keep_all + (int64_t)blockIdx.x * k;
  uint8_t* X = (keys ? K : V) + page * P.page_stride + h * P.head_stride + column * BYTES + lane * 16;
  float* scales = (keys ? K_scales : V_scales) + page * C.page + h * C.head;
  float* carried = keys && novelty != nullptr ? novelty + (int64_t)blockIdx.x * P.div.page : scales;
  struct Piece {
    v4u x[kSide];
    float s[kSide], n[kSide];
  } pieces[2];
  int from[2][kSide];
  auto index = [&](int (&i)[kSide], int j0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kSide; ++u) {
      const int j = j0 + u * kRows + row, found = keep[j < k ? j : k - 1];
      i[u] = j < k && found >= 0 && found < P.div.page ? found : -1;
    }
  };
  // (loads are made whether a row moves or not: how many are under way is known then)
  auto read = [&](Piece& p, const int (&i)[kSide]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kSide; ++u) {
      const int64_t r = i[u] < 0 ? 0 : i[u];
      p.x[u] = *reinterpret_cast<const v4u*>(X + r * P.row_stride);
      p.s[u] = scales[r];
      p.n[u] = carried[r];
    }
  };
  auto write = [&](const Piece& p, const int (&i)[kSide], int j0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kSide; ++u) asm volatile("" ::"v"(p.x[u]), "v"(p.s[u]), "v"(p.n[u]));          // (read, not just asked for)
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSide; ++u) {
      const int j = j0 + u * kRows + row;
      if (i[u] < 0 || i[u] == j) continue;
      *reinterpret_cast<v4u*>(X + j * P.row_stride) = p.x[u];
      if (scaled) {
        scales[j] = p.s[u];
        if (carried != scales) carried[j] = p.n[u];
      }
    }
  };
  index(from[0], 0);
  read(pieces[0], from[0]);
  index(from[1], kPiece);
  for (int j0 = 0; j0 < k; j0 += 2 * kPiece) {
    read(pieces[1], from[1]);
    write(pieces[0], from[0], j0);
    index(from[0], j0 + 2 * kPiece);
    if (j0 + kPiece >= k) break;
    read(pieces[0], from[0]);
    write(pieces[1], from[1], j0 + kPiece);
    index(from[1], j0 + 3 * kPiece);
  }
}

template <class T, int D, Turned MODE>
static void append_turned(const Paged& P, const Codes& C, int code, const Rotary& R, const Append<T>& N, hipStream_t s) {
  if (C.shift == 0) {
    launch(code == kInt8 ? append_tokens_kernel<T, kInt8, D, MODE> : append_tokens_kernel<T, kE4m3, D, MODE>, dim3((P.tokens + 3) / 4), dim3(256), s, P, C, R, N);
    return;
  }
  // Single tokens side by side: a workgroup each; long runs: none that finds nothing to begin.  (16384 tokens of 8 heads without rotation, blocks of 16 and 64, for 2048, 1024, 512, 256
  // workgroups: 33, 25, 25, 25 us and 84, 50, 36, 36.  Four waves instead of eight 24 and 33, but a decoding step of 64 sequences 8.3, 6.4 with eight.)
  int each = P.tokens / 512;
  if (each > 1 << C.shift) each = 1 << C.shift;
  if (each > 64) each = 64;
  if (each < 1) each = 1;
  while ((P.tokens + each - 1) / each > 1 << 21) each *= 2;            // (a launch has less than 2^32 threads; 2^25 tokens at most: each stays below 64)
  launch(append_blocks_kernel<T, D, MODE>, dim3((P.tokens + each - 1) / each, 2), dim3(64 * (P.Hkv < 8 ? P.Hkv : 8)), s, P, C, R, N, each);
}
template <class T>
static void append_of(const Paged& P, const Codes& C, int code, const Rotary& R, bool rope, const Append<T>& N, hipStream_t s) {
  const Turned how = turned_how(R, rope);
  auto of = P.d == 64 ? (how == kNot ? append_turned<T, 64, kNot> : how == kPieces ? append_turned<T, 64, kPieces> : append_turned<T, 64, kAnyhow>)
                      : (how == kNot ? append_turned<T, 128, kNot> : how == kPieces ? append_turned<T, 128, kPieces> : append_turned<T, 128, kAnyhow>);
  of(P, C, code, R, N, s);
}

void launch_append_codes(const Paged& P, const Codes& C, int code, int dtype, const Rotary* rope, const void* K_new, const void* V_new, const int32_t* slots,
                         const int32_t* positions, const uint64_t* turns, void* K, void* V, float* K_scales, float* V_scales, hipStream_t s) {
  const Rotary R = rope ? *rope : Rotary{};
  uint8_t *k = static_cast<uint8_t*>(K), *v = static_cast<uint8_t*>(V);
  if (dtype == 0)
    append_of<float>(P, C, code, R, rope != nullptr, {static_cast<const float*>(K_new), static_cast<const float*>(V_new), slots, positions, turns, k, v, K_scales, V_scales}, s);
  else
    append_of<uint16_t>(P, C, code, R, rope != nullptr, {static_cast<const uint16_t*>(K_new), static_cast<const uint16_t*>(V_new), slots, positions, turns, k, v, K_scales, V_scales},
                        s);
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

int attend_compute_units();

void launch_compact_codes(const Paged& P, const Codes& C, void* K, void* V, float* K_scales, float* V_scales, const int32_t* keep, int32_t k, float* novelty,
                          hipStream_t s) {
  uint8_t *x = static_cast<uint8_t*>(K), *y = static_cast<uint8_t*>(V);
  const unsigned units = (unsigned)(P.n_pages * P.Hkv);
  // (few pots: halves of rows, so that twice as many workgroups share them)
  if (P.d == 64 || (int64_t)units * 2 < attend_compute_units())
    launch(compact_codes_kernel<64>, dim3(units, 2 * P.d / 64), dim3(kCompactThreads), s, P, C, x, y, K_scales, V_scales, keep, k, novelty);
  else
    launch(compact_codes_kernel<128>, dim3(units, 2), dim3(kCompactThreads), s, P, C, x, y, K_scales, V_scales, keep, k, novelty);
}

}  // namespace ccd
