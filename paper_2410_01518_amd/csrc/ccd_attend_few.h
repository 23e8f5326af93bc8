// Few rows per unit, and fp32 caches: a workgroup per (unit, block of 16 or 32 rows, stretch of tokens).
//
// Decoding reads every key and value once for a handful of rows and is bound by memory.  So the work is cut along the tokens, fine
// enough to fill the chip evenly whatever the lengths, and a workgroup's waves go their own ways: wave w of W takes tiles w, w + W, ... of the
// stretch, keys straight from memory into the registers that the matrix instructions read (D[token][row] = K Q^T: the keys' lanes
// hold 16 bytes of a row, as they lie in memory), without a barrier.  The product with the values needs them transposed, D[d][row] = V^T
// W^T: bf16 values go through the wave's own piece of LDS and come back by transposing reads; fp32 values can be loaded as they are
// needed.  Weights need not move at all: a lane holds those of tokens 4g .. 4g + 3 of its row, which is an operand if the tokens of the
// product are counted in that order.  The waves join their sums at the end; stretches are joined by a second kernel.
//
// Measured, 32 query heads on 8 KV heads of 128 elements, bf16: one sequence of 131072 tokens 94 us (5.7 TB/s; the card reads 5.9), the join 6; 64
// sequences of 500 to 8192, cut evenly, 136 us (5.2 TB/s), the join 6; 4 of 200 to 500, whole, 9.4 a call among others.  fp32 chunks are bound by
// the fp32 matrix instructions, which are busy two thirds of the time: 1024 tokens over 4096, 16 heads of 128, 278 to 290 us (195 at the full rate).
#pragma once
#include "ccd_attend.h"

namespace ccd {

constexpr int kWaves = 4;

// Rows are read by quads of lanes, 64 bytes of a row each: a compute unit takes 125 bytes/ns of what L2 has so, but 38 where the matrix instructions'
// operand is read as it is, 16 bytes of 16 rows side by side (76 by pairs of lanes, 32 bytes).  Register s of lane j of N (4, or 2) lanes
// then has piece j of their row s, and has to have piece s of row j.
template <int CTRL>
__device__ __forceinline__ uint32_t from_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true); }
template <int CTRL>
__device__ __forceinline__ void exchange(v4u& a, v4u& b, bool second) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t of_a = from_lane<CTRL>(a[e]), of_b = from_lane<CTRL>(b[e]);
    a[e] = second ? of_b : a[e];
    b[e] = second ? b[e] : of_a;
  }
}
template <int N>
__device__ __forceinline__ void turn(v4u* r, int lane) {
  constexpr int kNext = 0xB1, kOver = 0x4E;                // quad_perm 1 0 3 2, 2 3 0 1
#pragma unroll
  for (int s = 0; s < N; s += 2) exchange<kNext>(r[s], r[s + 1], lane & 1);
  if constexpr (N == 4) {
    exchange<kOver>(r[0], r[2], lane & 2);
    exchange<kOver>(r[1], r[3], lane & 2);
  }
}
// the address that the s-th of the N lanes has
template <int N, int S>
__device__ __forceinline__ const char* of_row(const char* p) {
  constexpr int kCtrl = N == 4 ? 0x55 * S : 0xA0 + 0x55 * S;
  const uint64_t x = (uint64_t)p;
  return (const char*)((uint64_t)from_lane<kCtrl>((uint32_t)(x >> 32)) << 32 | from_lane<kCtrl>((uint32_t)x));
}
// N registers of 16 bytes: pieces first + (lane % N) of the rows of the N lanes, whose own row is at p
template <int N>
__device__ __forceinline__ void load_rows(v4u* r, const char* p, int first, int lane) {
  const int at = 16 * (first + (lane & (N - 1)));
  r[0] = *reinterpret_cast<const v4u*>(of_row<N, 0>(p) + at);
  r[1] = *reinterpret_cast<const v4u*>(of_row<N, 1>(p) + at);
  if constexpr (N == 4) {
    r[2] = *reinterpret_cast<const v4u*>(of_row<N, 2>(p) + at);
    r[3] = *reinterpret_cast<const v4u*>(of_row<N, 3>(p) + at);
  }
}

// sum + two weights as they are rounded to bf16.  The weights of the product with the values are rounded, their sum is not; a row that one token rules
// would be off by that token's rounding.  So the product is taken times l / lr in the end, lr being the sum of the rounded weights.
// (One query of 8 heads over 438 tokens: 3.0e-3 off in the norm where the output's own rounding is 1.8e-3; 1.9e-3 so.)
__device__ __forceinline__ float add_rounded(v8bf w, int pair, float sum) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(v2bf{w[2 * pair], w[2 * pair + 1]}, v2bf{(__bf16)1.f, (__bf16)1.f}, sum, false);
}
__device__ __forceinline__ float unrounded(float l, float lr) { return lr > 0.f ? l / lr : 1.f; }

template <class T, int D>
struct Tile;

// bf16: 32 tokens, halves of 16 (v_mfma_f32_16x16x32_bf16)
template <int D>
struct Tile<uint16_t, D> {
  using T = uint16_t;
  static constexpr int kTokens = 32, kHalves = 2, kSteps = D / 32, kBlocks = D / 16;
  static constexpr int kLdsBytes = kTokens * D * 2;
  static constexpr bool kValuesLate = false;         // values are out of the registers before the logits are computed
  struct Query { v8bf f[kSteps]; };
  struct Keys { v4u k[kHalves][kSteps]; };
  struct Values { v4u v[kHalves][kSteps]; };

  __device__ static void load_query(Query& q, const T* row, int lane, bool there) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      v4u w = {0, 0, 0, 0};
      if (there) w = *reinterpret_cast<const v4u*>(row + 8 * (kSteps * (lane >> 4) + s));
      q.f[s] = __builtin_bit_cast(v8bf, w);
    }
  }
  // off[h]: element offset of token 16 h + (lane & 15), negative where there is none
  __device__ static void load_keys(Keys& r, const T* K, const int64_t (&off)[kHalves], int lane) { load_pieces(r.k, K, off, lane); }
  __device__ static void load_values(Values& r, const T* V, const int64_t (&off)[kHalves], int lane) { load_pieces(r.v, V, off, lane); }
  __device__ static void load_pieces(v4u (&r)[kHalves][kSteps], const T* X, const int64_t (&off)[kHalves], int lane) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      const T* x = off[h] >= 0 ? X + off[h] : reinterpret_cast<const T*>(g_zero_row);
      load_rows<kSteps>(r[h], reinterpret_cast<const char*>(x), kSteps * (lane >> 4), lane);
    }
  }
  // 16-byte pieces of a row, exchanged in pairs by the row's number so that the rows a transposing read takes together (16 rows, one pair
  // of pieces) lie in different banks.  An exchange is an exclusive or of the piece's number, so a lane's places in a row differ by one, too.
  __device__ static int swap_of(int row) { return D == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1; }
  __device__ static void store_values(const Values& r, char* lds, int lane) {
    const int row = lane & 15 & ~(kSteps - 1), piece = kSteps * (lane >> 4) + (lane & (kSteps - 1));
    const int at = row * (D * 2) + ((piece ^ swap_of(row)) << 4);
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
      for (int s = 0; s < kSteps; ++s) *reinterpret_cast<v4u*>(lds + ((at ^ (swap_of(s) << 4)) + (16 * h + s) * (D * 2))) = r.v[h][s];
  }
  __device__ static void turn_keys(Keys& r, int lane) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) turn<kSteps>(r.k[h], lane);
  }
  // x[h][i]: logit of token 16 h + 4 (lane >> 4) + i for row lane & 15
  __device__ static void logits(v4f (&x)[kHalves], const Keys& r, const Query& q) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      x[h] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) x[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, r.k[h][s]), q.f[s], x[h], 0, 0, 0);
    }
  }
  struct Weights { v8bf w; };
  __device__ static Weights weights(const v4f (&x)[kHalves]) {
    const v4u w = {pack_bf16(x[0][0], x[0][1]), pack_bf16(x[0][2], x[0][3]), pack_bf16(x[1][0], x[1][1]), pack_bf16(x[1][2], x[1][3])};
    return {__builtin_bit_cast(v8bf, w)};
  }
  __device__ static float add_rounded(const Weights& w, float sum) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = ccd::add_rounded(w.w, i, sum);
    return sum;
  }
  // o[c][i] += element 16 c + 4 (lane >> 4) + i of the values, for row lane & 15
  template <int NQ>
  __device__ static void add_values(v4f (&o)[NQ][kBlocks], const Weights (&w)[NQ], const Values&, const char* lds, int lane) {
    const int row = 4 * (lane >> 4) + ((lane & 15) >> 2);
    const int at = row * (D * 2) + ((((lane & 3) >> 1) ^ swap_of(row)) << 4) + (lane & 1) * 8;
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
      v4s t[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        t[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(lds + ((at ^ (c << 5)) + 16 * h * (D * 2))));
      const v8bf a = __builtin_bit_cast(v8bf, __builtin_shufflevector(t[0], t[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int j = 0; j < NQ; ++j) o[j][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[j].w, o[j][c], 0, 0, 0);
    }
  }
  __device__ static int element(int c, int lane, int i) { return 16 * c + 4 * (lane >> 4) + i; }
};

// fp32: 16 tokens (v_mfma_f32_16x16x4_f32).  Elements of a row are counted in the products so that a lane's share of a row is 16 bytes:
// step (j, i) takes element 16 j + 4 g + i of lane group g.  (Read as the products take them: those take longer than the reading does.  By quads a
// step of ragged chunks took 60.5 us, not 57.6.)
template <int D>
struct Tile<float, D> {
  using T = float;
  static constexpr int kTokens = 16, kHalves = 1, kSteps = D / 16, kBlocks = D / 16;
  static constexpr int kLdsBytes = 0;
  static constexpr bool kValuesLate = true;
  struct Query { float4 f[kSteps]; };
  struct Keys { float4 k[kSteps]; };
  struct Values { float4 v[4][D / 64]; };

  __device__ static void load_query(Query& q, const T* row, int lane, bool there) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      q.f[s] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (there) q.f[s] = *reinterpret_cast<const float4*>(row + 16 * s + 4 * (lane >> 4));
    }
  }
  __device__ static void load_keys(Keys& r, const T* K, const int64_t (&off)[kHalves], int lane) {
    const T* k = off[0] >= 0 ? K + off[0] : reinterpret_cast<const T*>(g_zero_row);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) r.k[s] = *reinterpret_cast<const float4*>(k + 16 * s + 4 * (lane >> 4));
  }
  __device__ static void turn_keys(Keys&, int) {}
  // token 4 g + i, elements 64 c + 4 (lane & 15) ..
  __device__ static void load_values(Values& r, const T* V, const int64_t (&off)[kHalves], int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t at = __shfl(off[0], 4 * (lane >> 4) + i);
      const T* v = at >= 0 ? V + at : reinterpret_cast<const T*>(g_zero_row);
#pragma unroll
      for (int c = 0; c < D / 64; ++c) r.v[i][c] = *reinterpret_cast<const float4*>(v + 64 * c + 4 * (lane & 15));
    }
  }
  __device__ static void store_values(const Values&, char*, int) {}
  __device__ static void logits(v4f (&x)[kHalves], const Keys& r, const Query& q) {
    x[0] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      x[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(r.k[s].x, q.f[s].x, x[0], 0, 0, 0);
      x[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(r.k[s].y, q.f[s].y, x[0], 0, 0, 0);
      x[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(r.k[s].z, q.f[s].z, x[0], 0, 0, 0);
      x[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(r.k[s].w, q.f[s].w, x[0], 0, 0, 0);
    }
  }
  struct Weights { v4f w; };
  __device__ static Weights weights(const v4f (&x)[kHalves]) { return {x[0]}; }
  __device__ static float add_rounded(const Weights&, float sum) { return sum; }
  // o[4 c + e][i] += element 64 c + 4 (4 (lane >> 4) + i) + e
  template <int NQ>
  __device__ static void add_values(v4f (&o)[NQ][kBlocks], const Weights (&w)[NQ], const Values& r, const char*, int) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const float a[4] = {r.v[i][c].x, r.v[i][c].y, r.v[i][c].z, r.v[i][c].w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < NQ; ++j) o[j][4 * c + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], w[j].w[i], o[j][4 * c + e], 0, 0, 0);
      }
  }
  __device__ static int element(int c, int lane, int i) { return 64 * (c >> 2) + 4 * (4 * (lane >> 4) + i) + (c & 3); }
};

__device__ __forceinline__ void store_piece(float* to, const float (&x)[2]) { *reinterpret_cast<float2*>(to) = make_float2(x[0], x[1]); }
__device__ __forceinline__ void store_piece(uint16_t* to, const float (&x)[2]) { *reinterpret_cast<uint32_t*>(to) = pack_bf16(x[0], x[1]); }
__device__ __forceinline__ void store_piece(float* to, const float (&x)[4]) { *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void store_piece(float* to, const float (&x)[8]) {
  *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(to + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store_piece(uint16_t* to, const float (&x)[4]) {
  *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
}
__device__ __forceinline__ void store_piece(uint16_t* to, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// over the four lanes that hold a row
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// workgroups per compute unit, and so waves per SIMD, that the registers are cut for: what the rows of queries and of sums leave room for
template <class T, int D, int NQ>
constexpr int split_waves() { return NQ == 2 || D == 128 ? 2 : 3; }

template <class T, int D, int NQ, int WAVES = kWaves>
struct SplitLds {
  static constexpr int kRows = 16 * NQ, kPitch = D + 4;
  static constexpr int kWaveBytes = Tile<T, D>::kLdsBytes > 16 * kPitch * 4 ? Tile<T, D>::kLdsBytes : 16 * kPitch * 4;
  __align__(16) char wave[WAVES][kWaveBytes];
  float m[WAVES][kRows], l[WAVES][kRows];
};

// Rows r0 .. r1 - 1 of unit (b, hkv) over the tokens t_begin .. t_end - 1, by the workgroup.  whole_row: these are all tokens the rows see, the result
// is written; else (o, m, l) of row r go to entry part0 + (r - r0) of the workspace, or, part0 < 0, to those of part_no by the row's number.
// Returns whether the rows may have to be done again (bad_unseen says).
template <class T, int D, int NQ, int WAVES>
__device__ __forceinline__ bool attend_stretch(const Paged& P, const AttendArgs& A, SplitLds<T, D, NQ, WAVES>& L, const Sequence& sq, int b, int hkv, int r0, int r1,
                                               int t_begin, int t_end, bool whole_row, int64_t part0, int part_no) {
  using Tl = Tile<T, D>;
  constexpr int kPitch = SplitLds<T, D, NQ, WAVES>::kPitch, kStride = WAVES * Tl::kTokens;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t* pages = A.table + (int64_t)b * P.table_width;
  const T* Kh = static_cast<const T*>(A.K) + hkv * P.head_stride;
  const T* Vh = static_cast<const T*>(A.V) + hkv * P.head_stride;
  // Keys and values of a tile are asked for a tile ahead, the pages they are in two tiles ahead: a chain of two loads from memory
  // would not hide behind one tile's work.
  typename Tl::Keys keys;
  typename Tl::Values values;
  int64_t off[Tl::kHalves];
  int id[Tl::kHalves];
  auto look_up = [&](int t0) {
#pragma unroll
    for (int h = 0; h < Tl::kHalves; ++h) {
      const int t = t0 + 16 * h + (lane & 15);
      id[h] = t < t_end ? pages[page_of(P.div, t)] : -1;
    }
  };
  auto offsets = [&](int t0) {
#pragma unroll
    for (int h = 0; h < Tl::kHalves; ++h) {
      const int t = t0 + 16 * h + (lane & 15);
      off[h] = id[h] >= 0 && id[h] < P.n_pages ? id[h] * P.page_stride + (int64_t)(t - page_of(P.div, t) * P.div.page) * P.row_stride : -1;
    }
  };
  int t0 = t_begin + wave * Tl::kTokens;
  if (t0 < t_end) {
    look_up(t0);
    offsets(t0);
    Tl::load_keys(keys, Kh, off, lane);
    Tl::load_values(values, Vh, off, lane);
    look_up(t0 + kStride);
  }
  // the lane's rows
  typename Tl::Query q[NQ];
  int pos[NQ], low[NQ];                                    // position of the row, first position it sees
  const int pos_min = sq.base + r0 / P.G, low_max = first_seen(P, sq.base + (r1 - 1) / P.G);
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    const int r = r0 + 16 * j + (lane & 15), i = r / P.G;
    pos[j] = sq.base + i;
    low[j] = first_seen(P, pos[j]);
    Tl::load_query(q[j], static_cast<const T*>(A.Q) + b * P.q_b + (int64_t)(sq.first + i) * P.q_t + (int64_t)(hkv * P.G + r - i * P.G) * P.q_h, lane, r < r1);
  }
  float m[NQ], l[NQ], lr[NQ];
  v4f o[NQ][Tl::kBlocks];
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    m[j] = -INFINITY; l[j] = lr[j] = 0.f;
#pragma unroll
    for (int c = 0; c < Tl::kBlocks; ++c) o[j][c] = v4f{0.f, 0.f, 0.f, 0.f};
  }
  for (; t0 < t_end; t0 += kStride) {
    uint32_t there = (uint32_t)__ballot(off[0] >= 0) & 0xFFFFu;
    if constexpr (Tl::kHalves == 2) there |= (uint32_t)__ballot(off[Tl::kHalves - 1] >= 0) << 16;
    const bool whole = there == (Tl::kHalves == 2 ? 0xFFFFFFFFu : 0xFFFFu) && t0 + Tl::kTokens - 1 <= pos_min && t0 >= low_max;
    const bool more = t0 + kStride < t_end;
    if (more) offsets(t0 + kStride);
    // the next tile's rows are asked for as soon as this one's are out of their registers
    Tl::store_values(values, L.wave[wave], lane);
    if (more && !Tl::kValuesLate) Tl::load_values(values, Vh, off, lane);
    v4f x[NQ][Tl::kHalves];
    Tl::turn_keys(keys, lane);
#pragma unroll
    for (int j = 0; j < NQ; ++j) Tl::logits(x[j], keys, q[j]);
    if (more) {
      Tl::load_keys(keys, Kh, off, lane);
      if (!Tl::kValuesLate) look_up(t0 + 2 * kStride);
    }
    typename Tl::Weights w[NQ];
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      if (!whole) {
#pragma unroll
        for (int h = 0; h < Tl::kHalves; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = 16 * h + 4 * (lane >> 4) + i, t = t0 + at;
            if (!((there >> at) & 1u) || t > pos[j] || t < low[j]) x[j][h][i] = -INFINITY;
          }
      }
      float top = x[j][0][0];
#pragma unroll
      for (int h = 0; h < Tl::kHalves; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, x[j][h][i]);
      top *= P.scale_log2;
      if (__any(top > m[j] + kRaise)) {
        const float next = fmaxf(m[j], row_max(top));
        const float keep = next == -INFINITY ? 1.f : fast_exp2(m[j] - next);
        m[j] = next;
        l[j] *= keep;
        lr[j] *= keep;
#pragma unroll
        for (int c = 0; c < Tl::kBlocks; ++c) o[j][c] *= keep;
      }
      const float ref = m[j] == -INFINITY ? 0.f : m[j];
      float sum = 0.f;
#pragma unroll
      for (int h = 0; h < Tl::kHalves; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = fast_exp2(fmaf(x[j][h][i], P.scale_log2, -ref));
          x[j][h][i] = e;
          sum += e;
        }
      l[j] += sum;
      w[j] = Tl::weights(x[j]);
      lr[j] = Tl::add_rounded(w[j], lr[j]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    Tl::add_values(o, w, values, L.wave[wave], lane);
    __builtin_amdgcn_wave_barrier();
    if (more && Tl::kValuesLate) {
      Tl::load_values(values, Vh, off, lane);
      look_up(t0 + 2 * kStride);
    }
  }

  // the waves' sums together: all to the largest reference, 16 rows at a time through LDS
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    l[j] = row_sum(l[j]);
    lr[j] = row_sum(lr[j]);
    if (lane < 16) { L.m[wave][16 * j + lane] = m[j]; L.l[wave][16 * j + lane] = l[j]; }
  }
  __syncthreads();
  bool none = false;                                        // sums that are no numbers, of weights that are
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    float all = -INFINITY;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all = fmaxf(all, L.m[w][16 * j + (lane & 15)]);
    const float keep = m[j] == -INFINITY ? (l[j] == l[j] ? 0.f : l[j]) : fast_exp2(m[j] - all) * unrounded(l[j], lr[j]);
    float* mine = reinterpret_cast<float*>(L.wave[wave]) + (lane & 15) * kPitch;
    if (j > 0) __syncthreads();
#pragma unroll
    for (int c = 0; c < Tl::kBlocks; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) mine[Tl::element(c, lane, i)] = o[j][c][i] * keep;
    __syncthreads();
    // 16 rows of D elements by all threads
    constexpr int kPer = 16 * D / (64 * WAVES);           // 2, 4 or 8 elements a thread
    const int q_row = tid / (D / kPer), e0 = tid % (D / kPer) * kPer, r = r0 + 16 * j + q_row;
    float acc[kPer] = {}, top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float* from = reinterpret_cast<const float*>(L.wave[w]) + q_row * kPitch + e0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[e] += from[e];
      top = fmaxf(top, L.m[w][16 * j + q_row]);
    }
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float mw = L.m[w][16 * j + q_row], lw = L.l[w][16 * j + q_row];
      sum += mw == -INFINITY ? (lw == lw ? 0.f : lw) : lw * fast_exp2(mw - top);
    }
    if (r < r1) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) none = none || (acc[e] != acc[e] && sum == sum);
      const int i = r / P.G, head = hkv * P.G + r - i * P.G;
      const int64_t row = sq.first + i;
      if (whole_row) {
        const float inv = inverse_sum(sum);
        T* to = static_cast<T*>(A.out) + b * P.o_b + row * P.o_t + head * P.o_h + e0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] *= inv;
        store_piece(to, acc);
        if (A.lse != nullptr && e0 == 0) A.lse[b * P.l_b + row * P.l_t + head * P.l_h] = to_natural_lse(top, sum);
      } else {
        const int64_t at = part0 >= 0 ? part0 + (r - r0) : ((int64_t)part_no * P.tokens + row) * P.Hq + head;
        float* to = A.part.o + at * D + e0;
        store_piece(to, acc);
        if (e0 == 0) A.part.ml[at] = make_float2(top, sum);
      }
    }
  }
  // one new token alone sees all tokens of the stretch: what it has is its own
  return __syncthreads_or(none && r0 / P.G != (r1 - 1) / P.G);
}

// the call cut on a grid: (head, sequence, stretch, block of rows), or (head, stretch, block of the call)
// LISTED: the latter (not in the other kernels: the search costs 0.9 of 13 us).  By workgroup idx.
template <class T, int D, int NQ, int WAVES, bool LISTED>
__device__ __forceinline__ void attend_on_grid(const Paged& P, const AttendPlan& pl, const AttendArgs& A, SplitLds<T, D, NQ, WAVES>& L, int idx) {
  constexpr int kRows = 16 * NQ;
  const int hkv = idx % P.Hkv;
  idx /= P.Hkv;
  const int own_b = idx % P.B;
  if (!LISTED) idx /= P.B;
  const int part_no = idx % pl.parts, turn_no = LISTED ? idx / pl.parts : in_turn(pl, idx / pl.parts);
  auto blocks = [&](auto&& block) __attribute__((always_inline)) {
    int b = own_b, r0 = (pl.row_blocks - 1 - turn_no) * kRows, k = turn_no;                // the last rows see most: first
    while (!LISTED || find_block(P, pl, A, k, b, r0)) {
      const Sequence sq = load_sequence(P, b, A.q_start, A.kv_len);
      const int rows_all = sq.m * P.G;
      if (rows_all <= pl.few || r0 >= rows_all) break;
      const int r1 = r0 + kRows < rows_all ? r0 + kRows : rows_all;
      const Stretch st = cut_rows(P, sq, r0, r1, pl.parts, pl.chunk);
      const int t_begin = st.begin + part_no * st.chunk, t_end = t_begin + st.chunk < st.end ? t_begin + st.chunk : st.end;
      if (part_no < st.parts) block(sq, b, r0, r1, t_begin, t_end, st.parts == 1);
      r0 += pl.row_blocks * kRows;                         // (more rows than the host expected)
      k += pl.blocks;
    }
  };
  bool again = false;
  blocks([&](const Sequence& sq, int b, int r0, int r1, int t_begin, int t_end, bool whole) __attribute__((always_inline)) {
    again = attend_stretch<T, D, NQ, WAVES>(P, A, L, sq, b, hkv, r0, r1, t_begin, t_end, whole, -1, part_no) || again;
  });
  if (__builtin_expect(!again, 1)) return;
  blocks([&](const Sequence& sq, int b, int r0, int r1, int t_begin, int t_end, bool whole) __attribute__((always_inline)) {
    if (!bad_unseen<T, D>(P, A, sq, b, hkv, r0, r1, t_begin, t_begin, t_end)) return;
    for (int r = r0 + (int)(threadIdx.x >> 6); r < r1; r += WAVES) redo_row_of<T, D>(P, A, sq, b, hkv, r, t_begin, t_end, whole, part_no);
  });
}

constexpr int kAgain = -1;                                  // for a unit's number of stretches: its rows may have to be done again

// What all lanes have alike, into scalar registers (what comes from LDS the compiler takes to differ by lane).
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// The call cut evenly: the tokens of all units, one after the other, are dealt to the workgroups in equal stretches, so that one round of the chip
// has the same to read everywhere whatever the lengths.  A workgroup's stretch can end in one unit and go on in the next; a unit's rows are
// joined from the stretches of the workgroups `first` .. that share it.  Every workgroup sums up the lengths for itself.
constexpr int kEvenLeast = 256;          // tokens of a stretch, at least

// what sequence b has to read per KV head, to whole tiles: nothing if its rows are not for this kernel or see nothing
struct Span {
  int begin, end, padded;
};
__device__ __forceinline__ Span span_of(const Paged& P, const AttendPlan& pl, const Sequence& sq) {
  Span s{0, 0, 0};
  if (sq.m < 1 || (pl.only_few && sq.m * P.G > pl.few)) return s;
  const int64_t end = (int64_t)sq.base + sq.m;
  s.end = end < 0 ? 0 : end < sq.n ? (int)end : sq.n;
  const int low = first_seen(P, sq.base);
  s.begin = low < s.end ? low : s.end;
  s.padded = (s.end - s.begin + 31) & ~31;
  return s;
}

template <class T, int D, int NQ>
struct EvenLds {
  SplitLds<T, D, NQ> split;
  int64_t wave_sum[kWaves], found_at;
  int found_b;
};
// by workgroup me of wgs
template <class T, int D, int NQ>
__device__ __forceinline__ void attend_evenly(const Paged& P, const AttendPlan& pl, const AttendArgs& A, EvenLds<T, D, NQ>& E, int me, int wgs) {
  auto& L = E.split;
  constexpr int kRows = 16 * NQ, kThreads = 64 * kWaves;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto length = [&](int b) { return b < P.B ? span_of(P, pl, load_sequence(P, b, A.q_start, A.kv_len)).padded : 0; };
  // all tokens, and how many stand before the thread's sequences, which are neighbours
  const int each = (P.B + kThreads - 1) / kThreads, b_first = tid * each;
  int64_t run = 0;
  for (int j = 0; j < each; ++j) run += length(b_first + j);
  int64_t to = run;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const int64_t y = __shfl_up(to, s);
    if (lane >= s) to += y;
  }
  if (lane == 63) E.wave_sum[wave] = to;
  if (tid == 0) E.found_b = -1;
  __syncthreads();
  int64_t all = 0, before = to - run;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) { if (w < wave) before += E.wave_sum[w]; all += E.wave_sum[w]; }
  all = uniform(all) * P.Hkv;
  int64_t per = (all + wgs - 1) / wgs;
  per = per < kEvenLeast ? kEvenLeast : (per + 127) / 128 * 128;
  int64_t at = me * per;
  const int64_t stop = at + per < all ? at + per : all;
  // the sequence that the stretch begins in, and where that begins
  if (at < stop && run > 0 && before * P.Hkv <= at && at < (before + run) * P.Hkv) {
    int b = b_first;
    for (int n = length(b); at >= (before + n) * P.Hkv; n = length(++b)) before += n;
    E.found_b = b;
    E.found_at = before * P.Hkv;
  }
  // rows that see nothing
  int2* meta = A.part.meta;
  for (int b = me; b < P.B; b += wgs) {
    const Sequence sq = load_sequence(P, b, A.q_start, A.kv_len);
    const bool mine_too = sq.m > 0 && !(pl.only_few && sq.m * P.G > pl.few);
    if (!mine_too || span_of(P, pl, sq).padded > 0) continue;
    for (int h = tid; h < P.Hkv; h += kThreads) meta[b * P.Hkv + h] = make_int2(0, 1);
    for (int64_t x = tid; x < (int64_t)sq.m * P.Hq * (D / 4); x += kThreads) {
      const int e = (int)(x % (D / 4)) * 4, head = (int)(x / (D / 4) % P.Hq), i = (int)(x / (D / 4) / P.Hq);
      const float none[4] = {0.f, 0.f, 0.f, 0.f};
      store_piece(static_cast<T*>(A.out) + b * P.o_b + (int64_t)(sq.first + i) * P.o_t + head * P.o_h + e, none);
      if (A.lse != nullptr && e == 0) A.lse[b * P.l_b + (int64_t)(sq.first + i) * P.l_t + head * P.l_h] = -INFINITY;
    }
  }
  __syncthreads();
  int b = __builtin_amdgcn_readfirstlane(E.found_b);
  int64_t b_at = uniform(E.found_at);
  while (b >= 0 && at < stop) {
    const Sequence sq = load_sequence(P, b, A.q_start, A.kv_len);
    const Span sp = span_of(P, pl, sq);
    if (sp.padded == 0) { ++b; continue; }
    const int64_t b_end = b_at + (int64_t)sp.padded * P.Hkv;
    while (at < stop && at < b_end) {
      const int h = (int)((at - b_at) / sp.padded);
      const int64_t unit_at = b_at + (int64_t)h * sp.padded, unit_end = unit_at + sp.padded;
      const int64_t until = unit_end < stop ? unit_end : stop;
      const int first = (int)(unit_at / per), last = (int)((unit_end - 1) / per);
      const int rows_all = sq.m * P.G;
      // More rows than the host expected of any sequence: block after block and whole, by the workgroup that the unit begins in.
      const bool alone = rows_all > kRows;
      if (tid == 0 && first == me) meta[b * P.Hkv + h] = make_int2(first, alone ? 1 : last - first + 1);
      const int t_begin = sp.begin + (int)(at - unit_at), t_stop = sp.begin + (int)(until - unit_at);
      if (!alone || first == me)
        for (int r0 = 0; r0 < rows_all; r0 += kRows) {
          const int r1 = r0 + kRows < rows_all ? r0 + kRows : rows_all;
          Stretch st{t_begin, t_stop < sp.end ? t_stop : sp.end, 1, 0};
          if (alone) st = cut_rows(P, sq, r0, r1, 1, 1 << 30);               // what the block sees, which is not what the unit does
          const bool again = attend_stretch<T, D, NQ, kWaves>(P, A, L, sq, b, h, r0, r1, st.begin, st.end, alone || first == last, (int64_t)(2 * me + (first == me)) * kRows, 0);
          // (the kernel that joins sees to it, for those of several stretches without being told)
          if (again && (alone || first == last) && tid == 0) meta[b * P.Hkv + h].y = kAgain;
        }
      at = until;
    }
    b_at = b_end;
    ++b;
  }
}

}  // namespace ccd
