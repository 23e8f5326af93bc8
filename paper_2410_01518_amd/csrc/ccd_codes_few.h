// Few rows per unit over a cache of codes: the part of ccd_attend_few.h that reads it (included there).
//
// As with bf16 caches a workgroup's waves go their own ways through the tiles of a stretch, each with the heads that share a KV head as the rows of its products, and put
// their sums together in the end.  A tile is 32 tokens: quads of lanes read 64 bytes of a row, keys into registers and from there into the wave's piece of LDS, values
// straight into it, the next tile's while this one is worked on.  Keys come back as rows, values by the transposing read (ds_read_b64_tr_b8), and
// codes become bf16 numbers on their way into the matrix instructions, exactly.  A lane looks up one token of the tile, its page and its two scales.  The keys' scale is a
// factor of the logit, the values' one of the weight.  fp32 queries and weights are the sum of three bf16 numbers each: three products, and nothing rounded.
//
// Bound by the reading of the cache, d bytes and four of scale per token, head and side, and by the waves that are there to wait for it: a tile is half the bytes
// of a bf16 one.  So values take no registers on their way, and three waves share a SIMD.  Measured, bf16 queries, 32 heads on 8 of 128, int8: one sequence of 131072 tokens
// 59 - 61 us (4.5 - 4.7 TB/s), 64 of 500 .. 8192 100 us (4.4 TB/s; 115 with values through registers and two waves), 256 of them 316 us (4.9 TB/s; 357 so); fp32 queries, the 64 114 us, e4m3 105.  Tiles of 64 tokens spill: 135 us for the 64;
// tiles asked for two ahead change nothing.
#pragma once

namespace ccd {

// eight codes as an operand
template <int CODE>
__device__ __forceinline__ v8bf operand(uint32_t lo, uint32_t hi) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  v4u w;
  if constexpr (CODE == kInt8) {
    float x[4], y[4];
    numbers<CODE>(lo, x);
    numbers<CODE>(hi, y);
    // (whole numbers of 8 bits: the upper half of a float is all of it)
    auto upper = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302); };
    w = v4u{upper(x[0], x[1]), upper(x[2], x[3]), upper(y[0], y[1]), upper(y[2], y[3])};
  } else {
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const v2bf c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    w = v4u{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d)};
  }
  return __builtin_bit_cast(v8bf, w);
}

// x as a sum of bf16 numbers, the largest first: one (rounded), or three, which are all of an fp32 number
template <int PARTS>
__device__ __forceinline__ void cut(const float (&x)[8], v8bf (&f)[PARTS]) {
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = x[e];
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    const v4u w = {pack_bf16(rest[0], rest[1]), pack_bf16(rest[2], rest[3]), pack_bf16(rest[4], rest[5]), pack_bf16(rest[6], rest[7])};
    f[p] = __builtin_bit_cast(v8bf, w);
#pragma unroll
    for (int e = 0; e < 4 && p + 1 < PARTS; ++e) {
      rest[2 * e] -= __uint_as_float(w[e] << 16);
      rest[2 * e + 1] -= __uint_as_float(w[e] & 0xFFFF0000u);
    }
  }
}

// Part h, row r of a tile (LDS row 16 h + r) is its token kHalves r + h, so that a lane group's scales lie side by side, and a quad of lanes has row r of all parts.
template <class Q, int CODE, int D>
struct Tile<Coded<Q, CODE>, D> {
  static constexpr int kTokens = 32, kHalves = kTokens / 16, kBlocks = D / 16, kSteps = D / 32;                           // (steps of 32 elements)
  static constexpr int kPlanes = D / 64, kPlane = kTokens * 64, kLoads = kPlanes * kHalves;                               // LDS has planes of 64 bytes of every row
  static constexpr int kParts = sizeof(Q) == 4 ? 3 : 1;                            // bf16 numbers per element of a query, per weight
  static constexpr int kSide = kTokens * D;                                        // bytes of keys, or values
  static constexpr int kLdsBytes = 3 * kSide + 2 * kTokens * 4;                    // keys, values twice, scales
  struct Query { v8bf f[kSteps][kParts]; };
  struct Rows { v4u r[kLoads]; };

  // step 2 u + v: elements 16 (4 u + g) + 8 v .. of lane group g, as the codes of a piece give them
  __device__ static void load_query(Query& q, const Q* row, int lane, bool there) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int e0 = 16 * (4 * (s >> 1) + (lane >> 4)) + 8 * (s & 1);
      float x[8] = {};
      if (there) {
        if constexpr (sizeof(Q) == 2) {
          load_f32(*reinterpret_cast<const v4u*>(row + e0), x, row);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = row[e0 + e];
        }
      }
      cut(x, q.f[s]);
    }
  }
  // the lane's token, that of part h, row r, and a lane that has it
  __device__ static int own_token(int lane) { return kHalves * (lane >> 2) + lane % kHalves; }
  __device__ static int token_of(int h, int r) { return kHalves * r + h; }
  __device__ static int lane_of(int h, int r) { return 4 * r + h; }
  // The pieces of 16 bytes of a row's 64 change places by the row's number, so that what a read takes together lies in all banks: 16 rows of keys, one
  // piece; 16 rows of values, 4 g .. of two parts and two lane groups, one piece.
  __device__ static int key_swap(int row) { return (row >> 2) & 3; }
  __device__ static int value_swap(int row) { return ((row >> 2) & 1) | ((row >> 4) & 1) << 1; }
  // Load (u, h): 64 bytes, plane u, of row 16 h + quad.  own: the row of the lane's own token.
  __device__ static void load_keys(Rows& k, const char* own, int lane) {
    const int at = 16 * (lane & 3);
#pragma unroll
    for (int u = 0; u < kPlanes; ++u) {
      k.r[kHalves * u] = *reinterpret_cast<const v4u*>(of_row<4, 0>(own) + 64 * u + at);
      k.r[kHalves * u + 1] = *reinterpret_cast<const v4u*>(of_row<4, 1>(own) + 64 * u + at);
    }
  }
  __device__ static void store_keys(const Rows& k, char* lds, int lane) {
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      const int row = 16 * (n % kHalves) + (lane >> 2);
      *reinterpret_cast<v4u*>(lds + n / kHalves * kPlane + row * 64 + (((lane & 3) ^ key_swap(row)) << 4)) = k.r[n];
    }
  }
  // values straight into LDS
  __device__ static void load_values(uint32_t lds_addr, const char* own, int lane) {
#pragma unroll
    for (int u = 0; u < kPlanes; ++u) {
      load_to_lds(lds_addr + u * kPlane, of_row<4, 0>(own) + 64 * u + (((lane & 3) ^ value_swap(lane >> 2)) << 4));
      load_to_lds(lds_addr + u * kPlane + 1024, of_row<4, 1>(own) + 64 * u + (((lane & 3) ^ value_swap(16 + (lane >> 2))) << 4));
    }
  }
  // x[j][h][i] = <q, code> of token kHalves (4 g + i) + h, row lane & 15 of block j
  template <int NQ>
  __device__ static void logits(v4f (&x)[NQ][kHalves], const char* lds, const Query (&q)[NQ], int lane) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      const int row = 16 * h + (lane & 15);
#pragma unroll
      for (int j = 0; j < NQ; ++j) x[j][h] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < D / 64; ++u) {
        const v4u k = *reinterpret_cast<const v4u*>(lds + u * kPlane + row * 64 + (((lane >> 4) ^ key_swap(row)) << 4));
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const v8bf a = operand<CODE>(k[2 * v], k[2 * v + 1]);
#pragma unroll
          for (int j = 0; j < NQ; ++j)
#pragma unroll
            for (int p = kParts - 1; p >= 0; --p) x[j][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[j].f[2 * u + v][p], x[j][h], 0, 0, 0);
        }
      }
    }
  }
  struct Weights { v8bf w[kParts]; };
  // o[j][c][i] += element 16 c + 4 g + i of the values, for row lane & 15
  template <int NQ>
  __device__ static void add_values(v4f (&o)[NQ][kBlocks], const Weights (&w)[NQ], const char* lds, int lane) {
    typedef int v2i __attribute__((ext_vector_type(2)));
    const int at = (lane & 15) >> 1, row = 16 * (at >> 2) + 4 * (lane >> 4) + (at & 3);
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
      const char* piece = lds + (c >> 2) * kPlane + row * 64 + (((c & 3) ^ value_swap(row)) << 4) + (lane & 1) * 8;
      const v2i t = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) v2i*)piece);
      const v8bf a = operand<CODE>((uint32_t)t[0], (uint32_t)t[1]);
#pragma unroll
      for (int j = 0; j < NQ; ++j)
#pragma unroll
        for (int p = kParts - 1; p >= 0; --p) o[j][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[j].w[p], o[j][c], 0, 0, 0);
    }
  }
  __device__ static int element(int c, int lane, int i) { return 16 * c + 4 * (lane >> 4) + i; }
};

// attend_stretch over codes
template <class T, int D, int NQ, int WAVES>
__device__ __forceinline__ bool attend_stretch_codes(const Paged& P, const AttendArgs& A, SplitLds<T, D, NQ, WAVES>& L, const Sequence& sq, int b, int hkv, int r0, int r1,
                                                     int t_begin, int t_end, bool whole_row, int64_t part0, int part_no) {
  using Tl = Tile<T, D>;
  using Q = OutOf<T>;
  constexpr int kStride = WAVES * Tl::kTokens;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), group = lane >> 4;
  const int32_t* pages = A.table + (int64_t)b * P.table_width;
  const uint8_t* Kh = static_cast<const uint8_t*>(A.K) + hkv * P.head_stride;
  const uint8_t* Vh = static_cast<const uint8_t*>(A.V) + hkv * P.head_stride;
  const float* Ks = A.K_scales + hkv * A.codes.head;
  const float* Vs = A.V_scales + hkv * A.codes.head;
  char* keys_lds = L.wave[wave];
  float* scales_lds = reinterpret_cast<float*>(keys_lds + 3 * Tl::kSide);
  const uint32_t values_at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(keys_lds + Tl::kSide));
  // Keys, values and scales of a tile are asked for a tile ahead, the pages they are in two tiles ahead; values go straight into LDS, to the place that the tile before
  // the last left.
  typename Tl::Rows keys;
  float ks = 0.f, vs = 0.f;
  int id = -1, slot = 0;                                    // slot: of the values being asked for
  bool own_there = false;
  const int own = Tl::own_token(lane);
  auto look_up = [&](int t0) {
    const int t = t0 + own;
    id = t < t_end ? pages[page_of(P.div, t)] : -1;
  };
  auto ask = [&](int t0) {
    const int t = t0 + own, at = t - page_of(P.div, t) * P.div.page;
    own_there = id >= 0 && id < P.n_pages;
    ks = vs = 0.f;
    const char *k = reinterpret_cast<const char*>(g_zero_row), *v = k;
    if (own_there) {
      const int64_t s = id * A.codes.page + (at >> A.codes.shift), off = id * P.page_stride + (int64_t)at * P.row_stride;
      ks = Ks[s];
      vs = Vs[s];
      k = reinterpret_cast<const char*>(Kh + off);
      v = reinterpret_cast<const char*>(Vh + off);
    }
    Tl::load_values(__builtin_amdgcn_readfirstlane(values_at + slot), v, lane);
    Tl::load_keys(keys, k, lane);
  };
  int t0 = t_begin + wave * Tl::kTokens;
  if (t0 < t_end) {
    look_up(t0);
    ask(t0);
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
    Tl::load_query(q[j], static_cast<const Q*>(A.Q) + b * P.q_b + (int64_t)(sq.first + i) * P.q_t + (int64_t)(hkv * P.G + r - i * P.G) * P.q_h, lane, r < r1);
  }
  // l: sums of weights; ls, lr: of weights times the values' scales, as they are and as rounded for the product
  float m[NQ], l[NQ], ls[NQ], lr[NQ];
  v4f o[NQ][Tl::kBlocks];
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    m[j] = -INFINITY; l[j] = ls[j] = lr[j] = 0.f;
#pragma unroll
    for (int c = 0; c < Tl::kBlocks; ++c) o[j][c] = v4f{0.f, 0.f, 0.f, 0.f};
  }
  for (; t0 < t_end; t0 += kStride) {
    // what was asked for is there (loads into LDS do not arrive in the order they were asked for), and what the tile before read of LDS has been read
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    // (by lanes, all that have the token)
    const uint64_t there = __ballot(own_there);
    const bool whole = there == ~(uint64_t)0 && t0 + Tl::kTokens - 1 <= pos_min && t0 >= low_max;
    // (a value's scale that is no number makes a weight of 0 none: of tokens that are seen it has to, of others it must not)
    const bool guarded = !whole && __any(!(fabsf(vs) < INFINITY));
    auto unseen = [&](int j, int h, int i) {
      const int t = t0 + Tl::token_of(h, 4 * group + i);
      return !((there >> Tl::lane_of(h, 4 * group + i)) & 1u) || t > pos[j] || t < low[j];
    };
    const char* values_lds = keys_lds + Tl::kSide + slot;
    Tl::store_keys(keys, keys_lds, lane);
    scales_lds[own] = ks;
    scales_lds[Tl::kTokens + own] = vs;
    if (t0 + kStride < t_end) {
      slot ^= Tl::kSide;
      ask(t0 + kStride);
      look_up(t0 + 2 * kStride);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    v4f x[NQ][Tl::kHalves], sk[Tl::kHalves], sv[Tl::kHalves];       // scales of the group's tokens, 4 kHalves g ..
#pragma unroll
    for (int n = 0; n < Tl::kHalves; ++n) {
      sk[n] = *reinterpret_cast<const v4f*>(scales_lds + 4 * Tl::kHalves * group + 4 * n);
      sv[n] = *reinterpret_cast<const v4f*>(scales_lds + Tl::kTokens + 4 * Tl::kHalves * group + 4 * n);
    }
    auto scale_of = [](const v4f (&s)[Tl::kHalves], int h, int i) { return s[(Tl::kHalves * i + h) >> 2][(Tl::kHalves * i + h) & 3]; };
    Tl::logits(x, keys_lds, q, lane);
    typename Tl::Weights w[NQ];
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      float top = -INFINITY;
#pragma unroll
      for (int h = 0; h < Tl::kHalves; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[j][h][i] *= scale_of(sk, h, i);
          if (!whole && unseen(j, h, i)) x[j][h][i] = -INFINITY;
          top = fmaxf(top, x[j][h][i]);
        }
      top *= P.scale_log2;
      if (__any(top > m[j] + kRaise)) {
        const float next = fmaxf(m[j], row_max(top));
        const float keep = next == -INFINITY ? 1.f : fast_exp2(m[j] - next);
        m[j] = next;
        l[j] *= keep;
        ls[j] *= keep;
        lr[j] *= keep;
#pragma unroll
        for (int c = 0; c < Tl::kBlocks; ++c) o[j][c] *= keep;
      }
      const float ref = m[j] == -INFINITY ? 0.f : m[j];
      float e[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int h = k >> 2, i = k & 3;
        const float weight = fast_exp2(fmaf(x[j][h][i], P.scale_log2, -ref));
        l[j] += weight;
        e[k] = weight * scale_of(sv, h, i);
      }
      if (__builtin_expect(guarded, 0)) {
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = unseen(j, k >> 2, k & 3) ? 0.f : e[k];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) ls[j] += e[k];
      cut(e, w[j].w);
      if constexpr (Tl::kParts == 1) {
#pragma unroll
        for (int p = 0; p < 4; ++p) lr[j] = add_rounded(w[j].w[0], p, lr[j]);
      }
    }
    Tl::add_values(o, w, values_lds, lane);
    __builtin_amdgcn_wave_barrier();
  }
  float fix[NQ];
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    l[j] = row_sum(l[j]);
    fix[j] = Tl::kParts == 1 ? unrounded(row_sum(ls[j]), row_sum(lr[j])) : 1.f;
  }
  return join_waves<T, D, NQ, WAVES>(P, A, L, sq, b, hkv, r0, r1, whole_row, part0, part_no, m, l, fix, o);
}

}  // namespace ccd
