// ccd_paged_attend, few rows per unit and fp32 caches: a workgroup per (unit, block of 16, 32 or 64 rows, stretch of tokens).
//
// Decoding reads every key and value once for a handful of rows and is bound by memory.  So the work is cut along the tokens, fine
// enough to fill the chip evenly whatever the lengths, and a workgroup's waves go their own ways: wave w takes tiles w, w + 4, ... of the
// stretch, keys straight from memory into the registers that the matrix instructions read (D[token][row] = K Q^T: the keys' lanes
// hold 16 bytes of a row, as they lie in memory), without a barrier.  The product with the values needs them transposed, D[d][row] = V^T
// W^T: bf16 values go through the wave's own piece of LDS and come back by transposing reads; fp32 values can be loaded as they are
// needed.  Weights need not move at all: a lane holds those of tokens 4g .. 4g + 3 of its row, which is an operand if the tokens of the
// product are counted in that order.  The waves join their sums at the end; stretches are joined by a second kernel.
#include "ccd_attend.h"
#include "ccd_rotary.h"

namespace ccd {

constexpr int kWaves = 4;

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
      if (there) w = *reinterpret_cast<const v4u*>(row + 32 * s + 8 * (lane >> 4));
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
#pragma unroll
      for (int s = 0; s < kSteps; ++s) r[h][s] = *reinterpret_cast<const v4u*>(x + 32 * s + 8 * (lane >> 4));
    }
  }
  // 16-byte pieces of a row, exchanged in pairs by the row's number so that the rows a transposing read takes together (16 rows, one pair
  // of pieces) lie in different banks
  __device__ static int piece_at(int row, int piece) {
    const int swap = D == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1;
    return row * (D * 2) + ((piece ^ swap) << 4);
  }
  __device__ static void store_values(const Values& r, char* lds, int lane) {
#pragma unroll
    for (int h = 0; h < kHalves; ++h)
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        *reinterpret_cast<v4u*>(lds + piece_at(16 * h + (lane & 15), 4 * s + (lane >> 4))) = r.v[h][s];
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
  // o[c][i] += element 16 c + 4 (lane >> 4) + i of the values, for row lane & 15
  template <int NQ>
  __device__ static void add_values(v4f (&o)[NQ][kBlocks], const Weights (&w)[NQ], const Values&, const char* lds, int lane) {
    const int row = 4 * (lane >> 4) + ((lane & 15) >> 2);
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
      v4s t[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const char* p = lds + piece_at(16 * h + row, 2 * c + ((lane & 3) >> 1)) + (lane & 1) * 8;
        t[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(p));
      }
      const v8bf a = __builtin_bit_cast(v8bf, __builtin_shufflevector(t[0], t[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int j = 0; j < NQ; ++j) o[j][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w[j].w, o[j][c], 0, 0, 0);
    }
  }
  __device__ static int element(int c, int lane, int i) { return 16 * c + 4 * (lane >> 4) + i; }
};

// fp32: 16 tokens (v_mfma_f32_16x16x4_f32).  Elements of a row are counted in the products so that a lane's share of a row is 16 bytes:
// step (j, i) takes element 16 j + 4 g + i of lane group g.
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

// over the four lanes that hold a row
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// waves per SIMD that the registers are cut for: what the rows of queries and of sums leave room for
template <class T, int D, int NQ>
constexpr int split_waves() { return NQ == 4 ? 1 : NQ == 2 || (sizeof(T) == 4 && D == 128) ? 2 : D == 128 ? 3 : 4; }

template <class T, int D, int NQ>
__global__ __launch_bounds__(64 * kWaves, (split_waves<T, D, NQ>())) void attend_split_kernel(Paged P, AttendPlan pl, const T* __restrict__ Q, const T* __restrict__ K, const T* __restrict__ V,
                                                                     const int32_t* __restrict__ table, const int32_t* __restrict__ q_start,
                                                                     const int32_t* __restrict__ kv_len, T* __restrict__ out, float* __restrict__ lse,
                                                                     Partials part) {
  using Tl = Tile<T, D>;
  constexpr int kRows = 16 * NQ, kPitch = D + 4;
  constexpr int kWaveBytes = Tl::kLdsBytes > 16 * kPitch * 4 ? Tl::kLdsBytes : 16 * kPitch * 4;
  __shared__ __align__(16) char lds[kWaves][kWaveBytes];
  __shared__ float wave_m[kWaves][kRows], wave_l[kWaves][kRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int units = P.B * P.Hkv;
  int idx = blockIdx.x;
  const int unit = idx % units;
  idx /= units;
  const int part_no = idx % pl.parts, block0 = pl.row_blocks - 1 - idx / pl.parts;       // the last rows see most: first
  const int b = unit / P.Hkv, hkv = unit % P.Hkv;
  const Sequence sq = load_sequence(P, b, q_start, kv_len);
  const int rows_all = sq.m * P.G;
  const int32_t* pages = table + (int64_t)b * P.table_width;
  const T* Kh = K + hkv * P.head_stride;
  const T* Vh = V + hkv * P.head_stride;

  for (int r0 = block0 * kRows; r0 < rows_all; r0 += pl.row_blocks * kRows) {
    const int r1 = r0 + kRows < rows_all ? r0 + kRows : rows_all;
    const Stretch st = cut_rows(P, sq, r0, r1, pl.parts, pl.chunk);
    if (part_no >= st.parts) continue;
    const int t_begin = st.begin + part_no * st.chunk, t_end = t_begin + st.chunk < st.end ? t_begin + st.chunk : st.end;
    // the lane's rows
    typename Tl::Query q[NQ];
    int pos[NQ], low[NQ];                                    // position of the row, first position it sees
    const int pos_min = sq.base + r0 / P.G, low_max = first_seen(P, sq.base + (r1 - 1) / P.G);
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const int r = r0 + 16 * j + (lane & 15), i = r / P.G;
      pos[j] = sq.base + i;
      low[j] = first_seen(P, pos[j]);
      Tl::load_query(q[j], Q + b * P.q_b + (int64_t)(sq.first + i) * P.q_t + (int64_t)(hkv * P.G + r - i * P.G) * P.q_h, lane, r < r1);
    }
    float m[NQ], l[NQ];
    v4f o[NQ][Tl::kBlocks];
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      m[j] = -INFINITY; l[j] = 0.f;
#pragma unroll
      for (int c = 0; c < Tl::kBlocks; ++c) o[j][c] = v4f{0.f, 0.f, 0.f, 0.f};
    }
    auto offsets = [&](int t0, int64_t (&off)[Tl::kHalves]) {
#pragma unroll
      for (int h = 0; h < Tl::kHalves; ++h) {
        const int t = t0 + 16 * h + (lane & 15);
        off[h] = -1;
        if (t < t_end) {
          const int c = page_of(P.div, t), id = pages[c];
          if (id >= 0 && id < P.n_pages) off[h] = id * P.page_stride + (int64_t)(t - c * P.div.page) * P.row_stride;
        }
      }
    };
    typename Tl::Keys keys;
    typename Tl::Values values;
    int64_t off[Tl::kHalves];
    int t0 = t_begin + wave * Tl::kTokens;
    if (t0 < t_end) {
      offsets(t0, off);
      Tl::load_keys(keys, Kh, off, lane);
      Tl::load_values(values, Vh, off, lane);
    }
    for (; t0 < t_end; t0 += kWaves * Tl::kTokens) {
      uint32_t there = (uint32_t)__ballot(off[0] >= 0) & 0xFFFFu;
      if constexpr (Tl::kHalves == 2) there |= (uint32_t)__ballot(off[Tl::kHalves - 1] >= 0) << 16;
      const bool more = t0 + kWaves * Tl::kTokens < t_end;
      if (more) offsets(t0 + kWaves * Tl::kTokens, off);
      // the next tile's rows are asked for as soon as this one's are out of their registers
      Tl::store_values(values, lds[wave], lane);
      if (more && !Tl::kValuesLate) Tl::load_values(values, Vh, off, lane);
      v4f x[NQ][Tl::kHalves];
#pragma unroll
      for (int j = 0; j < NQ; ++j) Tl::logits(x[j], keys, q[j]);
      if (more) Tl::load_keys(keys, Kh, off, lane);
      const bool whole = there == (Tl::kHalves == 2 ? 0xFFFFFFFFu : 0xFFFFu) && t0 + Tl::kTokens - 1 <= pos_min && t0 >= low_max;
      typename Tl::Weights w[NQ];
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        float top = -INFINITY;
#pragma unroll
        for (int h = 0; h < Tl::kHalves; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float y = x[j][h][i] * P.scale_log2;
            if (!whole) {
              const int at = 16 * h + 4 * (lane >> 4) + i, t = t0 + at;
              if (!((there >> at) & 1u) || t > pos[j] || t < low[j]) y = -INFINITY;
            }
            x[j][h][i] = y;
            top = fmaxf(top, y);
          }
        if (__any(top > m[j] + kRaise)) {
          const float next = fmaxf(m[j], row_max(top));
          const float keep = next == -INFINITY ? 1.f : fast_exp2(m[j] - next);
          m[j] = next;
          l[j] *= keep;
#pragma unroll
          for (int c = 0; c < Tl::kBlocks; ++c) o[j][c] *= keep;
        }
        const float ref = m[j] == -INFINITY ? 0.f : m[j];
#pragma unroll
        for (int h = 0; h < Tl::kHalves; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float e = fast_exp2(x[j][h][i] - ref);
            x[j][h][i] = e;
            l[j] += e;
          }
        w[j] = Tl::weights(x[j]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      Tl::add_values(o, w, values, lds[wave], lane);
      __builtin_amdgcn_wave_barrier();
      if (more && Tl::kValuesLate) Tl::load_values(values, Vh, off, lane);
    }

    // the waves' sums together: all to the largest reference, 16 rows at a time through LDS
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      l[j] = row_sum(l[j]);
      if (lane < 16) { wave_m[wave][16 * j + lane] = m[j]; wave_l[wave][16 * j + lane] = l[j]; }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      float all = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) all = fmaxf(all, wave_m[w][16 * j + (lane & 15)]);
      const float keep = m[j] == -INFINITY ? (l[j] == l[j] ? 0.f : l[j]) : fast_exp2(m[j] - all);
      float* mine = reinterpret_cast<float*>(lds[wave]) + (lane & 15) * kPitch;
      if (j > 0) __syncthreads();
#pragma unroll
      for (int c = 0; c < Tl::kBlocks; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[Tl::element(c, lane, i)] = o[j][c][i] * keep;
      __syncthreads();
      // 16 rows of D elements by 256 threads
      constexpr int kPer = 16 * D / (64 * kWaves);           // 4 or 8 elements a thread
      const int q_row = tid / (D / kPer), e0 = tid % (D / kPer) * kPer, r = r0 + 16 * j + q_row;
      float acc[kPer] = {}, top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float* from = reinterpret_cast<const float*>(lds[w]) + q_row * kPitch + e0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] += from[e];
        top = fmaxf(top, wave_m[w][16 * j + q_row]);
      }
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float mw = wave_m[w][16 * j + q_row], lw = wave_l[w][16 * j + q_row];
        sum += mw == -INFINITY ? (lw == lw ? 0.f : lw) : lw * fast_exp2(mw - top);
      }
      if (r < r1) {
        const int i = r / P.G, head = hkv * P.G + r - i * P.G;
        const int64_t row = sq.first + i;
        if (st.parts == 1) {
          const float inv = inverse_sum(sum);
          T* to = out + b * P.o_b + row * P.o_t + head * P.o_h + e0;
#pragma unroll
          for (int e = 0; e < kPer; ++e) store_elem(to + e, acc[e] * inv);
          if (lse != nullptr && e0 == 0) lse[b * P.l_b + row * P.l_t + head * P.l_h] = to_natural_lse(top, sum);
        } else {
          const int64_t at = ((int64_t)part_no * P.tokens + row) * P.Hq + head;
          float* to = part.o + at * D + e0;
#pragma unroll
          for (int e = 0; e < kPer; ++e) to[e] = acc[e];
          if (e0 == 0) part.ml[at] = make_float2(top, sum);
        }
      }
    }
    __syncthreads();
  }
}

// joins the stretches of a row: one wave per (new token, query head)
template <class T, int D>
__global__ __launch_bounds__(256) void attend_join_kernel(Paged P, AttendPlan pl, Partials part, const int32_t* __restrict__ q_start,
                                                          const int32_t* __restrict__ kv_len, T* __restrict__ out, float* __restrict__ lse) {
  const int64_t at0 = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int row = (int)(at0 / P.Hq), head = (int)(at0 % P.Hq);
  if (row >= P.tokens || row < q_start[0] || row >= q_start[P.B]) return;
  int lo = 0, hi = P.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (q_start[mid] <= row) lo = mid; else hi = mid;
  }
  const Sequence sq = load_sequence(P, lo, q_start, kv_len);
  const int r = (row - sq.first) * P.G + head % P.G, r0 = r / pl.rows * pl.rows;
  const int rows_all = sq.m * P.G;
  if (r < 0 || r >= rows_all) return;
  const Stretch st = cut_rows(P, sq, r0, r0 + pl.rows < rows_all ? r0 + pl.rows : rows_all, pl.parts, pl.chunk);
  if (st.parts < 2) return;
  const int64_t step = (int64_t)P.tokens * P.Hq;
  float top = -INFINITY, sum = 0.f;
  for (int p = 0; p < st.parts; ++p) top = fmaxf(top, part.ml[at0 + p * step].x);
  float acc[D / 64] = {};
  for (int p = 0; p < st.parts; ++p) {
    const float2 ml = part.ml[at0 + p * step];
    const float keep = ml.x == -INFINITY ? (ml.y == ml.y ? 0.f : ml.y) : fast_exp2(ml.x - top);
    sum += ml.x == -INFINITY ? keep : ml.y * keep;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) acc[j] = fmaf(part.o[(at0 + p * step) * D + j * 64 + lane], keep, acc[j]);
  }
  const float inv = inverse_sum(sum);
#pragma unroll
  for (int j = 0; j < D / 64; ++j) store_elem(out + lo * P.o_b + row * P.o_t + head * P.o_h + j * 64 + lane, acc[j] * inv);
  if (lse != nullptr && lane == 0) lse[lo * P.l_b + row * P.l_t + head * P.l_h] = to_natural_lse(top, sum);
}

template <class T, int D>
static void split_launch(const Paged& P, const AttendPlan& pl, const void* Q, const void* K, const void* V, const int32_t* table,
                         const int32_t* q_start, const int32_t* kv_len, void* out, float* lse, Partials part, hipStream_t s) {
  const T *q = static_cast<const T*>(Q), *k = static_cast<const T*>(K), *v = static_cast<const T*>(V);
  T* o = static_cast<T*>(out);
  const dim3 grid((unsigned)((int64_t)P.B * P.Hkv * pl.parts * pl.row_blocks)), block(64 * kWaves);
  if (pl.rows == 16)      launch(attend_split_kernel<T, D, 1>, grid, block, s, P, pl, q, k, v, table, q_start, kv_len, o, lse, part);
  else if (pl.rows == 32) launch(attend_split_kernel<T, D, 2>, grid, block, s, P, pl, q, k, v, table, q_start, kv_len, o, lse, part);
  else                    launch(attend_split_kernel<T, D, 4>, grid, block, s, P, pl, q, k, v, table, q_start, kv_len, o, lse, part);
}

void launch_attend_split(const Paged& P, const AttendPlan& pl, int dtype, const void* Q, const void* K, const void* V, const int32_t* table,
                         const int32_t* q_start, const int32_t* kv_len, void* out, float* lse, Partials part, hipStream_t s) {
  if (dtype == 0) {
    if (P.d == 64) split_launch<float, 64>(P, pl, Q, K, V, table, q_start, kv_len, out, lse, part, s);
    else           split_launch<float, 128>(P, pl, Q, K, V, table, q_start, kv_len, out, lse, part, s);
  } else {
    if (P.d == 64) split_launch<uint16_t, 64>(P, pl, Q, K, V, table, q_start, kv_len, out, lse, part, s);
    else           split_launch<uint16_t, 128>(P, pl, Q, K, V, table, q_start, kv_len, out, lse, part, s);
  }
}

template <class T>
static void join_launch(const Paged& P, const AttendPlan& pl, Partials part, const int32_t* q_start, const int32_t* kv_len, void* out, float* lse,
                        hipStream_t s) {
  const dim3 grid((unsigned)(((int64_t)P.tokens * P.Hq + 3) / 4));
  if (P.d == 64) launch(attend_join_kernel<T, 64>, grid, dim3(256), s, P, pl, part, q_start, kv_len, static_cast<T*>(out), lse);
  else           launch(attend_join_kernel<T, 128>, grid, dim3(256), s, P, pl, part, q_start, kv_len, static_cast<T*>(out), lse);
}

void launch_attend_join(const Paged& P, const AttendPlan& pl, int dtype, Partials part, const int32_t* q_start, const int32_t* kv_len, void* out,
                        float* lse, hipStream_t s) {
  if (dtype == 0) join_launch<float>(P, pl, part, q_start, kv_len, out, lse, s);
  else            join_launch<uint16_t>(P, pl, part, q_start, kv_len, out, lse, s);
}

static AttendPlan plan_attend(const Paged& P, int dtype, int max_new, int max_len) {
  AttendPlan pl{};
  const int64_t rows = (int64_t)max_new * P.G;
  pl.by_rows = dtype != 0 && rows > 64;
  pl.rows = pl.by_rows ? 128 : rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  pl.row_blocks = (int)((rows + pl.rows - 1) / pl.rows);
  const int64_t units = (int64_t)P.B * P.Hkv * pl.row_blocks;
  int64_t len = max_len;
  if (P.window > 0 && len > (int64_t)P.window + max_new) len = (int64_t)P.window + max_new;
  // stretches: until some 1024 workgroups are under way (512 of the rows kernel), of 256 tokens at least
  int64_t parts = ((pl.by_rows ? 512 : 1024) + units - 1) / units;
  const int64_t most = (len + 255) / 256;
  if (parts > most) parts = most;
  if (parts > 64) parts = 64;
  if (parts < 1) parts = 1;
  pl.chunk = (int)(((len + parts - 1) / parts + 127) / 128 * 128);
  pl.parts = (int)((len + pl.chunk - 1) / pl.chunk);
  if (pl.parts < 1) pl.parts = 1;
  return pl;
}

size_t attend_workspace_bytes(const Paged& P, int dtype, int max_new, int max_len) {
  const AttendPlan pl = plan_attend(P, dtype, max_new, max_len);
  if (pl.parts < 2) return 256;
  const size_t rows = (size_t)P.tokens * P.Hq * pl.parts;
  return (rows * P.d * sizeof(float) + 255) / 256 * 256 + (rows * sizeof(float2) + 255) / 256 * 256;
}

void launch_attend(const Paged& P, int dtype, int max_new, int max_len, const void* Q, const void* K, const void* V, const int32_t* table,
                   const int32_t* q_start, const int32_t* kv_len, void* out, float* lse, void* workspace, hipStream_t s) {
  const AttendPlan pl = plan_attend(P, dtype, max_new, max_len);
  const size_t rows = (size_t)P.tokens * P.Hq * pl.parts;
  Partials part{static_cast<float*>(workspace),
                reinterpret_cast<float2*>(static_cast<char*>(workspace) + (rows * P.d * sizeof(float) + 255) / 256 * 256)};
  if (pl.by_rows) launch_attend_rows(P, pl, Q, K, V, table, q_start, kv_len, out, lse, part, s);
  else            launch_attend_split(P, pl, dtype, Q, K, V, table, q_start, kv_len, out, lse, part, s);
  if (pl.parts > 1) launch_attend_join(P, pl, dtype, part, q_start, kv_len, out, lse, s);
}

}  // namespace ccd
