// What the attention kernels share: how a call is cut, the tokens a block of rows sees, rows of pages, the running softmax.
//
//   out = sum_t w_t v_t / sum_t w_t,   w_t = 2^(scale log2(e) <q, k_t> - m)
// in one pass over the tokens.  m is a reference that only follows the largest logit at a distance: it is raised, and the sums so far
// scaled down by 2^(old - new), when a logit lies more than kRaise above it.  Weights are then at most 2^kRaise, far inside fp32, and most
// tiles cost no rescaling and no exchange between lanes.
//
// The rows of a unit (sequence, KV head) are its new tokens times the G query heads that share the head, row r = token r / G, head r % G:
// heads of one token lie side by side and see the same keys, and a block of rows is a narrow band of positions.
#pragma once
#include "ccd_codes.h"
#include "ccd_common.h"
#include "ccd_paged.h"
#include "ccd_rotary.h"

namespace ccd {

constexpr float kRaise = 8.f;

// What the kernels' T stands for: uint16_t and float, queries, cache and results of one type; Coded, a cache of codes under queries and results of type Q.
template <class Q, int CODE>
struct Coded {};
template <class T>
struct CacheOf {
  using Out = T;
  static constexpr bool kCoded = false;
};
template <class Q, int CODE_>
struct CacheOf<Coded<Q, CODE_>> {
  using Out = Q;
  static constexpr bool kCoded = true;
  static constexpr int kCode = CODE_;
};
template <class T>
using OutOf = typename CacheOf<T>::Out;

typedef short v4s __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

// How a call is cut.  On a grid: blocks of `rows` rows, each over at most `parts` stretches of its tokens; chunk: tokens per stretch, made longer where
// that gives more than `parts` (so the host's idea of the lengths only decides how well the work is spread); sequences of `few` rows or less
// are left to the even cut.  Evenly: `parts` workgroups, at most `rows` rows per unit; only_few: sequences of more than `few` rows are left to the grid.
// join: rows of a unit, as far as the host knows.
// turn: blocks of rows of the first half of one round (in_turn), 0: the call is more than one round.
// wide: workgroups of eight waves, not four.  sums: of the rounded weights, too (rows kernel).
// blocks: 0: the grid has row_blocks blocks of rows for every sequence; else it has these for all (find_block).
struct AttendPlan {
  int by_rows, rows, row_blocks, blocks, parts, chunk, few, only_few, turn, join, wide, sums;
};

// The last rows see most and come first.  Where the call is one round of two workgroups per compute unit, its second half runs the other way, so that
// a compute unit has a long one and a short one.
__device__ __forceinline__ int in_turn(const AttendPlan& pl, int turn_no) {
  return pl.turn > 0 && turn_no >= pl.turn ? pl.row_blocks - 1 - (turn_no - pl.turn) : turn_no;
}

// what a workgroup knows of its sequence
struct Sequence {
  int first, m, n, base;           // number of its first new token, new tokens, cached tokens, position of its first new token
};
__device__ __forceinline__ Sequence load_sequence(const Paged& P, int b, const int32_t* __restrict__ q_start, const int32_t* __restrict__ kv_len) {
  Sequence s;
  s.first = q_start[b];
  const int end = q_start[b + 1];
  int m = (end < P.tokens ? end : P.tokens) - s.first;         // rows that exist
  s.m = s.first < 0 || m < 0 ? 0 : m;
  const int n = kv_len[b];
  s.n = n < 0 ? 0 : n < P.max_len ? n : P.max_len;
  s.base = P.behind ? s.n : s.n - (end - s.first);
  return s;
}
// the first position that a query at position pos sees
__device__ __forceinline__ int first_seen(const Paged& P, int pos) {
  const int64_t low = (int64_t)pos - P.window + 1;
  return P.window > 0 && low > 0 ? (int)low : 0;
}
// the tokens begin .. end - 1 that some row of r0 .. r1 - 1 sees, and how they are cut
struct Stretch {
  int begin, end, parts, chunk;
};
__device__ __forceinline__ Stretch cut_rows(const Paged& P, const Sequence& s, int r0, int r1, int parts, int chunk) {
  Stretch c;
  const int64_t last = (int64_t)s.base + (r1 - 1) / P.G;
  const int first = first_seen(P, s.base + r0 / P.G);
  c.end = last + 1 < s.n ? (int)(last + 1) : s.n;
  if (c.end < 0) c.end = 0;
  c.begin = first < c.end ? first : c.end;
  const int len = c.end - c.begin;
  c.parts = (len + chunk - 1) / chunk;
  if (c.parts > parts) c.parts = parts;
  if (c.parts < 1) c.parts = 1;
  // (alike, but for whole tiles of the kernels)
  c.chunk = ((len + c.parts - 1) / c.parts + 63) / 64 * 64;
  if (c.chunk > 0) c.parts = (len + c.chunk - 1) / c.chunk;
  return c;
}

// A row of zeros: where rows that are not there are read (weights of 0 do not make good what a NaN beside them does to a product)
constexpr int kZeroBytes = 512;
static __device__ const uint4 g_zero_row[kZeroBytes / 16] = {};

// Sums of stretches in the workspace, scaled to their own references.  Entries: on a grid [parts][tokens * Hq]; of the even cut
// [workgroups][2][rows], the second for a unit that begins in the workgroup, the first for one that began before.
struct Partials {
  float* o;                        // [entries][d]
  float2* ml;                      // [entries]: reference, sum of weights
  int2* meta;                      // even cut, per unit: the first workgroup that has some of it, how many have
};

__device__ __forceinline__ float to_natural_lse(float m, float l) {
  return l > 0.f ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : l == l ? -INFINITY : l;
}
// 1 / sum of weights; a row that sees nothing has 0, one that sees a NaN keeps it
__device__ __forceinline__ float inverse_sum(float l) { return l > 0.f ? 1.f / l : l == l ? 0.f : l; }

struct AttendArgs {
  const void *Q, *K, *V;
  const int32_t *table, *q_start, *kv_len;
  void* out;
  float* lse;
  Partials part;
  // caches of codes
  Codes codes;
  const float *K_scales, *V_scales;
};

// Block k of the call's blocks of rows, counted from the last sequence's last: where the sequences' new tokens differ, a grid for the most of any
// would be workgroups without rows for the largest part.  By a wave: 64 sequences at a time.
__device__ __forceinline__ bool find_block(const Paged& P, const AttendPlan& pl, const AttendArgs& A, int k, int& b, int& r0) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < P.B; b0 += 64) {
    const int mine = P.B - 1 - (b0 + lane), rows = mine >= 0 ? load_sequence(P, mine, A.q_start, A.kv_len).m * P.G : 0;
    const int n = rows > pl.few ? (rows + pl.rows - 1) / pl.rows : 0;
    int to = n;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int y = __shfl_up(to, s);
      if (lane >= s) to += y;
    }
    const uint64_t past = __ballot(to > k);
    if (past != 0) {
      const int at = __builtin_ctzll(past);
      b = P.B - 1 - (b0 + at);
      r0 = (__builtin_amdgcn_readlane(to, at) - 1 - k) * pl.rows;
      return true;
    }
    k -= __builtin_amdgcn_readlane(to, 63);
  }
  return false;
}

// A weight of 0 takes a token out of a product only if its value is a number.  Where some rows see a token and others do not, and its value is infinite
// or NaN, the products carry NaN into rows that do not see it.  A row is therefore taken once more, over those tokens alone that it sees, if its sums come out
// as NaN and that can be why: its sum of weights is a number (weights of unseen tokens are 0 before they are summed up: where it is none, the row
// sees a key, or has a query, that is none), and an unseen value that went into the products is none.  Both are looked at because rows that see a NaN
// stay NaN, and a row by itself is slow, 5 ms over 32768 tokens of a bf16 cache: 2048 new tokens over 32768, with a NaN that all of them see,
// 1150 ms if every row is taken again, 1.1 so; 158 where the NaN is in the last token's value, for the rows of its block (a wave has 32 of them) before it.

// Of the tokens t_first .. t_end - 1: is a value that some of the rows r0 .. r1 - 1 do not see (nobody those before t_begin) infinite or NaN?  By the wave.
template <class T, int D>
__device__ __forceinline__ bool bad_unseen_rows(const Paged& P, const AttendArgs& A, const Sequence& sq, int b, int hkv, int r0, int r1, int t_first, int t_begin, int t_end) {
  const int low = first_seen(P, sq.base + (r1 - 1) / P.G), next = sq.base + r0 / P.G + 1, all_from = low > t_begin ? low : t_begin;
  const int32_t* pages = A.table + (int64_t)b * P.table_width;
  const T* V = static_cast<const T*>(A.V) + hkv * P.head_stride + (threadIdx.x & 63);
  bool bad = false;
  for (int t = t_first; t < t_end; ++t) {
    if (t >= all_from && t < next) t = next;                    // (all rows see those)
    if (t >= t_end) break;
    const int c = page_of(P.div, t), id = pages[c];
    if (id < 0 || id >= P.n_pages) continue;
    const T* v = V + id * P.page_stride + (int64_t)(t - c * P.div.page) * P.row_stride;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) bad = bad || !(fabsf(load_elem(v + j * 64)) < INFINITY);
  }
  return __any(bad);
}

// Row r over the tokens of t_begin .. t_end - 1 that it sees, by a wave, 64 tokens at a time: a lane has the logit of one of them, and then d / 64 elements of the sums.
// That is the result (whole_row), or the stretch's `entry` of the workspace.
template <class T, int D>
__device__ __forceinline__ void redo_row_rows(const Paged& P, const AttendArgs& A, const Sequence& sq, int b, int hkv, int r, int t_begin, int t_end,
                                         bool whole_row, int64_t entry) {
  constexpr int kPer = D / 64, kEPL = 16 / sizeof(T), kSide = 8;
  const int lane = threadIdx.x & 63;
  const int32_t* pages = A.table + (int64_t)b * P.table_width;
  const T* K = static_cast<const T*>(A.K) + hkv * P.head_stride;
  const T* V = static_cast<const T*>(A.V) + hkv * P.head_stride;
  const T* zero = reinterpret_cast<const T*>(g_zero_row);
  const int i = r / P.G, head = hkv * P.G + r - i * P.G, pos = sq.base + i, low = first_seen(P, pos);
  const int64_t row = sq.first + i;
  const T* from = static_cast<const T*>(A.Q) + b * P.q_b + row * P.q_t + head * P.q_h;
  const int begin = low > t_begin ? low : t_begin, end = pos + 1 < t_end ? pos + 1 : t_end;
  auto of_lane = [](float x, int u) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), u)); };
  float q[kPer], m = -INFINITY, l = 0.f, o[kPer] = {};
#pragma unroll
  for (int j = 0; j < kPer; ++j) q[j] = load_elem(from + j * 64 + lane);
  for (int t0 = begin; t0 < end; t0 += 64) {
    int64_t off = -1;                                           // of token t0 + lane
    if (t0 + lane < end) {
      const int t = t0 + lane, c = page_of(P.div, t), id = pages[c];
      if (id >= 0 && id < P.n_pages) off = id * P.page_stride + (int64_t)(t - c * P.div.page) * P.row_stride;
    }
    const T* k = off >= 0 ? K + off : zero;
    float x = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
#pragma unroll 2
      for (int p = 0; p < 64; p += kEPL) {
        float y[kEPL];
        load_f32(*reinterpret_cast<const v4u*>(k + j * 64 + p), y, static_cast<const T*>(nullptr));
#pragma unroll
        for (int e = 0; e < kEPL; ++e) x = fmaf(of_lane(q[j], p + e), y[e], x);
      }
    x = off >= 0 ? x * P.scale_log2 : -INFINITY;
    float next = fmaxf(m, x);
#pragma unroll
    for (int s = 32; s; s >>= 1) next = fmaxf(next, __shfl_xor(next, s));
    const float keep = next == -INFINITY ? 1.f : fast_exp2(m - next), w = fast_exp2(x - (next == -INFINITY ? 0.f : next));
    m = next;
    l = l * keep + w;
#pragma unroll
    for (int j = 0; j < kPer; ++j) o[j] *= keep;
    for (int u0 = 0; u0 < 64 && t0 + u0 < end; u0 += kSide) {
      float v[kSide][kPer];
#pragma unroll
      for (int u = 0; u < kSide; ++u) {
        const int64_t at = (int64_t)__builtin_amdgcn_readlane((int)(off >> 32), u0 + u) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)off, u0 + u);
        const T* from_v = at >= 0 ? V + at : zero;
#pragma unroll
        for (int j = 0; j < kPer; ++j) v[u][j] = load_elem(from_v + j * 64 + lane);
      }
#pragma unroll
      for (int u = 0; u < kSide; ++u)
#pragma unroll
        for (int j = 0; j < kPer; ++j) o[j] = fmaf(of_lane(w, u0 + u), v[u][j], o[j]);
    }
  }
#pragma unroll
  for (int s = 32; s; s >>= 1) l += __shfl_xor(l, s);
  if (whole_row) {
    const float inv = inverse_sum(l);
#pragma unroll
    for (int j = 0; j < kPer; ++j) store_elem(static_cast<T*>(A.out) + b * P.o_b + row * P.o_t + head * P.o_h + j * 64 + lane, o[j] * inv);
    if (A.lse != nullptr && lane == 0) A.lse[b * P.l_b + row * P.l_t + head * P.l_h] = to_natural_lse(m, l);
  } else {
#pragma unroll
    for (int j = 0; j < kPer; ++j) A.part.o[entry * D + j * 64 + lane] = o[j];
    if (lane == 0) A.part.ml[entry] = make_float2(m, l);
  }
}

// The same over a cache of codes.  int8: a code is a number, and a scale may be none; e4m3 has a code for what is none.
template <class T, int D>
__device__ __forceinline__ bool bad_unseen_codes(const Paged& P, const AttendArgs& A, const Sequence& sq, int b, int hkv, int r0, int r1, int t_first, int t_begin, int t_end) {
  const int low = first_seen(P, sq.base + (r1 - 1) / P.G), next = sq.base + r0 / P.G + 1, all_from = low > t_begin ? low : t_begin;
  const int32_t* pages = A.table + (int64_t)b * P.table_width;
  const uint8_t* V = static_cast<const uint8_t*>(A.V) + hkv * P.head_stride + (threadIdx.x & 63);
  bool bad = false;
  for (int t = t_first; t < t_end; ++t) {
    if (t >= all_from && t < next) t = next;                    // (all rows see those)
    if (t >= t_end) break;
    const int c = page_of(P.div, t), id = pages[c];
    if (id < 0 || id >= P.n_pages) continue;
    const int at = t - c * P.div.page;
    bad = bad || !(fabsf(A.V_scales[id * A.codes.page + hkv * A.codes.head + (at >> A.codes.shift)]) < INFINITY);
    const uint8_t* v = V + id * P.page_stride + at * P.row_stride;
#pragma unroll
    for (int j = 0; j < D / 64 && CacheOf<T>::kCode == kE4m3; ++j) bad = bad || (v[j * 64] & 0x7F) == 0x7F;
  }
  return __any(bad);
}

template <class T, int D>
__device__ __forceinline__ void redo_row_codes(const Paged& P, const AttendArgs& A, const Sequence& sq, int b, int hkv, int r, int t_begin, int t_end,
                                               bool whole_row, int64_t entry) {
  using Q = OutOf<T>;
  constexpr int kPer = D / 64, kCode = CacheOf<T>::kCode;
  const int lane = threadIdx.x & 63;
  const int32_t* pages = A.table + (int64_t)b * P.table_width;
  const uint8_t* K = static_cast<const uint8_t*>(A.K) + hkv * P.head_stride;
  const uint8_t* V = static_cast<const uint8_t*>(A.V) + hkv * P.head_stride;
  const uint8_t* zero = reinterpret_cast<const uint8_t*>(g_zero_row);
  const int i = r / P.G, head = hkv * P.G + r - i * P.G, pos = sq.base + i, low = first_seen(P, pos);
  const int64_t row = sq.first + i;
  const Q* from = static_cast<const Q*>(A.Q) + b * P.q_b + row * P.q_t + head * P.q_h;
  const int begin = low > t_begin ? low : t_begin, end = pos + 1 < t_end ? pos + 1 : t_end;
  auto of_lane = [](float x, int u) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), u)); };
  float q[kPer], m = -INFINITY, l = 0.f, o[kPer] = {};
#pragma unroll
  for (int j = 0; j < kPer; ++j) q[j] = load_elem(from + j * 64 + lane);
  for (int t0 = begin; t0 < end; t0 += 64) {
    int64_t off = -1;                                           // of token t0 + lane
    float ks = 0.f, vs = 0.f, x = 0.f;
    if (t0 + lane < end) {
      const int t = t0 + lane, c = page_of(P.div, t), id = pages[c], at = t - c * P.div.page;
      if (id >= 0 && id < P.n_pages) {
        off = id * P.page_stride + at * P.row_stride;
        const int64_t s = id * A.codes.page + hkv * A.codes.head + (at >> A.codes.shift);
        ks = A.K_scales[s];
        vs = A.V_scales[s];
      }
    }
    const uint8_t* k = off >= 0 ? K + off : zero;
#pragma unroll
    for (int j = 0; j < kPer; ++j)
#pragma unroll 2
      for (int p = 0; p < 64; p += 4) {
        float y[4];
        numbers<kCode>(*reinterpret_cast<const uint32_t*>(k + j * 64 + p), y);
#pragma unroll
        for (int e = 0; e < 4; ++e) x = fmaf(of_lane(q[j], p + e), y[e], x);
      }
    x = off >= 0 ? x * ks * P.scale_log2 : -INFINITY;
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
      const uint8_t* v = at >= 0 ? V + at : zero;
#pragma unroll
      for (int j = 0; j < kPer; ++j) o[j] = fmaf(of_lane(weight, u), number<kCode>(v[j * 64 + lane]), o[j]);
    }
  }
#pragma unroll
  for (int s = 32; s; s >>= 1) l += __shfl_xor(l, s);
  if (whole_row) {
    const float inv = inverse_sum(l);
#pragma unroll
    for (int j = 0; j < kPer; ++j) store_elem(static_cast<Q*>(A.out) + b * P.o_b + row * P.o_t + head * P.o_h + j * 64 + lane, o[j] * inv);
    if (A.lse != nullptr && lane == 0) A.lse[b * P.l_b + row * P.l_t + head * P.l_h] = to_natural_lse(m, l);
  } else {
#pragma unroll
    for (int j = 0; j < kPer; ++j) A.part.o[entry * D + j * 64 + lane] = o[j];
    if (lane == 0) A.part.ml[entry] = make_float2(m, l);
  }
}

template <class T, int D>
__device__ __forceinline__ bool bad_unseen(const Paged& P, const AttendArgs& A, const Sequence& sq, int b, int hkv, int r0, int r1, int t_first, int t_begin, int t_end) {
  if constexpr (CacheOf<T>::kCoded) return bad_unseen_codes<T, D>(P, A, sq, b, hkv, r0, r1, t_first, t_begin, t_end);
  else                              return bad_unseen_rows<T, D>(P, A, sq, b, hkv, r0, r1, t_first, t_begin, t_end);
}
template <class T, int D>
__device__ __forceinline__ void redo_row(const Paged& P, const AttendArgs& A, const Sequence& sq, int b, int hkv, int r, int t_begin, int t_end, bool whole_row,
                                         int64_t entry) {
  if constexpr (CacheOf<T>::kCoded) redo_row_codes<T, D>(P, A, sq, b, hkv, r, t_begin, t_end, whole_row, entry);
  else                              redo_row_rows<T, D>(P, A, sq, b, hkv, r, t_begin, t_end, whole_row, entry);
}
// the same for a grid's stretch part_no
template <class T, int D>
__device__ __forceinline__ void redo_row_of(const Paged& P, const AttendArgs& A, const Sequence& sq, int b, int hkv, int r, int t_begin, int t_end, bool whole_row, int part_no) {
  redo_row<T, D>(P, A, sq, b, hkv, r, t_begin, t_end, whole_row, ((int64_t)part_no * P.tokens + sq.first + r / P.G) * P.Hq + hkv * P.G + r % P.G);
}

inline unsigned grid_size(const Paged& P, const AttendPlan& pl) {
  return (unsigned)((int64_t)P.Hkv * pl.parts * (pl.blocks > 0 ? pl.blocks : (int64_t)P.B * pl.row_blocks));
}

// rows kernel (bf16 queries): a workgroup per (unit, block of 128 rows, stretch), its waves share the tiles; with it the even cut, if there is one
template <class T>
void launch_attend_rows(const Paged& P, const AttendPlan& pl, const AttendArgs& A, const AttendPlan& even, const Partials& even_part, hipStream_t s);
template <>
void launch_attend_rows<uint16_t>(const Paged& P, const AttendPlan& pl, const AttendArgs& A, const AttendPlan& even, const Partials& even_part, hipStream_t s);
template <>
void launch_attend_rows<Coded<uint16_t, kInt8>>(const Paged& P, const AttendPlan& pl, const AttendArgs& A, const AttendPlan& even, const Partials& even_part, hipStream_t s);
template <>
void launch_attend_rows<Coded<uint16_t, kE4m3>>(const Paged& P, const AttendPlan& pl, const AttendArgs& A, const AttendPlan& even, const Partials& even_part, hipStream_t s);

}  // namespace ccd
