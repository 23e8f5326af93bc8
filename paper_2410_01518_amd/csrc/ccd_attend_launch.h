// Kernels and launches of ccd_paged_attend and ccd_paged_attend_codes, by type of cache: those of few rows per unit and of fp32 caches (ccd_attend_few.h), and the joining of
// stretches.  How a call is cut is worked out in ccd_attend.hip.
#pragma once
#include "ccd_attend_few.h"

#include <type_traits>

namespace ccd {

template <class T, int D, int NQ, int WAVES>
__global__ __launch_bounds__(64 * WAVES, (WAVES == 8 ? 2 : split_waves<T, D, NQ>())) void attend_split_kernel(Paged P, AttendPlan pl, AttendArgs A) {
  __shared__ SplitLds<T, D, NQ, WAVES> L;
  attend_on_grid<T, D, NQ, WAVES, false>(P, pl, A, L, blockIdx.x);
}

template <class T, int D, int NQ>
__global__ __launch_bounds__(64 * kWaves, (split_waves<T, D, NQ>())) void attend_even_kernel(Paged P, AttendPlan pl, AttendArgs A) {
  __shared__ EvenLds<T, D, NQ> E;
  attend_evenly<T, D, NQ>(P, pl, A, E, blockIdx.x, gridDim.x);
}

// Chunks, and the sequences of few rows among them: their workgroups come last and fill what the others leave idle.  (Ragged chunks and single tokens
// in fp32, 869 rows of 12 heads with a window of 1024: 43.7 us, 58.0 one after the other.)
template <class T, int D, int NQ, bool LISTED>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_mixed_kernel(Paged P, AttendPlan grid, AttendPlan even, AttendArgs A, Partials even_part, int grid_wgs) {
  __shared__ __align__(16) char lds[sizeof(SplitLds<T, D, 2>) > sizeof(EvenLds<T, D, NQ>) ? sizeof(SplitLds<T, D, 2>) : sizeof(EvenLds<T, D, NQ>)];
  if ((int)blockIdx.x < grid_wgs) {
    attend_on_grid<T, D, 2, kWaves, LISTED>(P, grid, A, reinterpret_cast<SplitLds<T, D, 2>&>(lds), blockIdx.x);
  } else {
    A.part = even_part;
    attend_evenly<T, D, NQ>(P, even, A, reinterpret_cast<EvenLds<T, D, NQ>&>(lds), blockIdx.x - grid_wgs, even.parts);
  }
}

// Joins the stretches of a row: WAVES waves per (new token, query head).  A lane has the reference and the sum of one stretch, so 64 of them are
// there at once and their largest costs no chain of loads; the waves then take the stretches' sums in turn.  EVEN: the stretches of
// attend_even_kernel, `join` rows of every unit side by side; else those of a grid, rows counted through the call.
template <class T, int D, int WAVES, bool EVEN>
__global__ __launch_bounds__(256) void attend_join_kernel(Paged P, AttendPlan pl, AttendArgs A) {
  constexpr int kPer = D / 64;
  __shared__ float sums[WAVES > 1 ? WAVES : 1][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // row r of a unit of the even cut, whose products took in what the unit sees (those of a block of more rows than expected, less)
  auto again = [&](const Sequence& sq, int b, int hkv, int r) __attribute__((always_inline)) {
    const Span sp = span_of(P, pl, sq);
    const bool bad = bad_unseen<T, D>(P, A, sq, b, hkv, r, r + 1, sp.begin, sp.begin, sp.end);
    if (bad) redo_row<T, D>(P, A, sq, b, hkv, r, 0, sq.n, true, 0);
    return bad;
  };
  // entry of the first stretch, of the second less a step, distance of the others
  auto join = [&](const Sequence& sq, int b, int hkv, int r, int parts, int64_t part_first, int64_t part_0, int64_t part_step) __attribute__((always_inline)) {
    auto entry = [&](int p) { return p == 0 ? part_first : part_0 + p * part_step; };
    float top = -INFINITY, sum = 0.f, acc[kPer] = {};
    for (int p0 = 0; p0 < parts; p0 += 64) {
      const int here = parts - p0 < 64 ? parts - p0 : 64;
      const float2 ml = lane < here ? A.part.ml[entry(p0 + lane)] : make_float2(-INFINITY, 0.f);
      float next = fmaxf(top, ml.x);
#pragma unroll
      for (int s = 32; s; s >>= 1) next = fmaxf(next, __shfl_xor(next, s));
      const float keep = ml.x == -INFINITY ? (ml.y == ml.y ? 0.f : ml.y) : fast_exp2(ml.x - next);
      float more = ml.x == -INFINITY ? keep : ml.y * keep;
#pragma unroll
      for (int s = 32; s; s >>= 1) more += __shfl_xor(more, s);
      const float old = next == -INFINITY ? 1.f : fast_exp2(top - next);
      top = next;
      sum = sum * old + more;
#pragma unroll
      for (int j = 0; j < kPer; ++j) acc[j] *= old;
      for (int p = WAVES > 1 ? wave : 0; p < here; p += 8 * WAVES) {
        float v[8][kPer];
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
          for (int j = 0; j < kPer; ++j) v[u][j] = p + u * WAVES < here ? A.part.o[entry(p0 + p + u * WAVES) * D + j * 64 + lane] : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float k = __shfl(keep, (p + u * WAVES) & 63);
#pragma unroll
          for (int j = 0; j < kPer; ++j) acc[j] = p + u * WAVES < here ? fmaf(v[u][j], k, acc[j]) : acc[j];
        }
      }
    }
    if (WAVES > 1) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kPer; ++j) sums[wave][j * 64 + lane] = acc[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        acc[j] = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) acc[j] += sums[w][j * 64 + lane];
      }
      if (wave != 0) return;
    }
    bool none = false;
#pragma unroll
    for (int j = 0; j < kPer; ++j) none = none || (acc[j] != acc[j] && sum == sum);
    if (EVEN && sq.m > 1 && __builtin_expect(__any(none), 0) && again(sq, b, hkv, r)) return;
    const int row = sq.first + r / P.G, head = hkv * P.G + r % P.G;
    const float inv = inverse_sum(sum);
#pragma unroll
    for (int j = 0; j < kPer; ++j) store_elem(static_cast<OutOf<T>*>(A.out) + b * P.o_b + row * P.o_t + head * P.o_h + j * 64 + lane, acc[j] * inv);
    if (A.lse != nullptr && lane == 0) A.lse[b * P.l_b + row * P.l_t + head * P.l_h] = to_natural_lse(top, sum);
  };

  auto one = [&](int64_t at0) __attribute__((always_inline)) {
    if constexpr (EVEN) {
      const int unit = (int)(at0 / pl.join), hkv = unit % P.Hkv, b = unit / P.Hkv;
      if (b >= P.B) return;
      const Sequence sq = load_sequence(P, b, A.q_start, A.kv_len);
      const int rows_all = sq.m * P.G;
      if (rows_all < 1 || (pl.only_few && rows_all > pl.few)) return;
      const int2 cut = A.part.meta[unit];
      if (cut.y == 1 || (cut.y == kAgain && WAVES > 1 && wave != 0)) return;
      for (int r = (int)(at0 % pl.join); r < rows_all; r += pl.join) {
        if (cut.y == kAgain) { again(sq, b, hkv, r); continue; }
        join(sq, b, hkv, r, cut.y, (int64_t)(2 * cut.x + 1) * pl.rows + r, (int64_t)(2 * cut.x) * pl.rows + r, 2 * pl.rows);
      }
    } else {
      const int row = (int)(at0 / P.Hq), head = (int)(at0 % P.Hq);
      if (row >= P.tokens) return;
      int b = 0;                                                          // sequences that end at or before the row: counted, no chain of loads
      for (int b0 = 1; b0 <= P.B; b0 += 64) b += __popcll(__ballot(b0 + lane <= P.B && A.q_start[b0 + lane <= P.B ? b0 + lane : P.B] <= row));
      if (b >= P.B || row < A.q_start[0]) return;
      const Sequence sq = load_sequence(P, b, A.q_start, A.kv_len);
      const int r = (row - sq.first) * P.G + head % P.G, rows_all = sq.m * P.G;
      if (r < 0 || r >= rows_all || rows_all <= pl.few) return;
      const int r0 = r / pl.rows * pl.rows;
      const int parts = cut_rows(P, sq, r0, r0 + pl.rows < rows_all ? r0 + pl.rows : rows_all, pl.parts, pl.chunk).parts;
      if (parts > 1) join(sq, b, head / P.G, r, parts, at0, at0, (int64_t)P.tokens * P.Hq);
    }
  };
  if constexpr (WAVES > 1) {
    one(blockIdx.x);
  } else {
    const int64_t all = EVEN ? (int64_t)P.B * P.Hkv * pl.join : (int64_t)P.tokens * P.Hq;
    for (int64_t at0 = (int64_t)blockIdx.x * 4 + wave; at0 < all; at0 += (int64_t)gridDim.x * 4) one(at0);
  }
}

// ---- host side

// How a call is cut.  Few rows in every sequence (decoding, at most 32 rows per unit): evenly.  More: on a grid, with the sequences of
// few rows among them (a batch of chunks and single tokens) evenly by kernels of their own, as a block of 128 rows would walk their long
// caches alone.
struct AttendCuts {
  AttendPlan even, grid;           // rows == 0: not used
};

// dtype: that of Q and out
AttendCuts plan_attend(const Paged& P, int dtype, bool codes, int max_new, int max_len);

// the workspace: entries of the even cut and of the grid, (o, m, l) each, and the even cut's units
struct AttendSpace {
  size_t even_o, even_ml, meta, grid_o, grid_ml, total;
};
AttendSpace lay_out(const Paged& P, const AttendCuts& c);

constexpr int64_t kJoinMost = 1 << 22;      // workgroups

template <class T, int D, bool EVEN>
static void join_launch(const Paged& P, const AttendPlan& pl, const AttendArgs& A, hipStream_t s) {
  const int64_t rows = EVEN ? (int64_t)P.B * P.Hkv * pl.join : (int64_t)P.tokens * P.Hq;
  // (few rows, or many stretches: four waves each)
  if (rows <= 1024) launch(attend_join_kernel<T, D, 4, EVEN>, dim3((unsigned)rows), dim3(256), s, P, pl, A);
  else              launch(attend_join_kernel<T, D, 1, EVEN>, dim3((unsigned)(rows < kJoinMost * 4 ? (rows + 3) / 4 : kJoinMost)), dim3(256), s, P, pl, A);
}

template <class T, int D, int NQ>
static void mixed_launch(const Paged& P, const AttendCuts& c, const AttendArgs& grid, const Partials& even, hipStream_t s) {
  const int wgs = (int)grid_size(P, c.grid);
  const dim3 all((unsigned)(wgs + c.even.parts)), block(64 * kWaves);
  if (c.grid.blocks > 0) launch(attend_mixed_kernel<T, D, NQ, true>, all, block, s, P, c.grid, c.even, grid, even, wgs);
  else                   launch(attend_mixed_kernel<T, D, NQ, false>, all, block, s, P, c.grid, c.even, grid, even, wgs);
}

template <class T, int D>
static void attend_launch(const Paged& P, const AttendCuts& c, const AttendArgs& even, const AttendArgs& grid, hipStream_t s) {
  const dim3 block(64 * kWaves);
  if (c.grid.rows > 0 && c.grid.by_rows) {
    if constexpr (sizeof(OutOf<T>) == 2) launch_attend_rows<T>(P, c.grid, grid, c.even, even.part, s);
  } else if (c.grid.rows > 0 && (c.grid.blocks > 0 || c.even.rows > 0)) {
    if constexpr (sizeof(OutOf<T>) == 4) {
      if (c.even.rows == 32) mixed_launch<T, D, 2>(P, c, grid, even.part, s);
      else                   mixed_launch<T, D, 1>(P, c, grid, even.part, s);
    }
  } else if (c.grid.rows > 0) {
    const dim3 wgs(grid_size(P, c.grid));
    if (c.grid.wide && c.grid.rows == 16) launch(attend_split_kernel<T, D, 1, 8>, wgs, dim3(512), s, P, c.grid, grid);
    else if (c.grid.wide)                 launch(attend_split_kernel<T, D, 2, 8>, wgs, dim3(512), s, P, c.grid, grid);
    else if (c.grid.rows == 16)           launch(attend_split_kernel<T, D, 1, kWaves>, wgs, block, s, P, c.grid, grid);
    else                                  launch(attend_split_kernel<T, D, 2, kWaves>, wgs, block, s, P, c.grid, grid);
  } else if (c.even.rows == 16) {
    launch(attend_even_kernel<T, D, 1>, dim3((unsigned)c.even.parts), block, s, P, c.even, even);
  } else {
    launch(attend_even_kernel<T, D, 2>, dim3((unsigned)c.even.parts), block, s, P, c.even, even);
  }
  if (c.grid.rows > 0 && c.grid.parts > 1) join_launch<T, D, false>(P, c.grid, grid, s);
  if (c.even.rows > 0) join_launch<T, D, true>(P, c.even, even, s);
}

}  // namespace ccd
