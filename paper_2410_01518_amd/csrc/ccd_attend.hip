// ccd_paged_attend: the kernels of few rows per unit and of fp32 caches (ccd_attend_few.h), the joining of stretches, and how a call is cut.
#include "ccd_attend_few.h"
#include "ccd_attend_grid.h"

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
    for (int j = 0; j < kPer; ++j) store_elem(static_cast<T*>(A.out) + b * P.o_b + row * P.o_t + head * P.o_h + j * 64 + lane, acc[j] * inv);
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

template <class T, int D>
static int even_waves(int rows) { return rows == 16 ? split_waves<T, D, 1>() : split_waves<T, D, 2>(); }

int attend_compute_units();

// About the time (ns) of a grid that cuts `units` blocks of rows and heads into `parts` stretches each.  A workgroup takes `token` ns a token where it has a
// compute unit alone, and 250 tokens' time for itself; two that share one take `shared` times that (in between, while some have one alone:
// the rows kernel is bound by power).  Sums of stretches are written and read again by one more kernel.  The 250 tokens, the factors of a shared compute unit and of a
// round that is not full are fitted to what was measured, in us:
//   rows kernel, d 128, 32 heads of 8 groups, 8192 tokens, for 1, 2, 3, 4 stretches:  512 new tokens 160, 102, 101, 91;  1024: 162, 160, 168, 167;
//   1536: 213, 235, 250, 237;  64 new tokens, for 4, 8, 16, 32: 52, 35, 29, 33
//   fp32, 16 heads of 4 groups, 4096 tokens, for 1, 2, 3, 4, 6, 8:  d 64, 256 new tokens 111, 64, 71, 58, 77, 64;  d 128, 300: 167, 174, 128, 139, 140, 133
static double grid_time(const Paged& P, int by_rows, int64_t units, int64_t len, int64_t parts, int64_t cus) {
  const double token = by_rows ? (P.d == 64 ? 12 : 20) : (P.d == 64 ? 26 : 40), shared = by_rows || P.d == 64 ? 1.6 : 2.0;
  const int64_t wgs = units * parts, rounds = wgs / (2 * cus), rest = wgs % (2 * cus);
  const double last = rest == 0 ? 0 : rest <= cus ? 1 : by_rows && 2 * rest <= 3 * cus ? (1 + 3 * shared) / 4 : shared;
  const double sums = parts == 1 ? 0 : 8000 + (double)wgs * (by_rows ? 128 : 32) * P.d * 8 / 4000;
  return (rounds * shared + last) * ((double)len / parts + 250) * token + sums;
}

static AttendCuts plan_attend(const Paged& P, int dtype, int max_new, int max_len) {
  AttendCuts c{};
  const int64_t rows = (int64_t)max_new * P.G, cus = attend_compute_units();
  const bool many = rows > 32;
  int64_t len = max_len;
  if (P.window > 0 && len > (int64_t)P.window + max_new) len = (int64_t)P.window + max_new;
  if (!many || (P.B > 1 && P.G <= 32)) {
    AttendPlan& e = c.even;
    const int64_t most = many ? P.G : rows;
    e.rows = most <= 16 ? 16 : 32;
    e.only_few = many;
    e.few = e.rows;
    e.join = (int)(most < e.rows ? most : e.rows);
    const int waves = dtype == 0 ? (P.d == 64 ? even_waves<float, 64>(e.rows) : even_waves<float, 128>(e.rows))
                                 : (P.d == 64 ? even_waves<uint16_t, 64>(e.rows) : even_waves<uint16_t, 128>(e.rows));
    const int64_t units = (int64_t)P.B * P.Hkv;
    int64_t wgs = (units * len + kEvenLeast - 1) / kEvenLeast;
    if (wgs > cus * waves) wgs = cus * waves;
    e.parts = (int)(wgs < 1 ? 1 : wgs);
    // Short caches: workgroups that stay with one unit.  Not cut at all, which saves the second kernel, where one workgroup reads its unit in the time that
    // the second kernel costs and half of all units take at 5100 bytes/ns (half: lengths differ, and the host knows the longest alone).  A
    // workgroup reads 50 bytes/ns (d 64 32, fp32 35); of eight waves, where there is one per compute unit, 65 (60, 40).  Else cut as finely as there are
    // compute units to spare.  32 query heads of 8 groups, d 128, us uncut / uncut by eight waves / by 128 / by 256 / evenly: one sequence of 400 tokens
    // 10.4 / 9.7 / 12.0 / 12.3 / 17.9, of 1000 15.4 / 13.0 / 12.5 / 12.4 / 14.6, of 4000 29.7 / 24.3 / 13.7 / 13.3 / 18.3; 16 of 1000 17.3 /
    // 16.3 / 20.1 / 20.2 / 25.6; 32 of 2000 51.4 / 51.1 / 63 / 63 / 62; 256 of 100 .. 512 60 / - / 107 / 81 / 80.  By 1024, or 2048, and evenly: 16 of
    // 500 .. 4096 36.8, 36.8, d 64 19.9, 23.8; 8 of 16384 101, 104; but 32 of 500 .. 4096, two stretches each, 62, 57; fp32, 8 of 2000 .. 8192 76, 66.
    // Many rounds of units are dealt out as they end: 512 of 500 .. 4096, us whole and evenly, 616, 644, of 1 .. 16384 712, 801; but 256 of 500 .. 8192
    // 520, 513, and fp32, 512 of 100 .. 4000, 479, 426.
    const bool wide = units <= cus && len > 256;
    const int64_t row = 2 * (int64_t)P.d * (dtype == 0 ? 4 : 2), rate = wide ? (dtype == 0 ? 40 : P.d == 64 ? 60 : 65) : (dtype == 0 ? 35 : P.d == 64 ? 32 : 50);
    const bool uncut = (len <= 2048 && len * row / rate <= 6000 + units * len * row / 10200) || (dtype != 0 && units >= 16 * cus);
    for (int chunk = uncut ? (int)len : 128; !many && (uncut || chunk <= 2048); chunk *= 2) {
      const int64_t chunks = (len + chunk - 1) / chunk;
      if (!uncut && (chunks > 64 || units * chunks > (chunk <= 256 ? cus : cus * waves) || (chunk > 512 && (dtype == 0 || chunks < 4)))) continue;
      c.grid = e;
      c.grid.few = 0;
      c.grid.row_blocks = (int)((rows + e.rows - 1) / e.rows);
      c.grid.chunk = chunk;
      c.grid.parts = (int)(chunks < 1 ? 1 : chunks);
      c.grid.wide = uncut && wide;
      c.even.rows = c.even.parts = 0;
      break;
    }
  }
  if (many) {
    AttendPlan& g = c.grid;
    g.by_rows = dtype != 0;
    g.rows = g.by_rows ? 128 : 32;
    g.few = c.even.few;
    g.row_blocks = (int)((rows + g.rows - 1) / g.rows);
    // (as many blocks as there can be, not the most of any sequence for all: 512 slots of which one has 64 new tokens over 8192 637 us with a block for every slot, 50 so)
    const int64_t filled = ((int64_t)P.tokens * P.G + g.rows - 1) / g.rows, of_all = (int64_t)P.B * g.row_blocks;
    const int64_t listed = most_blocks(P.B, P.tokens, P.G, g.rows, g.few);
    if (of_all > listed) g.blocks = (int)listed;
    const int64_t units = P.Hkv * (filled < 1 ? 1 : filled < of_all ? filled : of_all);
    if (P.window > 0 && len > (int64_t)P.window + g.rows / P.G + 1) len = (int64_t)P.window + g.rows / P.G + 1;      // of one block
    const int64_t held = most_parts((of_all < listed ? of_all : listed) * P.Hkv, c.even.parts);
    int64_t most = len < 256 * 64 ? (len + 255) / 256 : 64;
    if (most > held) most = held;
    int64_t parts = 1;
    double least = 0;
    for (int64_t p = 1; p <= most; ++p) {
      const double t = grid_time(P, g.by_rows, units, len, p, cus);
      if (p == 1 || t < least) { least = t; parts = p; }
    }
    // Whether the products are put right by the sums of the weights as rounded (add_rounded).  That takes some of the error off at any length, and costs more the longer
    // the call: error in the norm against 64 bits (the output's own rounding 1.65e-3) and us, without and with, 32 heads on 8 of 128: 512 new tokens
    // over 512 1.78e-3, 1.76e-3 and 20.0, 20.7; over 1024 2.12e-3, 1.99e-3 and 30.2, 31.4; over 2048 1.75e-3, 1.70e-3 and 49.8, 51.2; over 4096 1.87e-3, 1.73e-3 and
    // 69, 72; 2048 over 4096 1.97e-3, 1.76e-3 and 118, 130; over 32768 2.08e-3, 1.86e-3 and 973, 1023.  So it is a matter of time: up to 1024 tokens it
    // is one microsecond, and there rows see the fewest tokens (one that a single token rules is off by all of that token's rounding).
    g.sums = g.by_rows && len <= 1024;
    g.chunk = (int)(((len + parts - 1) / parts + 127) / 128 * 128);
    g.parts = (int)((len + g.chunk - 1) / g.chunk);
    if (g.parts < 1) g.parts = 1;
    if (g.blocks == 0 && units * g.parts <= 2 * cus) g.turn = (g.row_blocks + 1) / 2;
  }
  return c;
}

// (the answer of the first device serves all: one GPU model per node)
int attend_compute_units() {
  static const int cus = [] {
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) == hipSuccess && hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && n > 0) return n;
    (void)hipGetLastError();                                 // none: sizes may be asked for where there is no device
    return 256;
  }();
  return cus;
}

// the workspace: entries of the even cut and of the grid, (o, m, l) each, and the even cut's units
struct AttendSpace {
  size_t even_o, even_ml, meta, grid_o, grid_ml, total;
};
static AttendSpace lay_out(const Paged& P, const AttendCuts& c) {
  AttendSpace w{};
  auto take = [&](size_t bytes) { const size_t at = w.total; w.total += (bytes + 255) / 256 * 256; return at; };
  if (c.even.rows > 0) {
    const size_t entries = (size_t)c.even.parts * 2 * c.even.rows;
    w.even_o = take(entries * P.d * sizeof(float));
    w.even_ml = take(entries * sizeof(float2));
    w.meta = take((size_t)P.B * P.Hkv * sizeof(int2));
  }
  if (c.grid.rows > 0 && c.grid.parts > 1) {
    const size_t entries = (size_t)P.tokens * P.Hq * c.grid.parts;
    w.grid_o = take(entries * P.d * sizeof(float));
    w.grid_ml = take(entries * sizeof(float2));
  }
  if (w.total == 0) w.total = 256;
  return w;
}

size_t attend_workspace_bytes(const Paged& P, int dtype, int max_new, int max_len) {
  return lay_out(P, plan_attend(P, dtype, max_new, max_len)).total;
}

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
    launch_attend_rows(P, c.grid, grid, c.even, even.part, s);
  } else if (c.grid.rows > 0 && (c.grid.blocks > 0 || c.even.rows > 0)) {
    if constexpr (sizeof(T) == 4) {
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

void launch_attend(const Paged& P, int dtype, int max_new, int max_len, const void* Q, const void* K, const void* V, const int32_t* table,
                   const int32_t* q_start, const int32_t* kv_len, void* out, float* lse, void* workspace, hipStream_t s) {
  const AttendCuts c = plan_attend(P, dtype, max_new, max_len);
  const AttendSpace w = lay_out(P, c);
  char* ws = static_cast<char*>(workspace);
  AttendArgs even{Q, K, V, table, q_start, kv_len, out, lse,
                  {reinterpret_cast<float*>(ws + w.even_o), reinterpret_cast<float2*>(ws + w.even_ml), reinterpret_cast<int2*>(ws + w.meta)}};
  AttendArgs grid = even;
  grid.part = {reinterpret_cast<float*>(ws + w.grid_o), reinterpret_cast<float2*>(ws + w.grid_ml), nullptr};
  if (dtype == 0 && P.d == 64) attend_launch<float, 64>(P, c, even, grid, s);
  else if (dtype == 0)         attend_launch<float, 128>(P, c, even, grid, s);
  else if (P.d == 64)          attend_launch<uint16_t, 64>(P, c, even, grid, s);
  else                         attend_launch<uint16_t, 128>(P, c, even, grid, s);
}

}  // namespace ccd
