// How a call of ccd_paged_attend or ccd_paged_attend_codes is cut; ccd_paged_attend's kernels (ccd_attend_launch.h).
#include "ccd_attend_grid.h"
#include "ccd_attend_launch.h"

namespace ccd {

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
//   rows kernel over codes (int8; two workgroups on a compute unit stand in each other's way less), d 128, 8192 tokens, for 1, 2, 3, 4 stretches:  512 new tokens 226, 140, 126, 107;
//   1024: 230, 188, 200, 195;  four of 128 over 4096: 124, 88, 84, 75;  64 new tokens, for 4, 8, 16, 32: 72, 46, 36, 42;  d 64, 512: 167, 104, 94, 77
static double grid_time(const Paged& P, int by_rows, bool codes, int64_t units, int64_t len, int64_t parts, int64_t cus) {
  codes = codes && by_rows;
  const double token = codes ? (P.d == 64 ? 20 : 26.5) : by_rows ? (P.d == 64 ? 12 : 20) : (P.d == 64 ? 26 : 40), shared = codes ? 1.4 : by_rows || P.d == 64 ? 1.6 : 2.0;
  const int64_t wgs = units * parts, rounds = wgs / (2 * cus), rest = wgs % (2 * cus);
  const double last = rest == 0 ? 0 : rest <= cus ? 1 : by_rows && 2 * rest <= 3 * cus ? (1 + 3 * shared) / 4 : shared;
  const double sums = parts == 1 ? 0 : 8000 + (codes ? (double)P.tokens * P.Hq * parts : (double)wgs * (by_rows ? 128 : 32)) * P.d * 8 / 4000;
  return (rounds * shared + last) * ((double)len / parts + 250) * token + sums;
}

AttendCuts plan_attend(const Paged& P, int dtype, bool codes, int max_new, int max_len) {
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
    const int waves = codes ? (!many && e.rows == 16 && (P.d == 64 || dtype != 0) ? 3 : 2) : dtype == 0 ? (P.d == 64 ? even_waves<float, 64>(e.rows) : even_waves<float, 128>(e.rows))
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
    // Codes have half the bytes, and are read at half the rate by a workgroup alone: its tiles take as long.  One sequence of 1000 and of 1500, 32 query heads, d 128: whole 13.6,
    // 17.3, cut 11.3, 11.4; 16 of 1000 14.8, 32 of 2000 27.6, 256 of 100 .. 512 40 (whole).
    const bool wide = units <= cus && len > 256;
    const int64_t row = 2 * (int64_t)P.d * (codes ? 1 : dtype == 0 ? 4 : 2), rate = codes ? (wide ? 33 : 25) : wide ? (dtype == 0 ? 40 : P.d == 64 ? 60 : 65) : (dtype == 0 ? 35 : P.d == 64 ? 32 : 50);
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
    // (over codes: as many tokens for every pot, as those of the catalyst prompt, are so many blocks, filled or not.  16 tokens over 32 pots, a block of 64 rows each, 119 us; 127 when taken for
    // half as many.  Lengths of sequences with several pages differ, and the longest decides: there more, shorter stretches are the safer choice, 17 of 519 .. 8192 201, 243 so)
    const bool alike = codes && g.by_rows && P.table_width == 1 && P.tokens == (int64_t)P.B * max_new;
    const int64_t units = P.Hkv * (alike ? of_all : filled < 1 ? 1 : filled < of_all ? filled : of_all);
    if (P.window > 0 && len > (int64_t)P.window + g.rows / P.G + 1) len = (int64_t)P.window + g.rows / P.G + 1;      // of one block
    const int64_t held = most_parts((of_all < listed ? of_all : listed) * P.Hkv, c.even.parts);
    int64_t most = len < 256 * 64 ? (len + 255) / 256 : 64;
    if (most > held) most = held;
    int64_t parts = 1;
    double least = 0;
    for (int64_t p = 1; p <= most; ++p) {
      const double t = grid_time(P, g.by_rows, codes, units, len, p, cus);
      if (p == 1 || t < least) { least = t; parts = p; }
    }
    // Whether the products are put right by the sums of the weights as rounded (add_rounded).  That takes some of the error off at any length, and costs more the longer
    // the call: error in the norm against 64 bits (the output's own rounding 1.65e-3) and us, without and with, 32 heads on 8 of 128: 512 new tokens
    // over 512 1.78e-3, 1.76e-3 and 20.0, 20.7; over 1024 2.12e-3, 1.99e-3 and 30.2, 31.4; over 2048 1.75e-3, 1.70e-3 and 49.8, 51.2; over 4096 1.87e-3, 1.73e-3 and
    // 69, 72; 2048 over 4096 1.97e-3, 1.76e-3 and 118, 130; over 32768 2.08e-3, 1.86e-3 and 973, 1023.  So it is a matter of time: up to 1024 tokens it
    // is one microsecond, and there rows see the fewest tokens (one that a single token rules is off by all of that token's rounding).  Over codes: 2048 new of 4096
    // tokens 2.3e-3 .. 2.6e-3 and 1.9e-3, 135 and 146 us; of 34816 1240 and 1350 us.
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

AttendSpace lay_out(const Paged& P, const AttendCuts& c) {
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
  return lay_out(P, plan_attend(P, dtype, false, max_new, max_len)).total;
}

void launch_attend(const Paged& P, int dtype, int max_new, int max_len, const void* Q, const void* K, const void* V, const int32_t* table,
                   const int32_t* q_start, const int32_t* kv_len, void* out, float* lse, void* workspace, hipStream_t s) {
  const AttendCuts c = plan_attend(P, dtype, false, max_new, max_len);
  const AttendSpace w = lay_out(P, c);
  char* ws = static_cast<char*>(workspace);
  AttendArgs even{Q, K, V, table, q_start, kv_len, out, lse,
                  {reinterpret_cast<float*>(ws + w.even_o), reinterpret_cast<float2*>(ws + w.even_ml), reinterpret_cast<int2*>(ws + w.meta)}, {}, nullptr, nullptr};
  AttendArgs grid = even;
  grid.part = {reinterpret_cast<float*>(ws + w.grid_o), reinterpret_cast<float2*>(ws + w.grid_ml), nullptr};
  if (dtype == 0 && P.d == 64) attend_launch<float, 64>(P, c, even, grid, s);
  else if (dtype == 0)         attend_launch<float, 128>(P, c, even, grid, s);
  else if (P.d == 64)          attend_launch<uint16_t, 64>(P, c, even, grid, s);
  else                         attend_launch<uint16_t, 128>(P, c, even, grid, s);
}

}  // namespace ccd
