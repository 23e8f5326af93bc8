// ccd_paged_attend, bf16 caches and many rows per unit (chunks of a prompt): a workgroup per (unit, block of 128 rows, stretch of tokens).
//
// Here the matrix cores are the bound, and next to them the vector ALUs: a logit costs 4 d flops but also an fma, an exp2, an addition and half a
// conversion.  Four waves have 32 rows each and walk the same tokens; tiles of 64 keys and values come from memory straight into LDS
// (global_load_lds, no registers), two deep, one barrier per tile.  Two workgroups share a compute unit.  Logits are computed as
// D[token][row] = K Q^T (v_mfma_f32_32x32x16_bf16): a lane has 16 of 32 tokens of one row, so a row's sum stays within a lane and its neighbour 32
// lanes on, and the weights are already the operand of D[d][row] = V^T W^T if that product counts its tokens in the same order; values
// are transposed by the LDS read (ds_read_b64_tr_b16).
//
// Measured, a chunk of 2048 tokens over 32768 cached ones, 32 query heads on 8 KV heads of 128 elements: 966 - 1049 us by the machine, 1.02 - 1.10 PFLOP/s,
// where a product of 8192^3 reaches 1.2 - 1.3.  The matrix cores are busy 52 % of the cycles and the clock is at 1.9 - 2.0 GHz: what is left is bound by power
// (removing all bank conflicts and a tenth of the instructions took 20 % of the cycles and 4 % of the time).  Waves of 64 rows, one per SIMD,
// read LDS half as often and keep 2.4 GHz, but a wave alone cannot cover its own waits: 1010 - 1040 us, and coarser blocks for short calls.
#include "ccd_attend_few.h"

#include <type_traits>

namespace ccd {

constexpr int kRowWaves = 4, kTile = 64;
constexpr float kFar = 256.f;            // sum of a lane's 16 weights above which the reference is raised
enum { kKeys = 1, kValues = 2 };

// 64 lanes x 16 bytes from memory into LDS, at lds_addr + 16 * lane
__device__ __forceinline__ void load_to_lds(uint32_t lds_addr, const void* p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_addr), "v"(p) : "memory");
}
// N such, to lds_addr + 1024 k + 16 * lane.  An instruction's own offset counts for both addresses: offset[k] is meant with it taken off, and what
// would then be negative is in the base (run_offset).
template <int N>
__device__ __forceinline__ void load_run_to_lds(uint32_t lds_addr, const uint32_t (&offset)[N], const void* base) {
  if constexpr (N == 4)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:0x400\n\t"
                 "global_load_lds_dwordx4 %3, %5 offset:0x800\n\tglobal_load_lds_dwordx4 %4, %5 offset:0xC00"
                 ::"s"(lds_addr), "v"(offset[0]), "v"(offset[1]), "v"(offset[2]), "v"(offset[3]), "s"(base) : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:0x400"
                 ::"s"(lds_addr), "v"(offset[0]), "v"(offset[1]), "s"(base) : "memory");
}
constexpr int kRunBack = 4096;
__device__ __forceinline__ uint32_t run_offset(int64_t bytes, int k) { return (uint32_t)(bytes + kRunBack - 1024 * k); }

__device__ __forceinline__ float largest(const v16f& x) {
  float top = x[0];
#pragma unroll
  for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
  return top;
}

// BANDED: pages of whole runs of 16 rows, so that a wave's 16 rows of a tile lie in one page, which is looked up 64 tiles ahead.  Else every row's page is looked
// up in its tile, and waited for: 2048 new tokens over 4096 in pages of 37 or 100 take 264 to 270 us where pages of 64 take 118, over 32768 2160 and 1045.
// SUMS: those of the rounded weights, too (add_rounded): calls over few tokens, where that costs little
template <int D>
struct RowsLds {
  __align__(1024) char tile[2][2][kTile * D * 2];                                  // [tile][keys, values]
  uint32_t here[2][kRowWaves];                                                     // [tile]: which of 16 tokens have a page
};
template <int D, bool BANDED, bool SUMS>
__device__ __forceinline__ void attend_rows(const Paged& P, const AttendPlan& pl, const AttendArgs& A, RowsLds<D>& L, int idx) {
  constexpr int kRows = 32 * kRowWaves, kRowB = D * 2, kPieces = D / 8;            // 16-byte pieces of a row
  constexpr int kPerLoad = 64 / kPieces, kLoads = 16 / kPerLoad;                   // rows per load instruction, loads of a wave's 16 rows
  constexpr int kTileB = kTile * kRowB, kSteps = D / 16, kBlocks = D / 32;
  auto& lds = L.tile;
  auto& here = L.here;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  const int hkv = idx % P.Hkv;
  idx /= P.Hkv;
  int b = idx % P.B;
  if (pl.blocks == 0) idx /= P.B;
  const int part_no = idx % pl.parts;
  int turn_no = in_turn(pl, idx / pl.parts);
  const uint16_t* Kh = static_cast<const uint16_t*>(A.K) + hkv * P.head_stride;
  const uint16_t* Vh = static_cast<const uint16_t*>(A.V) + hkv * P.head_stride;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)&lds[0][0][0];

  // Pieces change places by the row's number, so that what a read takes together lies in all banks: 16 lanes of a 16-byte read (16 rows of keys, one piece),
  // 32 lanes of a transposing one (four rows of values, two pairs of pieces).
  auto key_swap = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
  auto value_swap = [](int row) { return D == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2; };
  // what the lane loads of the wave's 16 rows: row kPerLoad * k + load_row, the piece that belongs at its place
  const int load_row = lane / kPieces, place = lane % kPieces;
  // what the lane reads: keys, row (lane & 31), piece 2 s + half; values, 4 tokens at 4 half + .., 16 elements at 16 ((lane >> 4) & 1)
  const int key_at = (lane & 31) * kRowB + ((half ^ key_swap(lane & 31)) << 4);
  const int value_row = 4 * half + ((lane & 15) >> 2);
  const int value_at = value_row * kRowB + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ value_swap(value_row)) << 4) + (lane & 1) * 8;
  // the lane's offsets in a run of 16 rows of one page
  uint32_t key_run[kLoads], value_run[kLoads];
#pragma unroll
  for (int k = 0; k < kLoads; ++k) {
    const int row = kPerLoad * k + load_row;
    key_run[k] = run_offset((int64_t)row * P.row_stride * 2 + ((place ^ key_swap(row)) << 4), k);
    value_run[k] = run_offset((int64_t)row * P.row_stride * 2 + ((place ^ value_swap(row)) << 4), k);
  }

  // (beyond row_blocks, or blocks: more rows than the host expected)
  for (int r0 = (pl.row_blocks - 1 - turn_no) * kRows;; r0 += pl.row_blocks * kRows, turn_no += pl.blocks) {
    if (pl.blocks > 0 && !find_block(P, pl, A, turn_no, b, r0)) break;
    const Sequence sq = load_sequence(P, b, A.q_start, A.kv_len);
    const int rows_all = sq.m * P.G;
    if (rows_all <= pl.few || r0 >= rows_all) break;
    const int32_t* pages = A.table + (int64_t)b * P.table_width;
    const int r1 = r0 + kRows < rows_all ? r0 + kRows : rows_all;
    const Stretch st = cut_rows(P, sq, r0, r1, pl.parts, pl.chunk);
    if (part_no >= st.parts) continue;
    const int t_begin = st.begin + part_no * st.chunk, t_end = t_begin + st.chunk < st.end ? t_begin + st.chunk : st.end;
    const int tile0 = t_begin & ~15, tiles = (t_end - tile0 + kTile - 1) / kTile;              // (tokens before t_begin are masked)
    // the lane's row, and the wave's rows (none if w0 >= r1)
    const int r = r0 + 32 * wave + (lane & 31), i_row = r / P.G, head = hkv * P.G + r - i_row * P.G;
    const int w0 = r0 + 32 * wave, w1 = w0 + 32 < r1 ? w0 + 32 : r1;
    const int pos = r < r1 ? sq.base + i_row : -1, low_row = first_seen(P, pos), low = low_row > t_begin ? low_row : t_begin;
    const int pos_min = sq.base + w0 / P.G, low_max = w0 < r1 ? first_seen(P, sq.base + (w1 - 1) / P.G) : 0, low_all = low_max > t_begin ? low_max : t_begin;
    v8bf q[kSteps];
    {
      const uint16_t* row = static_cast<const uint16_t*>(A.Q) + b * P.q_b + (int64_t)(sq.first + i_row) * P.q_t + (int64_t)head * P.q_h;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        v4u w = {0, 0, 0, 0};
        if (r < r1) w = *reinterpret_cast<const v4u*>(row + 16 * s + 8 * half);
        q[s] = __builtin_bit_cast(v8bf, w);
      }
    }
    float m = 0.f, l = 0.f, lr = 0.f;                          // reference (0 until the row has one), sums of weights (add_rounded)
    bool seen = r >= r1;                                       // has the row a reference?
    v16f o[kBlocks];
#pragma unroll
    for (int c = 0; c < kBlocks; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[c][e] = 0.f;

    // Pages of the wave's 16 rows, 64 tiles at once, a lane each: a scalar load per tile would be waited for with the first reads from LDS (they share a counter).
    int ids = -1;
    auto look_up = [&](int tile) __attribute__((always_inline)) {
      if (!BANDED) return -1;
      if ((tile & 63) == 0) {
        const int64_t tw = (int64_t)tile0 + (int64_t)(tile + lane) * kTile + 16 * wave;
        ids = tw + 16 <= t_end ? pages[page_of(P.div, (int)tw)] : -1;
      }
      return __builtin_amdgcn_readlane(ids, tile & 63);
    };
    // where the wave's 16 rows of a tile begin, if they are all there and in one page (else -1)
    auto run_of = [&](int tile) __attribute__((always_inline)) -> int64_t {
      const int page_id = look_up(tile), tw = tile0 + tile * kTile + 16 * wave;
      if (!BANDED || page_id < 0 || page_id >= P.n_pages) return -1;
      return page_id * P.page_stride + (int64_t)(tw - page_of(P.div, tw) * P.div.page) * P.row_stride;
    };
    // asks for the wave's 16 rows of a tile
    auto ask = [&](int tile, int slot, int what, int64_t run) __attribute__((always_inline)) {
      if (tile >= tiles) return;
      const int tw = tile0 + tile * kTile + 16 * wave;
      const uint32_t kd = lds0 + (slot * 2) * kTileB + 16 * wave * kRowB, vd = kd + kTileB;
      if (BANDED && run >= 0) {
        if (what & kKeys) load_run_to_lds<kLoads>(kd, key_run, reinterpret_cast<const char*>(Kh + run) - kRunBack);
        if (what & kValues) load_run_to_lds<kLoads>(vd, value_run, reinterpret_cast<const char*>(Vh + run) - kRunBack);
        if ((what & kKeys) && lane == 0) here[slot][wave] = 0xFFFFu;
        return;
      }
      auto row_at = [&](int t) __attribute__((always_inline)) -> int64_t {
        if (t >= t_end) return -1;
        const int c = page_of(P.div, t), id = pages[c];
        return id >= 0 && id < P.n_pages ? id * P.page_stride + (int64_t)(t - c * P.div.page) * P.row_stride : -1;
      };
      const uint16_t* zero = reinterpret_cast<const uint16_t*>(g_zero_row);
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        const int row = kPerLoad * k + load_row;
        const int64_t at = row_at(tw + row);
        if (what & kKeys) load_to_lds(kd + k * 1024, (at >= 0 ? Kh + at : zero) + ((place ^ key_swap(row)) << 3));
        if (what & kValues) load_to_lds(vd + k * 1024, (at >= 0 ? Vh + at : zero) + ((place ^ value_swap(row)) << 3));
      }
      if (what & kKeys) {
        const uint32_t mine = (uint32_t)__ballot(row_at(tw + (lane & 15)) >= 0) & 0xFFFFu;
        if (lane == 0) here[slot][wave] = mine;
      }
    };

    // The wave's pipeline, a step per 32 tokens (two steps a tile): while the weights of block j are worked out (vector ALUs), the matrix cores compute the
    // logits of block j + 1 and add the values of block j - 1; the three do not depend on each other.  Keys run a block ahead and values a block behind, so
    // tile t's second step needs the keys of tile t + 1 and the values of tile t, and one barrier a tile, before that step, is enough:
    // behind it the keys of tile t and the values of tile t - 1 are done with, and their places take those of t + 2 and t + 1.
    // Logits of block j and j + 1, weights of block j - 1 and j are two sets that change places with every step.
    v16f x0, x1;
    v8bf wa[2], wb[2];
    // masks block `at` (its first token; there: which of its tokens have a page) where not all of it is seen
    auto mask = [&](v16f& x, int at, uint32_t there) __attribute__((always_inline)) {
      if (__builtin_expect(there != ~0u || at + 31 > pos_min || at < low_all, 0)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int off = 8 * (e >> 2) + 4 * half + (e & 3), t = at + off;
          if (!((there >> off) & 1u) || t > pos || t < low) x[e] = -INFINITY;
        }
      }
    };
    auto weigh = [&](const v16f& x, v8bf (&w)[2]) __attribute__((always_inline)) {
      float sum = 0.f;
      v4u now[2];
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        const float e0 = fast_exp2(fmaf(x[2 * p], P.scale_log2, -m)), e1 = fast_exp2(fmaf(x[2 * p + 1], P.scale_log2, -m));
        now[p / 4][p % 4] = pack_bf16(e0, e1);
        sum += e0 + e1;
      }
      w[0] = __builtin_bit_cast(v8bf, now[0]);
      w[1] = __builtin_bit_cast(v8bf, now[1]);
      return sum;
    };
    // A block's largest logit is not looked for: all weights are positive, so as long as their sum is small no logit lies far above the reference.  Where
    // it is not (or is no number, or there is no reference yet) the reference is raised and the weights are worked out again.
    auto settle = [&](const v16f& x, v8bf (&w)[2], float& sum) __attribute__((always_inline)) {
      if (__builtin_expect(__any(!(sum <= kFar) || !seen), 0)) {
        const float top = largest(x) * P.scale_log2, next = fmaxf(top, __shfl_xor(top, 32));
        // a row without a reference takes the first finite one; until then it has no weights
        const float to = seen ? fmaxf(m, next) : next;
        if (to != -INFINITY) {
          const float keep = seen ? fast_exp2(m - to) : 0.f;
          l *= keep;
          if (SUMS) lr *= keep;
#pragma unroll
          for (int c = 0; c < kBlocks; ++c) o[c] *= keep;
          m = to;
          seen = true;
        }
        sum = weigh(x, w);
      }
      l += sum;
    };
    auto key_of = [&](const char* kt, int sub, int s) __attribute__((always_inline)) {
      return __builtin_bit_cast(v8bf, *reinterpret_cast<const v4u*>(kt + ((key_at ^ (s << 5)) + sub * 32 * kRowB)));
    };
    auto value_of = [&](const char* vt, int sub, int s, int c) __attribute__((always_inline)) {
      v4s t[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
        t[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(vt + ((value_at ^ (c << 6)) + (32 * sub + 16 * s + 8 * u) * kRowB)));
      return __builtin_bit_cast(v8bf, __builtin_shufflevector(t[0], t[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // the first blocks and the last ones, which have no neighbours: the step's parts by themselves
    auto logits = [&](v16f& x, const char* kt, int sub) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_of(kt, sub, s), q[s], x, 0, 0, 0);
    };
    auto weights = [&](const v16f& x, v8bf (&w)[2]) __attribute__((always_inline)) {
      float sum = weigh(x, w);
      settle(x, w, sum);
    };
    auto add_values = [&](const v8bf (&w)[2], const char* vt, int sub) __attribute__((always_inline)) {
#pragma unroll
      for (int p = 0; SUMS && p < 8; ++p) lr = add_rounded(w[p / 4], p % 4, lr);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value_of(vt, sub, s, c), w[s], o[c], 0, 0, 0);
    };
    // One step: weights `now` of block j (logits x), logits y of block j + 1 (keys kt, half sub; its first token next_at), values of block j - 1 (weights w, values
    // vt).  Left to itself the compiler puts the three one after the other and waits for every read from LDS where it is used.  So the order is laid down:
    // reads run kAhead products ahead, and behind every product stands its share of the vector work, which the products cover (a product takes the
    // matrix core 32 clocks and the issue port 4).  chained: the step's last reads are the first operands of the next, keys kt, half 1.
    constexpr int kProducts = kSteps + 2 * kBlocks, kAhead = 3;
    static_assert(kProducts % (kAhead + 1) == 0, "a step begins where the one before left the ring of operands");
    v8bf f[kAhead + 1];
    auto step = [&](const v16f& x, const v8bf (&w)[2], v16f& y, v8bf (&now)[2], const char* kt, const char* vt, int sub, int next_at, uint32_t next_there,
                    bool chained) __attribute__((always_inline)) {
      float sum = 0.f, v[2];
      v4u packed[2];
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = 0.f;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kProducts; ++i) {
        const int ahead = i + kAhead;
        if (ahead < kSteps) f[ahead % (kAhead + 1)] = key_of(kt, sub, ahead);
        else if (ahead < kProducts) f[ahead % (kAhead + 1)] = value_of(vt, sub, (ahead - kSteps) / kBlocks, (ahead - kSteps) % kBlocks);
        else if (chained) f[ahead % (kAhead + 1)] = key_of(kt, 1, ahead - kProducts);
        const v8bf a = f[i % (kAhead + 1)];
        if (i < kSteps) y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[i], y, 0, 0, 0);
        else o[(i - kSteps) % kBlocks] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, w[(i - kSteps) / kBlocks], o[(i - kSteps) % kBlocks], 0, 0, 0);
        // the product's share of block j - 1's weights, and of block j's 16 logits (as in weigh)
#pragma unroll
        for (int p = i * 8 / kProducts; SUMS && p < (i + 1) * 8 / kProducts; ++p) {
          lr = add_rounded(w[p / 4], p % 4, lr);
          asm volatile("" ::"v"(lr));
        }
#pragma unroll
        for (int e = i * 16 / kProducts; e < (i + 1) * 16 / kProducts; ++e) {
          v[e & 1] = fast_exp2(fmaf(x[e], P.scale_log2, -m));
          asm volatile("" ::"v"(v[e & 1]));
          if (e & 1) {
            const uint32_t two = pack_bf16(v[0], v[1]);
            sum += v[0] + v[1];
            asm volatile("" ::"v"(two), "v"(sum));
            packed[e / 8][e / 2 % 4] = two;
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      now[0] = __builtin_bit_cast(v8bf, packed[0]);
      now[1] = __builtin_bit_cast(v8bf, packed[1]);
      settle(x, now, sum);
      mask(y, next_at, next_there);
    };

    if (tiles > 0) {
      // (which tokens are there: one word per run of 16, read with the tile's keys)
      auto there_of = [&](int slot, int sub) __attribute__((always_inline)) { return here[slot][2 * sub] | here[slot][2 * sub + 1] << 16; };
      auto uniform = [](uint32_t u) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readfirstlane(u); };
      // loads into LDS are waited for all together: they do not arrive in the order they were asked for
      auto arrived = [&]() __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
      };
      ask(0, 0, kKeys | kValues, run_of(0));
      int64_t run1 = run_of(1);                                                // of the next tile: its keys are asked for, its values will be
      arrived();
      ask(1, 1, kKeys, run1);
      logits(x0, lds[0][0], 0);
      mask(x0, tile0, uniform(there_of(0, 0)));
      weights(x0, wa);
      logits(x0, lds[0][0], 1);
      mask(x0, tile0 + 32, uniform(there_of(0, 1)));
      auto turn = [&](auto even, int t) __attribute__((always_inline)) {
        constexpr int slot = decltype(even)::value ? 0 : 1, next = slot ^ 1;   // (places that the compiler knows: addresses without arithmetic)
        const int at = tile0 + (t + 1) * kTile;
        arrived();
        // (the first operands are on their way while the next tiles are asked for)
#pragma unroll
        for (int i = 0; i < kAhead; ++i) f[i] = key_of(lds[next][0], 0, i);
        const uint32_t here0 = there_of(next, 0), here1 = there_of(next, 1);
        __builtin_amdgcn_sched_barrier(0);
        const int64_t run2 = run_of(t + 2);
        ask(t + 1, next, kValues, run1);
        ask(t + 2, slot, kKeys, run2);
        run1 = run2;
        const uint32_t there0 = uniform(here0), there1 = uniform(here1);
        step(x0, wa, x1, wb, lds[next][0], lds[slot][1], 0, at, there0, true);
        // (its first operands: read at the end of the step before)
        step(x1, wb, x0, wa, lds[next][0], lds[slot][1], 1, at + 32, there1, false);
      };
      for (int t = 0; t + 1 < tiles; t += 2) {
        turn(std::true_type{}, t);
        if (t + 2 < tiles) turn(std::false_type{}, t + 1);
      }
      const char* vt = lds[(tiles - 1) & 1][1];
      arrived();
      add_values(wa, vt, 0);
      weights(x0, wb);
      add_values(wb, vt, 1);
    }

    l += __shfl_xor(l, 32);
    const float whole = SUMS ? unrounded(l, lr + __shfl_xor(lr, 32)) : 1.f;
    bool none = false;
#pragma unroll
    for (int c = 0; c < kBlocks; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) none = none || o[c][e] != o[c][e];
    none = none && l == l && r < r1;
    uint32_t again = 0;                                                        // the wave's rows that are taken once more (the tiles begin before the stretch)
    if (__builtin_expect(__any(none), 0) && bad_unseen<uint16_t, D>(P, A, sq, b, hkv, w0, w1, tile0, t_begin, t_end)) {
      const uint64_t lanes = __ballot(none);
      again = (uint32_t)lanes | (uint32_t)(lanes >> 32);
    }
    if (r < r1 && !((again >> (lane & 31)) & 1u)) {
      const int64_t row = sq.first + i_row;
      if (st.parts == 1) {
        const float inv = inverse_sum(l) * whole;
        uint16_t* to = static_cast<uint16_t*>(A.out) + b * P.o_b + row * P.o_t + (int64_t)head * P.o_h + 4 * half;
#pragma unroll
        for (int c = 0; c < kBlocks; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<uint2*>(to + 32 * c + 8 * e) = make_uint2(pack_bf16(o[c][4 * e] * inv, o[c][4 * e + 1] * inv),
                                                                         pack_bf16(o[c][4 * e + 2] * inv, o[c][4 * e + 3] * inv));
        if (A.lse != nullptr && half == 0) A.lse[b * P.l_b + row * P.l_t + head * P.l_h] = to_natural_lse(m, l);
      } else {
        const int64_t at = ((int64_t)part_no * P.tokens + row) * P.Hq + head;
        float* to = A.part.o + at * D + 4 * half;
#pragma unroll
        for (int c = 0; c < kBlocks; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<float4*>(to + 32 * c + 8 * e) = make_float4(o[c][4 * e] * whole, o[c][4 * e + 1] * whole, o[c][4 * e + 2] * whole, o[c][4 * e + 3] * whole);
        if (half == 0) A.part.ml[at] = make_float2(seen ? m : -INFINITY, l);
      }
    }
    for (; again != 0; again &= again - 1) redo_row_of<uint16_t, D>(P, A, sq, b, hkv, w0 + __builtin_ctz(again), t_begin, t_end, st.parts == 1, part_no);
    __syncthreads();
  }
}

template <int D, bool BANDED, bool SUMS>
__global__ __launch_bounds__(64 * kRowWaves, 2) void attend_rows_kernel(Paged P, AttendPlan pl, AttendArgs A) {
  __shared__ RowsLds<D> L;
  attend_rows<D, BANDED, SUMS>(P, pl, A, L, blockIdx.x);
}

// Chunks, and the sequences of few rows among them: their workgroups come last and fill what the others leave idle.  (17 sequences of 1 to 969 new tokens over
// 519 to 8192, 32 heads of 8 groups: 238 us, 266 one after the other.)
template <int D, bool BANDED, bool SUMS, int NQ>
__global__ __launch_bounds__(64 * kRowWaves, 2) void attend_rows_mixed_kernel(Paged P, AttendPlan grid, AttendPlan even, AttendArgs A, Partials even_part, int grid_wgs) {
  using Few = EvenLds<uint16_t, D, NQ>;
  __shared__ __align__(1024) char lds[sizeof(RowsLds<D>) > sizeof(Few) ? sizeof(RowsLds<D>) : sizeof(Few)];
  if ((int)blockIdx.x < grid_wgs) {
    attend_rows<D, BANDED, SUMS>(P, grid, A, reinterpret_cast<RowsLds<D>&>(lds), blockIdx.x);
  } else {
    A.part = even_part;
    attend_evenly<uint16_t, D, NQ>(P, even, A, reinterpret_cast<Few&>(lds), blockIdx.x - grid_wgs, even.parts);
  }
}

template <int D, bool BANDED, bool SUMS>
static void rows_launch(const Paged& P, const AttendPlan& pl, const AttendArgs& A, const AttendPlan& even, const Partials& even_part, hipStream_t s) {
  static_assert(kRowWaves == kWaves);
  const int wgs = (int)grid_size(P, pl);
  const dim3 all((unsigned)(wgs + even.parts)), block(64 * kRowWaves);
  if (even.rows == 0)       launch(attend_rows_kernel<D, BANDED, SUMS>, all, block, s, P, pl, A);
  else if (even.rows == 16) launch(attend_rows_mixed_kernel<D, BANDED, SUMS, 1>, all, block, s, P, pl, even, A, even_part, wgs);
  else                      launch(attend_rows_mixed_kernel<D, BANDED, SUMS, 2>, all, block, s, P, pl, even, A, even_part, wgs);
}
template <int D, bool BANDED>
static void rows_launch_of(const Paged& P, const AttendPlan& pl, const AttendArgs& A, const AttendPlan& even, const Partials& even_part, hipStream_t s) {
  if (pl.sums) rows_launch<D, BANDED, true>(P, pl, A, even, even_part, s);
  else         rows_launch<D, BANDED, false>(P, pl, A, even, even_part, s);
}

void launch_attend_rows(const Paged& P, const AttendPlan& pl, const AttendArgs& A, const AttendPlan& even, const Partials& even_part, hipStream_t s) {
  // (a lane's offset within the 16 rows of a run is 32 bits)
  const bool banded = P.div.page % 16 == 0 && P.row_stride * 2 * 16 < (int64_t)1 << 31;
  if (P.d == 64) banded ? rows_launch_of<64, true>(P, pl, A, even, even_part, s) : rows_launch_of<64, false>(P, pl, A, even, even_part, s);
  else           banded ? rows_launch_of<128, true>(P, pl, A, even, even_part, s) : rows_launch_of<128, false>(P, pl, A, even, even_part, s);
}

}  // namespace ccd
