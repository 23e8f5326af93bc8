// ccd_paged_attend, bf16 caches and many rows per unit (chunks of a prompt): a workgroup per (unit, block of 128 rows, stretch of tokens).
//
// Here the matrix cores are the bound, and next to them the vector ALUs: a logit costs 4 d flops but also an fma, an exp2, an addition and half a
// conversion.  Four waves have 32 rows each and walk the same tokens; tiles of 64 keys and values come from memory straight into LDS
// (global_load_lds, no registers), two buffers deep, one barrier per tile.  Two workgroups share a compute unit, so that one's softmax runs
// beside the other's products.  Logits are computed as D[token][row] = K Q^T (v_mfma_f32_32x32x16_bf16): a lane has 16 of 32 tokens of one row, so a row's
// largest logit and its sum stay within a lane and its neighbour 32 lanes on, and the weights are already the operand of D[d][row] = V^T W^T
// if that product counts its tokens in the same order; values are transposed by the LDS read (ds_read_b64_tr_b16).
#include "ccd_attend.h"
#include "ccd_rotary.h"

namespace ccd {

constexpr int kRowWaves = 4, kTile = 64;
enum { kKeys = 1, kValues = 2 };

// 64 lanes x 16 bytes from memory into LDS, at lds_addr + 16 * lane
__device__ __forceinline__ void load_to_lds(uint32_t lds_addr, const void* p) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_addr), "v"(p) : "memory");
}
__device__ __forceinline__ void load_to_lds(uint32_t lds_addr, uint32_t offset, const void* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_addr), "v"(offset), "s"(base) : "memory");
}

__device__ __forceinline__ float largest(const v16f& x) {
  float top = x[0];
#pragma unroll
  for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
  return top;
}

// BANDED: pages of whole runs of 16 rows, so that a wave's 16 rows of a tile lie in one page
template <int D, bool BANDED>
__global__ __launch_bounds__(64 * kRowWaves, 2) void attend_rows_kernel(Paged P, AttendPlan pl, const uint16_t* __restrict__ Q, const uint16_t* __restrict__ K,
                                                                       const uint16_t* __restrict__ V, const int32_t* __restrict__ table,
                                                                       const int32_t* __restrict__ q_start, const int32_t* __restrict__ kv_len,
                                                                       uint16_t* __restrict__ out, float* __restrict__ lse, Partials part) {
  constexpr int kRows = 32 * kRowWaves, kRowB = D * 2, kPieces = D / 8;            // 16-byte pieces of a row
  constexpr int kPerLoad = 64 / kPieces, kLoads = 16 / kPerLoad;                   // rows per load instruction, loads of a wave's 16 rows
  constexpr int kTileB = kTile * kRowB, kSteps = D / 16, kBlocks = D / 32;
  __shared__ __align__(1024) char lds[2][2][kTileB];                               // [buffer][keys, values]
  __shared__ uint32_t here[2][kRowWaves];                                          // [buffer]: which of 16 tokens have a page
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  const int units = P.B * P.Hkv;
  int idx = blockIdx.x;
  const int unit = idx % units;
  idx /= units;
  // The last rows see most and come first.  Where the call is one round of two workgroups per compute unit, its second half runs the other way, so that
  // a compute unit has a long one and a short one.
  int turn = idx / pl.parts;
  if (pl.turn > 0 && turn >= pl.turn) turn = pl.row_blocks - 1 - (turn - pl.turn);
  const int part_no = idx % pl.parts, block0 = pl.row_blocks - 1 - turn;
  const int b = unit / P.Hkv, hkv = unit % P.Hkv;
  const Sequence sq = load_sequence(P, b, q_start, kv_len);
  const int rows_all = sq.m * P.G;
  if (rows_all <= pl.few) return;
  const int32_t* pages = table + (int64_t)b * P.table_width;
  const uint16_t* Kh = K + hkv * P.head_stride;
  const uint16_t* Vh = V + hkv * P.head_stride;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)&lds[0][0][0];

  // Pieces change places by the row's number: keys so that the 8 or 16 rows of a 16-byte read lie in different banks, values so that the four rows
  // of a transposing read do.
  auto key_swap = [](int row) { return D == 128 ? row & 15 : (row >> 1) & 7; };
  auto value_swap = [](int row) { return D == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1; };
  // what the lane loads of the wave's 16 rows: row kPerLoad * k + load_row, the piece that belongs at its place
  const int load_row = lane / kPieces, place = lane % kPieces;
  // what the lane reads: keys, row (lane & 31), piece 2 s + half; values, 4 tokens at 4 half + .., 16 elements at 16 ((lane >> 4) & 1)
  const int key_at = (lane & 31) * kRowB + ((half ^ key_swap(lane & 31)) << 4);
  const int value_row = 4 * half + ((lane & 15) >> 2);
  const int value_at = value_row * kRowB + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ value_swap(value_row)) << 4) + (lane & 1) * 8;

  for (int r0 = block0 * kRows; r0 < rows_all; r0 += pl.row_blocks * kRows) {
    const int r1 = r0 + kRows < rows_all ? r0 + kRows : rows_all;
    const Stretch st = cut_rows(P, sq, r0, r1, pl.parts, pl.chunk);
    if (part_no >= st.parts) continue;
    const int t_begin = st.begin + part_no * st.chunk, t_end = t_begin + st.chunk < st.end ? t_begin + st.chunk : st.end;
    const int tile0 = t_begin & ~15;                                   // (tokens before t_begin are masked)
    // the lane's row
    const int r = r0 + 32 * wave + (lane & 31), i = r / P.G, head = hkv * P.G + r - i * P.G;
    const int pos = r < r1 ? sq.base + i : -1, low_row = first_seen(P, pos), low = low_row > t_begin ? low_row : t_begin;
    const int w0 = r0 + 32 * wave, w1 = w0 + 32 < r1 ? w0 + 32 : r1;   // the wave's rows (none if w0 >= r1)
    const int pos_min = sq.base + w0 / P.G, low_max = w0 < r1 ? first_seen(P, sq.base + (w1 - 1) / P.G) : 0, low_all = low_max > t_begin ? low_max : t_begin;
    v8bf q[kSteps];
    {
      const uint16_t* row = Q + b * P.q_b + (int64_t)(sq.first + i) * P.q_t + (int64_t)head * P.q_h;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        v4u w = {0, 0, 0, 0};
        if (r < r1) w = *reinterpret_cast<const v4u*>(row + 16 * s + 8 * half);
        q[s] = __builtin_bit_cast(v8bf, w);
      }
    }
    float m = -INFINITY, l = 0.f;
    v16f o[kBlocks];
#pragma unroll
    for (int c = 0; c < kBlocks; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[c][e] = 0.f;

    // the wave's 16 of the tile's 64 tokens; page_id: the page of the first of them, where it was looked up
    auto look_up = [&](int t0) {
      const int tw = t0 + 16 * wave;
      return BANDED && tw + 16 <= t_end ? pages[page_of(P.div, tw)] : -1;
    };
    auto request = [&](int t0, int buf, int what, int page_id) {
      const int tw = t0 + 16 * wave;
      const uint32_t kd = lds0 + (buf * 2) * kTileB + 16 * wave * kRowB, vd = kd + kTileB;
      if (BANDED && page_id >= 0 && page_id < P.n_pages) {
        const int64_t at = page_id * P.page_stride + (int64_t)(tw - page_of(P.div, tw) * P.div.page) * P.row_stride;
        const uint16_t *kb = Kh + at, *vb = Vh + at;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
          const int row = kPerLoad * k + load_row;
          if (what & kKeys) load_to_lds(kd + k * 1024, (uint32_t)(row * (int)P.row_stride + ((place ^ key_swap(row)) << 3)) * 2u, kb);
          if (what & kValues) load_to_lds(vd + k * 1024, (uint32_t)(row * (int)P.row_stride + ((place ^ value_swap(row)) << 3)) * 2u, vb);
        }
        if ((what & kKeys) && lane == 0) here[buf][wave] = 0xFFFFu;
        return;
      }
      auto row_at = [&](int t) -> int64_t {
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
        if (lane == 0) here[buf][wave] = mine;
      }
    };

    // The wave's pipeline, a step per 32 tokens (two steps a tile): while the weights of block j are worked out (vector ALUs), the matrix cores compute the
    // logits of block j + 1 and add the values of block j - 1; the three do not depend on each other.  Keys run a block ahead and values a block behind, so
    // tile t's second step needs the keys of tile t + 1 and the values of tile t, and one barrier a tile, before that step, is enough:
    // behind it the keys of tile t and the values of tile t - 1 are done with, and their buffers take those of t + 2 and t + 1.
    v16f x;                                                  // logits of block j, then of block j + 1
    v8bf w[2];                                               // weights of block j - 1, then of block j
    // masks block `at` (its first token) where not all of it is seen, and raises the reference where a logit calls for it
    auto settle = [&](int at, int buf, int sub, float top) {
      const uint32_t there = (uint32_t)__builtin_amdgcn_readfirstlane(here[buf][2 * sub] | here[buf][2 * sub + 1] << 16);
      const bool whole = there == ~0u && at + 31 <= pos_min && at >= low_all;
      if (!whole) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int off = 8 * (e >> 2) + 4 * half + (e & 3), t = at + off;
          if (!((there >> off) & 1u) || t > pos || t < low) x[e] = -INFINITY;
        }
        top = largest(x);
      }
      top *= P.scale_log2;
      if (__any(top > m + kRaise)) {
        // (a whole number: the weights in w, bf16 by now, are scaled without rounding)
        const float next = fmaxf(m, ceilf(fmaxf(top, __shfl_xor(top, 32))));
        const float keep = next == -INFINITY ? 1.f : fast_exp2(m - next);
        m = next;
        l *= keep;
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) o[c] *= keep;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int e = 0; e < 8; ++e) w[s][e] = (__bf16)((float)w[s][e] * keep);
      }
    };
    auto key_of = [&](const char* kt, int sub, int s) {
      return __builtin_bit_cast(v8bf, *reinterpret_cast<const v4u*>(kt + ((key_at ^ (s << 5)) + sub * 32 * kRowB)));
    };
    auto value_of = [&](const char* vt, int sub, int s, int c) {
      v4s t[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
        t[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(vt + ((value_at ^ (c << 6)) + (32 * sub + 16 * s + 8 * u) * kRowB)));
      return __builtin_bit_cast(v8bf, __builtin_shufflevector(t[0], t[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto logits = [&](const char* kt, int sub) {
      v16f y;
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = 0.f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_of(kt, sub, s), q[s], y, 0, 0, 0);
      return y;
    };
    auto add_values = [&](const char* vt, int sub) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value_of(vt, sub, s, c), w[s], o[c], 0, 0, 0);
    };
    auto weights = [&](v8bf (&to)[2]) {
      const float ref = m == -INFINITY ? 0.f : m;
      float sum = 0.f;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y[e] = fast_exp2(fmaf(x[8 * s + e], P.scale_log2, -ref));
          sum += y[e];
        }
        const v4u p = {pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
        to[s] = __builtin_bit_cast(v8bf, p);
      }
      l += sum;
    };
    // One step: weights of block j, logits of block j + 1 (keys: buffer kbuf, half sub), values of block j - 1 (buffer vbuf).  Left to itself the compiler puts
    // the three one after the other and waits for every read from LDS where it is used.  So the order is laid down: reads run kAhead products ahead,
    // and behind every product stands its share of the vector work, which the products cover (a product takes the matrix core 32 clocks and the issue
    // port 4).
    auto step = [&](int kbuf, int vbuf, int sub, int next_at) {
      constexpr int kProducts = kSteps + 2 * kBlocks, kAhead = 3;
      const char *kt = lds[kbuf][0], *vt = lds[vbuf][1];
      auto operand = [&](int i) { return i < kSteps ? key_of(kt, sub, i) : value_of(vt, sub, (i - kSteps) / kBlocks, (i - kSteps) % kBlocks); };
      const float ref = m == -INFINITY ? 0.f : m;
      v8bf f[kAhead + 1];
      v4u now[2];
      v16f y;
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = 0.f;
      float sum = 0.f, top = -INFINITY;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) f[i] = operand(i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kProducts; ++i) {
        if (i + kAhead < kProducts) f[(i + kAhead) % (kAhead + 1)] = operand(i + kAhead);
        const v8bf a = f[i % (kAhead + 1)];
        if (i < kSteps) y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[i], y, 0, 0, 0);
        else o[(i - kSteps) % kBlocks] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, w[(i - kSteps) / kBlocks], o[(i - kSteps) % kBlocks], 0, 0, 0);
        constexpr int kPairs = 8;                            // pairs of logits of block j
#pragma unroll
        for (int p = i * kPairs / kProducts; p < (i + 1) * kPairs / kProducts; ++p) {
          const float e0 = fast_exp2(fmaf(x[2 * p], P.scale_log2, -ref)), e1 = fast_exp2(fmaf(x[2 * p + 1], P.scale_log2, -ref));
          uint32_t packed = pack_bf16(e0, e1);
          sum += e0 + e1;
          asm volatile("" : "+v"(packed), "+v"(sum));
          now[p / 4][p % 4] = packed;
        }
        // block j + 1's largest logit, a few products behind its last one
        constexpr int kFrom = kSteps + 1, kLeft = kProducts - kFrom;
        if (i >= kFrom) {
#pragma unroll
          for (int e = (i - kFrom) * 16 / kLeft; e < (i - kFrom + 1) * 16 / kLeft; ++e) top = fmaxf(top, y[e]);
          asm volatile("" : "+v"(top));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      l += sum;
      w[0] = __builtin_bit_cast(v8bf, now[0]);
      w[1] = __builtin_bit_cast(v8bf, now[1]);
      x = y;
      settle(next_at, kbuf, sub, top);
    };

    const int tiles = (t_end - tile0 + kTile - 1) / kTile;
    if (tiles > 0) {
      request(tile0, 0, kKeys | kValues, __builtin_amdgcn_readfirstlane(look_up(tile0)));
      int id1 = __builtin_amdgcn_readfirstlane(look_up(tile0 + kTile)), id2 = __builtin_amdgcn_readfirstlane(look_up(tile0 + 2 * kTile));
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (tiles > 1) request(tile0 + kTile, 1, kKeys, id1);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) w[s][e] = (__bf16)0.f;
      x = logits(lds[0][0], 0);
      settle(tile0, 0, 0, largest(x));
      weights(w);
      x = logits(lds[0][0], 1);
      settle(tile0 + 32, 0, 1, largest(x));
      for (int t = 0; t + 1 < tiles; ++t) {
        const int at = tile0 + t * kTile, buf = t & 1;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        request(at + kTile, buf ^ 1, kValues, id1);
        if (t + 2 < tiles) request(at + 2 * kTile, buf, kKeys, id2);
        id1 = id2;
        id2 = __builtin_amdgcn_readfirstlane(look_up(at + 3 * kTile));        // (used a tile later: its latency is not waited for)
        step(buf ^ 1, buf, 0, at + kTile);
        step(buf ^ 1, buf, 1, at + kTile + 32);
      }
      const char* vt = lds[(tiles - 1) & 1][1];
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      add_values(vt, 0);
      weights(w);
      add_values(vt, 1);
    }

    l += __shfl_xor(l, 32);
    if (r < r1) {
      const int64_t row = sq.first + i;
      if (st.parts == 1) {
        const float inv = inverse_sum(l);
        uint16_t* to = out + b * P.o_b + row * P.o_t + (int64_t)head * P.o_h + 4 * half;
#pragma unroll
        for (int c = 0; c < kBlocks; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<uint2*>(to + 32 * c + 8 * e) = make_uint2(pack_bf16(o[c][4 * e] * inv, o[c][4 * e + 1] * inv),
                                                                         pack_bf16(o[c][4 * e + 2] * inv, o[c][4 * e + 3] * inv));
        if (lse != nullptr && half == 0) lse[b * P.l_b + row * P.l_t + head * P.l_h] = to_natural_lse(m, l);
      } else {
        const int64_t at = ((int64_t)part_no * P.tokens + row) * P.Hq + head;
        float* to = part.o + at * D + 4 * half;
#pragma unroll
        for (int c = 0; c < kBlocks; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) *reinterpret_cast<float4*>(to + 32 * c + 8 * e) = make_float4(o[c][4 * e], o[c][4 * e + 1], o[c][4 * e + 2], o[c][4 * e + 3]);
        if (half == 0) part.ml[at] = make_float2(m, l);
      }
    }
    __syncthreads();
  }
}

template <int D>
static void rows_launch(const Paged& P, const AttendPlan& pl, const void* Q, const void* K, const void* V, const int32_t* table, const int32_t* q_start,
                        const int32_t* kv_len, void* out, float* lse, Partials part, hipStream_t s) {
  const uint16_t *q = static_cast<const uint16_t*>(Q), *k = static_cast<const uint16_t*>(K), *v = static_cast<const uint16_t*>(V);
  const dim3 grid((unsigned)((int64_t)P.B * P.Hkv * pl.parts * pl.row_blocks)), block(64 * kRowWaves);
  // (a lane's offset within the 16 rows of a run is 32 bits)
  const bool banded = P.div.page % 16 == 0 && P.row_stride * 2 * 16 < (int64_t)1 << 31;
  if (banded) launch(attend_rows_kernel<D, true>, grid, block, s, P, pl, q, k, v, table, q_start, kv_len, static_cast<uint16_t*>(out), lse, part);
  else        launch(attend_rows_kernel<D, false>, grid, block, s, P, pl, q, k, v, table, q_start, kv_len, static_cast<uint16_t*>(out), lse, part);
}

void launch_attend_rows(const Paged& P, const AttendPlan& pl, const void* Q, const void* K, const void* V, const int32_t* table,
                        const int32_t* q_start, const int32_t* kv_len, void* out, float* lse, Partials part, hipStream_t s) {
  if (P.d == 64) rows_launch<64>(P, pl, Q, K, V, table, q_start, kv_len, out, lse, part, s);
  else           rows_launch<128>(P, pl, Q, K, V, table, q_start, kv_len, out, lse, part, s);
}

}  // namespace ccd
