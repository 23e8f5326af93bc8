// ccd_rope: rotary embedding of the queries and keys of a step, and ccd_paged_append, which embeds keys on their way into the
// pages.  Both move their rows once in and once out and are bound by memory; what could be in the way is the arithmetic of
// cosine and sine (about 35 instructions a pair), so a wave works them out once for a token and takes all its heads, four pieces of heads read before
// they are written.  Measured, bf16: 8192 tokens of 40 heads of 128 35.4 us (4.75 TB/s moved, a copy reaches 5.12), 16384 tokens of 8 heads appended with
// their keys embedded 29.5 us (4.55); 16 tokens 3.6 us and the launch.
#include "ccd_paged.h"
#include "ccd_rotary.h"

namespace ccd {

// where row h of a token goes: heads of a dense or strided tensor, or of a page
constexpr int kBatch = 4;

template <class T>
struct Rows {
  const T* src;
  T* dst;
  int64_t src_h, dst_h;
};

// one piece of the heads h, h + side, ... below h_end
template <class T>
__device__ __forceinline__ void copy_pieces(const Rows<T>& rows, int h, int h_end, int side, int e) {
  for (; h < h_end; h += kBatch * side) {
    v4u a[kBatch] = {};
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (h + u * side < h_end) a[u] = *reinterpret_cast<const v4u*>(rows.src + (h + u * side) * rows.src_h + e);
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (h + u * side < h_end) *reinterpret_cast<v4u*>(rows.dst + (h + u * side) * rows.dst_h + e) = a[u];
  }
}

// The heads h0, h0 + 1 .. of one token by one wave, in pieces of 16 bytes: `R.rot` elements turned, the rest copied.  A piece index
// runs over the turned pieces and then over the tail; 64 / pieces heads at a time.
template <class T, bool HALF>
__device__ __forceinline__ void rotate_heads(const Rotary& R, const Rows<T>& rows, int h_begin, int h_end, int lane, int position,
                                             const uint64_t* __restrict__ turns, bool copy_tail) {
  constexpr int kEPL = 16 / sizeof(T);
  const int turned = R.rot / (HALF ? 2 * kEPL : kEPL);
  const int pieces = turned + (copy_tail ? (R.d - R.rot) / kEPL : 0);
  // more than 64 pieces (rows of more than 1 KiB): several rounds of lanes
  for (int p0 = 0; p0 < pieces; p0 += 64) {
    const int width = pieces - p0 < 64 ? pieces - p0 : 64, side = 64 / width;
    const int piece = p0 + lane % width, h_lane = lane / width;
    if (h_lane >= side) continue;
    // (kBatch heads are read before the first is written: dst may be src, so the compiler would not move a load over a store)
    if (piece < turned) {
      const int e = piece * kEPL, e2 = e + R.rot / 2;
      RotaryLane<T, HALF> rot;
      for (int h0 = h_begin + h_lane; h0 < h_end; h0 += kBatch * side) {
        v4u a[kBatch] = {}, b[kBatch] = {};
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          if (h0 + u * side >= h_end) continue;
          const T* s = rows.src + (h0 + u * side) * rows.src_h;
          a[u] = *reinterpret_cast<const v4u*>(s + e);
          if constexpr (HALF) b[u] = *reinterpret_cast<const v4u*>(s + e2);
        }
        if (h0 == h_begin + h_lane) rot.angles(R, piece, position, turns);           // (while the first heads are on their way)
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          rot.rotate(a[u], b[u]);
          if (h0 + u * side < h_end) {
            T* o = rows.dst + (h0 + u * side) * rows.dst_h;
            *reinterpret_cast<v4u*>(o + e) = a[u];
            if constexpr (HALF) *reinterpret_cast<v4u*>(o + e2) = b[u];
          }
        }
      }
    } else {
      copy_pieces(rows, h_begin + h_lane, h_end, side, R.rot + (piece - turned) * kEPL);
    }
  }
}

// The same pair by pair, for a turned part that does not come in whole pieces of 16 bytes: as many heads side by side as lanes allow, kBatchPairs of them
// read before one is written; then the tail, element by element through all heads.  6437 tokens of 72 heads of 64, 60 turned: 45.5 us, 88 head
// after head (64 turned, by pieces: 28).
constexpr int kBatchPairs = 8;

template <class T, bool HALF>
__device__ __forceinline__ void rotate_heads_pairwise(const Rotary& R, const Rows<T>& rows, int h_begin, int h_end, int lane, int position,
                                                      const uint64_t* __restrict__ turns, bool copy_tail) {
  const int pairs = R.rot / 2;
  for (int i0 = 0; i0 < pairs; i0 += 64) {
    const int width = pairs - i0 < 64 ? pairs - i0 : 64, side = 64 / width;
    const int i = i0 + lane % width, h_lane = lane / width;
    if (h_lane >= side) continue;
    float c, s;
    cos_sin_of_phase((uint64_t)(uint32_t)position * turns[i], c, s);
    c *= R.amplitude;
    s *= R.inverse ? -R.amplitude : R.amplitude;
    const int e1 = HALF ? i : 2 * i, e2 = HALF ? i + pairs : 2 * i + 1;
    for (int h0 = h_begin + h_lane; h0 < h_end; h0 += kBatchPairs * side) {
      float x[kBatchPairs], z[kBatchPairs];
#pragma unroll
      for (int u = 0; u < kBatchPairs; ++u) {
        const T* src = rows.src + (int64_t)(h0 + u * side < h_end ? h0 + u * side : h0) * rows.src_h;
        if constexpr (HALF) {
          x[u] = load_elem(src + e1);
          z[u] = load_elem(src + e2);
        } else if constexpr (sizeof(T) == 2) {
          const uint32_t two = *reinterpret_cast<const uint32_t*>(src + e1);
          x[u] = __uint_as_float(two << 16);
          z[u] = __uint_as_float(two & 0xFFFF0000u);
        } else {
          const float2 two = *reinterpret_cast<const float2*>(src + e1);
          x[u] = two.x;
          z[u] = two.y;
        }
      }
#pragma unroll
      for (int u = 0; u < kBatchPairs; ++u) {
        if (h0 + u * side >= h_end) continue;
        T* dst = rows.dst + (int64_t)(h0 + u * side) * rows.dst_h;
        const float y1 = fmaf(-z[u], s, x[u] * c), y2 = fmaf(x[u], s, z[u] * c);
        if constexpr (HALF) {
          store_elem(dst + e1, y1);
          store_elem(dst + e2, y2);
        } else if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<uint32_t*>(dst + e1) = pack_bf16(y1, y2);
        } else {
          *reinterpret_cast<float2*>(dst + e1) = make_float2(y1, y2);
        }
      }
    }
  }
  if (!copy_tail || R.rot == R.d) return;
  const int tail = R.d - R.rot, all = tail * (h_end - h_begin);
  for (int k0 = lane; k0 < all; k0 += 64 * kBatchPairs) {
    T t[kBatchPairs];
    int h[kBatchPairs], e[kBatchPairs];
#pragma unroll
    for (int u = 0; u < kBatchPairs; ++u) {
      const int k = k0 + 64 * u < all ? k0 + 64 * u : k0;
      h[u] = h_begin + k / tail;
      e[u] = R.rot + k % tail;
      t[u] = rows.src[h[u] * rows.src_h + e[u]];
    }
#pragma unroll
    for (int u = 0; u < kBatchPairs; ++u)
      if (k0 + 64 * u < all) rows.dst[h[u] * rows.dst_h + e[u]] = t[u];
  }
}

enum { kHalves = 0, kPairsNext = 1, kHalvesPairwise = 2, kNextPairwise = 3 };

template <class T, int KIND>
__device__ __forceinline__ void rotate_any(const Rotary& R, const Rows<T>& rows, int h_begin, int h_end, int lane, int position,
                                           const uint64_t* __restrict__ turns, bool copy_tail) {
  if constexpr (KIND == kHalves) rotate_heads<T, true>(R, rows, h_begin, h_end, lane, position, turns, copy_tail);
  else if constexpr (KIND == kPairsNext) rotate_heads<T, false>(R, rows, h_begin, h_end, lane, position, turns, copy_tail);
  else rotate_heads_pairwise<T, KIND == kHalvesPairwise>(R, rows, h_begin, h_end, lane, position, turns, copy_tail);
}

// a wave per (token, group of heads)
template <class T, int KIND>
__global__ __launch_bounds__(256) void rotary_kernel(Rotary R, const T* X, const int32_t* __restrict__ positions,
                                                     const uint64_t* __restrict__ turns, T* Y, int heads_per_wave) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= R.tokens) return;
  const int position = positions[t];
  if (position < 0) return;
  const int h_begin = blockIdx.y * heads_per_wave;
  const int h_end = h_begin + heads_per_wave < R.heads ? h_begin + heads_per_wave : R.heads;
  const Rows<T> rows{X + t * R.x_t, Y + t * R.y_t, R.x_h, R.y_h};
  rotate_any<T, KIND>(R, rows, h_begin, h_end, lane, position, turns, (const void*)X != (const void*)Y);
}

// a wave per token: its keys (turned, or copied) and values into the row of its slot
template <class T, int KIND>
__global__ __launch_bounds__(256) void paged_append_kernel(Paged P, Rotary R, bool rope, const T* __restrict__ K_new, const T* __restrict__ V_new,
                                                           const int32_t* __restrict__ slots, const int32_t* __restrict__ positions,
                                                           const uint64_t* __restrict__ turns, T* K, T* V) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (t >= P.tokens) return;
  const int slot = slots[t], position = rope ? positions[t] : 0;
  if (slot < 0 || position < 0) return;
  const int page = page_of(P.div, slot), row = slot - page * P.div.page;
  if (page >= P.n_pages) return;
  const int64_t to = page * P.page_stride + row * P.row_stride, from = t * P.new_t;
  constexpr int kEPL = 16 / sizeof(T);
  const int pieces = P.d / kEPL;                       // 8, 16 or 32
  const int piece = lane % pieces, side = 64 / pieces;
  copy_pieces(Rows<T>{V_new + from, V + to, P.new_h, P.head_stride}, lane / pieces, P.Hkv, side, piece * kEPL);
  const Rows<T> rows{K_new + from, K + to, P.new_h, P.head_stride};
  if (rope) rotate_any<T, KIND>(R, rows, 0, P.Hkv, lane, position, turns, true);
  else      copy_pieces(rows, lane / pieces, P.Hkv, side, piece * kEPL);
}

template <class T, int KIND>
static void rotary_launch(const Rotary& R, const void* X, const int32_t* positions, const uint64_t* turns, void* Y, hipStream_t s) {
  // few tokens: the heads of a token are shared out until about 1024 waves are under way
  int groups = 1;
  while (groups * 2 <= R.heads && (int64_t)R.tokens * groups < 1024) groups *= 2;
  const int per = (R.heads + groups - 1) / groups;
  launch(rotary_kernel<T, KIND>, dim3((R.tokens + 3) / 4, (R.heads + per - 1) / per), dim3(256), s, R, static_cast<const T*>(X), positions, turns,
         static_cast<T*>(Y), per);
}

template <class T>
static void rotary_of(const Rotary& R, const void* X, const int32_t* positions, const uint64_t* turns, void* Y, hipStream_t s) {
  const bool whole = rotary_by_pieces(R.rot, R.half, sizeof(T));
  if (whole && R.half) rotary_launch<T, kHalves>(R, X, positions, turns, Y, s);
  else if (whole)      rotary_launch<T, kPairsNext>(R, X, positions, turns, Y, s);
  else if (R.half)     rotary_launch<T, kHalvesPairwise>(R, X, positions, turns, Y, s);
  else                 rotary_launch<T, kNextPairwise>(R, X, positions, turns, Y, s);
}

void launch_rotary(const Rotary& R, int dtype, const void* X, const int32_t* positions, const uint64_t* turns, void* Y, hipStream_t s) {
  if (dtype == 0) rotary_of<float>(R, X, positions, turns, Y, s);
  else            rotary_of<uint16_t>(R, X, positions, turns, Y, s);
}

template <class T, int KIND>
static void append_launch(const Paged& P, const Rotary* rope, const void* K_new, const void* V_new, const int32_t* slots, const int32_t* positions,
                          const uint64_t* turns, void* K, void* V, hipStream_t s) {
  launch(paged_append_kernel<T, KIND>, dim3((P.tokens + 3) / 4), dim3(256), s, P, rope ? *rope : Rotary{}, rope != nullptr, static_cast<const T*>(K_new),
         static_cast<const T*>(V_new), slots, positions, turns, static_cast<T*>(K), static_cast<T*>(V));
}

template <class T>
static void append_of(const Paged& P, const Rotary* rope, const void* K_new, const void* V_new, const int32_t* slots, const int32_t* positions,
                      const uint64_t* turns, void* K, void* V, hipStream_t s) {
  const bool whole = rope == nullptr || rotary_by_pieces(rope->rot, rope->half, sizeof(T)), half = rope == nullptr || rope->half;
  if (whole && half) append_launch<T, kHalves>(P, rope, K_new, V_new, slots, positions, turns, K, V, s);
  else if (whole)    append_launch<T, kPairsNext>(P, rope, K_new, V_new, slots, positions, turns, K, V, s);
  else if (half)     append_launch<T, kHalvesPairwise>(P, rope, K_new, V_new, slots, positions, turns, K, V, s);
  else               append_launch<T, kNextPairwise>(P, rope, K_new, V_new, slots, positions, turns, K, V, s);
}

void launch_paged_append(const Paged& P, int dtype, const Rotary* rope, const void* K_new, const void* V_new, const int32_t* slots,
                         const int32_t* positions, const uint64_t* turns, void* K, void* V, hipStream_t s) {
  if (dtype == 0) append_of<float>(P, rope, K_new, V_new, slots, positions, turns, K, V, s);
  else            append_of<uint16_t>(P, rope, K_new, V_new, slots, positions, turns, K, V, s);
}

}  // namespace ccd
