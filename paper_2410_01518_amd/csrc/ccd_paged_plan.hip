// ccd_paged_plan: block tables and slot maps of a step, built on the device from the sequences' lengths.
//
// Everything follows from three prefix sums over the sequences: pages taken, pages given back, new tokens.  A few thousand
// lengths are read and summed in about the time a second launch would take, so every workgroup does it for itself and then deals with its
// share of the tokens and of the table: one launch, and no workgroup waits for another.  Only what is given back needs an order
// of its own (entries that name no page are left out), which the first workgroup walks.  Bound by latency, a few dependent loads; so
// no workgroup has two kinds of work after one another: the first what is given back and the sums, others the table, others the tokens.
// Measured: 8 sequences 5 us and the launch, 512 of 512 entries with 205000 new tokens and 4455 pages given back 12.
#include "ccd_common.h"
#include "ccd_paged.h"

namespace ccd {

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64, kPlanGive = 8;

__device__ __forceinline__ int wave_inclusive(int x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}
__device__ __forceinline__ int64_t wave_inclusive(int64_t x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// the sequence whose range [first[b], first[b + 1]) holds i, for first[0] <= i < first[B]
__device__ __forceinline__ int find_sequence(const int* first, int B, int i) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

struct PlanArgs {
  const int32_t *before, *after, *table;
  int32_t *table_next, *ring, *cursor, *cursor_next, *q_start, *slots, *positions;
};

// CAP: sequences the workgroup's arrays hold
// table_wgs: workgroups that write the table; those behind them have the tokens
template <int CAP>
__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(Paged P, PlanArgs A, int table_wgs) {
  __shared__ int first_page[CAP + 1], first_gone[CAP + 1], first_token[CAP + 1];     // before sequence b: pages taken, given back, new tokens
  __shared__ int wave_take[kPlanWaves], wave_give[kPlanWaves];
  __shared__ int64_t wave_new[kPlanWaves];
  __shared__ int given;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = P.B, W = P.table_width;
  const bool in_place = A.table_next == A.table;
  constexpr int kPer = CAP / kPlanThreads > 0 ? CAP / kPlanThreads : 1;

  const int head = A.cursor[0], count = A.cursor[1];
  auto pages = [&](int len) { return len > 0 ? page_of(P.div, len - 1) + 1 : 0; };
  // the thread's sequences are neighbours
  int take = 0, give = 0;
  int64_t fresh = 0, short_of = 0;
  int takes[kPer], gives[kPer], news[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int b = tid * kPer + j;
    int len0 = 0, len1 = 0;
    if (b < B) { len0 = A.before[b] > 0 ? A.before[b] : 0; len1 = A.after[b] > 0 ? A.after[b] : 0; }
    const int want = pages(len1), p0 = pages(len0) < W ? pages(len0) : W, p1 = want < W ? want : W;
    takes[j] = p1 > p0 ? p1 - p0 : 0;
    gives[j] = p0 > p1 ? p0 - p1 : 0;
    news[j] = len1 > len0 ? len1 - len0 : 0;
    take += takes[j]; give += gives[j]; fresh += news[j];
    short_of += want - p1;
  }
  const int take_to = wave_inclusive(take, lane), give_to = wave_inclusive(give, lane);
  const int64_t new_to = wave_inclusive(fresh, lane);
  if (lane == 63) { wave_take[wave] = take_to; wave_give[wave] = give_to; wave_new[wave] = new_to; }
  if (tid == 0) given = 0;
  __syncthreads();
  int take_at = take_to - take, give_at = give_to - give;
  int64_t new_at = new_to - fresh;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w)
    if (w < wave) { take_at += wave_take[w]; give_at += wave_give[w]; new_at += wave_new[w]; }
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int b = tid * kPer + j;
    if (b <= B) {          // (behind the last sequence: the sums of all)
      first_page[b] = take_at; first_gone[b] = give_at;
      first_token[b] = new_at < 0x7FFFFFFF ? (int)new_at : 0x7FFFFFFF;
    }
    take_at += takes[j]; give_at += gives[j]; new_at += news[j];
  }
  if (B == CAP && tid == kPlanThreads - 1) {
    first_page[B] = take_at; first_gone[B] = give_at;
    first_token[B] = new_at < 0x7FFFFFFF ? (int)new_at : 0x7FFFFFFF;
  }
  __syncthreads();
  const int all_taken = first_page[B], all_gone = first_gone[B], all_new = first_token[B];
  const int free_now = count > 0 ? (count < P.n_pages ? count : P.n_pages) : 0;
  const int start = head >= 0 && head < P.n_pages ? head : 0;
  const int taken = all_taken < free_now ? all_taken : free_now;
  auto ring_at = [&](int i) {                                        // 0 <= i <= n_pages
    const int64_t at = (int64_t)start + i;
    return (int)(at < P.n_pages ? at : at - P.n_pages);
  };
  auto ring_behind = [&](int i) {                                    // of the free pages; more than the ring holds only where a table names pages twice
    int64_t at = (int64_t)ring_at(free_now) + i;
    if (at >= P.n_pages) at -= P.n_pages;
    return (int)(at < P.n_pages ? at : at % P.n_pages);
  };
  auto page_taken = [&](int rank) { return rank < free_now ? A.ring[ring_at(rank)] : -1; };
  auto p_before = [&](int b) { const int p = pages(A.before[b]); return p < W ? p : W; };

  if (blockIdx.x == 0) {
    for (int b = tid; b <= B; b += kPlanThreads) A.q_start[b] = first_token[b];
    // what is given back goes behind the free pages, in order, entries that name no page left out
    // (as few to a thread as they are: entries that follow one another, all searched for at once)
    const int each = (all_gone + kPlanThreads - 1) / kPlanThreads, per = each < kPlanGive ? each : kPlanGive;
    for (int r0 = 0; r0 < all_gone; r0 += kPlanThreads * per) {
      const int r_mine = r0 + tid * per, mine = all_gone - r_mine < per ? all_gone - r_mine : per;
      int ids[kPlanGive], of[kPlanGive] = {}, n = 0;
#pragma unroll
      for (int step = CAP / 2; step > 0; step >>= 1)
#pragma unroll
        for (int j = 0; j < kPlanGive; ++j) {
          const int next = of[j] + step;
          if (next < B && first_gone[next] <= r_mine + j) of[j] = next;
        }
#pragma unroll
      for (int j = 0; j < kPlanGive; ++j) {
        ids[j] = -1;
        if (j < mine) {
          const int64_t e = (int64_t)of[j] * W + p_before(of[j]) - (first_gone[of[j] + 1] - (r_mine + j));
          ids[j] = A.table[e];
          if (in_place) A.table_next[e] = -1;
        }
      }
#pragma unroll
      for (int j = 0; j < kPlanGive; ++j) {
        if (ids[j] < 0 || ids[j] >= P.n_pages) ids[j] = -1;
        n += ids[j] >= 0;
      }
      const int to = wave_inclusive(n, lane);
      if (lane == 63) wave_give[wave] = to;
      __syncthreads();
      int at = given + to - n, sum = 0;
#pragma unroll
      for (int w = 0; w < kPlanWaves; ++w) { if (w < wave) at += wave_give[w]; sum += wave_give[w]; }
#pragma unroll
      for (int j = 0; j < kPlanGive; ++j)
        if (ids[j] >= 0) A.ring[ring_behind(at++)] = ids[j];
      __syncthreads();
      if (tid == 0) given += sum;
      __syncthreads();
    }
    // the pages short: of the ring, and those a row of the table has no room for
    const int64_t over = wave_inclusive(short_of, lane);
    if (lane == 63) wave_new[wave] = over;
    __syncthreads();
    if (tid == 0) {
      int64_t missing = all_taken - taken;
      for (int w = 0; w < kPlanWaves; ++w) missing += wave_new[w];
      if (A.cursor_next != A.cursor) {
        A.cursor_next[0] = ring_at(taken);
        A.cursor_next[1] = free_now - taken + given;
        A.cursor_next[3] = 0;
      }
      A.cursor_next[2] = missing < 0x7FFFFFFF ? (int)missing : 0x7FFFFFFF;
    }
  }

  // the table: a wave per piece of 256 entries of a row
  const int wg = (int)blockIdx.x - 1, waves = table_wgs * kPlanWaves;
  const int pieces = (W + 255) / 256;
  for (int64_t it = wg * kPlanWaves + wave; wg >= 0 && wg < table_wgs && it < (int64_t)B * pieces; it += waves) {
    const int b = (int)(it / pieces), c0 = (int)(it % pieces) * 256;
    const int p0 = p_before(b), n_take = first_page[b + 1] - first_page[b], n_give = first_gone[b + 1] - first_gone[b];
    const int keep = p0 - n_give, p1 = p0 + n_take - n_give;
    const int64_t row = (int64_t)b * W;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = c0 + j * 64 + lane;
      if (c >= W) continue;
      if (c < keep) {
        if (!in_place) A.table_next[row + c] = A.table[row + c];
      } else if (c < p1) {
        A.table_next[row + c] = page_taken(first_page[b] + c - p0);
      } else if (!in_place) {
        A.table_next[row + c] = -1;
      }
    }
  }

  // the new tokens
  const int token_wgs = (int)gridDim.x - 1 - table_wgs;
  for (int64_t i = (int64_t)(wg - table_wgs) * kPlanThreads + tid; i >= 0 && i < P.tokens; i += (int64_t)token_wgs * kPlanThreads) {
    int slot = -1, pos = -1;
    if (i < all_new) {
      const int b = find_sequence(first_token, B, (int)i);
      const int len0 = A.before[b] > 0 ? A.before[b] : 0;
      pos = len0 + ((int)i - first_token[b]);
      const int c = page_of(P.div, pos), p0 = p_before(b);
      const int id = c >= W ? -1 : c < p0 ? A.table[(int64_t)b * W + c] : page_taken(first_page[b] + c - p0);
      if (id >= 0 && id < P.n_pages) slot = id * P.div.page + (pos - c * P.div.page);
    }
    A.slots[i] = slot;
    A.positions[i] = pos;
  }

  // A cursor that is moved in place: by whichever workgroup is the last to have read it.  The number of pages given back, which
  // only the first one knows, waits in q_start[0], which is 0 otherwise.
  if (A.cursor_next == A.cursor) {
    __syncthreads();
    if (tid == 0) {
      if (blockIdx.x == 0) atomicExch(&A.q_start[0], given);
      __threadfence();
      if (atomicAdd(&A.cursor[3], 1) == (int)gridDim.x - 1) {
        __threadfence();
        const int back = atomicExch(&A.q_start[0], 0);
        A.cursor[0] = ring_at(taken);
        A.cursor[1] = free_now - taken + back;
        A.cursor[3] = 0;
      }
    }
  }
}

void launch_paged_plan(const Paged& P, const int32_t* before, const int32_t* after, const int32_t* table, int32_t* table_next,
                       int32_t* ring, int32_t* cursor, int32_t* cursor_next, int32_t* q_start, int32_t* slots, int32_t* positions,
                       hipStream_t s) {
  const PlanArgs A{before, after, table, table_next, ring, cursor, cursor_next, q_start, slots, positions};
  const int64_t rows_wgs = ((int64_t)P.B * ((P.table_width + 255) / 256) + kPlanWaves - 1) / kPlanWaves;
  const int64_t tokens_wgs = ((int64_t)P.tokens + kPlanThreads - 1) / kPlanThreads;
  const int table_wgs = (int)(rows_wgs > 128 ? 128 : rows_wgs), token_wgs = (int)(tokens_wgs > 256 ? 256 : tokens_wgs);
  const dim3 grid((unsigned)(1 + table_wgs + token_wgs));
  if (P.B <= 512) launch(paged_plan_kernel<512>, grid, dim3(kPlanThreads), s, P, A, table_wgs);
  else            launch(paged_plan_kernel<kPlanMaxSequences>, grid, dim3(kPlanThreads), s, P, A, table_wgs);
}

}  // namespace ccd
