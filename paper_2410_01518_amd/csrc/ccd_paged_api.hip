// Host side of the paged cache's entry points: argument checks, everything before the launch.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/infinipot.h"
#include "ccd_launch.h"
#include "ccd_paged.h"

namespace ccd {

static bool on_16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
static int paged_status() { return hipGetLastError() == hipSuccess ? CCD_OK : CCD_ELAUNCH; }

constexpr int32_t kMostTokens = 1 << 25;               // of a launch of a wave each
enum PagedNeed { kPlan = 1, kCache = 2, kNew = 4, kAttend = 8 };

static int check_stride(int64_t stride, int64_t least, int64_t esz) {
  if (stride < least) return CCD_EINVAL;
  return (stride * esz) % 16 ? CCD_EALIGN : CCD_OK;
}

static int check_paged(const ccd_paged_t* c, int need) {
  if (c == nullptr) return CCD_EINVAL;
  if (c->tokens < 0 || c->page < 1 || c->n_pages < 1) return CCD_EINVAL;
  if ((int64_t)c->page * c->n_pages > 0x7FFFFFFF) return CCD_EINVAL;
  if (need & (kPlan | kAttend)) {
    if (c->B < 1 || c->table_width < 1 || (int64_t)c->B * c->table_width > 0x7FFFFFFF) return CCD_EINVAL;
    if ((int64_t)c->page * c->table_width > 1 << 30) return CCD_EINVAL;                // positions, and a tile past them, are counted in int32
  }
  if ((need & kPlan) && c->B > kPlanMaxSequences) return CCD_EUNSUPPORTED;
  if (!(need & kCache)) return CCD_OK;
  if (c->Hkv < 1 || c->Hkv > 65535) return CCD_EINVAL;
  if (c->dtype != CCD_FP32 && c->dtype != CCD_BF16) return CCD_EUNSUPPORTED;
  if (c->d != 64 && c->d != 128) return CCD_EUNSUPPORTED;
  const int64_t esz = c->dtype == CCD_FP32 ? 4 : 2;
  struct Stride { int64_t value, least; };
  Stride strides[10];
  int n = 0;
  strides[n++] = {c->page_stride, c->d}; strides[n++] = {c->head_stride, c->d}; strides[n++] = {c->row_stride, c->d};
  if ((need & kNew) && c->tokens > kMostTokens) return CCD_EUNSUPPORTED;
  if (need & kNew) { strides[n++] = {c->new_stride_t, c->d}; strides[n++] = {c->new_stride_h, c->d}; }
  if (need & kAttend) {
    if (c->Hq < 1 || c->Hq % c->Hkv != 0) return CCD_EINVAL;
    // (a launch has less than 2^32 threads)
    if ((int64_t)c->tokens * c->Hq > 1 << 28 || (int64_t)c->B * c->Hkv > 1 << 21) return CCD_EUNSUPPORTED;
    if (c->window < 0 || (c->behind != 0 && c->behind != 1) || c->max_new < 0 || c->max_len < 0) return CCD_EINVAL;
    if (!(c->scale >= 0.f) || isinf(c->scale)) return CCD_EINVAL;
    strides[n++] = {c->q_stride_b, 0}; strides[n++] = {c->q_stride_t, c->d}; strides[n++] = {c->q_stride_h, c->d};
    strides[n++] = {c->o_stride_b, 0}; strides[n++] = {c->o_stride_t, c->d}; strides[n++] = {c->o_stride_h, c->d};
    if (c->lse_stride_b < 0 || c->lse_stride_t < 1 || c->lse_stride_h < 1) return CCD_EINVAL;
  }
  for (int pass = 0; pass < 2; ++pass)                   // ranges before alignment, as in the other calls
    for (int i = 0; i < n; ++i) {
      const int rc = check_stride(strides[i].value, strides[i].least, esz);
      if (rc == (pass == 0 ? CCD_EINVAL : CCD_EALIGN)) return rc;
    }
  return CCD_OK;
}

static Paged make_paged(const ccd_paged_t* c) {
  Paged P{};
  P.B = c->B; P.tokens = c->tokens; P.Hq = c->Hq; P.Hkv = c->Hkv; P.G = c->Hkv > 0 ? c->Hq / c->Hkv : 0; P.d = c->d;
  P.n_pages = c->n_pages; P.table_width = c->table_width; P.window = c->window; P.behind = c->behind;
  P.div = make_page_div(c->page);
  const int64_t room = (int64_t)c->page * c->table_width;
  P.max_len = room < 0 ? 0 : room > 0x7FFFFFFF ? 0x7FFFFFFF : (int32_t)room;
  P.scale_log2 = (float)((c->scale > 0.f ? (double)c->scale : 1.0 / sqrt((double)(c->d > 0 ? c->d : 1))) * 1.4426950408889634074);
  P.page_stride = c->page_stride; P.head_stride = c->head_stride; P.row_stride = c->row_stride;
  P.new_t = c->new_stride_t; P.new_h = c->new_stride_h;
  P.q_b = c->q_stride_b; P.q_t = c->q_stride_t; P.q_h = c->q_stride_h;
  P.o_b = c->o_stride_b; P.o_t = c->o_stride_t; P.o_h = c->o_stride_h;
  P.l_b = c->lse_stride_b; P.l_t = c->lse_stride_t; P.l_h = c->lse_stride_h;
  return P;
}

// what the host knows of a step's lengths: its hints, where they are tighter than the tensors
static int hint_new(const ccd_paged_t* c) { return c->max_new > 0 && c->max_new < c->tokens ? c->max_new : c->tokens; }
static int hint_len(const ccd_paged_t* c, const Paged& P) { return c->max_len > 0 && c->max_len < P.max_len ? c->max_len : P.max_len; }

// rot, layout, inverse and amplitude: what turns a head of d elements
static int check_rotation(const ccd_rope_t* r, int d) {
  if (r->rot < 2 || r->rot % 2 != 0 || r->rot > d) return CCD_EINVAL;
  if (r->layout != CCD_ROPE_HALF && r->layout != CCD_ROPE_PAIRS) return CCD_EINVAL;
  if (r->inverse != 0 && r->inverse != 1) return CCD_EINVAL;
  if (!isfinite(r->amplitude)) return CCD_EINVAL;
  return CCD_OK;
}

static Rotary make_rotary(const ccd_rope_t* r) {
  Rotary R{};
  R.tokens = r->tokens; R.heads = r->heads; R.d = r->d; R.rot = r->rot;
  R.half = r->layout == CCD_ROPE_HALF; R.inverse = r->inverse;
  R.amplitude = r->amplitude == 0.f ? 1.f : r->amplitude;
  R.x_t = r->x_stride_t; R.x_h = r->x_stride_h; R.y_t = r->y_stride_t; R.y_h = r->y_stride_h;
  return R;
}

}  // namespace ccd

using namespace ccd;

extern "C" {

int ccd_paged_plan(const ccd_paged_t* paged, const int32_t* len_before, const int32_t* len_after, const int32_t* block_table,
                   int32_t* block_table_next, int32_t* free_pages, int32_t* cursor, int32_t* cursor_next, int32_t* q_start,
                   int32_t* slots, int32_t* positions, void* hip_stream) {
  const int rc = check_paged(paged, kPlan);
  if (rc != CCD_OK) return rc;
  if (len_before == nullptr || len_after == nullptr || block_table == nullptr || block_table_next == nullptr || free_pages == nullptr ||
      cursor == nullptr || cursor_next == nullptr || q_start == nullptr)
    return CCD_EINVAL;
  if (paged->tokens > 0 && (slots == nullptr || positions == nullptr)) return CCD_EINVAL;
  launch_paged_plan(make_paged(paged), len_before, len_after, block_table, block_table_next, free_pages, cursor, cursor_next, q_start, slots,
                    positions, static_cast<hipStream_t>(hip_stream));
  return paged_status();
}

int ccd_rope_turns(const ccd_rope_t* rope, uint64_t* turns) {
  if (rope == nullptr || turns == nullptr) return CCD_EINVAL;
  if (rope->rot < 2 || rope->rot % 2 != 0 || rope->rot > 1024) return CCD_EINVAL;
  if (rope->scaling < CCD_ROPE_PLAIN || rope->scaling > CCD_ROPE_PARTS) return CCD_EUNSUPPORTED;
  if (!(rope->base > 1.0) || rope->base > 18446744073709551616.0) return CCD_EINVAL;
  if (rope->scaling != CCD_ROPE_PLAIN && (!(rope->factor >= 1.0) || isinf(rope->factor))) return CCD_EINVAL;
  if (rope->scaling == CCD_ROPE_PARTS && (rope->context < 1 || !(rope->low < rope->high) || isinf(rope->low) || isinf(rope->high))) return CCD_EINVAL;
  const long double two_pi = 6.283185307179586476925286766559L, factor = rope->factor;
  long double base = rope->base;
  if (rope->scaling == CCD_ROPE_NTK && rope->rot > 2) base *= powl(factor, (long double)rope->rot / (rope->rot - 2));
  for (int i = 0; i < rope->rot / 2; ++i) {
    long double f = powl(base, -2.0L * i / rope->rot) / two_pi;            // turns per position, at most 1 / 2 pi
    if (rope->scaling == CCD_ROPE_LINEAR) f /= factor;
    if (rope->scaling == CCD_ROPE_PARTS) {
      const long double r = rope->context * f;
      long double keep = (r - rope->low) / ((long double)rope->high - rope->low);
      keep = keep < 0.0L ? 0.0L : keep > 1.0L ? 1.0L : keep;
      f *= keep + (1.0L - keep) / factor;
    }
    turns[i] = (uint64_t)(f * 18446744073709551616.0L + 0.5L);
  }
  return CCD_OK;
}

int ccd_rope(const ccd_rope_t* rope, const void* X, const int32_t* positions, const uint64_t* turns, void* Y, void* hip_stream) {
  if (rope == nullptr) return CCD_EINVAL;
  if (rope->tokens < 0 || rope->heads < 1 || rope->heads > 65535 || rope->d < 1) return CCD_EINVAL;
  if ((rope->dtype != CCD_FP32 && rope->dtype != CCD_BF16) || rope->tokens > kMostTokens) return CCD_EUNSUPPORTED;
  const int64_t esz = rope->dtype == CCD_FP32 ? 4 : 2;
  if (rope->d > 1024 || (rope->d * esz) % 16 != 0) return CCD_EUNSUPPORTED;
  int rc = check_rotation(rope, rope->d);
  if (rc != CCD_OK) return rc;
  if (rope->x_stride_t < rope->d || rope->x_stride_h < rope->d || rope->y_stride_t < rope->d || rope->y_stride_h < rope->d) return CCD_EINVAL;
  if (X != nullptr && X == Y && (rope->x_stride_t != rope->y_stride_t || rope->x_stride_h != rope->y_stride_h)) return CCD_EINVAL;
  if ((rope->x_stride_t * esz) % 16 || (rope->x_stride_h * esz) % 16 || (rope->y_stride_t * esz) % 16 || (rope->y_stride_h * esz) % 16) return CCD_EALIGN;
  if (rope->tokens == 0) return CCD_OK;
  if (X == nullptr || Y == nullptr || positions == nullptr || turns == nullptr) return CCD_EINVAL;
  if (!on_16(X) || !on_16(Y)) return CCD_EALIGN;
  launch_rotary(make_rotary(rope), rope->dtype, X, positions, turns, Y, static_cast<hipStream_t>(hip_stream));
  return paged_status();
}

int ccd_paged_append(const ccd_paged_t* paged, const ccd_rope_t* rope, const void* K_new, const void* V_new, const int32_t* slots,
                     const int32_t* positions, const uint64_t* turns, void* K_pages, void* V_pages, void* hip_stream) {
  int rc = check_paged(paged, kCache | kNew);
  if (rc != CCD_OK) return rc;
  if (rope != nullptr && (rc = check_rotation(rope, paged->d)) != CCD_OK) return rc;
  if (paged->tokens == 0) return CCD_OK;
  if (K_new == nullptr || V_new == nullptr || slots == nullptr || K_pages == nullptr || V_pages == nullptr) return CCD_EINVAL;
  if (rope != nullptr && (positions == nullptr || turns == nullptr)) return CCD_EINVAL;
  if (K_pages == V_pages || K_new == K_pages || V_new == V_pages) return CCD_EINVAL;
  if (!on_16(K_new) || !on_16(V_new) || !on_16(K_pages) || !on_16(V_pages)) return CCD_EALIGN;
  Rotary R{};
  if (rope != nullptr) {
    R = make_rotary(rope);
    R.d = paged->d;
  }
  launch_paged_append(make_paged(paged), paged->dtype, rope != nullptr ? &R : nullptr, K_new, V_new, slots, positions, turns, K_pages, V_pages,
                      static_cast<hipStream_t>(hip_stream));
  return paged_status();
}

size_t ccd_paged_workspace_bytes(const ccd_paged_t* paged) {
  if (check_paged(paged, kCache | kAttend) != CCD_OK) return 0;
  const Paged P = make_paged(paged);
  return attend_workspace_bytes(P, paged->dtype, hint_new(paged), hint_len(paged, P));
}

int ccd_paged_attend(const ccd_paged_t* paged, const void* Q, const void* K_pages, const void* V_pages, const int32_t* block_table,
                     const int32_t* q_start, const int32_t* kv_len, void* out, float* lse, void* workspace, size_t workspace_bytes,
                     void* hip_stream) {
  const int rc = check_paged(paged, kCache | kAttend);
  if (rc != CCD_OK) return rc;
  if (paged->tokens == 0) return CCD_OK;
  if (Q == nullptr || K_pages == nullptr || V_pages == nullptr || block_table == nullptr || q_start == nullptr || kv_len == nullptr || out == nullptr)
    return CCD_EINVAL;
  if (out == Q || out == K_pages || out == V_pages) return CCD_EINVAL;
  if (!on_16(Q) || !on_16(K_pages) || !on_16(V_pages) || !on_16(out)) return CCD_EALIGN;
  const Paged P = make_paged(paged);
  const int max_new = hint_new(paged), max_len = hint_len(paged, P);
  if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 ||
      workspace_bytes < attend_workspace_bytes(P, paged->dtype, max_new, max_len))
    return CCD_EWORKSPACE;
  launch_attend(P, paged->dtype, max_new, max_len, Q, K_pages, V_pages, block_table, q_start, kv_len, out, lse, workspace,
                static_cast<hipStream_t>(hip_stream));
  return paged_status();
}

}  // extern "C"
