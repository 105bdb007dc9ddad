// The cache handle, and the validation of an append and of an attention call against it: what every
// entry point checks before it enqueues anything.
#pragma once

#include <cmath>
#include <cstdint>
#include <string>

#include "cache_index.hpp"
#include "kernels.hpp"
#include "status.hpp"
#include "unstep.h"

// k, v: bf16 rows of 128 (256 bytes); with k_scale and v_scale, e4m3 rows (128 bytes) and their four
// scale bytes each.
struct unstep_cache {
  unstep::CacheIndex idx;
  int32_t B, H, D, grid_h, grid_w;
  int32_t slots;
  void* k;
  void* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  bool mx8() const { return k_scale != nullptr; }
};

namespace unstep {

// The entry points of one kind of cache refuse a handle of the other.
inline int need_kind(const unstep_cache* c, bool mx8, const char* where) {
  if (!c) return fail(UNSTEP_E_NULL, "%s: cache handle is NULL", where);
  if (c->mx8() == mx8) return UNSTEP_OK;
  return fail(UNSTEP_E_STATE, mx8 ? "%s: the cache holds bf16 rows" : "%s: the cache holds quantised rows", where);
}

struct AppendPlan {
  RopeAppendArgs args;
};

// Validation of an append.
inline int plan_append(const unstep_cache* c, int32_t f0, int32_t C, const void* q, const void* k, const void* v,
                       int64_t tok_stride, int64_t head_stride, const float* cos_t, const float* sin_t, void* q_rot,
                       AppendPlan* plan, const char* where) {
  if (!c) return fail(UNSTEP_E_NULL, "%s: cache handle is NULL", where);
  if (!k || !v || !cos_t || !sin_t) return fail(UNSTEP_E_NULL, "%s: k, v, cos_t or sin_t is NULL", where);
  if (q && !q_rot) return fail(UNSTEP_E_NULL, "%s: q given but q_rot is NULL", where);
  const CacheIndex& idx = c->idx;
  std::string why;
  int rc = idx.check_append(f0, C, &why);
  if (rc != UNSTEP_OK) return fail_msg(rc, where, why);
  if (head_stride < UNSTEP_HEAD_DIM || tok_stride < int64_t(c->H) * head_stride)
    return fail(UNSTEP_E_SHAPE, "%s: strides (tok %lld, head %lld) overlap for %d heads of 128", where,
                (long long)tok_stride, (long long)head_stride, c->H);
  if ((tok_stride % 8) || (head_stride % 8))
    return fail(UNSTEP_E_ALIGN, "%s: strides must be multiples of 8 elements", where);
  if (!aligned16(k) || !aligned16(v) || !aligned16(cos_t) || !aligned16(sin_t) || (q && !aligned16(q)) ||
      (q_rot && !aligned16(q_rot)))
    return fail(UNSTEP_E_ALIGN, "%s: pointers must be 16-byte aligned", where);
  RopeAppendArgs& a = plan->args;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.tok_stride = tok_stride;
  a.head_stride = head_stride;
  a.cos_t = cos_t;
  a.sin_t = sin_t;
  a.q_rot = q ? static_cast<uint16_t*>(q_rot) : nullptr;
  a.k_cache = static_cast<uint16_t*>(c->k);
  a.v_cache = static_cast<uint16_t*>(c->v);
  a.B = c->B;
  a.H = c->H;
  a.T = idx.T();
  a.C = C;
  a.slots = c->slots;
  a.f0 = f0;
  a.S = idx.S();
  a.R = idx.R();
  a.wq = nullptr;
  a.wk = nullptr;
  a.eps = 0.0;
  return UNSTEP_OK;
}

// Validation of an attention call with `newest` as the newest stored frame (which an append of the same
// call may reach).
inline int plan_attn(const unstep_cache* c, int32_t newest, int32_t f0, int32_t C, int32_t W, const void* q_rot,
                     void* out, float* lse, float scale, void* workspace, size_t ws_bytes, AttnArgs* a,
                     const char* where) {
  if (!c) return fail(UNSTEP_E_NULL, "%s: cache handle is NULL", where);
  if (!q_rot || !out) return fail(UNSTEP_E_NULL, "%s: q_rot or out is NULL", where);
  Segments logical;
  std::string why;
  int rc = c->idx.segments(f0, C, W, newest, &logical, &why);
  if (rc != UNSTEP_OK) return fail_msg(rc, where, why);
  const Segments seg = cache_order(logical);
  if (!aligned16(q_rot) || !aligned16(out) || (lse && (reinterpret_cast<uintptr_t>(lse) & 3u)) ||
      (workspace && !aligned16(workspace)))
    return fail(UNSTEP_E_ALIGN, "%s: pointers must be 16-byte aligned", where);
  const int32_t N = C * c->idx.T();
  // one 512-thread work-group per 256-query tile: the launch's work-item count must fit 32 bits
  if (int64_t(c->B) * c->H * ((int64_t(N) + 255) / 256) * 512 > int64_t(UINT32_MAX))
    return fail(UNSTEP_E_SHAPE, "%s: too many query tiles (batch x heads x chunk tokens / 256 >= 2^23)", where);
  a->q = static_cast<const uint16_t*>(q_rot);
  a->k_cache = static_cast<const uint16_t*>(c->k);
  a->v_cache = static_cast<const uint16_t*>(c->v);
  a->out = static_cast<uint16_t*>(out);
  a->lse = lse;
  a->B = c->B;
  a->N = N;
  a->H = c->H;
  a->slots = c->slots;
  a->n_keys = seg.total();
  a->n_seg = seg.n;
  int32_t l = 0;
  for (int i = 0; i < UNSTEP_MAX_SEGMENTS; ++i) {
    if (i < seg.n) {
      a->seg_l0[i] = l;
      a->seg_row0[i] = seg.row0[i];
      l += seg.len[i];
    } else {
      a->seg_l0[i] = INT32_MAX;
      a->seg_row0[i] = 0;
    }
  }
  a->seg_l0[UNSTEP_MAX_SEGMENTS] = INT32_MAX;
  a->scale = scale > 0.f ? scale : 1.0f / std::sqrt(float(UNSTEP_HEAD_DIM));
  const AttnPlan plan = (c->mx8() ? attn_plan_mx8 : attn_plan)(c->B, c->H, N, a->n_keys, workspace ? ws_bytes : 0);
  a->parts = 1;
  if (plan.workspace > 0) {
    a->groups = plan.groups;
    a->parts = plan.parts;
    a->part_o = static_cast<float*>(workspace);
    a->part_ml = static_cast<float*>(workspace) + plan.part_o_floats;
  } else {
    // one work-group per query tile over the whole key range: no scratch needed
    a->groups = plan.plain_groups;
    a->part_o = nullptr;
    a->part_ml = nullptr;
  }
  return UNSTEP_OK;
}

}  // namespace unstep
