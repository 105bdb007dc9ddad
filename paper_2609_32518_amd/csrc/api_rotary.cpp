// C ABI of the rotary options and the quantised cache (declared in include/unstep.h): tables with a split
// and a scaling of the caller's, the append in either layout, and the append, attention and read-back of
// a cache of e4m3 rows.  As everywhere, a call checks its arguments and the cache state before it
// enqueues anything, and nothing here reads device memory or synchronises.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <limits>

#include "kernels.hpp"
#include "plan.hpp"
#include "status.hpp"
#include "unstep.h"

namespace {

using unstep::aligned16;
using unstep::AppendPlan;
using unstep::fail;
using unstep::need_kind;
using unstep::ok;

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int check_rotary(const unstep_rotary* r, const char* where) {
  if (!r) return fail(UNSTEP_E_NULL, "%s: rotary is NULL", where);
  const int64_t rot = int64_t(r->dim_t) + r->dim_h + r->dim_w;
  if (r->dim_t < 0 || r->dim_h < 0 || r->dim_w < 0 || r->dim_t % 2 || r->dim_h % 2 || r->dim_w % 2 || rot < 16 ||
      rot > UNSTEP_HEAD_DIM || rot % 16)
    return fail(UNSTEP_E_SHAPE, "%s: dims (%d, %d, %d) must be even, with a sum that is a multiple of 16 up to 128", where,
                r->dim_t, r->dim_h, r->dim_w);
  if (!(r->theta > 1.0) || !std::isfinite(r->theta)) return fail(UNSTEP_E_RANGE, "%s: theta must be > 1", where);
  if (r->scaling < UNSTEP_ROTARY_UNSCALED || r->scaling > UNSTEP_ROTARY_PARTS)
    return fail(UNSTEP_E_RANGE, "%s: unknown scaling %d", where, r->scaling);
  if (!(r->amplitude >= 0.0) || !std::isfinite(r->amplitude))
    return fail(UNSTEP_E_RANGE, "%s: amplitude must be finite and >= 0 (0: the scaling's own)", where);
  if (r->scaling == UNSTEP_ROTARY_UNSCALED) return UNSTEP_OK;
  if (!(r->factor >= 1.0) || !std::isfinite(r->factor)) return fail(UNSTEP_E_RANGE, "%s: factor must be >= 1", where);
  if (r->scaling == UNSTEP_ROTARY_PARTS &&
      (!(r->trained_frames > 0.0) || !std::isfinite(r->trained_frames) || !(r->turns_slow >= 0.0) ||
       !(r->turns_fast > r->turns_slow) || !std::isfinite(r->turns_fast)))
    return fail(UNSTEP_E_RANGE, "%s: trained_frames must be > 0 and turns_fast > turns_slow >= 0", where);
  return UNSTEP_OK;
}

// Angle per position of every pair, and the tables' amplitude.  w_k = theta^(-2k/d) is a chain of extended
// products (64 fraction bits; the 63rd is within 2^-56 before its rounding to binary64): one power an axis, where one
// a pair took 1.6 of a small call's 5.9 us.
void frequencies(const unstep_rotary& r, unstep::RotaryTableArgs* a) {
  static_assert(std::numeric_limits<long double>::digits >= 64, "the chain needs guard bits");
  const int32_t dims[3] = {r.dim_t, r.dim_h, r.dim_w};
  double* w = a->freq;
  for (int axis = 0; axis < 3; ++axis) {
    const int32_t d = dims[axis];
    if (d == 0) continue;
    long double theta = r.theta;
    if (axis == 0 && r.scaling == UNSTEP_ROTARY_BASE && d > 2) theta *= std::pow((long double)r.factor, (long double)d / (d - 2));
    const long double ratio = std::pow(theta, -2.0L / d);
    long double x = 1.0L;
    for (int32_t k = 0; k < d / 2; ++k, x *= ratio) {
      double f = double(x);
      if (axis == 0 && r.scaling == UNSTEP_ROTARY_LINEAR) f /= r.factor;
      if (axis == 0 && r.scaling == UNSTEP_ROTARY_PARTS) {
        const double turns = r.trained_frames * f / (2.0 * M_PI);
        const double keep = std::min(1.0, std::max(0.0, (turns - r.turns_slow) / (r.turns_fast - r.turns_slow)));
        f *= keep + (1.0 - keep) / r.factor;
      }
      *w++ = f;
    }
  }
  a->amplitude = r.amplitude > 0.0 ? r.amplitude
                 : r.scaling == UNSTEP_ROTARY_PARTS ? 0.1 * std::log(r.factor) + 1.0
                                                    : 1.0;
}

// The options of a rotating append, on top of plan_append's checks.
int plan_rotary(const unstep_cache* c, int32_t layout, int32_t rot, bool with_q, const void* wq, const void* wk, double eps,
                AppendPlan* p, unstep::RotaryAppendArgs* r, const char* where) {
  if (layout != UNSTEP_ROTARY_INTERLEAVED && layout != UNSTEP_ROTARY_HALF)
    return fail(UNSTEP_E_RANGE, "%s: unknown layout %d", where, layout);
  if (rot < 16 || rot > UNSTEP_HEAD_DIM || rot % 16)
    return fail(UNSTEP_E_SHAPE, "%s: rot_dim %d must be a multiple of 16 up to 128", where, rot);
  if (p->args.tok_stride > UINT32_MAX || p->args.head_stride > UINT32_MAX)
    return fail(UNSTEP_E_SHAPE, "%s: strides above 2^32 elements", where);
  // the pass numbers the 16-byte pieces of one batch's chunk in 32 bits
  if (int64_t(p->args.C) * p->args.T * c->H * (UNSTEP_HEAD_DIM / 8) > INT32_MAX)
    return fail(UNSTEP_E_SHAPE, "%s: too many tokens x heads in one chunk", where);
  if (wk || wq) {
    if (!wk || (with_q && !wq))
      return fail(UNSTEP_E_NULL, "%s: k_norm_weight (and q_norm_weight when q is given) is NULL", where);
    if (c->H > unstep::kNormMaxHeads)
      return fail(UNSTEP_E_SHAPE, "%s: %d heads; the normalising pass handles at most %d", where, c->H, unstep::kNormMaxHeads);
    if (!(eps >= 0.0) || !std::isfinite(eps)) return fail(UNSTEP_E_RANGE, "%s: norm_eps must be finite and >= 0", where);
    if (!aligned16(wk) || (with_q && !aligned16(wq))) return fail(UNSTEP_E_ALIGN, "%s: norm weights must be 16-byte aligned", where);
    p->args.wq = with_q ? static_cast<const uint16_t*>(wq) : nullptr;
    p->args.wk = static_cast<const uint16_t*>(wk);
    p->args.eps = eps;
  }
  *r = unstep::RotaryAppendArgs{};
  r->a = p->args;
  r->half = layout == UNSTEP_ROTARY_HALF;
  r->rot = rot;
  return UNSTEP_OK;
}

int plan_append_mx8(const unstep_cache* c, int32_t f0, int32_t C, const void* q, const void* k, const void* v, int64_t ts,
                    int64_t hs, const float* cos_t, const float* sin_t, int32_t layout, int32_t rot, const void* wq,
                    const void* wk, double eps, float scale, void* q8, void* q_scale, unstep::RotaryAppendArgs* r,
                    const char* where) {
  AppendPlan p;
  if (int rc = need_kind(c, true, where)) return rc;
  if (q && (!q8 || !q_scale)) return fail(UNSTEP_E_NULL, "%s: q given but q8 or q_scale is NULL", where);
  if (int rc = unstep::plan_append(c, f0, C, q, k, v, ts, hs, cos_t, sin_t, q8, &p, where)) return rc;
  if (q && !aligned4(q_scale)) return fail(UNSTEP_E_ALIGN, "%s: q_scale must be 4-byte aligned", where);
  if (!std::isfinite(scale)) return fail(UNSTEP_E_RANGE, "%s: softmax_scale must be finite", where);
  if (int rc = plan_rotary(c, layout, rot, q != nullptr, wq, wk, eps, &p, r, where)) return rc;
  r->a.q_rot = r->a.k_cache = r->a.v_cache = nullptr;
  r->q8 = q ? static_cast<uint8_t*>(q8) : nullptr;
  r->q_scale = q ? static_cast<uint8_t*>(q_scale) : nullptr;
  r->k8 = static_cast<uint8_t*>(c->k);
  r->v8 = static_cast<uint8_t*>(c->v);
  r->k_scale = c->k_scale;
  r->v_scale = c->v_scale;
  const double s = scale > 0.f ? double(scale) : 1.0 / std::sqrt(double(UNSTEP_HEAD_DIM));
  r->q_mul = float(s * 1.4426950408889634);
  return UNSTEP_OK;
}

int plan_attn_mx8(const unstep_cache* c, int32_t newest, int32_t f0, int32_t C, int32_t W, const void* q8, const void* q_scale,
                  void* out, float* lse, void* workspace, size_t ws_bytes, unstep::Mx8AttnArgs* m, const char* where) {
  if (int rc = need_kind(c, true, where)) return rc;
  if (!q_scale) return fail(UNSTEP_E_NULL, "%s: q_scale is NULL", where);
  if (int rc = unstep::plan_attn(c, newest, f0, C, W, q8, out, lse, 0.f, workspace, ws_bytes, &m->a, where)) return rc;
  if (!aligned4(q_scale)) return fail(UNSTEP_E_ALIGN, "%s: q_scale must be 4-byte aligned", where);
  m->a.q = m->a.k_cache = m->a.v_cache = nullptr;
  m->a.scale = 0.69314718f;                                // scores are exponents of two
  m->q8 = static_cast<const uint8_t*>(q8);
  m->q_scale = static_cast<const uint8_t*>(q_scale);
  m->k8 = static_cast<const uint8_t*>(c->k);
  m->v8 = static_cast<const uint8_t*>(c->v);
  m->k_scale = c->k_scale;
  m->v_scale = c->v_scale;
  return UNSTEP_OK;
}

}  // namespace

extern "C" {

int unstep_rotary_tables(int32_t start_frame, int32_t n_frames, int32_t grid_h, int32_t grid_w, const unstep_rotary* rotary,
                         float* cos_out, float* sin_out, void* hip_stream) {
  return unstep::guarded("unstep_rotary_tables", [&]() -> int {
    const char* where = "unstep_rotary_tables";
    if (!cos_out || !sin_out) return fail(UNSTEP_E_NULL, "%s: cos_out/sin_out is NULL", where);
    if (int rc = check_rotary(rotary, where)) return rc;
    if (n_frames < 1 || grid_h < 1 || grid_w < 1)
      return fail(UNSTEP_E_SHAPE, "%s: n_frames, grid_h, grid_w must be >= 1", where);
    // one 256-thread work-group holds at least one token: the launch's work-items must fit 32 bits
    if (int64_t(n_frames) * grid_h > (int64_t(1) << 23) || int64_t(n_frames) * grid_h * grid_w > (int64_t(1) << 23))
      return fail(UNSTEP_E_SHAPE, "%s: table too large (more than 2^23 tokens)", where);
    if (start_frame < 0 || int64_t(start_frame) + n_frames > INT32_MAX) return fail(UNSTEP_E_RANGE, "%s: bad start_frame", where);
    if (!aligned16(cos_out) || !aligned16(sin_out)) return fail(UNSTEP_E_ALIGN, "%s: pointers must be 16-byte aligned", where);
    unstep::RotaryTableArgs a{};
    frequencies(*rotary, &a);
    a.cos_t = cos_out;
    a.sin_t = sin_out;
    a.f0 = start_frame;
    a.frames = n_frames;
    a.grid_h = grid_h;
    a.grid_w = grid_w;
    a.pairs_t = rotary->dim_t / 2;
    a.pairs_h = rotary->dim_h / 2;
    a.pairs_w = rotary->dim_w / 2;
    const hipError_t e = unstep::launch_rotary_tables(a, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return fail(UNSTEP_E_HIP, "%s: %s", where, hipGetErrorString(e));
    return ok();
  });
}

int unstep_kv_append_rotary(unstep_cache* c, int32_t start_frame, int32_t n_frames, const void* q, const void* k, const void* v,
                            int64_t tok_stride, int64_t head_stride, const float* cos_t, const float* sin_t, int32_t layout,
                            int32_t rot_dim, const void* q_norm_weight, const void* k_norm_weight, double norm_eps,
                            void* q_rot, void* hip_stream) {
  return unstep::guarded("unstep_kv_append_rotary", [&]() -> int {
    const char* where = "unstep_kv_append_rotary";
    if (int rc = need_kind(c, false, where)) return rc;
    AppendPlan p;
    if (int rc = unstep::plan_append(c, start_frame, n_frames, q, k, v, tok_stride, head_stride, cos_t, sin_t, q_rot, &p, where))
      return rc;
    unstep::RotaryAppendArgs r;
    if (int rc = plan_rotary(c, layout, rot_dim, q != nullptr, q_norm_weight, k_norm_weight, norm_eps, &p, &r, where)) return rc;
    const hipError_t e = unstep::launch_rotary_append(r, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return fail(UNSTEP_E_HIP, "%s: %s", where, hipGetErrorString(e));
    c->idx.commit_append(start_frame, n_frames);
    return ok();
  });
}

int unstep_cache_create_mx8(unstep_cache** out, int32_t batch, int32_t n_heads, int32_t head_dim, int32_t grid_h, int32_t grid_w,
                            int32_t sink_frames, int32_t ring_frames, void* k8, void* k_scale, void* v8, void* v_scale) {
  return unstep::guarded("unstep_cache_create_mx8", [&]() -> int {
    if (!k_scale || !v_scale) return fail(UNSTEP_E_NULL, "unstep_cache_create_mx8: NULL argument");
    if (!aligned16(k_scale) || !aligned16(v_scale))
      return fail(UNSTEP_E_ALIGN, "unstep_cache_create_mx8: cache buffers must be 16-byte aligned");
    if (int rc = unstep_cache_create(out, batch, n_heads, head_dim, grid_h, grid_w, sink_frames, ring_frames, k8, v8)) return rc;
    (*out)->k_scale = static_cast<uint8_t*>(k_scale);
    (*out)->v_scale = static_cast<uint8_t*>(v_scale);
    return ok();
  });
}

int unstep_kv_append_mx8(unstep_cache* c, int32_t start_frame, int32_t n_frames, const void* q, const void* k, const void* v,
                         int64_t tok_stride, int64_t head_stride, const float* cos_t, const float* sin_t, int32_t layout,
                         int32_t rot_dim, const void* q_norm_weight, const void* k_norm_weight, double norm_eps,
                         float softmax_scale, void* q8, void* q_scale, void* hip_stream) {
  return unstep::guarded("unstep_kv_append_mx8", [&]() -> int {
    const char* where = "unstep_kv_append_mx8";
    unstep::RotaryAppendArgs r;
    if (int rc = plan_append_mx8(c, start_frame, n_frames, q, k, v, tok_stride, head_stride, cos_t, sin_t, layout, rot_dim,
                                 q_norm_weight, k_norm_weight, norm_eps, softmax_scale, q8, q_scale, &r, where))
      return rc;
    const hipError_t e = unstep::launch_rotary_append(r, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return fail(UNSTEP_E_HIP, "%s: %s", where, hipGetErrorString(e));
    c->idx.commit_append(start_frame, n_frames);
    return ok();
  });
}

int unstep_window_attn_mx8(const unstep_cache* c, int32_t start_frame, int32_t n_frames, int32_t window_frames, const void* q8,
                           const void* q_scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                           void* hip_stream) {
  return unstep::guarded("unstep_window_attn_mx8", [&]() -> int {
    const char* where = "unstep_window_attn_mx8";
    if (!c) return fail(UNSTEP_E_NULL, "%s: cache handle is NULL", where);
    unstep::Mx8AttnArgs m;
    if (int rc = plan_attn_mx8(c, c->idx.newest(), start_frame, n_frames, window_frames, q8, q_scale, out, lse, workspace,
                               workspace_bytes, &m, where))
      return rc;
    const hipError_t e = unstep::launch_mx8_attn(m, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return fail(UNSTEP_E_HIP, "%s: %s", where, hipGetErrorString(e));
    return ok();
  });
}

int unstep_step_mx8(unstep_cache* c, int32_t start_frame, int32_t n_frames, int32_t window_frames, const void* q, const void* k,
                    const void* v, int64_t tok_stride, int64_t head_stride, const float* cos_t, const float* sin_t,
                    int32_t layout, int32_t rot_dim, const void* q_norm_weight, const void* k_norm_weight, double norm_eps,
                    float softmax_scale, void* q8, void* q_scale, void* out, float* lse, void* workspace,
                    size_t workspace_bytes, void* hip_stream) {
  return unstep::guarded("unstep_step_mx8", [&]() -> int {
    const char* where = "unstep_step_mx8";
    if (!q) return fail(UNSTEP_E_NULL, "%s: q is NULL", where);
    unstep::RotaryAppendArgs r;
    if (int rc = plan_append_mx8(c, start_frame, n_frames, q, k, v, tok_stride, head_stride, cos_t, sin_t, layout, rot_dim,
                                 q_norm_weight, k_norm_weight, norm_eps, softmax_scale, q8, q_scale, &r, where))
      return rc;
    unstep::Mx8AttnArgs m;
    const int32_t newest = std::max(c->idx.newest(), start_frame + n_frames - 1);
    if (int rc = plan_attn_mx8(c, newest, start_frame, n_frames, window_frames, q8, q_scale, out, lse, workspace,
                               workspace_bytes, &m, where))
      return rc;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipError_t e = unstep::launch_rotary_append(r, st);
    if (e != hipSuccess) return fail(UNSTEP_E_HIP, "%s (append): %s", where, hipGetErrorString(e));
    c->idx.commit_append(start_frame, n_frames);
    e = unstep::launch_mx8_attn(m, st);
    if (e != hipSuccess) return fail(UNSTEP_E_HIP, "%s (attention): %s", where, hipGetErrorString(e));
    return ok();
  });
}

int unstep_kv_read_mx8(const unstep_cache* c, int32_t start_frame, int32_t n_frames, void* k_out, void* v_out, void* hip_stream) {
  return unstep::guarded("unstep_kv_read_mx8", [&]() -> int {
    const char* where = "unstep_kv_read_mx8";
    if (int rc = need_kind(c, true, where)) return rc;
    if (!k_out || !v_out) return fail(UNSTEP_E_NULL, "%s: k_out or v_out is NULL", where);
    if (n_frames < 1) return fail(UNSTEP_E_SHAPE, "%s: empty chunk (n_frames < 1)", where);
    if (start_frame < 0 || int64_t(start_frame) + n_frames > INT32_MAX) return fail(UNSTEP_E_RANGE, "%s: bad start_frame", where);
    const int32_t end = start_frame + n_frames, missing = c->idx.first_missing(start_frame, end, c->idx.newest());
    if (missing != end) return fail(UNSTEP_E_STATE, "%s: frame %d is not in the cache", where, missing);
    const int64_t rows = int64_t(c->B) * c->H * n_frames * c->idx.T();
    if (rows > (int64_t(1) << 27)) return fail(UNSTEP_E_SHAPE, "%s: more than 2^27 rows", where);
    if (!aligned16(k_out) || !aligned16(v_out)) return fail(UNSTEP_E_ALIGN, "%s: pointers must be 16-byte aligned", where);
    unstep::Mx8ReadArgs a{};
    a.x8 = static_cast<const uint8_t*>(c->k);
    a.x_scale = c->k_scale;
    a.out = static_cast<uint16_t*>(k_out);
    a.y8 = static_cast<const uint8_t*>(c->v);
    a.y_scale = c->v_scale;
    a.y_out = static_cast<uint16_t*>(v_out);
    a.rows = rows;
    a.B = c->B;
    a.H = c->H;
    a.T = c->idx.T();
    a.C = n_frames;
    a.slots = c->slots;
    a.f0 = start_frame;
    a.S = c->idx.S();
    a.R = c->idx.R();
    const hipError_t e = unstep::launch_mx8_read(a, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return fail(UNSTEP_E_HIP, "%s: %s", where, hipGetErrorString(e));
    return ok();
  });
}

int unstep_mx8_dequantize(const void* x8, const void* scale, void* out, int64_t rows, void* hip_stream) {
  return unstep::guarded("unstep_mx8_dequantize", [&]() -> int {
    const char* where = "unstep_mx8_dequantize";
    if (!x8 || !scale || !out) return fail(UNSTEP_E_NULL, "%s: NULL tensor", where);
    if (rows < 0 || rows > (int64_t(1) << 27)) return fail(UNSTEP_E_SHAPE, "%s: rows must lie in [0, 2^27]", where);
    if (!aligned16(x8) || !aligned16(out)) return fail(UNSTEP_E_ALIGN, "%s: pointers must be 16-byte aligned", where);
    if (rows == 0) return ok();
    unstep::Mx8ReadArgs a{};
    a.x8 = static_cast<const uint8_t*>(x8);
    a.x_scale = static_cast<const uint8_t*>(scale);
    a.out = static_cast<uint16_t*>(out);
    a.rows = rows;
    const hipError_t e = unstep::launch_mx8_read(a, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return fail(UNSTEP_E_HIP, "%s: %s", where, hipGetErrorString(e));
    return ok();
  });
}

}  // extern "C"
