// Attention of quantised queries, 16 per work-group, over the retained rows of a quantised cache: the call of a
// single-token stream, and of small chunks.  Bound by memory: 16 queries read every retained row once (264
// bytes of K and V) and cost the same as one; a short range by its chain of loads and products, 1.3-1.6 us per
// 256 keys.
//
// Work-group: 8 waves, each walking a slice of its own of the work-group's key range, 32 keys at a time.  No wave
// waits for another before the end.  Rows are loaded when they are needed: a step ahead they cost 55 registers and
// were 2-9% slower on every shape (12 heads x 1 query x 32768 keys 22.5 and 21.9 us, 24 x 160 x 960 12.4 and 11.5).
//   S^T = K Q^T with v_mfma_f32_16x16x32_bf16, keys on the M side: lane l holds 32 bytes of row l % 16, the block
//   l / 16, so a block's scale is a lane's; the bytes become bf16 exactly, and the products and sums have fp32
//   accuracy (unlike the 8-bit instruction's, whose cut shows where a call has few keys to average over).
//   O^T += V^T P^T with the same instruction: V rows become bf16 on their way to a wave's own 8 KB of LDS, from
//   which the transposing read takes 4 keys of a dimension at a time; the 8 contraction slots of a lane are
//   the keys whose scores it holds.
// Running maximum, rescaled when it grows.  At the end the waves' sums meet in LDS, in one order.
// One query, 12 heads x 32768 keys (104 MB): 18.5 us in 252 work-groups (5.6 TB/s) and the merge's 3-4.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "attn_schedule.hpp"
#include "kernels.hpp"
#include "mx8.hpp"
#include "seg_table.hpp"

namespace unstep {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr int kTile = 32;                      // keys per step of a wave
constexpr int kRow8 = kHeadDim, kRow16 = kHeadDim * 2;
constexpr int kXcds = 8;
constexpr int kMaxQ = kMx8FewQueries;
static_assert(kMaxQ == 16, "one MFMA column per query");

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4_t;

__device__ __forceinline__ int swz(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }

// 8 e4m3 values (two words) times a power of two
__device__ __forceinline__ u32x4_t to_bf16(uint32_t a, uint32_t b, float s) {
  const bf16x2_t v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, true)};
  return u32x4_t{__builtin_bit_cast(uint32_t, v[0]), __builtin_bit_cast(uint32_t, v[1]), __builtin_bit_cast(uint32_t, v[2]),
                 __builtin_bit_cast(uint32_t, v[3])};
}

// Combines a value over the lanes l, l ^ 16, l ^ 32, l ^ 48 (those of one query).
template <class F>
__device__ __forceinline__ float over_groups(float x, F f) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// 32 keys as a lane loads them: 32 bytes of rows l % 16 and 16 + l % 16 of K, 16 bytes of rows 8 i + l / 8 of V.
struct Rows {
  u32x4_t k[2][2], v[4];
  uint32_t ks[2], vs[4];
};

struct Source {
  const uint8_t *k8, *v8, *ks, *vs;
  SegTable seg;
  int32_t end;                                 // of the wave's slice
};

__device__ __forceinline__ void load(Rows& r, const Source& s, int32_t key0) {
  const int lane = threadIdx.x & 63, g = lane >> 4;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t row = uint32_t(s.seg.row(min(key0 + 16 * i + (lane & 15), s.end - 1)));
#pragma unroll
    for (int j = 0; j < 2; ++j)
      r.k[i][j] = *reinterpret_cast<const u32x4_t*>(s.k8 + (row * uint32_t(kRow8) + 32 * g + 16 * j));
    r.ks[i] = s.ks[row * uint32_t(kMxBlocks) + g];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t row = uint32_t(s.seg.row(min(key0 + 8 * i + (lane >> 3), s.end - 1)));
    r.v[i] = *reinterpret_cast<const u32x4_t*>(s.v8 + (row * uint32_t(kRow8) + 16 * (lane & 7)));
    r.vs[i] = s.vs[row * uint32_t(kMxBlocks) + ((lane & 7) >> 1)];
  }
}

struct State {
  f32x4_t o[8];                                // O^T: dims 16 d + 4 (l / 16) .. + 3 of query l % 16
  float m, l;                                  // running maximum of the query, this lane's part of its sum
};

__device__ __forceinline__ void step(State& a, const Rows& r, const u32x4_t (&q)[4], uint8_t* vt, int32_t key0, int32_t end) {
  const int lane = threadIdx.x & 63, g = lane >> 4;
  f32x4_t s[2] = {};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float sc = mx8_scale(r.ks[i]);
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      const u32x4_t w = r.k[i][st >> 1];
      const u32x4_t f = to_bf16(w[2 * (st & 1)], w[2 * (st & 1) + 1], sc);
      s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, f), __builtin_bit_cast(bf16x8_t, q[st]), s[i], 0, 0, 0);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 8 * i + (lane >> 3), piece = 2 * (lane & 7);
    const float sc = mx8_scale(r.vs[i]);
    *reinterpret_cast<u32x4_t*>(vt + row * kRow16 + ((piece ^ swz(row)) * 16)) = to_bf16(r.v[i][0], r.v[i][1], sc);
    *reinterpret_cast<u32x4_t*>(vt + row * kRow16 + (((piece + 1) ^ swz(row)) * 16)) = to_bf16(r.v[i][2], r.v[i][3], sc);
  }
  float top = a.m;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (key0 + 16 * i + 4 * g + e >= end) s[i][e] = -INFINITY;
      top = fmaxf(top, s[i][e]);
    }
  top = over_groups(top, [](float x, float y) { return fmaxf(x, y); });
  if (__any(top > a.m)) {
    const float shrink = __builtin_amdgcn_exp2f(a.m - top);
    a.l *= shrink;
#pragma unroll
    for (int d = 0; d < 8; ++d) a.o[d] *= shrink;
    a.m = top;
  }
  bf16x8_t p;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float e = __builtin_amdgcn_exp2f(s[i >> 2][i & 3] - a.m);
    a.l += e;
    p[i] = (__bf16)e;
  }
#pragma unroll
  for (int d = 0; d < 8; ++d) {
    u32x2_t f[2];
#pragma unroll
    for (int up = 0; up < 2; ++up) {
      const int row = 16 * up + 4 * g + ((lane & 15) >> 2), piece = 2 * d + ((lane & 3) >> 1);
      f[up] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                              (lds_i16x4_t*)(vt + row * kRow16 + ((piece ^ swz(row)) * 16) + 8 * (lane & 1))));
    }
    a.o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, u32x4_t{f[0].x, f[0].y, f[1].x, f[1].y}), p,
                                                     a.o[d], 0, 0, 0);
  }
}

__global__ __launch_bounds__(kThreads) void mx8_attn_few_kernel(Mx8AttnArgs m) {
  // the waves' V tiles, then their sums [wave][query][dim]
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kWaves * kTile * kRow16];
  __shared__ float part_m[kWaves][kMaxQ], part_l[kWaves][kMaxQ];
  static_assert(sizeof(lds) >= kWaves * kMaxQ * kHeadDim * sizeof(float), "the sums must fit the tiles");
  const AttnArgs& a = m.a;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t N = a.N, H = a.H, G = gridDim.x, tiles = (N + kMaxQ - 1) / kMaxQ;
  // as in the general kernel: an XCD's work-groups are consecutive, so that a head's query tiles share its L2
  const int32_t xcd = blockIdx.x % kXcds;
  const int32_t grp = xcd * (G / kXcds) + min(xcd, G % kXcds) + blockIdx.x / kXcds;
  const Segment sg = part_segment((a.n_keys + kAttnBlockK - 1) / kAttnBlockK, a.parts, grp);
  const int32_t bh = int32_t(sg.t) / tiles, q0 = (int32_t(sg.t) - bh * tiles) * kMaxQ, h = bh % H, b = bh / H;
  const int32_t here = min(N - q0, kMaxQ);                 // queries of this work-group
  const int64_t row0 = int64_t(bh) * a.slots;
  const int32_t k_begin = sg.k0 * kAttnBlockK, k_end = min(a.n_keys, sg.k1 * kAttnBlockK);
  const int32_t slice = ((k_end - k_begin + kWaves * kTile - 1) / (kWaves * kTile)) * kTile;
  const int32_t begin = k_begin + wave * slice;
  Source src{m.k8 + row0 * kRow8, m.v8 + row0 * kRow8, m.k_scale + row0 * kMxBlocks, m.v_scale + row0 * kMxBlocks,
             SegTable{a.seg_l0[1], a.seg_l0[2], a.seg_l0[3], a.seg_row0[0], a.seg_row0[1], a.seg_row0[2], a.seg_row0[3]},
             min(begin + slice, k_end)};
  State st;
  st.m = -FLT_MAX;                             // finite: scores of -infinity weigh nothing, also before any other
  st.l = 0.f;
#pragma unroll
  for (int d = 0; d < 8; ++d) st.o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (begin < src.end) {
    u32x4_t q[4];
    {
      const int64_t qrow = (int64_t(b) * N + min(q0 + (lane & 15), N - 1)) * H + h;
      const u32x4_t* qp = reinterpret_cast<const u32x4_t*>(m.q8 + qrow * kRow8 + 32 * g);
      const float sc = mx8_scale(m.q_scale[qrow * kMxBlocks + g]);
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = to_bf16(qp[i >> 1][2 * (i & 1)], qp[i >> 1][2 * (i & 1) + 1], sc);
    }
    uint8_t* const vt = lds + wave * kTile * kRow16;
    for (int32_t k = begin; k < src.end; k += kTile) {
      Rows r;
      load(r, src, k);
      step(st, r, q, vt, k, src.end);
    }
  }
  st.l = over_groups(st.l, [](float x, float y) { return x + y; });
  if (lane < kMaxQ) {
    part_m[wave][lane] = st.m;
    part_l[wave][lane] = st.l;
  }
  __syncthreads();                             // and every wave has finished with its V tile
  const int qi = lane & 15;
  float top = part_m[0][qi];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) top = fmaxf(top, part_m[w][qi]);
  const float f = __builtin_amdgcn_exp2f(st.m - top);
  float* const sums = reinterpret_cast<float*>(lds);
  if (qi < here) {
#pragma unroll
    for (int d = 0; d < 8; ++d)
      *reinterpret_cast<f32x4_t*>(sums + (wave * kMaxQ + qi) * kHeadDim + 16 * d + 4 * g) = st.o[d] * f;
  }
  __syncthreads();
  // a thread finishes four dimensions of a query
  for (int i = tid; i < here * (kHeadDim / 4); i += kThreads) {
    const int n = i / (kHeadDim / 4), d4 = i % (kHeadDim / 4);
    float mm = part_m[0][n], l = 0.f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mm = fmaxf(mm, part_m[w][n]);
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      l += part_l[w][n] * __builtin_amdgcn_exp2f(part_m[w][n] - mm);
      o += *reinterpret_cast<const f32x4_t*>(sums + (w * kMaxQ + n) * kHeadDim + 4 * d4);
    }
    o *= a.parts == 1 || l > 0.f ? 1.f / l : 0.f;         // a part may hold nothing but scores of -infinity
    if (a.parts == 1) {
      bf16x4_t v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (__bf16)o[e];
      *reinterpret_cast<bf16x4_t*>(a.out + ((int64_t(b) * N + q0 + n) * H + h) * kHeadDim + 4 * d4) = v;
      if (a.lse && d4 == 0) a.lse[(int64_t(b) * H + h) * N + q0 + n] = mm * a.scale + logf(l);
    } else {
      // the merge's layout: a work-group's partials per 256-query tile and part
      const int32_t tile = bh * ((N + kAttnBlockQ - 1) / kAttnBlockQ) + q0 / kAttnBlockQ;
      const int64_t prow = (int64_t(tile) * a.parts + (grp - int32_t(sg.t) * a.parts)) * 2 * kAttnBlockQ + q0 % kAttnBlockQ + n;
      *reinterpret_cast<f32x4_t*>(a.part_o + prow * kHeadDim + 4 * d4) = o;
      if (d4 == 0) {
        a.part_ml[prow * 2] = mm;
        a.part_ml[prow * 2 + 1] = l;
      }
    }
  }
}

}  // namespace

hipError_t launch_mx8_attn_few(const Mx8AttnArgs& m, hipStream_t stream) {
  hipLaunchKernelGGL(mx8_attn_few_kernel, dim3(unsigned(m.a.groups)), dim3(kThreads), 0, stream, m);
  return hipGetLastError();
}

}  // namespace unstep
