// Attention of a chunk's quantised queries over the retained rows of a quantised cache (mx8.hpp's format):
// out = sum_m w_m v_m / sum_m w_m, w_m = 2^(q k_m), q holding the softmax scale times log2 e.
//
// QK is v_mfma_scale_f32_32x32x64_f8f6f4 on the bytes as they are, at twice the bf16 rate: keys on the
// M side, the wave's 32 queries on N.  Of the 64 dimensions of one such product, two blocks of 32, lane l
// holds bytes 16 (l / 32) .. + 15 of each block of its row, and the scale of block l / 32.  The
// instruction adds the 16 products of such a group after cutting each below 2^-13 of the largest
// (measured), so a score is off by about 2^-14 of its largest product: for normalised queries and
// keys (products below 16, mostly below 1) less than the probabilities' rounding.  PV is v_mfma_f32_32x32x16_bf16: the probabilities, at most 1 and rounded to
// bf16 (a relative 2^-9 each, averaged over the keys), times the values, which a tile's load turns into
// bf16 exactly.  Sums, maxima and accumulators are fp32.
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
constexpr int kBlockK = kAttnBlockK;
constexpr int kBlockQ = kAttnBlockQ;
constexpr int kRow8 = kHeadDim;               // bytes of a quantised row
constexpr int kRow16 = kHeadDim * 2;          // bytes of a bf16 row
constexpr int kXcds = 8;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4_t;

__device__ __forceinline__ int swz16(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }
__device__ __forceinline__ int swz8(int row) { return (row >> 1) & 7; }

__device__ __forceinline__ u32x2_t lds_read_tr(const uint8_t* p) {
  const i16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(p));
  return __builtin_bit_cast(u32x2_t, v);
}

// 16 e4m3 values times one power of two, in bf16
__device__ __forceinline__ void to_bf16(u32x4_t x, float s, u32x4_t (&o)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], s, false);
    const bf16x2_t hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], s, true);
    o[i >> 1][2 * (i & 1)] = __builtin_bit_cast(uint32_t, lo);
    o[i >> 1][2 * (i & 1) + 1] = __builtin_bit_cast(uint32_t, hi);
  }
}

__device__ __forceinline__ i32x8_t join(u32x4_t a, u32x4_t b) {
  return i32x8_t{int(a.x), int(a.y), int(a.z), int(a.w), int(b.x), int(b.y), int(b.z), int(b.w)};
}

__global__ __launch_bounds__(kThreads) void mx8_attn_kernel(Mx8AttnArgs m) {
  __shared__ __attribute__((aligned(1024))) uint8_t kt[kBlockK * kRow8];
  __shared__ __attribute__((aligned(1024))) uint8_t vt[kBlockK * kRow16];
  __shared__ uint32_t ks[kBlockK];
  const AttnArgs& a = m.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, col = lane & 31;
  const int32_t N = a.N, H = a.H, G = gridDim.x;
  const int32_t xcd = blockIdx.x % kXcds;
  const int32_t g = xcd * (G / kXcds) + min(xcd, G % kXcds) + blockIdx.x / kXcds;
  int32_t qtiles;
  const Schedule sc = make_schedule(a, &qtiles);
  SegTable seg{a.seg_l0[1], a.seg_l0[2], a.seg_l0[3], a.seg_row0[0], a.seg_row0[1], a.seg_row0[2], a.seg_row0[3]};

  const int64_t u_begin = sc.start(g);
  int64_t u_hi = sc.start(int64_t(g) + 1);
  do {
    const Segment sg = take_segment(sc, u_begin, u_hi);
    const int32_t t = int32_t(sg.t), qt = t % qtiles, bh = t / qtiles, h = bh % H, b = bh / H;
    const int64_t row0 = int64_t(bh) * a.slots;
    const int32_t k_begin = sg.k0 * kBlockK, k_end = min(a.n_keys, sg.k1 * kBlockK);
    const int32_t r = wave * 32 + col, qi = qt * kBlockQ + r;
    i32x8_t qf[2];
    uint32_t qs;
    {
      const int64_t qrow = (int64_t(b) * N + min(qi, N - 1)) * H + h;
      const u32x4_t* qp = reinterpret_cast<const u32x4_t*>(m.q8 + qrow * kRow8 + 16 * half);
      qf[0] = join(qp[0], qp[2]);
      qf[1] = join(qp[4], qp[6]);
      qs = *reinterpret_cast<const uint32_t*>(m.q_scale + qrow * kMxBlocks) >> (8 * half);
    }
    f32x16_t o[4] = {};
    float l = 0.f, mx = -INFINITY;
    for (int32_t k0 = k_begin; k0 < k_end; k0 += kBlockK) {
      __syncthreads();
      {
        const int tr = tid >> 3, ts = tid & 7;
        const int64_t row = row0 + seg.row(min(k0 + tr, k_end - 1));
        const u32x4_t kx = *reinterpret_cast<const u32x4_t*>(m.k8 + row * kRow8 + 16 * ts);
        const u32x4_t vx = *reinterpret_cast<const u32x4_t*>(m.v8 + row * kRow8 + 16 * ts);
        u32x4_t vb[2];
        to_bf16(vx, mx8_scale(m.v_scale[row * kMxBlocks + (ts >> 1)]), vb);
        *reinterpret_cast<u32x4_t*>(kt + tr * kRow8 + ((ts ^ swz8(tr)) * 16)) = kx;
#pragma unroll
        for (int i = 0; i < 2; ++i)
          *reinterpret_cast<u32x4_t*>(vt + tr * kRow16 + (((2 * ts + i) ^ swz16(tr)) * 16)) = vb[i];
        if (ts == 0) ks[tr] = *reinterpret_cast<const uint32_t*>(m.k_scale + row * kMxBlocks);
      }
      __syncthreads();
      f32x16_t s[2] = {};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int row = 32 * kb + col;
        const uint32_t sc8 = ks[row] >> (8 * half);
        const u32x4_t* base = reinterpret_cast<const u32x4_t*>(kt + row * kRow8);
        const int x = swz8(row);
        const i32x8_t f0 = join(base[half ^ x], base[(2 + half) ^ x]);
        const i32x8_t f1 = join(base[(4 + half) ^ x], base[(6 + half) ^ x]);
        s[kb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f0, qf[0], s[kb], 0, 0, 0, int(sc8), 0, int(qs));
        s[kb] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f1, qf[1], s[kb], 0, 0, 2, int(sc8), 2, int(qs));
      }
      float top = mx;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (k0 + 32 * kb + 8 * (i >> 2) + 4 * half + (i & 3) >= k_end) s[kb][i] = -INFINITY;
          top = fmaxf(top, s[kb][i]);
        }
      top = fmaxf(top, __shfl_xor(top, 32));
      const float shrink = __builtin_amdgcn_exp2f(mx - top);
      mx = top;
      l *= shrink;
      bf16x8_t p[2][2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float e = __builtin_amdgcn_exp2f(s[kb][i] - top);
          l += e;
          p[kb][i >> 3][i & 7] = (__bf16)e;
        }
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] *= shrink;
      const int e = (lane & 15) >> 2, q = lane & 3, g16 = lane >> 4;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            u32x2_t f[2];
#pragma unroll
            for (int up = 0; up < 2; ++up) {
              const int row = 32 * kb + 16 * st + 8 * up + 4 * half + e;
              const int piece = 4 * d + 2 * (g16 & 1) + (q >> 1);
              f[up] = lds_read_tr(vt + row * kRow16 + (piece ^ swz16(row)) * 16 + (q & 1) * 8);
            }
            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                __builtin_bit_cast(bf16x8_t, u32x4_t{f[0].x, f[0].y, f[1].x, f[1].y}), p[kb][st], o[d], 0, 0, 0);
          }
    }
    const float l_tot = l + __shfl_xor(l, 32);
    if (qi < N) {
      if (sg.full) {
        const float inv = 1.f / l_tot;
        uint16_t* op = a.out + ((int64_t(b) * N + qi) * H + h) * kHeadDim + 4 * half;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int gg = 0; gg < 4; ++gg) {
            bf16x4_t rr;
#pragma unroll
            for (int e = 0; e < 4; ++e) rr[e] = (__bf16)(o[d][4 * gg + e] * inv);
            *reinterpret_cast<bf16x4_t*>(op + d * 32 + 8 * gg) = rr;
          }
        if (a.lse && half == 0) a.lse[(int64_t(b) * H + h) * N + qi] = mx * a.scale + logf(l_tot);
      } else {
        const int64_t prow = (int64_t(g) * 2 + sg.slot) * kBlockQ + r;
        const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
        float* op = a.part_o + prow * kHeadDim + 4 * half;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int gg = 0; gg < 4; ++gg)
            *reinterpret_cast<float4*>(op + d * 32 + 8 * gg) =
                make_float4(o[d][4 * gg] * inv, o[d][4 * gg + 1] * inv, o[d][4 * gg + 2] * inv, o[d][4 * gg + 3] * inv);
        if (half == 0) {
          a.part_ml[prow * 2] = l_tot > 0.f ? mx : -INFINITY;
          a.part_ml[prow * 2 + 1] = l_tot;
        }
      }
    }
  } while (u_hi > u_begin);
}

}  // namespace

hipError_t launch_mx8_attn(const Mx8AttnArgs& m, hipStream_t stream) {
  hipLaunchKernelGGL(mx8_attn_kernel, dim3(unsigned(m.a.groups)), dim3(kThreads), 0, stream, m);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? launch_attn_combine(m.a, stream) : e;
}

}  // namespace unstep
