// Rotary embedding of a chunk's queries and keys in the interleaved or the half layout, over the whole
// head or its first `rot` dimensions, optionally after the RMS normalisation, and the write into a
// bf16 cache or a quantised one: one bandwidth-bound pass over q, k and v.
//
// Pair j < rot / 2 is (x_2j, x_2j+1) (interleaved) or (x_j, x_j+rot/2) (half); with the table entries c, s
// of its token, y_a = x_a c - x_b s and y_b = x_a s + x_b c, every product and sum a binary32 operation of
// its own (contraction is off).  Dimensions from rot on are left as they are.  The bf16 outputs are y
// rounded to nearest even; the quantised ones are y (the queries times q_mul, a binary32 product) in
// e4m3 blocks of 32 (mx8.hpp), rounded once from binary32.
//
// A thread owns one 16-byte piece (8 values) of a head vector; the 16 pieces of a vector sit in 16
// consecutive lanes, so the half layout's partner piece, rot / 2 values on or back, comes from another
// lane, a block's maximum is that of 4 neighbouring lanes and a row's four scale bytes are joined by two
// rotations within the 16.  Nothing but q, k, v, the tables and the outputs moves through memory.
#include <hip/hip_runtime.h>

#include "kernels.hpp"
#include "mx8.hpp"
#include "seg_table.hpp"

namespace unstep {
namespace {

constexpr int kThreads = 256;
constexpr int kPieces = kHeadDim / 8;   // pieces of a head vector, one lane each
// pieces per lane of the normalising kernel (a wave per token): 3 cover 12 heads, 8 cover kNormMaxHeads
constexpr int kNormPiecesSmall = 3;
constexpr int kNormPiecesLarge = kNormMaxHeads * kPieces / 64;

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

struct F8 {
  float v[8];
};

__device__ __forceinline__ F8 widen(u32x4_t x) {
  F8 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    y.v[2 * e] = bf16_lo(x[e]);
    y.v[2 * e + 1] = bf16_hi(x[e]);
  }
  return y;
}

// What a piece needs of its token's tables: 4 entries of cos and of sin (interleaved) or 8 (half).
template <bool kHalf>
struct Turn {
  f32x4_t c[kHalf ? 2 : 1], s[kHalf ? 2 : 1];
};

// The table entries of piece p; a piece that is not rotated reads entry 0 and does not use it.
template <bool kHalf>
__device__ __forceinline__ Turn<kHalf> load_turn(const RotaryAppendArgs& r, int64_t n, int32_t p) {
  const int32_t hp = r.rot >> 4;                          // pieces per half of the rotated part
  const int64_t at = n * (r.rot >> 1) + (p >= 2 * hp ? 0 : kHalf ? 8 * (p >= hp ? p - hp : p) : 4 * p);
  Turn<kHalf> t;
#pragma unroll
  for (int i = 0; i < (kHalf ? 2 : 1); ++i) {
    t.c[i] = *reinterpret_cast<const f32x4_t*>(r.a.cos_t + at + 4 * i);
    t.s[i] = *reinterpret_cast<const f32x4_t*>(r.a.sin_t + at + 4 * i);
  }
  return t;
}

// Piece p of a head vector, rotated.  The 16 lanes of the vector are in this together.
template <bool kHalf>
__device__ __forceinline__ F8 rotate(u32x4_t x, const Turn<kHalf>& t, const RotaryAppendArgs& r, int32_t p) {
#pragma clang fp contract(off)
  const int32_t hp = r.rot >> 4;
  const F8 own = widen(x);
  F8 y = own;
  if constexpr (kHalf) {
    const int lane = threadIdx.x & 63;
    const int from = p >= 2 * hp ? lane : p >= hp ? lane - hp : lane + hp;
    u32x4_t o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = uint32_t(__shfl(int(x[e]), from));
    const F8 other = widen(o);
    if (p < 2 * hp) {
      // first half: x_a c - x_b s, second: x_b c + x_a s (= x_a s + x_b c, addition commutes)
      const bool second = p >= hp;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float a = own.v[i] * t.c[i >> 2][i & 3];
        const float b = other.v[i] * t.s[i >> 2][i & 3];
        y.v[i] = second ? a + b : a - b;
      }
    }
  } else if (p < 2 * hp) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float xe = own.v[2 * e], xo = own.v[2 * e + 1], c = t.c[0][e], s = t.s[0][e];
      const float a = xe * c, b = xo * s, d = xe * s, g = xo * c;
      y.v[2 * e] = a - b;
      y.v[2 * e + 1] = d + g;
    }
  }
  return y;
}

__device__ __forceinline__ u32x4_t to_bf16(const F8& y) {
  u32x4_t o;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    bf16x2_t w;
    w[0] = (__bf16)y.v[2 * e];
    w[1] = (__bf16)y.v[2 * e + 1];
    o[e] = __builtin_bit_cast(uint32_t, w);
  }
  return o;
}

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(x), kCtrl, 0xf, 0xf, false));
}

// Stores piece p of the head vector at row `row`: eight e4m3 bytes, and (lane of piece 0) the row's
// scale bytes.  The 16 lanes of the vector are in this together.
__device__ __forceinline__ void store_mx8(const F8& y, uint8_t* x8, uint8_t* scale, int64_t row, int32_t p) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t m = __float_as_uint(y.v[i]) & 0x7fffffffu;
    top = max(top, m < 0x7f800000u ? m : 0u);
  }
  top = max(top, dpp<0xb1>(top));                         // quad_perm 1,0,3,2
  top = max(top, dpp<0x4e>(top));                         // quad_perm 2,3,0,1
  const int32_t byte = mx8_byte(top);
  const float inv = mx8_inverse(byte);
  float z[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t m = __float_as_uint(y.v[i]) & 0x7fffffffu;
    z[i] = m < 0x7f800000u ? y.v[i] * inv : __uint_as_float(0x7fc00000u);
  }
  u32x2_t w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int d = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * i], z[4 * i + 1], 0, false);
    d = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * i + 2], z[4 * i + 3], d, true);
    w[i] = uint32_t(d);
  }
  __builtin_nontemporal_store(w, reinterpret_cast<u32x2_t*>(x8 + row * kHeadDim + p * 8));
  uint32_t bytes = uint32_t(byte) << (8 * (p >> 2));
  bytes |= dpp<0x124>(bytes);                             // row_ror 4
  bytes |= dpp<0x128>(bytes);                             // row_ror 8
  if (p == 0) *reinterpret_cast<uint32_t*>(scale + row * kMxBlocks) = bytes;
}

// Places of token n of batch b, head h: row of the chunk's outputs, and of the cache.
struct Place {
  int64_t chunk_row, cache_row;
};
__device__ __forceinline__ Place place(const RopeAppendArgs& a, int32_t b, int32_t n, int32_t h) {
  const int32_t fi = n / a.T, t = n - fi * a.T;
  const int32_t slot = frame_slot(a.f0 + fi, a.S, a.R);
  return Place{(int64_t(b) * (int64_t(a.C) * a.T) + n) * a.H + h,
               (int64_t(b) * a.H + h) * a.slots + int64_t(slot) * a.T + t};
}

template <bool kHalf, bool kMx8, bool kQuery>
__device__ __forceinline__ void put_rotated(const RotaryAppendArgs& r, const F8& y, const Place& at, int32_t p) {
  if constexpr (kMx8) {
    if constexpr (kQuery) {
      F8 m;
#pragma unroll
      for (int i = 0; i < 8; ++i) m.v[i] = y.v[i] * r.q_mul;
      store_mx8(m, r.q8, r.q_scale, at.chunk_row, p);
    } else {
      store_mx8(y, r.k8, r.k_scale, at.cache_row, p);
    }
  } else {
    uint16_t* const o = kQuery ? r.a.q_rot + at.chunk_row * kHeadDim : r.a.k_cache + at.cache_row * kHeadDim;
    __builtin_nontemporal_store(to_bf16(y), reinterpret_cast<u32x4_t*>(o + p * 8));
  }
}

template <bool kMx8>
__device__ __forceinline__ void put_value(const RotaryAppendArgs& r, u32x4_t v, const Place& at, int32_t p) {
  if constexpr (kMx8)
    store_mx8(widen(v), r.v8, r.v_scale, at.cache_row, p);
  else
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(r.a.v_cache + at.cache_row * kHeadDim + p * 8));
}

template <bool kWithQ, bool kHalf, bool kMx8>
__global__ __launch_bounds__(kThreads) void rotary_append_kernel(RotaryAppendArgs r) {
  const RopeAppendArgs& a = r.a;
  const uint32_t u = blockIdx.x * kThreads + threadIdx.x;
  const uint32_t hv = u / kPieces;                        // (token, head) of the chunk
  if (hv >= uint32_t(a.C) * a.T * a.H) return;            // whole head vectors: 16 lanes each
  const int32_t p = u % kPieces;
  const int32_t n = hv / uint32_t(a.H), h = hv - uint32_t(n) * a.H;
  const int32_t b = blockIdx.y;
  const int64_t src = (int64_t(b) * (int64_t(a.C) * a.T) + n) * a.tok_stride + int64_t(h) * a.head_stride + p * 8;
  const u32x4_t kx = *reinterpret_cast<const u32x4_t*>(a.k + src);
  const u32x4_t vx = *reinterpret_cast<const u32x4_t*>(a.v + src);
  u32x4_t qx = {};
  if (kWithQ) qx = *reinterpret_cast<const u32x4_t*>(a.q + src);
  const Turn<kHalf> t = load_turn<kHalf>(r, n, p);
  const Place at = place(a, b, n, h);
  put_rotated<kHalf, kMx8, false>(r, rotate<kHalf>(kx, t, r, p), at, p);
  put_value<kMx8>(r, vx, at, p);
  if (kWithQ) put_rotated<kHalf, kMx8, true>(r, rotate<kHalf>(qx, t, r, p), at, p);
}

// ---- with the RMS normalisation: one wave per token, lane l owning the pieces l, l + 64, ... of its heads.
// x'_j = bf16(fp32((x_j rr) w_j)), rr = 1 / sqrt(sum x^2 / channels + eps) in fp64 (each bf16 square is exact).
template <int kPer>
__device__ __forceinline__ double sum_sq(const u32x4_t (&x)[kPer], int n) {
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (i >= n) break;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double lo = bf16_lo(x[i][e]), hi = bf16_hi(x[i][e]);
      s += lo * lo;
      s += hi * hi;
    }
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
  return s;
}

// The binary32 value is kept opaque to the optimiser, which would fold the two roundings into one.
__device__ __forceinline__ u32x4_t normalise8(u32x4_t x, u32x4_t w, double rr) {
  u32x4_t y;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float lo = (float)(((double)bf16_lo(x[e]) * rr) * (double)bf16_lo(w[e]));
    float hi = (float)(((double)bf16_hi(x[e]) * rr) * (double)bf16_hi(w[e]));
    asm volatile("" : "+v"(lo), "+v"(hi));
    bf16x2_t pr;
    pr[0] = (__bf16)lo;
    pr[1] = (__bf16)hi;
    y[e] = __builtin_bit_cast(uint32_t, pr);
  }
  return y;
}

template <bool kWithQ, bool kHalf, bool kMx8, int kPer>
__global__ __launch_bounds__(kThreads) void rotary_norm_append_kernel(RotaryAppendArgs r) {
  const RopeAppendArgs& a = r.a;
  const int32_t N = a.C * a.T;
  const int32_t n = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (n >= N) return;                                     // whole wave
  const int lane = threadIdx.x & 63;
  const int b = blockIdx.y;
  const int32_t pieces = a.H * kPieces;
  const int np = (pieces - lane + 63) / 64;               // the same for the 16 lanes of a head vector
  const int32_t p = lane % kPieces;
  u32x4_t kx[kPer], vx[kPer], qx[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (i >= np) break;
    const int32_t h = (lane + 64 * i) / kPieces;
    const int64_t src = (int64_t(b) * N + n) * a.tok_stride + int64_t(h) * a.head_stride + p * 8;
    kx[i] = *reinterpret_cast<const u32x4_t*>(a.k + src);
    vx[i] = *reinterpret_cast<const u32x4_t*>(a.v + src);
    if (kWithQ) qx[i] = *reinterpret_cast<const u32x4_t*>(a.q + src);
  }
  const Turn<kHalf> t = load_turn<kHalf>(r, n, p);
  const double inv_c = 1.0 / double(a.H * kHeadDim);
  const double rk = 1.0 / sqrt(sum_sq(kx, np) * inv_c + a.eps);
  double rq = 0.0;
  if (kWithQ) rq = 1.0 / sqrt(sum_sq(qx, np) * inv_c + a.eps);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (i >= np) break;
    const int32_t h = (lane + 64 * i) / kPieces;
    const Place at = place(a, b, n, h);
    const int32_t ch = h * kHeadDim + p * 8;
    const u32x4_t wk = *reinterpret_cast<const u32x4_t*>(a.wk + ch);
    put_rotated<kHalf, kMx8, false>(r, rotate<kHalf>(normalise8(kx[i], wk, rk), t, r, p), at, p);
    put_value<kMx8>(r, vx[i], at, p);
    if (kWithQ) {
      const u32x4_t wq = *reinterpret_cast<const u32x4_t*>(a.wq + ch);
      put_rotated<kHalf, kMx8, true>(r, rotate<kHalf>(normalise8(qx[i], wq, rq), t, r, p), at, p);
    }
  }
}

template <bool kWithQ, bool kHalf, bool kMx8>
void launch(const RotaryAppendArgs& r, hipStream_t stream) {
  const RopeAppendArgs& a = r.a;
  if (a.wk) {
    const int32_t N = a.C * a.T;
    const dim3 grid(unsigned((N + kThreads / 64 - 1) / (kThreads / 64)), unsigned(a.B));
    if (a.H * kPieces <= 64 * kNormPiecesSmall)
      hipLaunchKernelGGL((rotary_norm_append_kernel<kWithQ, kHalf, kMx8, kNormPiecesSmall>), grid, dim3(kThreads), 0, stream, r);
    else
      hipLaunchKernelGGL((rotary_norm_append_kernel<kWithQ, kHalf, kMx8, kNormPiecesLarge>), grid, dim3(kThreads), 0, stream, r);
    return;
  }
  const int64_t units = int64_t(a.C) * a.T * a.H * kPieces;
  const dim3 grid(unsigned((units + kThreads - 1) / kThreads), unsigned(a.B));
  hipLaunchKernelGGL((rotary_append_kernel<kWithQ, kHalf, kMx8>), grid, dim3(kThreads), 0, stream, r);
}

template <bool kHalf, bool kMx8>
void launch(const RotaryAppendArgs& r, hipStream_t stream) {
  r.a.q ? launch<true, kHalf, kMx8>(r, stream) : launch<false, kHalf, kMx8>(r, stream);
}

}  // namespace

hipError_t launch_rotary_append(const RotaryAppendArgs& r, hipStream_t stream) {
  if (r.k8)
    r.half ? launch<true, true>(r, stream) : launch<false, true>(r, stream);
  else
    r.half ? launch<true, false>(r, stream) : launch<false, false>(r, stream);
  return hipGetLastError();
}

}  // namespace unstep
