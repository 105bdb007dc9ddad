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

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short i16x2_t __attribute__((ext_vector_type(2)));

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

template <int kCtrl>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(x), kCtrl, 0xf, 0xf, false));
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
    if (r.rot == kHeadDim) {                              // the whole head: 8 lanes on or back within the 16
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = dpp<0x128>(x[e]);   // row_ror 8
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = uint32_t(__shfl(int(x[e]), from));
    }
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

// The scale byte of the block (4 lanes) that this lane's 8 values belong to.  A value that is not finite does not
// count: a maximum leaves NaN out by itself, and one that is infinite (or nothing but NaN) sends the lane through
// its values again.
__device__ __forceinline__ int32_t block_byte(const F8& y) {
  float most = __builtin_fabsf(y.v[0]);
#pragma unroll
  for (int i = 1; i < 8; ++i) most = __builtin_fmaxf(most, __builtin_fabsf(y.v[i]));
  uint32_t top = __float_as_uint(most);
  if (__builtin_expect(top >= 0x7f800000u, 0)) {
    top = 0;
    for (int i = 0; i < 8; ++i) {
      const uint32_t m = __float_as_uint(y.v[i]) & 0x7fffffffu;
      top = m < 0x7f800000u ? max(top, m) : top;
    }
  }
  top = max(top, dpp<0xb1>(top));                         // quad_perm 1,0,3,2
  top = max(top, dpp<0x4e>(top));                         // quad_perm 2,3,0,1
  return mx8_byte(top);
}

// Stores piece p of the head vector at row `row`: eight e4m3 bytes (the conversion divides by the power of
// two and rounds once; infinities become NaN), and (lane of piece 0) the row's scale bytes.  The 16 lanes of the
// vector are in this together.
__device__ __forceinline__ void store_mx8(const F8& y, uint8_t* x8, uint8_t* scale, int64_t row, int32_t p) {
  const int32_t byte = block_byte(y);
  const float s = mx8_scale(uint32_t(byte));
  u32x2_t w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    i16x2_t d = {};
    d = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(d, y.v[4 * i], y.v[4 * i + 1], s, false);
    d = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(d, y.v[4 * i + 2], y.v[4 * i + 3], s, true);
    w[i] = __builtin_bit_cast(uint32_t, d);
  }
  // kept in the caches: what follows an append reads them (with a read-back 30.2 us instead of 33.5 for 4680 tokens x
  // 12 heads, a step the same; the append alone 0.2 to 0.9 more)
  *reinterpret_cast<u32x2_t*>(x8 + row * kHeadDim + p * 8) = w;
  uint32_t bytes = uint32_t(byte) << (8 * (p >> 2));
  bytes |= dpp<0x124>(bytes);                             // row_ror 4
  bytes |= dpp<0x128>(bytes);                             // row_ror 8
  if (p == 0) *reinterpret_cast<uint32_t*>(scale + row * kMxBlocks) = bytes;
}

// Places of token n of batch b, head h: row of the chunk's outputs, and of the cache.
struct Place {
  int64_t chunk_row, cache_row;
};
__device__ __forceinline__ Place place(const RotaryAppendArgs& r, int32_t b, uint32_t n, uint32_t h) {
  const RopeAppendArgs& a = r.a;
  const uint32_t fi = divide(n, r.by_t), t = n - fi * uint32_t(a.T);
  const int32_t f = a.f0 + int32_t(fi), g = f - a.S;       // frame, and which of the ring's
  const uint32_t slot = g < 0 ? uint32_t(f) : uint32_t(a.S) + uint32_t(g) - divide(uint32_t(g), r.by_r) * uint32_t(a.R);
  const uint32_t N = uint32_t(a.C) * uint32_t(a.T);
  return Place{int64_t(b) * N * a.H + (n * uint32_t(a.H) + h),
               int64_t(b) * a.H * a.slots + int64_t(uint64_t(h) * uint32_t(a.slots) + (slot * uint32_t(a.T) + t))};
}
// Element offset of piece p of token n, head h in the inputs of batch b.
__device__ __forceinline__ int64_t source(const RopeAppendArgs& a, int32_t b, uint32_t n, uint32_t h, uint32_t p) {
  const uint32_t N = uint32_t(a.C) * uint32_t(a.T);
  return int64_t(b) * N * a.tok_stride + int64_t(uint64_t(n) * uint32_t(a.tok_stride) + uint64_t(h) * uint32_t(a.head_stride) + p * 8);
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
  const uint32_t n = divide(hv, r.by_h), h = hv - n * uint32_t(a.H);
  const int32_t b = blockIdx.y;
  const int64_t src = source(a, b, n, h, p);
  const u32x4_t kx = *reinterpret_cast<const u32x4_t*>(a.k + src);
  const u32x4_t vx = *reinterpret_cast<const u32x4_t*>(a.v + src);
  u32x4_t qx = {};
  if (kWithQ) qx = *reinterpret_cast<const u32x4_t*>(a.q + src);
  const Turn<kHalf> t = load_turn<kHalf>(r, n, p);
  const Place at = place(r, b, n, h);
  put_rotated<kHalf, kMx8, false>(r, rotate<kHalf>(kx, t, r, p), at, p);
  put_value<kMx8>(r, vx, at, p);
  if (kWithQ) put_rotated<kHalf, kMx8, true>(r, rotate<kHalf>(qx, t, r, p), at, p);
}

// ---- with the RMS normalisation: a token's head vectors on ceil(heads / 4) waves, one piece per lane as above.
// x'_j = bf16(fp32(x_j r w_j)), r = 1 / sqrt(sum x^2 / channels + eps) in fp64 (each bf16 square is exact), summed
// over a wave by exchanges and over the token's waves through LDS, in one order.
// What bounds it is memory and, between a token's loads and its stores, the statistic: 4680 tokens x 12 heads take
// 15.8 us into the quantised cache (67.7 MB; 12.4 without the normalisation, the rate of a copy) and 14.9 into the bf16
// one (88.7 MB; 14.3).  Before: fp64 products per channel and a wave per token 21.4; binary32 pairs 17.5; one piece per
// lane, divisions by multiplication and two Newton steps for the root 16.0; 64 registers, so that 8 waves fit a SIMD,
// and the values stored before the statistic is known 15.8; with stores that stay in the caches 16.5; two operations
// a product instead of four and no branches around the loads 15.8.
__device__ __forceinline__ double sum_sq(u32x4_t x) {
  double s = 0.0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const double lo = bf16_lo(x[e]), hi = bf16_hi(x[e]);
    s += lo * lo;
    s += hi * hi;
  }
  return s;
}

// 1 / sqrt(x), as it is and as a sum of two binary32 numbers.
struct Rms {
  float hi, lo;
  double r;
  bool plain;                                             // 2^-51 < r < 2^51, the same for the whole wave
};
// The binary32 reciprocal root (2^-22) and two Newton steps in fp64 for ordinary x: within two units of the
// last place of fp64, for a quarter of the instructions of the square root and division.
__device__ __forceinline__ double inverse_root(double x) {
  if (__builtin_expect(!(x > 0x1p-100 && x < 0x1p100), 0)) return 1.0 / sqrt(x);
  double y = (double)__builtin_amdgcn_rsqf((float)x);
  const double h = 0.5 * x;
  y = y * (1.5 - h * y * y);
  return y * (1.5 - h * y * y);
}
__device__ __forceinline__ double lane_value(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane(uint32_t(u), lane), hi = __builtin_amdgcn_readlane(uint32_t(u >> 32), lane);
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}
__device__ __forceinline__ Rms rms_of(double r) {
  Rms m;
  m.r = r;
  m.hi = (float)r;
  m.lo = (float)(r - (double)m.hi);
  m.plain = r > 0x1p-51 && r < 0x1p51;
  return m;
}
template <int kCtrl>
__device__ __forceinline__ double dpp(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, uint64_t(dpp<kCtrl>(uint32_t(u >> 32))) << 32 | dpp<kCtrl>(uint32_t(u)));
}
// Both sums of a wave in one reduction: its lower half takes the keys', the upper the queries', so that the
// steps after the first, and the root later, are done once for the two.
__device__ __forceinline__ double wave_sums(double k, double q) {
  const bool upper = (threadIdx.x & 32) != 0;
  double s = (upper ? q : k) + __shfl_xor(upper ? k : q, 32);
  s += dpp<0xb1>(s);                                      // quad_perm 1,0,3,2
  s += dpp<0x4e>(s);                                      // quad_perm 2,3,0,1
  s += dpp<0x141>(s);                                     // row_half_mirror: the other quad of 8
  s += dpp<0x140>(s);                                     // row_mirror: the other 8 of 16
  return s + __shfl_xor(s, 16);
}

// bf16(fp32(x r w)) for the 8 channels of a piece.  x w is exact in binary32 (8 and 8 bits); its product with
// hi + lo, formed as fma(x w, hi, x w lo), is within 2^-47 of the exact one before its only rounding to
// binary32, as the fp64 product is within 2^-52: two binary32 operations instead of five conversions and
// products in fp64, which the pass's time went into.  The binary32 value is kept opaque, or the two roundings
// would be folded into one.
__device__ __forceinline__ u32x4_t normalise8(u32x4_t x, u32x4_t w, const Rms& m) {
#pragma clang fp contract(off)
  const F8 xs = widen(x), ws = widen(w);
  F8 v;
  if (__builtin_expect(m.plain, 1)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = xs.v[i] * ws.v[i];
      v.v[i] = __builtin_fmaf(t, m.hi, t * m.lo);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v.v[i] = (float)(((double)xs.v[i] * m.r) * (double)ws.v[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(v.v[i]));
  return to_bf16(v);
}

constexpr int kNormMaxWaves = kNormMaxHeads * kPieces / 64;   // of a token, and of a work-group
static_assert(kNormMaxWaves == 8, "");

// waves: of a token; tokens: of a work-group.  Lanes past the last head or token load and compute what the last one's
// do, and neither count nor store.
template <bool kWithQ, bool kHalf, bool kMx8>
__global__ __launch_bounds__(kNormMaxWaves * 64, 8) void rotary_norm_append_kernel(RotaryAppendArgs r, uint32_t waves,
                                                                                   uint32_t tokens, FastDiv by_waves) {
  const RopeAppendArgs& a = r.a;
  __shared__ double sums[kNormMaxWaves][2];
  const uint32_t last = uint32_t(a.C) * uint32_t(a.T) - 1;
  const int lane = threadIdx.x & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t tok = divide(wave, by_waves), part = wave - tok * waves;    // of the work-group; wave of the token
  const uint32_t n0 = blockIdx.x * tokens + tok, n = min(n0, last);
  const int32_t b = blockIdx.y, h0 = int32_t(4 * part) + (lane >> 4), h = min(h0, a.H - 1), p = lane % kPieces;
  const bool here = n0 == n && h0 == h;                                      // the same for a head vector's 16 lanes
  const int64_t src = source(a, b, n, h, p);
  const u32x4_t kx = *reinterpret_cast<const u32x4_t*>(a.k + src);
  u32x4_t qx = {}, wq = {};
  if (kWithQ) qx = *reinterpret_cast<const u32x4_t*>(a.q + src);
  const Turn<kHalf> t = load_turn<kHalf>(r, n, p);
  const u32x4_t vx = *reinterpret_cast<const u32x4_t*>(a.v + src);
  const u32x4_t wk = *reinterpret_cast<const u32x4_t*>(a.wk + h * kHeadDim + p * 8);
  if (kWithQ) wq = *reinterpret_cast<const u32x4_t*>(a.wq + h * kHeadDim + p * 8);
  const double sk = sum_sq(kx), sq = kWithQ ? sum_sq(qx) : 0.0;
  const double s = wave_sums(here ? sk : 0.0, here ? sq : 0.0);
  if ((lane & 31) == 0) sums[wave][lane >> 5] = s;
  const Place at = place(r, b, n, h);
  if (here) put_value<kMx8>(r, vx, at, p);                // the values need no statistic
  __syncthreads();
  double ss = 0.0;
  for (uint32_t i = 0; i < waves; ++i) ss += sums[tok * waves + i][lane >> 5];
  const double rr = inverse_root(ss * r.inv_channels + a.eps);
  const Rms rk = rms_of(lane_value(rr, 0)), rq = rms_of(lane_value(rr, 32));
  if (!here) return;
  put_rotated<kHalf, kMx8, false>(r, rotate<kHalf>(normalise8(kx, wk, rk), t, r, p), at, p);
  if (kWithQ) put_rotated<kHalf, kMx8, true>(r, rotate<kHalf>(normalise8(qx, wq, rq), t, r, p), at, p);
}

template <bool kWithQ, bool kHalf, bool kMx8>
void launch(const RotaryAppendArgs& r, hipStream_t stream) {
  const RopeAppendArgs& a = r.a;
  if (a.wk) {
    const uint32_t waves = uint32_t(a.H + 3) / 4, tokens = waves < 4 ? 4 / waves : 1;  // of a token; tokens of a work-group
    const dim3 grid((uint32_t(a.C * a.T) + tokens - 1) / tokens, unsigned(a.B));
    hipLaunchKernelGGL((rotary_norm_append_kernel<kWithQ, kHalf, kMx8>), grid, dim3(waves * tokens * 64), 0, stream, r, waves,
                       tokens, fast_div(waves));
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

hipError_t launch_rotary_append(const RotaryAppendArgs& args, hipStream_t stream) {
  RotaryAppendArgs r = args;
  r.by_h = fast_div(uint32_t(r.a.H));
  r.by_t = fast_div(uint32_t(r.a.T));
  r.by_r = fast_div(uint32_t(r.a.R));
  r.inv_channels = 1.0 / double(r.a.H * kHeadDim);
  if (r.k8)
    r.half ? launch<true, true>(r, stream) : launch<false, true>(r, stream);
  else
    r.half ? launch<true, false>(r, stream) : launch<false, false>(r, stream);
  return hipGetLastError();
}

}  // namespace unstep
