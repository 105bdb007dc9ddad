// Quantised rows read back as bf16: value = e4m3 * 2^(byte - 127), exact in bf16 for what the
// quantising append writes.  A thread turns 8 values (8 bytes and their block's scale byte) into 16
// bytes; consecutive threads cover a row, then the next output row, so the writes, two thirds of the
// bytes, stream contiguously.
#include <hip/hip_runtime.h>

#include "kernels.hpp"
#include "mx8.hpp"
#include "seg_table.hpp"

namespace unstep {
namespace {

constexpr int kThreads = 256;
constexpr int kPieces = kHeadDim / 8;

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ u32x4_t values(u32x2_t x, uint32_t byte) {
  const float s = mx8_scale(byte);
  u32x4_t o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2_t v = (i & 1) ? __builtin_amdgcn_cvt_pk_f32_fp8(int(x[i >> 1]), true)
                              : __builtin_amdgcn_cvt_pk_f32_fp8(int(x[i >> 1]), false);
    bf16x2_t w;
    w[0] = (__bf16)(v[0] * s);
    w[1] = (__bf16)(v[1] * s);
    o[i] = __builtin_bit_cast(uint32_t, w);
  }
  return o;
}

template <bool kCache>
__global__ __launch_bounds__(kThreads) void mx8_read_kernel(Mx8ReadArgs a) {
  const int64_t u = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  const int64_t row = u / kPieces;
  if (row >= a.rows) return;
  const int32_t p = int32_t(u % kPieces);
  int64_t from = row;
  if (kCache) {
    const int64_t tok = row / a.H;
    const int32_t h = int32_t(row - tok * a.H), N = a.C * a.T;
    const int32_t b = int32_t(tok / N), n = int32_t(tok - int64_t(b) * N);
    const int32_t fi = n / a.T;
    from = (int64_t(b) * a.H + h) * a.slots + int64_t(frame_slot(a.f0 + fi, a.S, a.R)) * a.T + (n - fi * a.T);
  }
  const u32x2_t x = *reinterpret_cast<const u32x2_t*>(a.x8 + from * kHeadDim + p * 8);
  const uint32_t xs = a.x_scale[from * kMxBlocks + (p >> 2)];
  if (kCache) {
    const u32x2_t y = *reinterpret_cast<const u32x2_t*>(a.y8 + from * kHeadDim + p * 8);
    const uint32_t ys = a.y_scale[from * kMxBlocks + (p >> 2)];
    __builtin_nontemporal_store(values(y, ys), reinterpret_cast<u32x4_t*>(a.y_out + row * kHeadDim + p * 8));
  }
  __builtin_nontemporal_store(values(x, xs), reinterpret_cast<u32x4_t*>(a.out + row * kHeadDim + p * 8));
}

}  // namespace

hipError_t launch_mx8_read(const Mx8ReadArgs& a, hipStream_t stream) {
  const dim3 grid(unsigned((a.rows * kPieces + kThreads - 1) / kThreads));
  if (a.T > 0)
    hipLaunchKernelGGL(mx8_read_kernel<true>, grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(mx8_read_kernel<false>, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace unstep
