// Quantised rows read back as bf16: value = e4m3 * 2^(byte - 127), exact in bf16 for what the
// quantising append writes.  Bound by memory: 132 bytes in and 256 out per row.  A thread turns 8 values (8 bytes
// and their block's scale byte) into 16 bytes; consecutive threads cover a row, then the next output row, so
// that a wave's store is one run of 1 KB (16 values a thread, in two stores of every other 16 bytes: 9.5 us
// instead of 6.8 for 4680 tokens x 12 heads of both tensors
// in the Infinity Cache; 9 behind an append that has just written them, 43.6 MB at 4.8 TB/s).
#include <hip/hip_runtime.h>

#include "kernels.hpp"
#include "mx8.hpp"
#include "seg_table.hpp"

namespace unstep {
namespace {

constexpr int kThreads = 256;
constexpr int kPieces = kHeadDim / 8;   // 8-byte pieces of a quantised row, one thread each

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void put(uint16_t* out, u32x2_t x, uint32_t byte) {
  const float s = mx8_scale(byte);
  u32x4_t o;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t w = x[e >> 1];
    const bf16x2_t v = (e & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)
                               : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false);
    o[e] = __builtin_bit_cast(uint32_t, v);
  }
  __builtin_nontemporal_store(o, reinterpret_cast<u32x4_t*>(out));
}

template <bool kCache>
__global__ __launch_bounds__(kThreads) void mx8_read_kernel(Mx8ReadArgs a) {
  const uint32_t u = blockIdx.x * kThreads + threadIdx.x, row = u / kPieces, p = u % kPieces;
  if (row >= uint32_t(a.rows)) return;
  int64_t from = row;
  if (kCache) {
    const uint32_t tok = divide(row, a.by_h), h = row - tok * uint32_t(a.H);
    const uint32_t frame = divide(tok, a.by_t), t = tok - frame * uint32_t(a.T);   // of all batches
    const uint32_t b = divide(frame, a.by_c), f = uint32_t(a.f0) + (frame - b * uint32_t(a.C));
    const int32_t g = int32_t(f) - a.S;
    const uint32_t slot = g < 0 ? f : uint32_t(a.S) + uint32_t(g) - divide(uint32_t(g), a.by_r) * uint32_t(a.R);
    from = int64_t(uint64_t(b * uint32_t(a.H) + h) * uint32_t(a.slots) + (slot * uint32_t(a.T) + t));
  }
  const u32x2_t x = *reinterpret_cast<const u32x2_t*>(a.x8 + from * kHeadDim + p * 8);
  const uint32_t xs = a.x_scale[from * kMxBlocks + (p >> 2)];
  if (kCache) {
    const u32x2_t y = *reinterpret_cast<const u32x2_t*>(a.y8 + from * kHeadDim + p * 8);
    const uint32_t ys = a.y_scale[from * kMxBlocks + (p >> 2)];
    put(a.y_out + int64_t(row) * kHeadDim + p * 8, y, ys);
  }
  put(a.out + int64_t(row) * kHeadDim + p * 8, x, xs);
}

}  // namespace

hipError_t launch_mx8_read(const Mx8ReadArgs& args, hipStream_t stream) {
  Mx8ReadArgs a = args;
  const dim3 grid(unsigned((a.rows * kPieces + kThreads - 1) / kThreads));
  if (a.T > 0) {
    a.by_h = fast_div(uint32_t(a.H));
    a.by_t = fast_div(uint32_t(a.T));
    a.by_c = fast_div(uint32_t(a.C));
    a.by_r = fast_div(uint32_t(a.R));
    hipLaunchKernelGGL(mx8_read_kernel<true>, grid, dim3(kThreads), 0, stream, a);
  } else {
    hipLaunchKernelGGL(mx8_read_kernel<false>, grid, dim3(kThreads), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace unstep
