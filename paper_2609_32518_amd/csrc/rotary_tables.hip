// cos/sin tables of a chunk on the device, for rotary embeddings whose pairs are split over (frame,
// row, column) in any proportion and whose frame axis may be scaled for clips longer than the trained
// ones: the scaling is in the frequencies, which the host computes in 64 bits.
//
// table[n][j] = fp32(amplitude * cos(p w_j)), p the absolute frame index, the row or the column of token
// n, w_j = freq[j]; the angle, cos and sin in double precision (the angle of a far frame has lost its
// fraction in fp32: at frame 60000 the first pair's fp32 angle is off by up to 2e-3).
//
// What bounds it: the fp64 sincos, of which a chunk needs few (frames * pairs_t + rows * pairs_h +
// columns * pairs_w) against the N * pairs entries it writes.  A work-group is kCols tokens of one row of
// one frame: one sincos per thread at most for up to 256 distinct angles (22 + 21 + 8 * 21 of the video
// model's split), kept in LDS, then the tokens' entries written with consecutive threads on consecutive
// entries.  Small groups keep the latency at one sincos and make enough of them for the chip.
// 4680 tokens x 64 pairs (2.4 MB): 3.9 us; one token: 1.9.
#include <hip/hip_runtime.h>

#include "kernels.hpp"

namespace unstep {
namespace {

constexpr int kThreads = 256;
constexpr int kCols = 8;
constexpr int kMaxPairs = kHeadDim / 2;

__global__ __launch_bounds__(kThreads) void rotary_tables_kernel(RotaryTableArgs a) {
  __shared__ float2 cs[kMaxPairs * kCols];               // frame and row pairs, then each column's
  const int32_t groups = (a.grid_w + kCols - 1) / kCols;   // of columns, per row
  const int32_t fr = int32_t(blockIdx.x) / groups, fi = fr / a.grid_h, row = fr - fi * a.grid_h;
  const int32_t col0 = (int32_t(blockIdx.x) - fr * groups) * kCols;
  const int32_t cols = min(kCols, a.grid_w - col0);
  const int32_t shared_pairs = a.pairs_t + a.pairs_h, pairs = shared_pairs + a.pairs_w;
  const int32_t angles = shared_pairs + cols * a.pairs_w;
  for (int32_t i = threadIdx.x; i < angles; i += kThreads) {
    const int32_t c = i < shared_pairs ? 0 : (i - shared_pairs) / a.pairs_w;
    const int32_t j = i < shared_pairs ? i : shared_pairs + (i - shared_pairs) - c * a.pairs_w;
    const int32_t p = j < a.pairs_t ? a.f0 + fi : j < shared_pairs ? row : col0 + c;
    double s, co;
    sincos(double(p) * a.freq[j], &s, &co);
    cs[i] = make_float2(float(a.amplitude * co), float(a.amplitude * s));
  }
  __syncthreads();
  const int64_t n0 = (int64_t(fi) * a.grid_h + row) * a.grid_w + col0;
  float* const cos_t = a.cos_t + n0 * pairs;
  float* const sin_t = a.sin_t + n0 * pairs;
  for (int32_t i = threadIdx.x; i < cols * pairs; i += kThreads) {
    const int32_t c = i / pairs, j = i - c * pairs;
    const float2 v = cs[j < shared_pairs ? j : j + c * a.pairs_w];
    cos_t[i] = v.x;
    sin_t[i] = v.y;
  }
}

}  // namespace

hipError_t launch_rotary_tables(const RotaryTableArgs& a, hipStream_t stream) {
  const int64_t groups = int64_t(a.frames) * a.grid_h * ((a.grid_w + kCols - 1) / kCols);
  hipLaunchKernelGGL(rotary_tables_kernel, dim3(unsigned(groups)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace unstep
