// The quantised cache's number format on the device: blocks of 32 values along the head, each an e4m3
// value (at most 448, steps of 2^-9 below 2^-6) times one power of two 2^(byte - 127).
//
// A block's exponent is the smallest e >= -100 with max|y| 2^-e <= 448: a power of two costs no
// precision (scaling is exact, so the only rounding is e4m3's own, at most half a step) and keeps every
// held value exact in bf16, which the attention's product with the values relies on.  The bound of -100
// keeps the smallest held value, 2^-109, a normal number.  A value that is not finite is held as NaN and
// does not count towards its block's maximum.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace unstep {

constexpr int kMxBlock = 32;
constexpr int kMxBlocks = 4;             // per row of 128
constexpr int32_t kMxMinByte = 27;       // 2^-100

// The scale byte of a block from the bits of its largest finite |y|: 1.f 2^k takes k - 8 where
// 1.f <= 1.75 = 448 / 256, else k - 7 (the sum carries into the exponent).
__device__ __forceinline__ int32_t mx8_byte(uint32_t top) {
  return max(int32_t((top + 0x1fffffu) >> 23) - 8, kMxMinByte);
}
__device__ __forceinline__ float mx8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace unstep
