// kv4_device.cuh -- what the kernels over the paged 4-bit cache share.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv8_device.cuh"

namespace dptq {

// Scales are 0 to 9344, the largest that append makes of a finite value; anything else is no number (binary16 holds 7
// times 9344).
__device__ __forceinline__ bool kv4_bad(uint32_t scale_bits) { return scale_bits > 0x4612u; }
__device__ __forceinline__ float bf16_float(uint16_t s) { return __uint_as_float((uint32_t)s << 16); }

// Eight codes (two's complement nibbles of a word) to four pairs of binary16, in the order 0 4, 1 5, 2 6, 3 7.  A
// nibble with its sign flipped is code + 8; under the exponent of 1024 it reads 1032 + code, four bits higher
// 1024 + 16 (code + 8): one subtraction or fma, exact, takes the offset off.
__device__ __forceinline__ void widen8(uint32_t w, __half2 (&r)[4]) {
  const __half2 off = __half2half2(__ushort_as_half(0x6408));      // 1032
  const __half2 sixteenth = __half2half2(__ushort_as_half(0x2C00)), off16 = __half2half2(__ushort_as_half(0xD480));   // 1 / 16, -72
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t v = k ? w >> 8 : w;
    const uint32_t lo = (v & 0x000F000Fu) ^ 0x64086408u, hi = (v & 0x00F000F0u) ^ 0x64806480u;
    r[2 * k] = __hsub2(*reinterpret_cast<const __half2*>(&lo), off);
    r[2 * k + 1] = __hfma2(*reinterpret_cast<const __half2*>(&hi), sixteenth, off16);
  }
}

}  // namespace dptq
