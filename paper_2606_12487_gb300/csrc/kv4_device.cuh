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

// Below 2^-17 a scale itself is no binary16 number.
__device__ __forceinline__ bool kv4_tiny(uint32_t scale_bits) { return scale_bits != 0 && scale_bits < 0x3700u; }

// Eight codes (two's complement nibbles of a word) times a scale to 16 bytes of binary16, in the order 0 4, 1 5, 2 6,
// 3 7.  A nibble with its sign flipped is code + 8; under the exponent of 1024 it reads 1032 + code, four bits higher
// 1024 + 16 (code + 8): one subtraction or fma, exact, takes the offset off.
__device__ __forceinline__ uint4 widen8(uint32_t w, __half2 s) {
  const __half2 off = __half2half2(__ushort_as_half(0x6408));                                                         // 1032
  const __half2 sixteenth = __half2half2(__ushort_as_half(0x2C00)), off16 = __half2half2(__ushort_as_half(0xD480));   // 1 / 16, -72
  uint32_t r[4];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t v = k ? w >> 8 : w, a = (v & 0x000F000Fu) ^ 0x64086408u, b = (v & 0x00F000F0u) ^ 0x64806480u;
    const __half2 lo = __hmul2(__hsub2(*reinterpret_cast<const __half2*>(&a), off), s);
    const __half2 hi = __hmul2(__hfma2(*reinterpret_cast<const __half2*>(&b), sixteenth, off16), s);
    r[2 * k] = *reinterpret_cast<const uint32_t*>(&lo);
    r[2 * k + 1] = *reinterpret_cast<const uint32_t*>(&hi);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}
// The same for scales that binary16 does not hold: each product in fp32, rounded once.
__device__ __forceinline__ uint4 widen8_slow(uint32_t w, float s) {
  auto value = [&](int e) { return s * (float)((int)(w << (28 - 4 * e)) >> 28); };
  return make_uint4(pack_half2(value(0), value(4)), pack_half2(value(1), value(5)), pack_half2(value(2), value(6)),
                    pack_half2(value(3), value(7)));
}

}  // namespace dptq
