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
__device__ __forceinline__ float bf16_float(uint32_t s) { return __uint_as_float(s << 16); }

__device__ __forceinline__ float rcp_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Below 2^-17 a scale itself is no binary16 number, and from 8192 on -8 times it is none (a code that append does not make,
// but that unused memory may hold).
__device__ __forceinline__ bool kv4_odd(uint32_t scale_bits) { return scale_bits - 1u < 0x36FFu || scale_bits - 0x4600u < 0x100u; }

// The nibbles of a word of eight codes, two a register, in the order 0 4, 1 5, 2 6, 3 7.  A nibble with its sign flipped is
// code + 8.  With its constants in registers a mask and the flip are one instruction.
struct Nibbles {
  uint32_t lo, hi, wide_lo, wide_hi;
  __device__ __forceinline__ Nibbles() {
    asm("mov.b32 %0, 0x000F000F;" : "=r"(lo));
    asm("mov.b32 %0, 0x00F000F0;" : "=r"(hi));
    asm("mov.b32 %0, 0x64086408;" : "=r"(wide_lo));
    asm("mov.b32 %0, 0x64806480;" : "=r"(wide_hi));
  }
  static __device__ __forceinline__ uint32_t and_xor(uint32_t w, uint32_t mask, uint32_t flip) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0x6A;" : "=r"(d) : "r"(w), "r"(mask), "r"(flip));
    return d;
  }
  // The codes as binary16: under the exponent of 1024 a nibble reads 1032 + code, four bits higher 1024 + 16 (code + 8); one
  // subtraction or fma, exact, takes the offset off.
  __device__ __forceinline__ void codes(uint32_t w, __half2 (&r)[4]) const {
    const __half2 off = __half2half2(__ushort_as_half(0x6408));                                                         // 1032
    const __half2 sixteenth = __half2half2(__ushort_as_half(0x2C00)), off16 = __half2half2(__ushort_as_half(0xD480));   // 1 / 16, -72
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t v = k ? w >> 8 : w, a = and_xor(v, lo, wide_lo), b = and_xor(v, hi, wide_hi);
      r[2 * k] = __hsub2(*reinterpret_cast<const __half2*>(&a), off);
      r[2 * k + 1] = __hfma2(*reinterpret_cast<const __half2*>(&b), sixteenth, off16);
    }
  }
  // The codes times a scale that binary16 holds.
  __device__ __forceinline__ uint4 values(uint32_t w, __half2 s) const {
    __half2 r[4];
    codes(w, r);
    uint32_t v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      r[k] = __hmul2(r[k], s);
      v[k] = *reinterpret_cast<const uint32_t*>(&r[k]);
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
  }
};
// The values for any scale: each product in fp32, rounded once.  FINITE: at most the largest number of binary16 (NaN stays:
// it marks the K rows of keys whose scale is no number, and fmin and fmax would lose it).
template <bool FINITE>
__device__ __forceinline__ uint4 values_slow(uint32_t w, float s) {
  auto value = [&](int e) {
    const float v = s * (float)((int)(w << (28 - 4 * e)) >> 28);
    return FINITE && fabsf(v) > 65504.f ? copysignf(65504.f, v) : v;
  };
  return make_uint4(pack_half2(value(0), value(4)), pack_half2(value(1), value(5)), pack_half2(value(2), value(6)),
                    pack_half2(value(3), value(7)));
}

}  // namespace dptq
