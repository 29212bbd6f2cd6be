// kv8_device.cuh -- what the kernels over the paged int8 cache share: the checked view of a
// sequence, page lookups and the exact quantizer of a value.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "dptq_device.cuh"
#include "dptq_internal.h"

namespace dptq {

// A sequence of the call: its n new tokens are rows tok0 .. tok0 + n - 1 and stand at the
// positions start .. start + n - 1 (start = len - n; below zero for tokens that a sequence
// shorter than its rows has no place for).
struct Seq {
  int tok0, n, len, start;
};
// False (and, from the thread that `tells`, the error word) where the arrays contradict what
// the call declared: such a sequence is left alone, so no index is made from its numbers.
__device__ __forceinline__ bool load_seq(const Kv8Args& c, int s, Seq& q, bool tells) {
  const int a = ld_plain(c.cu + s), b = ld_plain(c.cu + s + 1), len = ld_plain(c.lens + s);
  const bool ok = a >= 0 && b >= a && b <= c.tokens && b - a <= c.max_tokens && len >= 0 && len <= c.max_len;
  q.tok0 = a;
  q.n = b - a;
  q.len = len;
  q.start = len - q.n;
  if (!ok && tells) atomicCAS(c.bad, 0, kDevBadBatch);
  return ok;
}

// The page that holds position p of sequence s, or -1 (and the error word) if the table has
// none.  p < max_len <= table_stride * page, checked on the host and by load_seq.
__device__ __forceinline__ int load_page(const Kv8Args& c, int s, int page) {
  const int b = ld_plain(c.table + (long long)s * c.table_stride + page);
  if (b >= 0 && b < c.num_blocks) return b;
  atomicCAS(c.bad, 0, kDevBadPage);
  return -1;
}

// Whether the query at position p sees the key at position j.
__device__ __forceinline__ bool kv8_sees(int p, int j, int window, int sinks) {
  return j <= p && (window == 0 || j > p - window || j < sinks);
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t less_1152(uint32_t h) {
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&h), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Four codes to two pairs of binary16: values 0, 1 and 2, 3.
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  w ^= 0x80808080u;
  lo = less_1152(__byte_perm(w, 0x64646464u, 0x4140));
  hi = less_1152(__byte_perm(w, 0x64646464u, 0x4342));
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace dptq
