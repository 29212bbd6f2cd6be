// norm_quant.cu -- residual addition, RMS norm and the per-token symmetric quantizer in one
// kernel: what the projections that read the residual stream take as their codes.
//   h = fp16(x + r),  p_k = h_k g_k,  s' = max|p| fl(1 / qmax),  c_k = rint(p_k / s'),
//   scale = s' / sqrt(mean(h^2) + eps).
// p is exact in fp32 (11 + 11 bits), and the norm's factor is one positive number for the
// whole token, so it goes into the scale alone: the codes are a function of h and g, whatever
// order the squares are summed in.
//
// Two bytes in twice, two and one out: bytes bound it.  A token is read once and stays in
// registers (16 bytes a thread and vector) between the reduction and its codes.  A CTA takes
// one token, with as few vectors a thread as 512 threads allow: four such CTAs fit an SM (32
// registers a thread), so that one's loads run under another's reduction, and a call of few
// tokens is as long as its chain of one load, one reduction and one store.  Tokens that
// registers do not hold (K > 16384) are read again from the second-level cache.
// 8192 x 8192 (470 MB): 71 us, 6.6 TB/s (4-bit codes, 436 MB: 70 us); 2048 x 28672 (411 MB and a second
// read): 111 us.  At 8192 x 8192, CTAs of 1024 threads: 92 us; three of 512 an SM: 86 us; a resident wave of
// CTAs that ask for their next token before they reduce this one: 100 us (the second token's
// registers cost a resident CTA and more).
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "dptq_device.cuh"
#include "dptq_internal.h"

namespace dptq {

__device__ __forceinline__ __half2 h2(uint32_t v) { return *reinterpret_cast<const __half2*>(&v); }
__device__ __forceinline__ uint32_t u2(__half2 v) { return *reinterpret_cast<const uint32_t*>(&v); }

// The CTA's sum and maximum, in every thread: warps first, then one warp's worth of partials.
__device__ __forceinline__ void norm_reduce(float& sq, float& am, float (&red)[2][32]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nw = blockDim.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sq += __shfl_xor_sync(0xffffffffu, sq, o);
    am = fmaxf(am, __shfl_xor_sync(0xffffffffu, am, o));
  }
  if (nw == 1) return;
  if (lane == 0) red[0][warp] = sq, red[1][warp] = am;
  __syncthreads();
  sq = lane < nw ? red[0][lane] : 0.f;
  am = lane < nw ? red[1][lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sq += __shfl_xor_sync(0xffffffffu, sq, o);
    am = fmaxf(am, __shfl_xor_sync(0xffffffffu, am, o));
  }
}

// h of eight values (written where there is a residual), their squares and largest |p|.
__device__ __forceinline__ uint4 norm_take(const NormArgs& a, size_t at, int k, const uint4 x, const uint4 r, const uint4 g,
                                           float& sq, float& am) {
  uint32_t h[4] = {x.x, x.y, x.z, x.w};
  const uint32_t rr[4] = {r.x, r.y, r.z, r.w}, gg[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (a.residual) h[e] = u2(__hadd2(h2(h[e]), h2(rr[e])));   // (one rounding: the sum of two binary16)
    const float2 f = __half22float2(h2(h[e]));
    sq = fmaf(f.x, f.x, fmaf(f.y, f.y, sq));
    float2 p = f;
    if (a.gamma) {
      const float2 w = __half22float2(h2(gg[e]));
      p.x *= w.x;
      p.y *= w.y;
    }
    am = fmaxf(am, fmaxf(fabsf(p.x), fabsf(p.y)));
  }
  const uint4 v = make_uint4(h[0], h[1], h[2], h[3]);
  if (a.residual) *reinterpret_cast<uint4*>(a.residual_out + at + k) = v;
  return v;
}

__device__ __forceinline__ void norm_put(const NormArgs& a, size_t at, int k, const uint4 v, const uint4 g, float s,
                                         float r) {
  const uint32_t h[4] = {v.x, v.y, v.z, v.w}, gg[4] = {g.x, g.y, g.z, g.w};
  int c[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float2 p = __half22float2(h2(h[e]));
    if (a.gamma) {
      const float2 w = __half22float2(h2(gg[e]));
      p.x *= w.x;
      p.y *= w.y;
    }
    c[2 * e] = quant_code(p.x, s, r);
    c[2 * e + 1] = quant_code(p.y, s, r);
  }
  if (a.bits == 8) {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e >> 2] |= (uint32_t)(c[e] & 0xFF) << (8 * (e & 3));
    *reinterpret_cast<uint2*>(a.codes + at + k) = make_uint2(w[0], w[1]);
  } else {
    uint32_t w = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= (uint32_t)(c[e] & 0xF) << (4 * e);
    *reinterpret_cast<uint32_t*>(a.codes + (at + k) / 2) = w;
  }
}

// The step and its reciprocal, and the token's scale from thread 0.
__device__ __forceinline__ void norm_scale(const NormArgs& a, int row, float sq, float am, float& s, float& r) {
  s = __fmul_rn(am, a.bits == 4 ? 1.f / 7.f : 1.f / 127.f);
  r = s > 0.f ? __frcp_rn(s) : 0.f;
  // (no square, however small h is, rounds to zero: a sum of zero is a token of zeros, whose factor is 1 / 0
  // without eps)
  if (threadIdx.x == 0)
    a.scales[row] = sq == 0.f ? 0.f : s * __frcp_rn(__fsqrt_rn(__fdiv_rn(sq, (float)a.K) + a.eps));
}

// A token of at most 8 V blockDim values, in registers.
constexpr int kNormThreads = 512;
constexpr int norm_ctas(int v) { return v == 4 ? 2 : 4; }   // of 512 threads, an SM
template <int V>
__global__ void __launch_bounds__(kNormThreads, norm_ctas(V)) norm_quant_kernel(const NormArgs a) {
  __shared__ float red[2][32];
  const int row = blockIdx.x;
  const size_t at = (size_t)row * a.K;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  pdl_launch_dependents();
  pdl_wait();
  uint4 x[V], r[V];
  float sq = 0.f, am = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    // (threads past the row's end read its last vector: a load in a branch would wait for its data)
    const int k = min(8 * (int)(threadIdx.x + i * blockDim.x), a.K - 8);
    x[i] = *reinterpret_cast<const uint4*>(a.x + at + k);
    r[i] = a.residual ? *reinterpret_cast<const uint4*>(a.residual + at + k) : zero;
  }
  auto weight = [&](int k) { return a.gamma ? ld_plain(reinterpret_cast<const uint4*>(a.gamma + k)) : zero; };
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int k = 8 * (threadIdx.x + i * blockDim.x);
    if (k < a.K) x[i] = norm_take(a, at, k, x[i], r[i], weight(k), sq, am);
  }
  norm_reduce(sq, am, red);
  float s, inv;
  norm_scale(a, row, sq, am, s, inv);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int k = 8 * (threadIdx.x + i * blockDim.x);
    if (k < a.K) norm_put(a, at, k, x[i], weight(k), s, inv);
  }
}

__global__ void __launch_bounds__(1024, 1) norm_quant_long_kernel(const NormArgs a) {
  __shared__ float red[2][32];
  const int row = blockIdx.x;
  const size_t at = (size_t)row * a.K;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  pdl_launch_dependents();
  pdl_wait();
  float sq = 0.f, am = 0.f;
  for (int k = 8 * threadIdx.x; k < a.K; k += 8 * blockDim.x) {
    const uint4 x = *reinterpret_cast<const uint4*>(a.x + at + k);
    const uint4 r = a.residual ? *reinterpret_cast<const uint4*>(a.residual + at + k) : zero;
    const uint4 g = a.gamma ? ld_plain(reinterpret_cast<const uint4*>(a.gamma + k)) : zero;
    norm_take(a, at, k, x, r, g, sq, am);
  }
  norm_reduce(sq, am, red);
  float s, r;
  norm_scale(a, row, sq, am, s, r);
  // (a thread reads back what it wrote itself)
  const __half* h = a.residual ? a.residual_out : a.x;
  for (int k = 8 * threadIdx.x; k < a.K; k += 8 * blockDim.x)
    norm_put(a, at, k, *reinterpret_cast<const uint4*>(h + at + k),
             a.gamma ? ld_plain(reinterpret_cast<const uint4*>(a.gamma + k)) : zero, s, r);
}

cudaError_t launch_norm_quant(const NormArgs& a, cudaStream_t s) {
  const int vecs = a.K / 8, v = ceil_div(vecs, kNormThreads);
  const int V = v == 3 ? 4 : v, threads = round_up(ceil_div(vecs, V), 32);
  const auto fn = V == 1 ? norm_quant_kernel<1> : V == 2 ? norm_quant_kernel<2> : norm_quant_kernel<4>;
  return V <= 4 ? launch_after(fn, a.M, threads, 0, s, 1, a) : launch_after(norm_quant_long_kernel, a.M, 1024, 0, s, 1, a);
}

}  // namespace dptq
