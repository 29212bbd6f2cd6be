// norm_quant.cu -- residual addition, RMS norm and the per-token symmetric quantizer in one
// kernel: what the projections that read the residual stream take as their codes.
//   h = fp16(x + r),  p_k = h_k g_k,  s' = max|p| fl(1 / qmax),  c_k = rint(p_k / s'),
//   scale = s' / sqrt(mean(h^2) + eps).
// p is exact in fp32 (11 + 11 bits), and the norm's factor is one positive number for the
// whole token, so it goes into the scale alone: the codes are a function of h and g, whatever
// order the squares are summed in.
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "dptq_internal.h"

namespace dptq {

constexpr int kNormThreads = 256;

__global__ void __launch_bounds__(kNormThreads) norm_quant_kernel(const NormArgs a) {
  __shared__ float red[2][kNormThreads / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const size_t row = (size_t)blockIdx.x * a.K;
  const __half* h = a.residual ? a.residual_out : a.x;
  float sq = 0.f, am = 0.f;
  for (int k = tid; k < a.K; k += kNormThreads) {
    float v = __half2float(a.x[row + k]);
    if (a.residual) {
      const __half u = __float2half_rn(v + __half2float(a.residual[row + k]));
      a.residual_out[row + k] = u;
      v = __half2float(u);
    }
    sq = fmaf(v, v, sq);
    am = fmaxf(am, fabsf(a.gamma ? v * __half2float(a.gamma[k]) : v));
  }
  for (int o = 16; o > 0; o >>= 1) {
    sq += __shfl_xor_sync(0xffffffffu, sq, o);
    am = fmaxf(am, __shfl_xor_sync(0xffffffffu, am, o));
  }
  if (lane == 0) red[0][warp] = sq, red[1][warp] = am;
  __syncthreads();
  sq = 0.f;
  am = 0.f;
  for (int w = 0; w < kNormThreads / 32; ++w) sq += red[0][w], am = fmaxf(am, red[1][w]);
  const float s = __fmul_rn(am, a.bits == 4 ? 1.f / 7.f : 1.f / 127.f);
  if (tid == 0) a.scales[blockIdx.x] = s * __frcp_rn(__fsqrt_rn(__fdiv_rn(sq, (float)a.K) + a.eps));
  for (int k = 2 * tid; k < a.K; k += 2 * kNormThreads) {
    int c[2];
    for (int e = 0; e < 2; ++e) {
      const float v = __half2float(h[row + k + e]);
      const float p = a.gamma ? v * __half2float(a.gamma[k + e]) : v;
      c[e] = s > 0.f ? __float2int_rn(__fdiv_rn(p, s)) : 0;
    }
    if (a.bits == 4) {
      a.codes[(row + k) / 2] = (uint8_t)((c[0] & 15) | ((c[1] & 15) << 4));
    } else {
      a.codes[row + k] = (uint8_t)c[0];
      a.codes[row + k + 1] = (uint8_t)c[1];
    }
  }
}

cudaError_t launch_norm_quant(const NormArgs& a, int num_sms, cudaStream_t s) {
  (void)num_sms;
  norm_quant_kernel<<<a.M, kNormThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace dptq
