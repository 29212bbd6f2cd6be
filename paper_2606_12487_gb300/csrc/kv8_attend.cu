// kv8_attend.cu -- causal attention over the paged int8 cache.
//   logit_j = scale sk[page of j] (q . ck_j),  out = sum_j softmax(logit)_j sv[page of j] cv_j
// over the keys that the query sees; zero where it sees none.  Running maximum, sum and
// weighted values in fp32.
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv8_device.cuh"

namespace dptq {

constexpr int kAttendWarps = 4;

// One CTA per (new token, query head): the warps take every fourth key, a lane D / 32 dims.
template <int D>
__global__ void __launch_bounds__(kAttendWarps * 32) kv8_attend_kernel(const Kv8AttendArgs a) {
  constexpr int E = D / 32;
  __shared__ float sm[kAttendWarps], sl[kAttendWarps], so[kAttendWarps][D];
  const Kv8Args& c = a.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, head = blockIdx.y, kvh = head / a.group;
  Seq q;
  if (!load_seq(c, blockIdx.z, q, threadIdx.x == 0 && blockIdx.x == 0 && head == 0) || (int)blockIdx.x >= q.n) return;
  const int pos = q.start + blockIdx.x;
  const size_t tok = q.tok0 + blockIdx.x;
  float qv[E], o[E], m = -INFINITY, l = 0.f;
  for (int e = 0; e < E; ++e) {
    qv[e] = __half2float(a.q[tok * a.q_stride + (size_t)head * D + lane * E + e]);
    o[e] = 0.f;
  }
  for (int j = warp; j <= pos; j += kAttendWarps) {
    if (!kv8_sees(pos, j, a.window, a.sinks)) continue;
    const int blk = load_page(c, blockIdx.z, j >> c.log2_page);
    if (blk < 0) continue;
    const size_t hb = (size_t)blk * c.kv_heads + kvh;
    const size_t row = ((hb << c.log2_page) + (j & ((1 << c.log2_page) - 1))) * D + lane * E;
    float d = 0.f;
    for (int e = 0; e < E; ++e) d = fmaf(qv[e], (float)c.codes[0][row + e], d);
    for (int w = 16; w > 0; w >>= 1) d += __shfl_xor_sync(0xffffffffu, d, w);
    d *= a.scale * c.scales[0][hb];
    const float mn = fmaxf(m, d), f = m == -INFINITY ? 0.f : expf(m - mn), p = expf(d - mn), pv = p * c.scales[1][hb];
    l = l * f + p;
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + pv * (float)c.codes[1][row + e];
    m = mn;
  }
  if (lane == 0) sm[warp] = m, sl[warp] = l;
  for (int e = 0; e < E; ++e) so[warp][lane * E + e] = o[e];
  __syncthreads();
  if (warp == 0) {
    float M = -INFINITY, L = 0.f;
    for (int w = 0; w < kAttendWarps; ++w) M = fmaxf(M, sm[w]);
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    for (int w = 0; w < kAttendWarps; ++w) {
      if (sl[w] == 0.f) continue;
      const float f = expf(sm[w] - M);
      L += f * sl[w];
      for (int e = 0; e < E; ++e) o[e] += f * so[w][lane * E + e];
    }
    for (int e = 0; e < E; ++e)
      a.out[tok * a.out_stride + (size_t)head * D + lane * E + e] = __float2half_rn(L == 0.f ? 0.f : o[e] / L);
  }
}

cudaError_t launch_kv8_attend(const Kv8AttendArgs& a, int num_sms, cudaStream_t s) {
  (void)num_sms;
  const dim3 grid(a.c.max_tokens, a.q_heads, a.c.seqs);
  if (a.c.head_dim == 64)
    kv8_attend_kernel<64><<<grid, kAttendWarps * 32, 0, s>>>(a);
  else
    kv8_attend_kernel<128><<<grid, kAttendWarps * 32, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace dptq
