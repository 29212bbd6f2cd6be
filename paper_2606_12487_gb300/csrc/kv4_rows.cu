// kv4_rows.cu -- attention over the paged 4-bit cache: a warp a row of a query head, one pass over the keys with
// the running maximum and sum in fp32.
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv4_device.cuh"

namespace dptq {

template <int D>
__global__ void __launch_bounds__(256) kv4_rows_kernel(const Kv4AttendArgs A) {
  constexpr int E = D / 32;
  const Kv8Args& c = A.k.c;
  const int lane = threadIdx.x & 31, head = blockIdx.z, row = blockIdx.x * 8 + (threadIdx.x >> 5);
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(c, blockIdx.y, q, threadIdx.x == 0 && blockIdx.x == 0 && head == 0) || row >= q.n) return;
  const int pos = q.start + row, P1 = (1 << c.log2_page) - 1, kvh = head / A.group;
  const __half* src = A.q + (size_t)(q.tok0 + row) * A.q_stride + (size_t)head * D + E * lane;
  float x[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = __half2float(ld_plain(src + e)), o[e] = 0.f;
  for (int j = 0; j <= pos; ++j) {
    if (!kv8_sees(pos, j, A.window, A.sinks)) {
      j = max(j, pos - A.window);
      continue;
    }
    const int b = load_page(c, blockIdx.y, j >> c.log2_page);
    if (b < 0) continue;
    const size_t at = (((size_t)b * c.kv_heads + kvh) << c.log2_page) + (j & P1);
    float k[E], v[E];
    const float sk = bf16_float(ld_plain(A.k.scales[0] + at)), sv = bf16_float(ld_plain(A.k.scales[1] + at));
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const int w = ld_plain(A.k.codes[kv] + at * (D / 2) + (E * lane + e) / 2);
        (kv ? v : k)[e] = (float)((w << 28) >> 28);
        (kv ? v : k)[e + 1] = (float)((w << 24) >> 28);
      }
    float t = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) t = fmaf(x[e], k[e], t);
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) t += __shfl_xor_sync(0xffffffffu, t, w);
    t *= isfinite(sk) && isfinite(sv) ? sk * A.scale : NAN;
    const float mn = t > m ? t : m, f = m == -INFINITY ? 0.f : __expf(m - mn), p = t == -INFINITY ? 0.f : __expf(t - mn);
    m = mn;
    l = fmaf(l, f, p);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(o[e], f, p * (isfinite(sv) ? sv * v[e] : 0.f));
  }
  __half* dst = A.out + (size_t)(q.tok0 + row) * A.out_stride + (size_t)head * D + E * lane;
#pragma unroll
  for (int e = 0; e < E; ++e) dst[e] = __float2half_rn(l == 0.f ? 0.f : o[e] / l);
}

cudaError_t launch_kv4_rows(const Kv4AttendArgs& a, int num_sms, cudaStream_t s) {
  const dim3 grid(ceil_div(a.k.c.max_tokens, 8), a.k.c.seqs, a.q_heads);
  return a.k.c.head_dim == 64 ? launch_after(kv4_rows_kernel<64>, grid, 256, 0, s, 1, a)
                              : launch_after(kv4_rows_kernel<128>, grid, 256, 0, s, 1, a);
}

}  // namespace dptq
