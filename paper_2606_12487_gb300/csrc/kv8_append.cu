// kv8_append.cu -- new K and V rows into a paged cache of int8 codes, one scale for each page
// and head.  A page keeps the scale of its largest value: new rows quantize with
// s1 = max(s0, max|x| fl(1 / 127)), s0 the scale of the page's earlier rows, whose codes are
// rescaled, rint(c s0 / s1), where s1 is larger.
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv8_device.cuh"

namespace dptq {

constexpr int kAppendThreads = 128;

__global__ void __launch_bounds__(kAppendThreads) kv8_append_kernel(const Kv8AppendArgs a) {
  __shared__ float red[kAppendThreads / 32];
  const Kv8Args& c = a.c;
  const int tid = threadIdx.x, kv = blockIdx.y & 1, head = blockIdx.y >> 1, D = c.head_dim, P = 1 << c.log2_page;
  Seq q;
  if (!load_seq(c, blockIdx.z, q, tid == 0 && blockIdx.x == 0 && blockIdx.y == 0) || q.len == 0 || q.n == 0) return;
  const int first = q.start > 0 ? q.start : 0;             // position of the first stored row
  const int page = (first >> c.log2_page) + blockIdx.x;
  const int p0 = page << c.log2_page;
  if (p0 >= q.len) return;
  const int lo = first > p0 ? first - p0 : 0;              // rows of the page: earlier ones below lo,
  const int hi = q.len - p0 < P ? q.len - p0 : P;          // new ones up to hi
  const int blk = load_page(c, blockIdx.z, page);
  if (blk < 0) return;
  const __half* src = a.rows[kv] + (size_t)(q.tok0 + p0 - q.start) * a.stride + (size_t)head * D;
  int8_t* dst = c.codes[kv] + ((size_t)blk * c.kv_heads + head) * P * D;
  float* scale = c.scales[kv] + (size_t)blk * c.kv_heads + head;
  float am = 0.f;
  for (int i = lo * D + tid; i < hi * D; i += kAppendThreads)
    am = fmaxf(am, fabsf(__half2float(src[(long long)(i / D) * a.stride + i % D])));
  for (int o = 16; o > 0; o >>= 1) am = fmaxf(am, __shfl_xor_sync(0xffffffffu, am, o));
  if ((tid & 31) == 0) red[tid >> 5] = am;
  const float s0 = lo > 0 ? *scale : 0.f;
  __syncthreads();
  for (int w = 0; w < kAppendThreads / 32; ++w) am = fmaxf(am, red[w]);
  const float s1 = fmaxf(s0, __fmul_rn(am, 1.f / 127.f));
  if (s1 > s0)
    for (int i = tid; i < lo * D; i += kAppendThreads) dst[i] = (int8_t)quant_code(__fmul_rn((float)dst[i], s0), s1);
  for (int i = lo * D + tid; i < hi * D; i += kAppendThreads)
    dst[i] = (int8_t)quant_code(__half2float(src[(long long)(i / D) * a.stride + i % D]), s1);
  if (tid == 0) *scale = s1;
}

cudaError_t launch_kv8_append(const Kv8AppendArgs& a, cudaStream_t s) {
  const int pages = ((a.c.max_tokens - 1) >> a.c.log2_page) + 2;
  kv8_append_kernel<<<dim3(pages, 2 * a.c.kv_heads, a.c.seqs), kAppendThreads, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace dptq
