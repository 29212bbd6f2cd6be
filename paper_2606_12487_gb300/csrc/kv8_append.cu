// kv8_append.cu -- new K and V rows into a paged cache of int8 codes, one scale for each page
// and head.  A page keeps the scale of its largest value: new rows quantize with
// s1 = max(s0, max|x| fl(1 / 127)), s0 the scale of the page's earlier rows, whose codes are
// rescaled, rint(fl(c s0) / s1), where s1 is larger.
//
// Two bytes in, one out: bytes bound it for prompts, the launch for single tokens.
//   * Prompts: a CTA takes a page of one head (of K or V): 16-byte loads, all of a thread's
//     four before the first is used, the maximum, 8-byte stores.  Neighbouring CTAs take
//     neighbouring heads, whose rows stand side by side in a token.
//   * Few tokens a sequence (kAppendFew at most): a warp takes a (sequence, head), its pages one
//     after the other; with a CTA a page almost all of its threads would have no row.
// Four prompts up to 2048 tokens, 8 heads of 128 (39.6 MB): 9.4 us in a graph, 4.2 TB/s; one token of each of 32
// sequences, 32 heads: 2.6 us (a CTA a page for those too: 8.2 against 5.6 us a call).
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv8_device.cuh"

namespace dptq {

constexpr int kAppendVecs = 4;    // 16-byte vectors of a thread
constexpr int kAppendFew = 8;     // (8 tokens of each of 128 sequences, 32 heads: 7.3 us a call; a CTA a page: 30.8)

// The new rows of a page of a sequence.
struct PageRows {
  int p0;         // the page's first position
  int lo, hi;     // its rows: earlier ones below lo, new ones up to hi
};
__device__ __forceinline__ PageRows page_rows(const Seq& q, int first, int page, int log2_page) {
  const int p0 = page << log2_page, P = 1 << log2_page;
  return {p0, first > p0 ? first - p0 : 0, q.len - p0 < P ? q.len - p0 : P};
}
// The largest |x| so far, two binary16 side by side (a NaN loses against a number).
__device__ __forceinline__ __half2 abs_max8(const uint4& v, __half2 am) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) am = __hmax2(am, __habs2(*reinterpret_cast<const __half2*>(&w[e])));
  return am;
}
__device__ __forceinline__ float widest(__half2 am) { return fmaxf(__low2float(am), __high2float(am)); }
__device__ __forceinline__ uint2 pack_codes(const int (&c)[8]) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e >> 2] |= (uint32_t)(c[e] & 0xFF) << (8 * (e & 3));
  return make_uint2(w[0], w[1]);
}
// Eight codes as quant_code makes them, two values an instruction: t = x r + 1.5 2^23 holds
// rint(x r) in its low byte, and x r - rint(x r), from one fma, says whether the quotient itself has to
// decide (or a NaN has turned up).  One value at a time took 12.0 us in a graph for four prompts
// (39.6 MB), this takes 9.4 us.
__device__ __forceinline__ uint2 quant8(const uint4& v, float s, float r) {
  constexpr float kMagic = 12582912.f;   // 1.5 2^23
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  const uint64_t r2 = f2_pack(r, r), magic = f2_pack(kMagic, kMagic), n2 = f2_pack(-r, -r);
  float t[8], d = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[e]));
    const uint64_t x2 = f2_pack(f.x, f.y), t2 = f2_fma(x2, r2, magic);
    float d0, d1;
    f2_unpack(f2_fma(x2, n2, f2_sub(t2, magic)), d0, d1);   // rint(x r) - x r
    asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(d) : "f"(fabsf(d0)), "f"(fabsf(d1)));
    f2_unpack(t2, t[2 * e], t[2 * e + 1]);
  }
  if (!(d < 0.5f - 0x1p-15f)) {
    int c[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[e]));
      c[2 * e] = quant_code(f.x, s, r);
      c[2 * e + 1] = quant_code(f.y, s, r);
    }
    return pack_codes(c);
  }
  uint32_t b[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] = __byte_perm(__float_as_uint(t[2 * e]), __float_as_uint(t[2 * e + 1]), 0x0040);
  return make_uint2(__byte_perm(b[0], b[1], 0x5410), __byte_perm(b[2], b[3], 0x5410));
}
__device__ __forceinline__ uint2 rescale8(const uint2& v, float s0, float s1, float r) {
  int c[8];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    c[e] = quant_code(__fmul_rn((float)(int8_t)((e < 4 ? v.x : v.y) >> (8 * (e & 3))), s0), s1, r);
  return pack_codes(c);
}

__global__ void __launch_bounds__(512, 3) kv8_append_pages_kernel(const Kv8AppendArgs a) {
  __shared__ float red[16];
  const Kv8Args& c = a.c;
  const int tid = threadIdx.x, kv = blockIdx.x & 1, head = blockIdx.x >> 1;
  const int vecs = c.head_dim / 8, log2v = c.head_dim == 64 ? 3 : 4;   // vectors of a row
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(c, blockIdx.z, q, tid == 0 && blockIdx.x == 0 && blockIdx.y == 0) || q.len == 0 || q.n == 0) return;
  const int first = q.start > 0 ? q.start : 0, page = (first >> c.log2_page) + blockIdx.y;
  if (page << c.log2_page >= q.len) return;
  const PageRows pr = page_rows(q, first, page, c.log2_page);
  // (looked at after the rows are asked for)
  const int entry = ld_plain(c.table + (long long)blockIdx.z * c.table_stride + page);
  const __half* src = (kv ? a.rows[1] : a.rows[0]) + (q.tok0 + pr.p0 - (long long)q.start) * a.stride +
                      (size_t)head * c.head_dim;
  uint4 x[kAppendVecs];
  __half2 am2 = __half2half2(__ushort_as_half(0));
#pragma unroll
  for (int i = 0; i < kAppendVecs; ++i) {
    // (always a row that is there: a load in a branch would wait for its own data; rows twice do
    // not change the maximum)
    const int v = tid + i * blockDim.x, row = min(max(v >> log2v, pr.lo), pr.hi - 1);
    x[i] = ld_plain(reinterpret_cast<const uint4*>(src + row * a.stride) + (v & (vecs - 1)));
  }
  if (entry < 0 || entry >= c.num_blocks) {
    atomicCAS(c.bad, 0, kDevBadPage);
    return;
  }
  const size_t hb = (size_t)entry * c.kv_heads + head;
  int8_t* dst = (kv ? c.codes[1] : c.codes[0]) + (hb << c.log2_page) * c.head_dim;
  float* scale = (kv ? c.scales[1] : c.scales[0]) + hb;
  const float s0 = pr.lo > 0 ? *scale : 0.f;
#pragma unroll
  for (int i = 0; i < kAppendVecs; ++i) am2 = abs_max8(x[i], am2);
  float am = widest(am2);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) am = fmaxf(am, __shfl_xor_sync(0xffffffffu, am, o));
  if ((tid & 31) == 0) red[tid >> 5] = am;
  __syncthreads();   // (every thread has read s0 as well)
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) am = fmaxf(am, red[w]);
  const float s1 = fmaxf(s0, __fmul_rn(am, 1.f / 127.f)), r = s1 > 0.f ? __frcp_rn(s1) : 0.f;
#pragma unroll
  for (int i = 0; i < kAppendVecs; ++i) {
    const int v = tid + i * blockDim.x, row = v >> log2v;
    uint2* p = reinterpret_cast<uint2*>(dst) + v;
    if (row >= pr.lo && row < pr.hi)
      *p = quant8(x[i], s1, r);
    else if (row < pr.lo && s1 > s0)
      *p = rescale8(*p, s0, s1, r);
  }
  if (tid == 0) *scale = s1;
}

__global__ void __launch_bounds__(256) kv8_append_few_kernel(const Kv8AppendArgs a) {
  const Kv8Args& c = a.c;
  const int lane = threadIdx.x & 31, item = blockIdx.x * 8 + (threadIdx.x >> 5), kv = item & 1, head = item >> 1;
  const int vecs = c.head_dim / 8, log2v = c.head_dim == 64 ? 3 : 4;
  if (head >= c.kv_heads) return;
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(c, blockIdx.y, q, lane == 0 && item == 0) || q.len == 0 || q.n == 0) return;
  const int first = q.start > 0 ? q.start : 0, per = 32 >> log2v;   // rows side by side in the warp
  for (int page = first >> c.log2_page; page << c.log2_page < q.len; ++page) {
    const PageRows pr = page_rows(q, first, page, c.log2_page);
    const int blk = load_page(c, blockIdx.y, page);
    if (blk < 0) continue;
    const size_t hb = (size_t)blk * c.kv_heads + head;
    const __half* src = (kv ? a.rows[1] : a.rows[0]) + (q.tok0 + pr.p0 - (long long)q.start) * a.stride +
                        (size_t)head * c.head_dim;
    uint2* dst = reinterpret_cast<uint2*>((kv ? c.codes[1] : c.codes[0]) + (hb << c.log2_page) * c.head_dim);
    float* scale = (kv ? c.scales[1] : c.scales[0]) + hb;
    const float s0 = pr.lo > 0 ? *scale : 0.f;
    constexpr int kRounds = kAppendFew / 2;   // (at least two rows a round)
    uint4 x[kRounds];
    __half2 am2 = __half2half2(__ushort_as_half(0));
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int row = min(pr.lo + i * per + (lane >> log2v), pr.hi - 1);   // (a row that is there)
      x[i] = ld_plain(reinterpret_cast<const uint4*>(src + row * a.stride) + (lane & (vecs - 1)));
    }
#pragma unroll
    for (int i = 0; i < kRounds; ++i) am2 = abs_max8(x[i], am2);
    float am = widest(am2);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) am = fmaxf(am, __shfl_xor_sync(0xffffffffu, am, o));
    const float s1 = fmaxf(s0, __fmul_rn(am, 1.f / 127.f)), r = s1 > 0.f ? __frcp_rn(s1) : 0.f;
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      const int row = pr.lo + i * per + (lane >> log2v);
      if (row < pr.hi) dst[(row << log2v) + (lane & (vecs - 1))] = quant8(x[i], s1, r);
    }
    if (s1 > s0)
      for (int v = lane; v < pr.lo << log2v; v += 32) dst[v] = rescale8(dst[v], s0, s1, r);
    __syncwarp();
    if (lane == 0) *scale = s1;
  }
}

cudaError_t launch_kv8_append(const Kv8AppendArgs& a, cudaStream_t s) {
  if (a.c.max_tokens <= kAppendFew)
    return launch_after(kv8_append_few_kernel, dim3(ceil_div(2 * a.c.kv_heads, 8), a.c.seqs), 256, 0, s, 1, a);
  const int pages = ((a.c.max_tokens - 1) >> a.c.log2_page) + 2;
  const int threads = (a.c.head_dim << a.c.log2_page) / (8 * kAppendVecs);   // 32 to 512
  return launch_after(kv8_append_pages_kernel, dim3(2 * a.c.kv_heads, pages, a.c.seqs), threads, 0, s, 1, a);
}

}  // namespace dptq
