// kv4_cache.cu -- K and V rows into the paged 4-bit cache and back.
//
//   append: s = bf16(max|x| fl(1 / 7)) for each token and head, codes rint(x / s)
//   read:   binary16(s c)
// A bfloat16 scale has 8 significant bits and a code at most 3, so s c is a binary16 number (from s = 2^-17
// on, where binary16's own steps of 2^-24 begin to be coarser): what the cache stands for is the same in
// every kernel and format, and the scales cost half of fp32's bytes.
//
// Every token and head stands alone, so a group of D / 8 lanes takes a row of a head: 16-byte loads of
// binary16, 4-byte words of codes.  Bytes bound both for prompts, the launch for single tokens.
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv4_device.cuh"

namespace dptq {

constexpr int kRowThreads = 256;

// A vector of 8 values of the batch's rows: of token `row` of a sequence, K or V, a head, its place there.
struct Vec {
  int row, kv, head, at;
};
// Vector v of a sequence's rows, in the order of a token's K heads, its V heads, then the next token's.
template <int D>
__device__ __forceinline__ Vec vec_of(unsigned v, int kv_heads) {
  constexpr unsigned kVecs = D / 8;
  const unsigned item = v / kVecs, per = 2u * kv_heads, row = item / per, h = item - row * per;
  const int kv = h >= (unsigned)kv_heads;
  return {(int)row, kv, (int)h - kv * kv_heads, (int)(v % kVecs)};
}
// Where a row of codes (and its scale) of position p stands, in rows of the cache; -1: no such page.
__device__ __forceinline__ long long cache_row(const Kv8Args& c, int s, int p, int head) {
  const int b = load_page(c, s, p >> c.log2_page);
  return b < 0 ? -1 : ((((long long)b * c.kv_heads + head) << c.log2_page) + (p & ((1 << c.log2_page) - 1)));
}

template <int D, int V>   // V: vectors of a thread
__global__ void __launch_bounds__(kRowThreads) kv4_append_kernel(const Kv4RowsArgs a) {
  const Kv8Args& c = a.k.c;
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(c, blockIdx.y, q, threadIdx.x == 0 && blockIdx.x == 0)) return;
  const int first = max(-q.start, 0);
  const unsigned all = (unsigned)(max(q.n - first, 0)) * 2u * c.kv_heads * (D / 8);
  const unsigned v0 = blockIdx.x * (unsigned)(kRowThreads * V) + threadIdx.x;
  if (blockIdx.x * (unsigned)(kRowThreads * V) >= all) return;
  uint4 x[V];
  long long to[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    // (groups of lanes past the end read the last row: a load in a branch would wait for its own data)
    const unsigned v = v0 + i * kRowThreads, w = v < all ? v : all - (D / 8) + (v % (D / 8));
    const Vec p = vec_of<D>(w, c.kv_heads);
    const __half* src = (p.kv ? a.rows[1] : a.rows[0]) + (long long)(q.tok0 + first + p.row) * a.stride + p.head * D;
    x[i] = ld_plain(reinterpret_cast<const uint4*>(src) + p.at);
    to[i] = cache_row(c, blockIdx.y, q.start + first + p.row, p.head);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    __half2 am = __half2half2(__ushort_as_half(0));
#pragma unroll
    for (int e = 0; e < 4; ++e) am = __hmax2(am, __habs2(*reinterpret_cast<const __half2*>(&w[e])));
    float m = fmaxf(__low2float(am), __high2float(am));
#pragma unroll
    for (int o = D / 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const __nv_bfloat16 sb = __float2bfloat16_rn(__fmul_rn(m, 1.f / 7.f));
    const float s = __bfloat162float(sb), r = s > 0.f ? __frcp_rn(s) : 0.f;
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[e]));
      codes |= (uint32_t)(quant_code(f.x, s, r) & 15) << (8 * e);
      codes |= (uint32_t)(quant_code(f.y, s, r) & 15) << (8 * e + 4);
    }
    const unsigned v = v0 + i * kRowThreads;
    if (v >= all || to[i] < 0) continue;
    const Vec p = vec_of<D>(v, c.kv_heads);
    *reinterpret_cast<uint32_t*>((p.kv ? a.k.codes[1] : a.k.codes[0]) + to[i] * (D / 2) + 4 * p.at) = codes;
    if (p.at == 0) (p.kv ? a.k.scales[1] : a.k.scales[0])[to[i]] = __bfloat16_as_ushort(sb);
  }
}

template <int D, int V>
__global__ void __launch_bounds__(kRowThreads) kv4_read_kernel(const Kv4RowsArgs a) {
  const Kv8Args& c = a.k.c;
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(c, blockIdx.y, q, threadIdx.x == 0 && blockIdx.x == 0)) return;
  const int first = max(-q.start, 0);
  const unsigned all = (unsigned)(max(q.n - first, 0)) * 2u * c.kv_heads * (D / 8);
  const unsigned v0 = blockIdx.x * (unsigned)(kRowThreads * V) + threadIdx.x;
  if (blockIdx.x * (unsigned)(kRowThreads * V) >= all) return;
  long long from[V];
  uint32_t codes[V];
  uint16_t scale[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const unsigned v = v0 + i * kRowThreads;
    const Vec p = vec_of<D>(v < all ? v : all - 1, c.kv_heads);
    from[i] = cache_row(c, blockIdx.y, q.start + first + p.row, p.head);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const unsigned v = v0 + i * kRowThreads;
    const Vec p = vec_of<D>(v < all ? v : all - 1, c.kv_heads);
    const long long at = from[i] < 0 ? 0 : from[i];   // (a row that is there; nothing is written from it)
    codes[i] = ld_plain(reinterpret_cast<const uint32_t*>((p.kv ? a.k.codes[1] : a.k.codes[0]) + at * (D / 2)) + p.at);
    scale[i] = ld_plain((p.kv ? a.k.scales[1] : a.k.scales[0]) + at);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const unsigned v = v0 + i * kRowThreads;
    if (v >= all || from[i] < 0) continue;
    const Vec p = vec_of<D>(v, c.kv_heads);
    const float s = bf16_float(scale[i]);
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = s * (float)((int)(codes[i] << (28 - 4 * e)) >> 28);
    __half* dst = (p.kv ? a.rows[1] : a.rows[0]) + (long long)(q.tok0 + first + p.row) * a.stride + p.head * D;
    *(reinterpret_cast<uint4*>(dst) + p.at) =
        make_uint4(pack_half2(f[0], f[1]), pack_half2(f[2], f[3]), pack_half2(f[4], f[5]), pack_half2(f[6], f[7]));
  }
}

template <class Fn>
static cudaError_t launch_rows(Fn fn, const Kv4RowsArgs& a, int vecs, cudaStream_t s) {
  const long long all = (long long)a.k.c.max_tokens * 2 * a.k.c.kv_heads * (a.k.c.head_dim / 8);
  return launch_after(fn, dim3(ceil_div(all, (long long)kRowThreads * vecs), a.k.c.seqs), kRowThreads, 0, s, 1, a);
}

cudaError_t launch_kv4_append(const Kv4RowsArgs& a, int num_sms, cudaStream_t s) {
  return a.k.c.head_dim == 64 ? launch_rows(kv4_append_kernel<64, 1>, a, 1, s) : launch_rows(kv4_append_kernel<128, 1>, a, 1, s);
}
cudaError_t launch_kv4_read(const Kv4RowsArgs& a, int num_sms, cudaStream_t s) {
  return a.k.c.head_dim == 64 ? launch_rows(kv4_read_kernel<64, 1>, a, 1, s) : launch_rows(kv4_read_kernel<128, 1>, a, 1, s);
}

}  // namespace dptq
