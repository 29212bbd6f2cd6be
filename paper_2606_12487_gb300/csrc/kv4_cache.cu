// kv4_cache.cu -- K and V rows into the paged 4-bit cache and back.
//
//   append: s = bf16(max|x| fl(1 / 7)) for each token and head, codes rint(x / s)
//   read:   binary16(s c)
// A bfloat16 scale has 8 significant bits and a code at most 3, so s c is a binary16 number (from s = 2^-17
// on, where binary16's own steps of 2^-24 begin to be coarser): what the cache stands for is the same in
// every kernel and format, and the scales cost half of fp32's bytes.
//
// Every token and head stands alone, so a group of D / 8 lanes takes a row of a head: 16-byte loads of
// binary16, 4-byte words of codes.  Bytes bound both for prompts, the launch for single tokens.  A thread keeps its place
// in a token (K or V, head, 8 values) and takes V tokens one after the other, all of them asked for before the first is
// used: their pages are two at most.
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv4_device.cuh"

namespace dptq {

constexpr int kRowThreads = 256;
constexpr int kRowTokens = 8;   // tokens of a thread, of prompts

// What a thread works on: place `at` of a row of a head, K or V, and its tokens row0 + i step, i < V, of the sequence's
// rows (rows past the last one are not there).
struct Work {
  int kv, head, at, row0, step, end;
};
// False for threads without work (whole groups of lanes).
template <int D, int V>
__device__ __forceinline__ bool work_of(const Kv8Args& c, const Seq& q, Work& w) {
  constexpr int kVecs = D / 8;
  const int items = 2 * c.kv_heads * kVecs, side = items < kRowThreads ? kRowThreads / items : 1;   // tokens side by side
  const int t = items < kRowThreads ? threadIdx.x / items : 0;
  const int item = items < kRowThreads ? threadIdx.x - t * items : blockIdx.x * kRowThreads + threadIdx.x;
  const int h = item / kVecs;
  w.at = item % kVecs;
  w.kv = h >= c.kv_heads;
  w.head = h - w.kv * c.kv_heads;
  w.step = side;
  w.row0 = max(-q.start, 0) + blockIdx.z * side * V + t;   // (rows at negative positions come first)
  w.end = q.n;
  return item < items && t < side && w.row0 < w.end;
}
// Where the rows of codes (and the scales) of its tokens stand, in rows of the cache; -1: no such page.
template <int V>
__device__ __forceinline__ void cache_rows(const Kv8Args& c, const Seq& q, const Work& w, long long (&to)[V]) {
  int entry[V];
#pragma unroll
  for (int i = 0; i < V; ++i)   // (all asked for before the first is looked at)
    entry[i] = ld_plain(c.table + (long long)blockIdx.y * c.table_stride +
                        ((q.start + min(w.row0 + i * w.step, w.end - 1)) >> c.log2_page));
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int p = q.start + min(w.row0 + i * w.step, w.end - 1);
    const bool held = entry[i] >= 0 && entry[i] < c.num_blocks;
    if (!held) atomicCAS(c.bad, 0, kDevBadPage);
    to[i] = held ? ((((long long)entry[i] * c.kv_heads + w.head) << c.log2_page) + (p & ((1 << c.log2_page) - 1))) : -1;
  }
}

// Eight codes of a row, a nibble each.
__device__ __forceinline__ uint32_t quant8_nibbles(const uint4& v, float s, float r) {
  float t[8];
  uint32_t codes = 0;
  if (rounded8(v, r, t)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) codes |= (__float_as_uint(t[e]) & 15u) << (4 * e);
    return codes;
  }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll 1
  for (int e = 0; e < 8; ++e) {
    const uint32_t h = (e < 4 ? (e < 2 ? w[0] : w[1]) : (e < 6 ? w[2] : w[3])) >> (16 * (e & 1));
    codes |= (uint32_t)(quant_code(__half2float(__ushort_as_half((unsigned short)h)), s, r) & 15) << (4 * e);
  }
  return codes;
}

template <int D, int V>
__global__ void __launch_bounds__(kRowThreads) kv4_append_kernel(const Kv4RowsArgs a) {
  const Kv8Args& c = a.k.c;
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(c, blockIdx.y, q, threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.z == 0)) return;
  Work w;
  const bool on = work_of<D, V>(c, q, w);
  const unsigned lanes = __ballot_sync(0xffffffffu, on);
  if (!on) return;
  const __half* src = (w.kv ? a.rows[1] : a.rows[0]) + (long long)q.tok0 * a.stride + w.head * D + 8 * w.at;
  uint4 x[V];
#pragma unroll
  for (int i = 0; i < V; ++i)   // (past the last row it once more: a load in a branch would wait for its own data)
    x[i] = ld_plain(reinterpret_cast<const uint4*>(src + min(w.row0 + i * w.step, w.end - 1) * a.stride));
  long long to[V];
  cache_rows(c, q, w, to);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float m = widest(abs_max8(x[i], __half2half2(__ushort_as_half(0))));
#pragma unroll
    for (int o = D / 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(lanes, m, o));
    const __nv_bfloat16 sb = __float2bfloat16_rn(__fmul_rn(m, 1.f / 7.f));
    const float s = __bfloat162float(sb);
    const uint32_t codes = quant8_nibbles(x[i], s, s > 0.f ? __frcp_rn(s) : 0.f);
    if (w.row0 + i * w.step < w.end && to[i] >= 0) {
      *reinterpret_cast<uint32_t*>((w.kv ? a.k.codes[1] : a.k.codes[0]) + to[i] * (D / 2) + 4 * w.at) = codes;
      if (w.at == 0) (w.kv ? a.k.scales[1] : a.k.scales[0])[to[i]] = __bfloat16_as_ushort(sb);
    }
  }
}

template <int D, int V>
__global__ void __launch_bounds__(kRowThreads) kv4_read_kernel(const Kv4RowsArgs a) {
  const Kv8Args& c = a.k.c;
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(c, blockIdx.y, q, threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.z == 0)) return;
  Work w;
  if (!work_of<D, V>(c, q, w)) return;
  long long from[V];
  cache_rows(c, q, w, from);
  const uint8_t* src = (w.kv ? a.k.codes[1] : a.k.codes[0]) + 4 * w.at;
  const uint16_t* scales = w.kv ? a.k.scales[1] : a.k.scales[0];
  uint32_t codes[V];
  uint16_t scale[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const long long at = from[i] < 0 ? 0 : from[i];   // (a row that is there; nothing is written from it)
    codes[i] = ld_plain(reinterpret_cast<const uint32_t*>(src + at * (D / 2)));
    scale[i] = ld_plain(scales + at);
  }
  __half* dst = (w.kv ? a.rows[1] : a.rows[0]) + (long long)q.tok0 * a.stride + w.head * D + 8 * w.at;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int row = w.row0 + i * w.step;
    const float s = bf16_float(scale[i]);
    const uint4 v = kv4_tiny(scale[i]) || kv4_bad(scale[i]) ? widen8_slow(codes[i], s) : widen8(codes[i], __float2half2_rn(s));
    if (row < w.end && from[i] >= 0)   // (from the order 0 4, 1 5, 2 6, 3 7)
      *reinterpret_cast<uint4*>(dst + row * a.stride) =
          make_uint4(__byte_perm(v.x, v.y, 0x5410), __byte_perm(v.z, v.w, 0x5410), __byte_perm(v.x, v.y, 0x7632),
                     __byte_perm(v.z, v.w, 0x7632));
  }
}

template <int V, class Fn>
static cudaError_t launch_rows(Fn fn, const Kv4RowsArgs& a, cudaStream_t s) {
  const int items = 2 * a.k.c.kv_heads * (a.k.c.head_dim / 8), side = items < kRowThreads ? kRowThreads / items : 1;
  return launch_after(fn, dim3(ceil_div(items, kRowThreads), a.k.c.seqs, ceil_div(a.k.c.max_tokens, side * V)), kRowThreads, 0,
                      s, 1, a);
}

cudaError_t launch_kv4_append(const Kv4RowsArgs& a, cudaStream_t s) {
  const bool few = a.k.c.max_tokens < kRowTokens;
  if (a.k.c.head_dim == 64) return few ? launch_rows<1>(kv4_append_kernel<64, 1>, a, s) : launch_rows<kRowTokens>(kv4_append_kernel<64, kRowTokens>, a, s);
  return few ? launch_rows<1>(kv4_append_kernel<128, 1>, a, s) : launch_rows<kRowTokens>(kv4_append_kernel<128, kRowTokens>, a, s);
}
cudaError_t launch_kv4_read(const Kv4RowsArgs& a, cudaStream_t s) {
  const bool few = a.k.c.max_tokens < kRowTokens;
  if (a.k.c.head_dim == 64) return few ? launch_rows<1>(kv4_read_kernel<64, 1>, a, s) : launch_rows<kRowTokens>(kv4_read_kernel<64, kRowTokens>, a, s);
  return few ? launch_rows<1>(kv4_read_kernel<128, 1>, a, s) : launch_rows<kRowTokens>(kv4_read_kernel<128, kRowTokens>, a, s);
}

}  // namespace dptq
