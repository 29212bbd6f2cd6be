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
// used.
// Four prompts up to 2048 tokens, 8 heads of 128 (27.6 MB): append 10.6, read 8.7 us in a graph (floor 4.1: lengths, table and rows are three
// latencies in a row); a token of each of 32 sequences, 32 heads: 2.4 and 2.7 us.  Read of 32 sequences up to 4096 tokens, 32 heads (1.45
// GB): 244 us, 5.9 TB/s.
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv4_device.cuh"

namespace dptq {

constexpr int kRowThreads = 256;
// Tokens of a thread, of prompts: append of the four 12.9 / 10.6 / 11.7 / 11.7 us with 1 / 2 / 4 / 8; read with 4 / 8 / 16 of them 8.7 / 9.3 /
// 9.4, of three sequences up to 1500 tokens, 8 heads 6.5 / 6.5 / 7.8, of the 32 sequences 244 / 244 / 237.
constexpr int kAppendTokens = 2, kReadTokens = 4;

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
// Where the rows of codes (and the scales) of its tokens stand, in rows of the cache (fewer than 2^32, checked on the host);
// returns the tokens that are there and have a page, a bit each (the others' row is one that is there).
template <int V>
__device__ __forceinline__ uint32_t cache_rows(const Kv8Args& c, const Seq& q, const Work& w, uint32_t (&to)[V]) {
  const int* table = c.table + (long long)blockIdx.y * c.table_stride;
  const int p0 = q.start + w.row0, last = q.start + w.end - 1;
  int entry[V];
#pragma unroll
  for (int i = 0; i < V; ++i) entry[i] = ld_plain(table + (min(p0 + i * w.step, last) >> c.log2_page));   // (all before the first is looked at)
  uint32_t held = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int p = p0 + i * w.step;
    const bool ok = (unsigned)entry[i] < (unsigned)c.num_blocks;
    if (!ok) atomicCAS(c.bad, 0, kDevBadPage);
    if (ok && p <= last) held |= 1u << i;
    to[i] = ok ? (((unsigned)entry[i] * c.kv_heads + w.head) << c.log2_page) + (min(p, last) & ((1 << c.log2_page) - 1)) : 0u;
  }
  return held;
}

// Eight codes rint(x / s) of a row, a nibble each; r = 1 / s within a unit in its last place.
// Exact ties are common (x = (k + 1/2) s with x of 11 bits and s of 8), and nothing else comes near one: with x = X 2^a,
// s = S 2^b a quotient that is no tie differs from k + 1/2 by a multiple of 2^min(a + 1, b) / (2 S 2^b), that is by 1 / 2 S > 2^-9,
// or, where a + 1 < b, by 2^(a - b) / S, and 2^(a - b) > 0.4 S / X next to a tie: by more than 0.4 / X > 2^-12.4.  x r is
// within 2^-19 of the quotient, which is 7.03 at most.  So x r rounded to a multiple of 2^-13 is the tie itself where there
// is one and on the quotient's side of it elsewhere, and rint of that is rint of the quotient.  (With a check for near ties and a
// division behind it, two of three warps divided, and the append of four prompts took 16 us in a graph instead of 11.)
// nan: one of the values is.
__device__ __forceinline__ uint32_t quant8_nibbles(const uint4& v, float s, float r, bool nan) {
  constexpr float kGrid = 1536.f, kMagic = 12582912.f;   // 1.5 2^10 and 1.5 2^23, where fp32 has steps of 2^-13 and 1
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t t[8];
  const uint64_t r2 = f2_pack(r, r), grid = f2_pack(kGrid, kGrid), magic = f2_pack(kMagic, kMagic);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[e]));
    float a, b;
    f2_unpack(f2_add(f2_sub(f2_fma(f2_pack(f.x, f.y), r2, grid), grid), magic), a, b);
    t[2 * e] = __float_as_uint(a);
    t[2 * e + 1] = __float_as_uint(b);
  }
  const uint32_t even = __byte_perm(__byte_perm(t[0], t[2], 0x0040), __byte_perm(t[4], t[6], 0x0040), 0x5410);
  const uint32_t odd = __byte_perm(__byte_perm(t[1], t[3], 0x0040), __byte_perm(t[5], t[7], 0x0040), 0x5410);
  uint32_t codes = (even & 0x0F0F0F0Fu) | ((odd << 4) & 0xF0F0F0F0u);
  if (nan || !isfinite(s)) {   // NaN takes the code 0, and so does a row with an infinite value
    for (int e = 0; e < 8; ++e) {
      const uint32_t h = (w[e >> 1] >> (16 * (e & 1))) & 0x7FFFu;
      if (!isfinite(s) || h > 0x7C00u) codes &= ~(15u << (4 * e));
    }
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
  const __half* src = (w.kv ? a.rows[1] : a.rows[0]) + (q.tok0 + w.row0) * a.stride + (w.head * D + 8 * w.at);
  const long long step = w.step * a.stride;
  uint4 x[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {   // (past the last row it once more: a load in a branch would wait for its own data)
    x[i] = ld_plain(reinterpret_cast<const uint4*>(src));
    if (w.row0 + (i + 1) * w.step < w.end) src += step;
  }
  uint32_t to[V], nan = 0;
  const uint32_t held = cache_rows(c, q, w, to);
  float m[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t v[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    __half2 am = __habs2(*reinterpret_cast<const __half2*>(&v[0]));
#pragma unroll
    for (int e = 1; e < 4; ++e) am = __hmax2_nan(am, __habs2(*reinterpret_cast<const __half2*>(&v[e])));
    m[i] = widest(am);
    if (__hisnan(__hmax_nan(__low2half(am), __high2half(am)))) {   // it counts for nothing in the maximum
      nan |= 1u << i;
      m[i] = widest(abs_max8(x[i], __half2half2(__ushort_as_half(0))));
    }
  }
#pragma unroll
  for (int o = D / 16; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < V; ++i) m[i] = fmaxf(m[i], __shfl_xor_sync(lanes, m[i], o));
  uint8_t* codes = (w.kv ? a.k.codes[1] : a.k.codes[0]) + 4 * w.at;
  uint16_t* scales = w.kv ? a.k.scales[1] : a.k.scales[0];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const __nv_bfloat16 sb = __float2bfloat16_rn(__fmul_rn(m[i], 1.f / 7.f));
    const float s = __bfloat162float(sb);
    const uint32_t eight = quant8_nibbles(x[i], s, s > 0.f ? rcp_fast(s) : 0.f, nan >> i & 1u);
    if (held >> i & 1u) {
      *reinterpret_cast<uint32_t*>(codes + (unsigned long long)to[i] * (D / 2)) = eight;
      if (w.at == 0) scales[to[i]] = __bfloat16_as_ushort(sb);
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
  uint32_t from[V];
  const uint32_t held = cache_rows(c, q, w, from);
  const uint8_t* src = (w.kv ? a.k.codes[1] : a.k.codes[0]) + 4 * w.at;
  const uint16_t* scales = w.kv ? a.k.scales[1] : a.k.scales[0];
  const Nibbles nib;
  uint32_t codes[V];
  uint16_t scale[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    codes[i] = ld_plain(reinterpret_cast<const uint32_t*>(src + (unsigned long long)from[i] * (D / 2)));
    scale[i] = ld_plain(scales + from[i]);
  }
  __half* dst = (w.kv ? a.rows[1] : a.rows[0]) + (q.tok0 + w.row0) * a.stride + (w.head * D + 8 * w.at);
  const long long step = w.step * a.stride;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float s = bf16_float(scale[i]);
    const uint4 v = kv4_odd(scale[i]) || kv4_bad(scale[i]) ? values_slow<false>(codes[i], s) : nib.values(codes[i], __float2half2_rn(s));
    if (held >> i & 1u)   // (from the order 0 4, 1 5, 2 6, 3 7)
      *reinterpret_cast<uint4*>(dst + i * step) =
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

// (the kernel for V tokens a thread, or for one where no sequence has as many)
#define DPTQ_LAUNCH_ROWS(kernel, V)                                                                              \
  do {                                                                                                           \
    const bool few = a.k.c.max_tokens < V;                                                                       \
    if (a.k.c.head_dim == 64) return few ? launch_rows<1>(kernel<64, 1>, a, s) : launch_rows<V>(kernel<64, V>, a, s); \
    return few ? launch_rows<1>(kernel<128, 1>, a, s) : launch_rows<V>(kernel<128, V>, a, s);                    \
  } while (0)
cudaError_t launch_kv4_append(const Kv4RowsArgs& a, cudaStream_t s) { DPTQ_LAUNCH_ROWS(kv4_append_kernel, kAppendTokens); }
cudaError_t launch_kv4_read(const Kv4RowsArgs& a, cudaStream_t s) { DPTQ_LAUNCH_ROWS(kv4_read_kernel, kReadTokens); }
#undef DPTQ_LAUNCH_ROWS

}  // namespace dptq
