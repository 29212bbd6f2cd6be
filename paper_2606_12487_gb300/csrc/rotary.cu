// rotary.cu -- rotary positions of query and key rows: pair i of a head's first `rot` values is turned by
// p f_i, p the row's position.
//
// Angles: a position times a 64-bit fraction of a turn, modulo 2^64, is the exact angle modulo whole
// turns in one integer multiplication; as a signed number it is the angle between -1/2 and 1/2 turn, which
// converts to fp32 half turns with a relative error of 2^-24, however far the position is.  (fp32
// products of positions and radians are 2^-24 of the whole angle off: 0.004 rad at position 65536.  fp64,
// the other way out, runs at 1 / 64 of the fp32 rate here.)
//
// Two bytes in, two out a value: bytes bound it.  The angles of a row serve all of its heads, so a CTA makes
// them once in shared memory; a thread then keeps the eight of its place in a head and goes over the heads with
// 16-byte loads and stores.  8192 rows of 72 heads of 128 (302 MB): 46.1 us in a graph, 6.5 TB/s; 1333 rows of 80, half of each head
// turned, the other half copied: 12.1 us, 4.5 TB/s; one row of 40: 2.3 us (2.7 from HBM).
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv8_device.cuh"

namespace dptq {

constexpr int kRotThreads = 256, kRotMost = 256;   // most pairs of a head

// cos and sin of the pairs of `rows` rows from position `pos` on.
__device__ __forceinline__ void make_angles(const RotaryArgs& a, int pos, int rows, float* cs, float* sn) {
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < rows * half; i += blockDim.x) {
    const int r = i / half, k = i - r * half;
    const uint64_t turn = (uint64_t)(pos + r) * ld_plain(a.turns + k);   // (modulo whole turns)
    float c, s;
    sincospif((float)(long long)turn * 0x1p-63f, &s, &c);
    cs[i] = c * a.amplitude;
    sn[i] = s * a.amplitude;
  }
}
__device__ __forceinline__ void turn_pair(float& x, float& y, float c, float s) {
  const float u = x * c - y * s, v = x * s + y * c;
  x = u;
  y = v;
}
__device__ __forceinline__ void to_floats(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[e]));
    f[2 * e] = p.x;
    f[2 * e + 1] = p.y;
  }
}
__device__ __forceinline__ uint4 to_halves(const float (&f)[8]) {
  return make_uint4(pack_half2(f[0], f[1]), pack_half2(f[2], f[3]), pack_half2(f[4], f[5]), pack_half2(f[6], f[7]));
}

// Whole units of 16 values: rot and head_dim are multiples of 16.  A CTA takes ROWS rows of a sequence and a part
// (blockIdx.z) of their heads, a thread one unit of every `side`-th head; the first kAhead of them are asked for before
// the angles are made.
constexpr int kAhead = 2;
// Two rows a CTA where that leaves kRotFull CTAs an SM, one otherwise.  One / two / four rows, us in a graph: 8192 rows of 72 heads 49.0 /
// 46.1 / 47.3 (6.5 TB/s), 2500 of 40 12.6 / 11.4 / 12.6, 4 x 1000 of 72 21.1 / 20.1 / 21.1; 1333 of 80, half of each head, in place of the one that
// the rule takes (12.1), two 13.3.
constexpr int kRotRows = 2, kRotFull = 8;
template <int ROWS>
__global__ void __launch_bounds__(kRotThreads) rotary_units_kernel(const RotaryArgs a) {
  __shared__ float cs[ROWS * kRotMost], sn[ROWS * kRotMost];
  constexpr int kLane = kRotThreads / ROWS;   // threads of a row
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(a.c, blockIdx.y, q, threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.z == 0)) return;
  const int first = max(-q.start, 0), row0 = first + blockIdx.x * ROWS;   // (rows at negative positions come first)
  if (row0 >= q.n) return;
  const int rows = min(ROWS, q.n - row0);
  const int turned = a.rot / 16, all = a.x == a.out ? turned : a.head_dim / 16;   // units of a head that change; that are written
  const int r = threadIdx.x / kLane, at = threadIdx.x % kLane;
  const int side = kLane / all, u = at % all;   // heads side by side
  const int per = (a.heads + gridDim.z - 1) / gridDim.z, h1 = min((blockIdx.z + 1) * per, a.heads);
  int h = r < rows && at < side * all ? blockIdx.z * per + at / all : h1;
  const size_t tok = (size_t)(q.tok0 + row0 + (r < rows ? r : 0));
  const __half* x = a.x + tok * a.x_stride;
  __half* y = a.out + tok * a.out_stride;
  // A unit: 8 pairs, or (u >= turned) 16 values of the rest of a head.
  const bool near = a.interleaved || u >= turned;
  const int d0 = near ? 16 * u : 8 * u, d1 = near ? d0 + 8 : d0 + a.rot / 2;
  uint4 v0[kAhead], v1[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    // (threads without a head read the last one: a load in a branch would wait for its own data)
    const int d = min(h + k * side, h1 - 1) * a.head_dim;
    v0[k] = ld_plain(reinterpret_cast<const uint4*>(x + d + d0));
    v1[k] = ld_plain(reinterpret_cast<const uint4*>(x + d + d1));
  }
  make_angles(a, q.start + row0, rows, cs, sn);
  __syncthreads();
  float c[8], s[8];
  if (u < turned && r < rows) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      c[e] = cs[r * (a.rot / 2) + 8 * u + e];
      s[e] = sn[r * (a.rot / 2) + 8 * u + e];
    }
  }
  while (h < h1) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      uint4 w0 = v0[k], w1 = v1[k];
      const int now = h + k * side;
      if (now + kAhead * side < h1) {
        const int d = (now + kAhead * side) * a.head_dim;
        v0[k] = ld_plain(reinterpret_cast<const uint4*>(x + d + d0));
        v1[k] = ld_plain(reinterpret_cast<const uint4*>(x + d + d1));
      }
      if (now >= h1) break;
      if (u < turned) {
        float f[8], g[8];
        to_floats(w0, f);
        to_floats(w1, g);
        if (a.interleaved) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            turn_pair(f[2 * e], f[2 * e + 1], c[e], s[e]);
            turn_pair(g[2 * e], g[2 * e + 1], c[4 + e], s[4 + e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) turn_pair(f[e], g[e], c[e], s[e]);
        }
        w0 = to_halves(f);
        w1 = to_halves(g);
      }
      *reinterpret_cast<uint4*>(y + now * a.head_dim + d0) = w0;
      *reinterpret_cast<uint4*>(y + now * a.head_dim + d1) = w1;
    }
    h += kAhead * side;
  }
}

// Any even rot: pairs cross 16-byte vectors in any way, so a CTA takes a part of a row through shared memory, whole vectors in and
// out, a thread a pair in between: 8192 rows of 72 heads, 20 of 128 values, 60 us (with 256 threads a part 73, 64 and half a
// part 63; a thread a pair from and to global memory 162).
constexpr int kPairThreads = 128, kPairValues = 4096;   // values of a part: whole heads
__global__ void __launch_bounds__(kPairThreads) rotary_pairs_kernel(const RotaryArgs a) {
  __shared__ float cs[kRotMost], sn[kRotMost];
  __shared__ __align__(16) __half row_s[kPairValues];
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(a.c, blockIdx.y, q, threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.z == 0)) return;
  const int row = max(-q.start, 0) + blockIdx.x;
  if (row >= q.n) return;
  const int per = kPairValues / a.head_dim, h0 = blockIdx.z * per, heads = min(per, a.heads - h0);
  const __half* x = a.x + (size_t)(q.tok0 + row) * a.x_stride + (size_t)h0 * a.head_dim;
  __half* y = a.out + (size_t)(q.tok0 + row) * a.out_stride + (size_t)h0 * a.head_dim;
  // vectors of a head that change or are copied, of its head_dim / 8
  const int all = a.head_dim / 8, vecs = a.x == a.out ? (a.rot + 7) / 8 : all, half = a.rot / 2;
  for (int i = threadIdx.x; i < heads * vecs; i += kPairThreads) {
    const int h = i / vecs, v = h * all + i - h * vecs;
    reinterpret_cast<uint4*>(row_s)[v] = ld_plain(reinterpret_cast<const uint4*>(x) + v);
  }
  make_angles(a, q.start + row, 1, cs, sn);
  __syncthreads();
  for (int i = threadIdx.x; i < heads * half; i += kPairThreads) {
    const int h = i / half, k = i - h * half, d0 = h * a.head_dim + (a.interleaved ? 2 * k : k), d1 = d0 + (a.interleaved ? 1 : half);
    float u = __half2float(row_s[d0]), v = __half2float(row_s[d1]);
    turn_pair(u, v, cs[k], sn[k]);
    row_s[d0] = __float2half_rn(u);
    row_s[d1] = __float2half_rn(v);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < heads * vecs; i += kPairThreads) {
    const int h = i / vecs, v = h * all + i - h * vecs;
    reinterpret_cast<uint4*>(y)[v] = reinterpret_cast<const uint4*>(row_s)[v];
  }
}

template <int ROWS>
static cudaError_t launch_units(const RotaryArgs& a, int parts, cudaStream_t s) {
  return launch_after(rotary_units_kernel<ROWS>, dim3(ceil_div(a.c.max_tokens, ROWS), a.c.seqs, parts), kRotThreads, 0, s,
                      1, a);
}

cudaError_t launch_rotary(const RotaryArgs& a, int num_sms, cudaStream_t s) {
  const long long rows = (long long)a.c.max_tokens * a.c.seqs;   // (most of them)
  if (a.rot % 16 != 0 || a.head_dim % 16 != 0)
    return launch_after(rotary_pairs_kernel, dim3(a.c.max_tokens, a.c.seqs, ceil_div(a.heads, kPairValues / a.head_dim)),
                        kPairThreads, 0, s, 1, a);
  if (a.c.max_tokens >= kRotRows && rows >= (long long)kRotRows * kRotFull * num_sms) return launch_units<kRotRows>(a, 1, s);
  // Few rows: their heads over as many CTAs as there are SMs, while a thread has more than it asks for ahead (one row of 640 heads:
  // 2.4 us, in one CTA 5.9; of 80: 2.2 and 2.5).
  long long parts = ceil_div((long long)a.heads * (a.head_dim / 16), kAhead * kRotThreads);
  if (parts > num_sms / rows) parts = num_sms / rows;
  return launch_units<1>(a, parts > 1 ? (int)parts : 1, s);
}

}  // namespace dptq
