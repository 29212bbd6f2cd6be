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
// 16-byte loads and stores.
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv8_device.cuh"

namespace dptq {

constexpr int kRotThreads = 256, kRotMost = 256;   // most pairs of a head

// cos and sin of the pairs of `rows` rows from position `pos` on.
__device__ __forceinline__ void make_angles(const RotaryArgs& a, int pos, int rows, float* cs, float* sn) {
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < rows * half; i += kRotThreads) {
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
// (blockIdx.z) of their heads.
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
  make_angles(a, q.start + row0, rows, cs, sn);
  __syncthreads();
  const int units = a.head_dim / 16, turned = a.rot / 16, all = turned + (a.x == a.out ? 0 : units - turned);
  const int r = threadIdx.x / kLane, at = threadIdx.x % kLane;
  const int side = kLane / all;   // heads at a time
  const int u = at % all, per = (a.heads + gridDim.z - 1) / gridDim.z, h0 = blockIdx.z * per, h1 = min(h0 + per, a.heads);
  if (r >= rows || at >= side * all) return;
  const size_t tok = (size_t)(q.tok0 + row0 + r);
  const __half* x = a.x + tok * a.x_stride;
  __half* y = a.out + tok * a.out_stride;
  if (u >= turned) {   // the rest of a head
    for (int h = h0 + at / all; h < h1; h += side) {
      const int d = h * a.head_dim + 16 * u;
      const uint4 v0 = ld_plain(reinterpret_cast<const uint4*>(x + d)), v1 = ld_plain(reinterpret_cast<const uint4*>(x + d) + 1);
      *reinterpret_cast<uint4*>(y + d) = v0;
      *(reinterpret_cast<uint4*>(y + d) + 1) = v1;
    }
    return;
  }
  float c[8], s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    c[e] = cs[r * (a.rot / 2) + 8 * u + e];
    s[e] = sn[r * (a.rot / 2) + 8 * u + e];
  }
  const int d0 = a.interleaved ? 16 * u : 8 * u, d1 = a.interleaved ? d0 + 8 : d0 + a.rot / 2;
#pragma unroll 2
  for (int h = h0 + at / all; h < h1; h += side) {
    const int d = h * a.head_dim;
    float f[8], g[8];
    to_floats(ld_plain(reinterpret_cast<const uint4*>(x + d + d0)), f);
    to_floats(ld_plain(reinterpret_cast<const uint4*>(x + d + d1)), g);
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
    *reinterpret_cast<uint4*>(y + d + d0) = to_halves(f);
    *reinterpret_cast<uint4*>(y + d + d1) = to_halves(g);
  }
}

// Any even rot: a thread a pair, or a value of the rest of a head.
__global__ void __launch_bounds__(kRotThreads) rotary_pairs_kernel(const RotaryArgs a) {
  __shared__ float cs[kRotMost], sn[kRotMost];
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(a.c, blockIdx.y, q, threadIdx.x == 0 && blockIdx.x == 0)) return;
  const int row = max(-q.start, 0) + blockIdx.x;
  if (row >= q.n) return;
  make_angles(a, q.start + row, 1, cs, sn);
  __syncthreads();
  const __half* x = a.x + (size_t)(q.tok0 + row) * a.x_stride;
  __half* y = a.out + (size_t)(q.tok0 + row) * a.out_stride;
  const int half = a.rot / 2, items = half + (a.x == a.out ? 0 : a.head_dim - a.rot);
  for (int i = threadIdx.x; i < a.heads * items; i += kRotThreads) {
    const int h = i / items, k = i - h * items, d = h * a.head_dim;
    if (k >= half) {
      y[d + half + k] = ld_plain(x + d + half + k);
      continue;
    }
    const int d0 = d + (a.interleaved ? 2 * k : k), d1 = d0 + (a.interleaved ? 1 : half);
    float u = __half2float(ld_plain(x + d0)), v = __half2float(ld_plain(x + d1));
    turn_pair(u, v, cs[k], sn[k]);
    y[d0] = __float2half_rn(u);
    y[d1] = __float2half_rn(v);
  }
}

cudaError_t launch_rotary(const RotaryArgs& a, int num_sms, cudaStream_t s) {
  const int n = a.c.max_tokens;
  if (a.rot % 16 != 0 || a.head_dim % 16 != 0)
    return launch_after(rotary_pairs_kernel, dim3(n, a.c.seqs), kRotThreads, 0, s, 1, a);
  const dim3 grid(n, a.c.seqs, 1);
  return launch_after(rotary_units_kernel<1>, grid, kRotThreads, 0, s, 1, a);
}

}  // namespace dptq
