// kv8_decode.cu -- attention of a few rows (at most 16 for each sequence and KV head) over the
// paged int8 cache: decode steps and a few speculative tokens.
//
// The call is a stream over the visible K and V codes (one byte a value, read once) with
// 4 R multiply-adds a byte pair for R rows, so bytes bound it.  Work is cut into steps of 32
// keys of one (sequence, KV head); the CTAs of one resident wave take equal, contiguous
// shares of all steps whatever the lengths are (they are read from the device), and a
// (sequence, head) that several CTAs share is joined by the last of them to finish.
// Inside a CTA the warps take every fourth step; each keeps its own running maximum, sum and
// accumulators, joined through shared memory once per share.
//
// A warp multiplies with 16 x 8 x 16 register MMAs (rows of q x keys, then rows x dims): with
// one row tile of at most 16 rows there is nothing for tcgen05's 128-row tiles to do, and the
// fragments come straight from global memory into registers, without shared memory:
//   * logits: the B fragment of key g takes any order of the dims as long as q has the same,
//     so a lane takes 16 consecutive bytes of its key's row, 64 bytes a quad and load;
//   * values: the B fragment of dim g takes any order of the dims across its tiles, so a lane
//     takes D / 8 consecutive bytes of four keys, a whole row for eight lanes.
// int8 -> binary16 is exact: a byte c + 128 under the exponent of 1024 is 1152 + c.
//
// Softmax in base 2 on x_j = log2(e) scale sk (q . ck_j) + log2(sv): the weights that go into
// the second product are then p_j sv_j relative to the largest of them, and binary16 loses
// nothing to pages whose scales are far apart; the denominator takes each back by 1 / sv.
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv8_device.cuh"

namespace dptq {

constexpr int kDecWarps = 4, kDecThreads = 32 * kDecWarps;
constexpr int kDecKeys = 32;        // keys of a step
constexpr int kDecMinSteps = 16;    // fewest steps that a CTA is started for

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t less_1152(uint32_t h) {
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&h), __half2half2(__ushort_as_half(0x6480)));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Four codes to two pairs of binary16: values 0, 1 and 2, 3.
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  w ^= 0x80808080u;
  lo = less_1152(__byte_perm(w, 0x64646464u, 0x4140));
  hi = less_1152(__byte_perm(w, 0x64646464u, 0x4342));
}
// Four codes of two keys to four pairs (key a, key b).
__device__ __forceinline__ void widen_pairs(uint32_t a, uint32_t b, uint32_t (&r)[4]) {
  const uint32_t lo = __byte_perm(a, b, 0x5140) ^ 0x80808080u, hi = __byte_perm(a, b, 0x7362) ^ 0x80808080u;
  r[0] = less_1152(__byte_perm(lo, 0x64646464u, 0x4140));
  r[1] = less_1152(__byte_perm(lo, 0x64646464u, 0x4342));
  r[2] = less_1152(__byte_perm(hi, 0x64646464u, 0x4140));
  r[3] = less_1152(__byte_perm(hi, 0x64646464u, 0x4342));
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// The steps of a sequence: `sink` steps from key 0, then steps from key `from`.
struct Steps {
  int sink, from, count;
};
__device__ __forceinline__ Steps seq_steps(const Seq& q, int window, int sinks) {
  Steps r{0, 0, 0};
  if (q.n == 0 || q.len == 0) return r;
  if (window > 0) {
    const int first = (q.start > 0 ? q.start : 0) - window + 1;   // the first row's oldest key
    if (first >= kDecKeys) {
      r.from = first & ~(kDecKeys - 1);
      r.sink = sinks < r.from ? (sinks + kDecKeys - 1) / kDecKeys : r.from / kDecKeys;
    }
  }
  r.count = r.sink + (q.len - r.from + kDecKeys - 1) / kDecKeys;
  return r;
}

// Steps of sequences 0 .. s - 1 (of one head each): the CTA sums them chunk by chunk.
__device__ __forceinline__ int block_scan(int v, int* red, int& total) {   // exclusive prefix over the CTA's threads
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) red[warp] = x;
  __syncthreads();
  int base = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kDecWarps; ++w) {
    if (w < warp) base += red[w];
    total += red[w];
  }
  return base + x - v;
}

// One step's loads of a warp.
template <int D>
struct StepRegs {
  uint4 k[4][D / 64];       // [8-key tile][64-dim chunk]
  uint4 v[2][4];            // [16-key group][key]  (D = 64: the low half)
  float a[2], b[2], inv[2];   // per 16 keys: logit factor, log2(sv), 1 / sv
};

template <int D, int RT>   // RT: 8-row halves of the row tile that hold rows (1 or 2)
__global__ void __launch_bounds__(kDecThreads, RT == 1 ? kDecodeCtas8 : kDecodeCtas16) kv8_decode_kernel(const Kv8AttendArgs A) {
  constexpr int VB = D / 8;                       // bytes of a V row for one lane; n-tiles of the second product
  constexpr int R = 8 * RT, kSlot = R * D + 2 * R;   // floats of a partial result
  extern __shared__ __align__(16) float sm[];     // [warps][R][D], then maxima and sums [warps][R] each
  __shared__ int red[kDecWarps], found[3];
  __shared__ uint32_t arrived;
  float* so = sm;
  float* s_m = sm + kDecWarps * R * D;
  float* s_l = s_m + kDecWarps * R;
  const Kv8Args& c = A.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int P = 1 << c.log2_page;

  // ---- this CTA's share
  long long total = 0;
  bool none = false;   // a sequence of rows without a key
  for (int s0 = 0; s0 < c.seqs; s0 += kDecThreads) {
    Seq q;
    int n = 0, all;
    if (s0 + tid < c.seqs && load_seq(c, s0 + tid, q, blockIdx.x == 0)) {
      n = seq_steps(q, A.window, A.sinks).count;
      none |= n == 0 && q.n > 0;
    }
    block_scan(n, red, all);
    total += all;
  }
  total *= c.kv_heads;
  long long ctas = (total + kDecMinSteps - 1) / kDecMinSteps;
  if (ctas > gridDim.x) ctas = gridDim.x;
  // (such a sequence has no step: zeros, from CTA 0)
  if (blockIdx.x == 0 && __syncthreads_or(none)) {
    for (int s = 0; s < c.seqs; ++s) {
      Seq q;
      if (!load_seq(c, s, q, false) || q.len > 0) continue;
      for (int i = 0; i < q.n; ++i)
        for (int k = tid; k < A.q_heads * D; k += kDecThreads)
          A.out[(size_t)(q.tok0 + i) * A.out_stride + k] = __ushort_as_half(0);
    }
  }
  if (blockIdx.x >= ctas) return;
  const long long begin = blockIdx.x * total / ctas, end = (blockIdx.x + 1) * total / ctas;
  // the sequence that holds step `begin`
  long long before = 0;
  for (int s0 = 0; s0 < c.seqs; s0 += kDecThreads) {
    Seq q;
    int n = 0, all;
    if (s0 + tid < c.seqs && load_seq(c, s0 + tid, q, false)) n = seq_steps(q, A.window, A.sinks).count;
    const long long at = before + (long long)block_scan(n, red, all) * c.kv_heads;
    if (n > 0 && at <= begin && begin < at + (long long)n * c.kv_heads) {
      found[0] = s0 + tid;
      found[1] = (int)((begin - at) / n);
      found[2] = (int)((begin - at) % n);
    }
    before += (long long)all * c.kv_heads;
    __syncthreads();
    if (before > begin) break;
  }
  int s = found[0], head = found[1], i0 = found[2];

  Seq q;
  load_seq(c, s, q, false);
  Steps st = seq_steps(q, A.window, A.sinks);
  for (long long it = begin; it < end;) {
    const int i1 = (int)(end - it < st.count - i0 ? i0 + (end - it) : st.count);
    const int rows = q.n * A.group;

    // ---- this share's rows of q, in the order of the dims that the keys' bytes have
    uint32_t qf[D / 16][2 * RT];
    int pos[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int row = g + 8 * r, tok = row / A.group, hh = row - tok * A.group;
      pos[r] = row < rows ? q.start + tok : -1;
      const __half* src = A.q + (size_t)(q.tok0 + tok) * A.q_stride + (size_t)(head * A.group + hh) * D;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        uint2 v = make_uint2(0u, 0u);
        if (row < rows) v = __ldg(reinterpret_cast<const uint2*>(src + (k >> 2) * 64 + 16 * t + 4 * (k & 3)));
        qf[k][r] = v.x;
        qf[k][RT + r] = v.y;
      }
    }
    float o[VB][2 * RT], m[RT], l[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) m[r] = -INFINITY, l[r] = 0.f;
#pragma unroll
    for (int j = 0; j < VB; ++j)
#pragma unroll
      for (int e = 0; e < 2 * RT; ++e) o[j][e] = 0.f;

    // ---- the steps of this warp
    auto key_of = [&](int i) { return i < st.sink ? i * kDecKeys : st.from + (i - st.sink) * kDecKeys; };
    // whether any row sees one of the 16 keys from `k` on (pages that none does are not looked up)
    auto group_seen = [&](int k) {
      return k < q.len && (A.window == 0 || k + 15 > (q.start > 0 ? q.start : 0) - A.window || k < A.sinks);
    };
    auto pages_of = [&](int i, int (&blk)[2]) {
      blk[0] = blk[1] = -1;
      if (i >= i1) return;
      const int key = key_of(i);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (group_seen(key + 16 * h)) blk[h] = load_page(c, s, (key + 16 * h) >> c.log2_page);
    };
    auto load_k = [&](int i, const int (&blk)[2], StepRegs<D>& x) {
      const int in = key_of(i) & (P - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const size_t hb = (size_t)(blk[h] < 0 ? 0 : blk[h]) * c.kv_heads + head;
        const int r0 = (in + 16 * h) & (P - 1);
        const int8_t* src = c.codes[0] + ((hb << c.log2_page) + r0 + g) * D + 16 * t;
        x.a[h] = x.b[h] = x.inv[h] = 0.f;
        if (blk[h] >= 0) {
          x.a[h] = __ldg(c.scales[0] + hb);
          x.b[h] = __ldg(c.scales[1] + hb);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int ch = 0; ch < D / 64; ++ch)
            x.k[2 * h + u][ch] = blk[h] >= 0 ? __ldg(reinterpret_cast<const uint4*>(src + 8 * u * D + 64 * ch))
                                             : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    auto load_v = [&](int i, const int (&blk)[2], StepRegs<D>& x) {
      const int in = key_of(i) & (P - 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const size_t hb = (size_t)(blk[h] < 0 ? 0 : blk[h]) * c.kv_heads + head;
        const int r0 = (in + 16 * h) & (P - 1);
        const int8_t* src = c.codes[1] + ((hb << c.log2_page) + r0 + 2 * t) * D + VB * g;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int8_t* p = src + ((u >> 1) * 8 + (u & 1)) * D;
          x.v[h][u] = make_uint4(0u, 0u, 0u, 0u);
          if (blk[h] >= 0) {
            if constexpr (D == 128) {
              x.v[h][u] = __ldg(reinterpret_cast<const uint4*>(p));
            } else {
              const uint2 y = __ldg(reinterpret_cast<const uint2*>(p));
              x.v[h][u].x = y.x;
              x.v[h][u].y = y.y;
            }
          }
        }
      }
    };

    StepRegs<D> x;
    int blk[2], next[2];
    int i = i0 + warp;
    pages_of(i, blk);
    if (i < i1) {
      load_k(i, blk, x);
      load_v(i, blk, x);
    }
    for (; i < i1; i += kDecWarps) {
      pages_of(i + kDecWarps, next);
      const int key = key_of(i);
      float sc[4][4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[n][e] = 0.f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint4& w4 = x.k[n][k >> 2];
          const uint32_t w = (k & 3) == 0 ? w4.x : (k & 3) == 1 ? w4.y : (k & 3) == 2 ? w4.z : w4.w;
          uint32_t b0, b1;
          widen4(w, b0, b1);
          if constexpr (RT == 1)
            mma_16816(sc[n], qf[k][0], 0u, qf[k][1], 0u, b0, b1);
          else
            mma_16816(sc[n], qf[k][0], qf[k][1], qf[k][2], qf[k][3], b0, b1);
        }
      }
      // x_j, per 16 keys one factor and one addend
      float fa[2], fb[2], inv[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float sv = fmaxf(x.b[h], 0x1p-40f);   // (below, 127 sv is no binary16 any more)
        fa[h] = x.a[h] * (A.scale * 1.4426950408889634f);
        fb[h] = __log2f(sv);
        inv[h] = __frcp_rn(sv);
      }
      const bool held0 = blk[0] >= 0, held1 = blk[1] >= 0;
      if (i + kDecWarps < i1) load_k(i + kDecWarps, next, x);
      float top[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) top[r] = m[r];
      // every row sees every key of the step
      const bool all = held0 && held1 && key + kDecKeys - 1 <= q.start &&
                       (A.window == 0 || key > q.len - 1 - A.window || key + kDecKeys <= A.sinks);
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float& v = sc[n][2 * r + e];
            v = fmaf(v, fa[n >> 1], fb[n >> 1]);
            if (!all) {
              const int j = key + 8 * n + 2 * t + e;
              if (!((n < 2 ? held0 : held1) && kv8_sees(pos[r], j, A.window, A.sinks))) v = -INFINITY;
            }
            top[r] = fmaxf(top[r], v);
          }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
        top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
        if (__any_sync(0xffffffffu, top[r] != m[r])) {
          const float f = top[r] == m[r] ? 1.f : exp2_fast(m[r] - top[r]);
          l[r] *= f;
#pragma unroll
          for (int j = 0; j < VB; ++j) o[j][2 * r] *= f, o[j][2 * r + 1] *= f;
          m[r] = top[r];
        }
      }
      uint32_t pf[2][2 * RT];   // A fragments of the weights, per 16 keys
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const float mm = m[r] == -INFINITY ? 0.f : m[r];
          float p[4], sum = 0.f;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              p[2 * u + e] = exp2_fast(sc[2 * h + u][2 * r + e] - mm);
              sum += p[2 * u + e];
            }
          l[r] = fmaf(sum, inv[h], l[r]);
          pf[h][r] = pack_half2(p[0], p[1]);
          pf[h][RT + r] = pack_half2(p[2], p[3]);
        }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int w = 0; w < VB / 4; ++w) {
          uint32_t b0[4], b1[4];
          auto word = [&](const uint4& v) { return w == 0 ? v.x : w == 1 ? v.y : w == 2 ? v.z : v.w; };
          widen_pairs(word(x.v[h][0]), word(x.v[h][1]), b0);
          widen_pairs(word(x.v[h][2]), word(x.v[h][3]), b1);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float (&acc)[2 * RT] = o[4 * w + e];
            if constexpr (RT == 1) {
              float d[4] = {acc[0], acc[1], 0.f, 0.f};
              mma_16816(d, pf[h][0], 0u, pf[h][1], 0u, b0[e], b1[e]);
              acc[0] = d[0];
              acc[1] = d[1];
            } else {
              mma_16816(acc, pf[h][0], pf[h][1], pf[h][2], pf[h][3], b0[e], b1[e]);
            }
          }
        }
      if (i + kDecWarps < i1) load_v(i + kDecWarps, next, x);
      blk[0] = next[0];
      blk[1] = next[1];
    }

    // ---- the CTA's warps joined
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
      float* dst = so + (warp * R + g + 8 * r) * D;
#pragma unroll
      for (int j = 0; j < VB; ++j) {
        dst[2 * t * VB + j] = o[j][2 * r];
        dst[(2 * t + 1) * VB + j] = o[j][2 * r + 1];
      }
      if (t == 0) {
        s_m[warp * R + g + 8 * r] = m[r];
        s_l[warp * R + g + 8 * r] = l[r];
      }
    }
    __syncthreads();
    const bool whole = i0 == 0 && i1 == st.count;
    const long long seg0 = it - i0;   // the (sequence, head)'s steps: seg0 .. seg0 + count - 1
    float* slot = A.ws + (size_t)(2 * blockIdx.x + (i0 == 0 ? 1 : 0)) * kSlot;
    for (int k = tid; k < rows * D; k += kDecThreads) {
      const int row = k / D, d = k - row * D;
      float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) M = fmaxf(M, s_m[w * R + row]);
      const float mm = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) {
        const float f = exp2_fast(s_m[w * R + row] - mm);
        L = fmaf(f, s_l[w * R + row], L);
        O = fmaf(f, so[(w * R + row) * D + d], O);
      }
      if (whole) {
        const int tok = row / A.group, hh = row - tok * A.group;
        A.out[(size_t)(q.tok0 + tok) * A.out_stride + (size_t)(head * A.group + hh) * D + d] =
            __float2half_rn(L == 0.f ? 0.f : O / L);
      } else {
        slot[k] = O;
        if (d == 0) {
          slot[R * D + row] = M;
          slot[R * D + R + row] = L;
        }
      }
    }
    if (!whole) {
      // CTA b holds steps b total / ctas ..: the one that holds step i is ((i + 1) ctas - 1) / total
      const int c0 = (int)(((seg0 + 1) * ctas - 1) / total), c1 = (int)(((seg0 + st.count) * ctas - 1) / total);
      __syncthreads();
      if (tid == 0) arrived = atom_add_acq_rel_gpu(A.counters + c0, 1u);
      __syncthreads();
      if (arrived == (uint32_t)(c1 - c0)) {
        __threadfence();
        for (int k = tid; k < rows * D; k += kDecThreads) {
          const int row = k / D, d = k - row * D;
          float M = -INFINITY, L = 0.f, O = 0.f;
          for (int b = c0; b <= c1; ++b)
            M = fmaxf(M, __ldcg(A.ws + (size_t)(2 * b + (b == c0 ? 1 : 0)) * kSlot + R * D + row));
          const float mm = M == -INFINITY ? 0.f : M;
#pragma unroll 4
          for (int b = c0; b <= c1; ++b) {
            const float* p = A.ws + (size_t)(2 * b + (b == c0 ? 1 : 0)) * kSlot;
            const float f = exp2_fast(__ldcg(p + R * D + row) - mm);
            L = fmaf(f, __ldcg(p + R * D + R + row), L);
            O = fmaf(f, __ldcg(p + k), O);
          }
          const int tok = row / A.group, hh = row - tok * A.group;
          A.out[(size_t)(q.tok0 + tok) * A.out_stride + (size_t)(head * A.group + hh) * D + d] =
              __float2half_rn(L == 0.f ? 0.f : O / L);
        }
        if (tid == 0) A.counters[c0] = 0u;
      }
    }
    __syncthreads();

    // ---- on to the next (sequence, head)
    it += i1 - i0;
    i0 = 0;
    if (it < end && ++head == c.kv_heads) {
      head = 0;
      do {
        ++s;
        st.count = load_seq(c, s, q, false) ? (st = seq_steps(q, A.window, A.sinks)).count : 0;
      } while (st.count == 0);
    }
  }
}

template <int D, int RT>
static cudaError_t launch_decode(const Kv8AttendArgs& a, int num_sms, cudaStream_t s) {
  const auto fn = kv8_decode_kernel<D, RT>;
  const size_t smem = sizeof(float) * kDecWarps * (8 * RT * D + 2 * 8 * RT);
  fn<<<num_sms * (RT == 1 ? kDecodeCtas8 : kDecodeCtas16), kDecThreads, smem, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_kv8_decode(const Kv8AttendArgs& a, int num_sms, cudaStream_t s) {
  const bool one = a.c.max_tokens * a.group <= 8;
  if (a.c.head_dim == 64) return one ? launch_decode<64, 1>(a, num_sms, s) : launch_decode<64, 2>(a, num_sms, s);
  return one ? launch_decode<128, 1>(a, num_sms, s) : launch_decode<128, 2>(a, num_sms, s);
}

}  // namespace dptq
