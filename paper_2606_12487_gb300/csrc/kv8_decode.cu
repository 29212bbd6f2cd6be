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
// one row tile of at most 16 rows there is nothing for tcgen05's 128-row tiles to do.  Each
// warp keeps its own ring of steps in shared memory, filled by asynchronous 16-byte copies
// (no barrier between warps), and reads fragments in whatever order suits 16-byte reads:
//   * logits: the B fragment of key g takes any order of the dims as long as q has the same,
//     so a lane takes 16 consecutive bytes of its key's row at a time;
//   * values: the B fragment of dim g takes any order of the dims across its tiles, so a lane
//     takes D / 8 consecutive bytes of four keys.
// Each 16-byte chunk of a 128-byte line stands at its place xor the line's number mod 8, so
// that neither read meets a bank twice.
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
constexpr int kDecJoin = 12;        // most partial results joined at once
constexpr int kDecJoinMost = 32;    // of a group, and groups: sqrt of a grid of 1024 CTAs at most

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

// A warp's ring: steps of 32 K rows, then 32 V rows, and what goes with a step.
template <int D>
struct alignas(128) Ring {
  static constexpr int kStages = 256 / D;            // 16 KB a warp
  static constexpr int kHalf = kDecKeys * D;         // bytes of K (and of V)
  uint8_t kv[kStages][2 * kHalf];
  float scale[kStages][4];                           // sk of the two 16-key groups, then sv
  int blk[kStages][2];                               // their pages, -1: none
};
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(on ? 4 : 0) : "memory");
}
// Where byte `at` (a multiple of 8) of a half of a step stands.
__device__ __forceinline__ uint32_t swz(uint32_t at) { return at ^ (((at >> 7) & 7u) << 4); }

template <int D, int RT>   // RT: 8-row halves of the row tile that hold rows (1 or 2)
__global__ void __launch_bounds__(kDecThreads, RT == 1 ? kDecodeCtas8 : kDecodeCtas16) kv8_decode_kernel(const Kv8AttendArgs A) {
  constexpr int VB = D / 8;                       // bytes of a V row for one lane; n-tiles of the second product
  constexpr int R = 8 * RT, kSlot = R * D + 2 * R;   // floats of a partial result
  constexpr int NS = Ring<D>::kStages, H = Ring<D>::kHalf;
  extern __shared__ __align__(128) uint8_t sm[];
  __shared__ float s_m[kDecWarps][R], s_l[kDecWarps][R];
  __shared__ int red[kDecWarps], found[3];
  __shared__ float j_m[kDecJoinMost][R], j_l[kDecJoinMost][R];
  __shared__ uint32_t arrived;
  Ring<D>* rings = reinterpret_cast<Ring<D>*>(sm);   // (each warp's becomes its weighted values [R][D] at a share's end)
  const Kv8Args& c = A.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int P = 1 << c.log2_page;
  Ring<D>& ring = rings[warp];

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
        if (row < rows) v = __ldg(reinterpret_cast<const uint2*>(src + D / 4 * t + 4 * k));
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
    // copies step i into its stage; always one group, so that the waits can count
    auto issue = [&](int i, int stage, const int (&blk)[2]) {
      if (i < i1) {
        const int in = key_of(i) & (P - 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bool on = blk[h] >= 0;
          const size_t hb = (size_t)(on ? blk[h] : 0) * c.kv_heads + head;
          const size_t row = ((hb << c.log2_page) + ((in + 16 * h) & (P - 1))) * D + 16 * lane;
#pragma unroll
          for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int u = 0; u < D / 32; ++u)
              copy16(smem_u32(ring.kv[stage]) + kv * H + swz(16 * D * h + 512 * u + 16 * lane),
                     c.codes[kv] + row + 512 * u, on);
          if (lane < 2) copy4(smem_u32(&ring.scale[stage][2 * lane + h]), c.scales[lane] + hb, on);
          if (lane == 0) ring.blk[stage][h] = blk[h];
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };

    int blk[2], i = i0 + warp, stage = 0;
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      pages_of(i + k * kDecWarps, blk);
      issue(i + k * kDecWarps, k, blk);
    }
    for (; i < i1; i += kDecWarps) {
      pages_of(i + NS * kDecWarps, blk);   // (used after this step)
      asm volatile("cp.async.wait_group %0;" ::"n"(NS - 1) : "memory");
      __syncwarp();
      const uint8_t* sk = ring.kv[stage];
      const uint8_t* sv = sk + H;
      const bool held0 = ring.blk[stage][0] >= 0, held1 = ring.blk[stage][1] >= 0;
      const float4 scl = *reinterpret_cast<const float4*>(ring.scale[stage]);
      const int key = key_of(i);
      float sc[4][4];
#pragma unroll
      for (int n = 0; n < 4; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[n][e] = 0.f;
        uint4 kw[D / 64];
#pragma unroll
        for (int ch = 0; ch < D / 64; ++ch)
          kw[ch] = *reinterpret_cast<const uint4*>(sk + swz((8 * n + g) * D + D / 4 * t + 16 * ch));
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint4& w4 = kw[k >> 2];
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
        const float v = fmaxf(h ? scl.w : scl.z, 0x1p-40f);   // (below, 127 sv is no binary16 any more)
        fa[h] = (h ? scl.y : scl.x) * (A.scale * 1.4426950408889634f);
        fb[h] = __log2f(v);
        inv[h] = __frcp_rn(v);
      }
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
{
          uint32_t vw[4][VB / 4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const uint8_t* p = sv + swz((16 * h + 2 * t + (u >> 1) * 8 + (u & 1)) * D + VB * g);
            if constexpr (D == 128) {
              const uint4 v = *reinterpret_cast<const uint4*>(p);
              vw[u][0] = v.x, vw[u][1] = v.y, vw[u][2] = v.z, vw[u][3] = v.w;
            } else {
              const uint2 v = *reinterpret_cast<const uint2*>(p);
              vw[u][0] = v.x, vw[u][1] = v.y;
            }
          }
#pragma unroll
          for (int w = 0; w < VB / 4; ++w) {
            uint32_t b0[4], b1[4];
            widen_pairs(vw[0][w], vw[1][w], b0);
            widen_pairs(vw[2][w], vw[3][w], b1);
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
        }
      __syncwarp();
      issue(i + NS * kDecWarps, stage, blk);
      stage = stage + 1 == NS ? 0 : stage + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();

    // ---- the CTA's warps joined
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
      float* dst = reinterpret_cast<float*>(&ring) + (g + 8 * r) * D;
#pragma unroll
      for (int j = 0; j < VB; ++j) {
        dst[2 * t * VB + j] = o[j][2 * r];
        dst[(2 * t + 1) * VB + j] = o[j][2 * r + 1];
      }
      if (t == 0) {
        s_m[warp][g + 8 * r] = m[r];
        s_l[warp][g + 8 * r] = l[r];
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
      for (int w = 0; w < kDecWarps; ++w) M = fmaxf(M, s_m[w][row]);
      const float mm = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) {
        const float f = exp2_fast(s_m[w][row] - mm);
        L = fmaf(f, s_l[w][row], L);
        O = fmaf(f, reinterpret_cast<const float*>(&rings[w])[k], O);
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
      const int n = c1 - c0 + 1;
      auto slot_of = [&](int b) { return A.ws + (size_t)(2 * b + (b == c0 ? 1 : 0)) * kSlot; };
      // The last of the CTAs joins their results, from as many as fit one round of loads; more
      // are joined in about sqrt(n) groups first, each by its own last.
      auto last_of = [&](uint32_t* counter, int of) {
        __syncthreads();
        if (tid == 0) arrived = atom_add_acq_rel_gpu(counter, 1u);
        __syncthreads();
        if (arrived != (uint32_t)(of - 1)) return false;
        __threadfence();
        if (tid == 0) *counter = 0u;
        return true;
      };
      auto join = [&](int b0, int step, int cnt, bool final) {
        for (int k = tid; k < cnt * rows; k += kDecThreads) {
          const float* p = slot_of(b0 + (k / rows) * step) + R * D + k % rows;
          j_m[k / rows][k % rows] = __ldcg(p);
          j_l[k / rows][k % rows] = __ldcg(p + R);
        }
        __syncthreads();
        float M = -INFINITY, L = 0.f;
        if (tid < rows) {
          for (int b = 0; b < cnt; ++b) M = fmaxf(M, j_m[b][tid]);
          const float mm = M == -INFINITY ? 0.f : M;
          for (int b = 0; b < cnt; ++b) {
            const float f = exp2_fast(j_m[b][tid] - mm);
            j_m[b][tid] = f;
            L = fmaf(f, j_l[b][tid], L);
          }
          j_l[0][tid] = L;
        }
        __syncthreads();
        float* dst = slot_of(b0);
        for (int k = 4 * tid; k < rows * D; k += 4 * kDecThreads) {
          const int row = k / D, d = k - row * D;
          float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
          for (int b = 0; b < cnt; ++b) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(slot_of(b0 + b * step) + k));
            const float f = j_m[b][row];
            O.x = fmaf(f, v.x, O.x);
            O.y = fmaf(f, v.y, O.y);
            O.z = fmaf(f, v.z, O.z);
            O.w = fmaf(f, v.w, O.w);
          }
          if (final) {
            const float sum = j_l[0][row], r = sum == 0.f ? 0.f : __frcp_rn(sum);
            const int tok = row / A.group, hh = row - tok * A.group;
            __half* y = A.out + (size_t)(q.tok0 + tok) * A.out_stride + (size_t)(head * A.group + hh) * D + d;
            *reinterpret_cast<uint2*>(y) = make_uint2(pack_half2(O.x * r, O.y * r), pack_half2(O.z * r, O.w * r));
          } else {
            *reinterpret_cast<float4*>(dst + k) = O;
          }
        }
        if (!final && tid < rows) {
          dst[R * D + tid] = M;
          dst[R * D + R + tid] = L;
        }
      };
      int per = n;
      if (n > kDecJoin) {
        per = 1;
        while (per * per < n) ++per;
        const int b0 = c0 + ((int)blockIdx.x - c0) / per * per, cnt = c1 - b0 + 1 < per ? c1 - b0 + 1 : per;
        // (a CTA may start one group of an earlier head and the first group of its last head)
        if (!last_of(A.counters + (b0 == c0 ? 2 : 1) * gridDim.x + b0, cnt)) per = 0;
        if (per) join(b0, 1, cnt, false);
      }
      if (per && last_of(A.counters + c0, n > kDecJoin ? (n + per - 1) / per : n))
        join(c0, n > kDecJoin ? per : 1, n > kDecJoin ? (n + per - 1) / per : n, true);
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
  const size_t smem = sizeof(Ring<D>) * kDecWarps;
  const cudaError_t e = ensure_max_dyn_smem(fn);
  if (e != cudaSuccess) return e;
  static_assert(kDecodeCtas8 * 256 <= kDecJoinMost * kDecJoinMost, "groups of a join");   // (up to 256 SMs)
  if (num_sms > 256) return cudaErrorInvalidValue;
  fn<<<num_sms * (RT == 1 ? kDecodeCtas8 : kDecodeCtas16), kDecThreads, smem, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_kv8_decode(const Kv8AttendArgs& a, int num_sms, cudaStream_t s) {
  const bool one = a.c.max_tokens * a.group <= 8;
  if (a.c.head_dim == 64) return one ? launch_decode<64, 1>(a, num_sms, s) : launch_decode<64, 2>(a, num_sms, s);
  return one ? launch_decode<128, 1>(a, num_sms, s) : launch_decode<128, 2>(a, num_sms, s);
}

}  // namespace dptq
