// kv_decode.cuh -- what the decode kernels of both paged caches share: the rows' work cut into equal shares, the
// register MMA, and the join of partial results.
//
// Work is cut into steps of KEYS keys of one (sequence, KV head); the CTAs of one resident wave take equal,
// contiguous shares of all steps whatever the lengths are (they are read from the device), and a
// (sequence, head) that several CTAs share is joined by the last of them to finish.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv8_device.cuh"

namespace dptq {

constexpr int kDecWarps = 4, kDecThreads = 32 * kDecWarps;
// Most partial results of a group, or groups: sqrt of a grid of 1024 CTAs at most.
constexpr int kDecJoinMost = 32;

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// What a (sequence, head) costs a CTA beyond its steps (its rows of q, the first copies' latency,
// the join): shares of 16 steps and more are cut as if every one had so many steps more, which
// come first.  With 6 / without, us: 32 ragged MHA sequences (7 to 128 steps a head) 98.8 / 121.0, the same with heads
// of 64 68.0 / 88.2, 64 with a window over 8 heads 90.4 / 95.0, 16 up to 8000 tokens over 8 heads 39.0 / 40.9, 64
// of 8000 tokens over 8 heads, two rows each, 210 / 208 (equal lengths).
constexpr int kDecExtra = 6, kDecExtraFrom = 16;

// The steps of a sequence: `sink` steps from key 0, then steps from key `from`.
struct Steps {
  int sink, from, count;
};
template <int KEYS>
__device__ __forceinline__ Steps seq_steps(const Seq& q, int window, int sinks) {
  Steps r{0, 0, 0};
  if (q.n == 0 || q.len == 0) return r;
  if (window > 0) {
    const int first = (q.start > 0 ? q.start : 0) - window + 1;   // the first row's oldest key
    if (first >= KEYS) {
      r.from = first & ~(KEYS - 1);
      r.sink = sinks < r.from ? (sinks + KEYS - 1) / KEYS : r.from / KEYS;
    }
  }
  r.count = r.sink + (q.len - r.from + KEYS - 1) / KEYS;
  return r;
}

// The exclusive prefix of v over the CTA's threads, and its sum over all of them.
__device__ __forceinline__ int block_scan(int v, int* red, int& total) {
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

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(on ? 4 : 0) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {   // of binary16, two of a row in each lane
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Of a CTA: each warp's running maxima and sums at a share's end, and what is joined.
template <int R>
struct JoinShared {
  float m[kDecWarps][R], l[kDecWarps][R];
  int red[kDecWarps], found[3];
  int3 sums[kDecWarps];
  float part_m[kDecJoinMost][R], part_l[kDecJoinMost][R];
  uint32_t arrived;
};

// Runs body(q, s, st, head, i0, i1) for each run of steps i0 .. i1 - 1 of a (sequence s, KV head) in this CTA's share.
// Every warp leaves its rows' weighted values [R][D] in its own memory (at `mem`, `pitch` bytes apart), and
// maxima and sums in S; they are joined here, across CTAs too, and written.
// MIN: fewest steps that a CTA is started for.  JOIN: most partial results joined at once.
// ALIGN: calls that do not fill the grid are cut by (sequence, head) instead: CTAs of MIN or 2 MIN steps of one head, as long as its
// results are joined at once.  A head's steps are then counted up to a multiple of that, the ones that are none first.
template <int D, int R, int KEYS, int MIN, int JOIN, bool ALIGN, class Args, class Body>
__device__ __forceinline__ void decode_shares(const Kv8Args& c, const Args& A, JoinShared<R>& S, const uint8_t* mem,
                                              size_t pitch, Body body) {
  constexpr int kSlot = R * D + 2 * R;   // floats of a partial result
  static_assert(JOIN <= kDecJoinMost, "results joined at once");
  const int tid = threadIdx.x;
  // ---- this CTA's share
  long long total = 0;
  int some = 0;   // sequences with steps
  bool none = false;   // a sequence of rows without a key
  int mine = 0, ahead = 0;   // this thread's sequence of the last 128: its steps, those before it
  int most = 0, ctas1 = 0, ctas2 = 0;   // (ALIGN) the most steps of a head, CTAs of MIN and 2 MIN steps for one head of each sequence
  for (int s0 = 0; s0 < c.seqs; s0 += kDecThreads) {
    Seq q;
    int n = 0, all;
    if (s0 + tid < c.seqs && load_seq(c, s0 + tid, q, blockIdx.x == 0)) {
      n = seq_steps<KEYS>(q, A.window, A.sinks).count;
      none |= n == 0 && q.n > 0;
    }
    ahead = block_scan(n, S.red, all);
    mine = n;
    total += all;
    if constexpr (ALIGN) {
      most = max(most, n);
      ctas1 += (n + MIN - 1) / MIN;
      ctas2 += (n + 2 * MIN - 1) / (2 * MIN);
    }
    some += __syncthreads_count(n > 0);
  }
  total *= c.kv_heads;
  long long ctas = (total + MIN - 1) / MIN;
  if (ctas > gridDim.x) ctas = gridDim.x;
  const int extra = total >= (long long)kDecExtraFrom * ctas ? kDecExtra : 0;
  int unit = 0;   // steps of a CTA of a call that is cut by heads
  if constexpr (ALIGN) {
    // (of up to 128 sequences: their steps are at hand)
    most = __reduce_max_sync(0xffffffffu, most);
    ctas1 = __reduce_add_sync(0xffffffffu, ctas1);
    ctas2 = __reduce_add_sync(0xffffffffu, ctas2);
    if ((tid & 31) == 0) S.sums[tid >> 5] = make_int3(most, ctas1, ctas2);
    __syncthreads();
    most = ctas1 = ctas2 = 0;
#pragma unroll
    for (int w = 0; w < kDecWarps; ++w) {
      most = max(most, S.sums[w].x);
      ctas1 += S.sums[w].y;
      ctas2 += S.sums[w].z;
    }
    if (c.seqs <= kDecThreads && most > 0) {
      const bool fit1 = (long long)ctas1 * c.kv_heads <= gridDim.x, fit2 = (long long)ctas2 * c.kv_heads <= gridDim.x;
      if (fit2 && most <= 2 * MIN) unit = 2 * MIN;        // one CTA a head, nothing to join
      else if (fit1 && most <= JOIN * MIN) unit = MIN;
      else if (fit2 && most <= JOIN * 2 * MIN) unit = 2 * MIN;
      if (unit) ctas = (long long)(unit == MIN ? ctas1 : ctas2) * c.kv_heads;
    }
  }
  // A head's steps as they are cut.
  auto counted = [&](int n) {
    if (ALIGN && unit) return (n + unit - 1) & -unit;
    return n > 0 ? n + extra : 0;
  };
  total = ALIGN && unit ? ctas * unit : total + (long long)extra * some * c.kv_heads;
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
  auto find = [&](int s, int n, long long at) {   // n: steps of a head with the extra ones
    if (n > 0 && at <= begin && begin < at + (long long)n * c.kv_heads) {
      S.found[0] = s;
      S.found[1] = (int)((begin - at) / n);
      S.found[2] = (int)((begin - at) % n);
    }
    __syncthreads();
  };
  if (ALIGN && unit) {
    int all;
    const int n = counted(mine), at = block_scan(n, S.red, all);
    find(tid, n, (long long)at * c.kv_heads);
  } else if (c.seqs <= kDecThreads && (extra == 0 || some == c.seqs)) {   // from the sums at hand
    find(tid, mine > 0 ? mine + extra : 0, ((long long)ahead + (long long)extra * tid) * c.kv_heads);
  } else {
    long long before = 0;
    for (int s0 = 0; s0 < c.seqs; s0 += kDecThreads) {
      Seq q;
      int n = 0, all;
      if (s0 + tid < c.seqs && load_seq(c, s0 + tid, q, false)) n = seq_steps<KEYS>(q, A.window, A.sinks).count;
      n += n > 0 ? extra : 0;
      find(s0 + tid, n, before + (long long)block_scan(n, S.red, all) * c.kv_heads);
      before += (long long)all * c.kv_heads;
      if (before > begin) break;
    }
  }
  int s = S.found[0], head = S.found[1], v0 = S.found[2];   // (v: steps as they are counted)

  Seq q;
  load_seq(c, s, q, false);
  Steps st = seq_steps<KEYS>(q, A.window, A.sinks);
  for (long long it = begin; it < end;) {
    const int vs = counted(st.count), pad = vs - st.count, v1 = (int)(end - it < vs - v0 ? v0 + (end - it) : vs);
    const int i0 = v0 > pad ? v0 - pad : 0, i1 = v1 - pad;
    if (i1 > i0) {
      const int rows = q.n * A.group;
      body(q, s, st, head, i0, i1);
      __syncthreads();
      const bool whole = i0 == 0 && i1 == st.count;
      const long long seg0 = it - v0 + pad;   // the (sequence, head)'s steps: seg0 .. seg0 + count - 1
      float* slot = A.ws + (size_t)(2 * blockIdx.x + (i0 == 0 ? 1 : 0)) * kSlot;
      for (int k = tid; k < rows * D; k += kDecThreads) {
        const int row = k / D, d = k - row * D;
        float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
        for (int w = 0; w < kDecWarps; ++w) M = fmaxf(M, S.m[w][row]);
        const float mm = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int w = 0; w < kDecWarps; ++w) {
          const float f = exp2_fast(S.m[w][row] - mm);
          L = fmaf(f, S.l[w][row], L);
          O = fmaf(f, reinterpret_cast<const float*>(mem + w * pitch)[k], O);
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
          if (tid == 0) S.arrived = atom_add_acq_rel_gpu(counter, 1u);
          __syncthreads();
          if (S.arrived != (uint32_t)(of - 1)) return false;
          __threadfence();
          if (tid == 0) *counter = 0u;
          return true;
        };
        auto join = [&](int b0, int step, int cnt, bool final) {
          for (int k = tid; k < cnt * rows; k += kDecThreads) {
            const float* p = slot_of(b0 + (k / rows) * step) + R * D + k % rows;
            S.part_m[k / rows][k % rows] = __ldcg(p);
            S.part_l[k / rows][k % rows] = __ldcg(p + R);
          }
          __syncthreads();
          float M = -INFINITY, L = 0.f;
          if (tid < rows) {
            for (int b = 0; b < cnt; ++b) M = fmaxf(M, S.part_m[b][tid]);
            const float mm = M == -INFINITY ? 0.f : M;
            for (int b = 0; b < cnt; ++b) {
              const float f = exp2_fast(S.part_m[b][tid] - mm);
              S.part_m[b][tid] = f;
              L = fmaf(f, S.part_l[b][tid], L);
            }
            S.part_l[0][tid] = L;
          }
          __syncthreads();
          float* dst = slot_of(b0);
          for (int k = 4 * tid; k < rows * D; k += 4 * kDecThreads) {
            const int row = k / D, d = k - row * D;
            float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
            for (int b = 0; b < cnt; ++b) {
              const float4 v = __ldcg(reinterpret_cast<const float4*>(slot_of(b0 + b * step) + k));
              const float f = S.part_m[b][row];
              O.x = fmaf(f, v.x, O.x);
              O.y = fmaf(f, v.y, O.y);
              O.z = fmaf(f, v.z, O.z);
              O.w = fmaf(f, v.w, O.w);
            }
            if (final) {
              const float sum = S.part_l[0][row], r = sum == 0.f ? 0.f : __frcp_rn(sum);
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
        if (n > JOIN) {
          per = 1;
          while (per * per < n) ++per;
          const int b0 = c0 + ((int)blockIdx.x - c0) / per * per, cnt = c1 - b0 + 1 < per ? c1 - b0 + 1 : per;
          // (a CTA may start one group of an earlier head and the first group of its last head)
          if (!last_of(A.counters + (b0 == c0 ? 2 : 1) * gridDim.x + b0, cnt)) per = 0;
          if (per) join(b0, 1, cnt, false);
        }
        if (per && last_of(A.counters + c0, n > JOIN ? (n + per - 1) / per : n))
          join(c0, n > JOIN ? per : 1, n > JOIN ? (n + per - 1) / per : n, true);
      }
      __syncthreads();
    }

    // ---- on to the next (sequence, head)
    it += v1 - v0;
    v0 = 0;
    if (it < end && ++head == c.kv_heads) {
      head = 0;
      do {
        ++s;
        st.count = load_seq(c, s, q, false) ? (st = seq_steps<KEYS>(q, A.window, A.sinks)).count : 0;
      } while (st.count == 0);
    }
  }
}

}  // namespace dptq
