// kv8_decode.cu -- attention of a few rows (at most 16 for each sequence and KV head) over the
// paged int8 cache: decode steps and a few speculative tokens.
//
// The call is a stream over the visible K and V codes (one byte a value, read once) with
// 2 R multiply-adds (4 R flops) a pair of bytes for R rows, so bytes bound it.  Work is cut into steps of 32
// keys of one (sequence, KV head); the CTAs of one resident wave take equal, contiguous
// shares of all steps whatever the lengths are (they are read from the device), and a
// (sequence, head) that several CTAs share is joined by the last of them to finish.
// Inside a CTA the warps take every fourth step; each keeps its own running maximum, sum and
// accumulators, joined through shared memory once per share.
//
// A warp multiplies with 16 x 8 x 16 register MMAs, codes first (keys x rows of q, then dims x
// rows: eight rows are then no padding): with at most 16 rows there is nothing for tcgen05's
// 128-row tiles to do.  Each warp keeps its own ring of steps in shared memory, filled by
// asynchronous 16-byte copies (no barrier between warps), and reads fragments in whatever
// order suits 16-byte reads:
//   * logits: the A fragment of key g takes any order of the dims as long as q has the same,
//     so a lane takes 16 consecutive bytes of its keys' rows at a time;
//   * values: the A fragment of dim g takes any order of the dims across its tiles, so a lane
//     takes D / 8 consecutive bytes of four keys.
// Each 16-byte chunk of a 128-byte line stands at its place xor the line's number mod 8, so
// that neither read meets a bank twice.
// int8 -> binary16 is exact: a byte c + 128 under the exponent of 1024 is 1152 + c.
//
// Softmax in base 2 on x_j = log2(e) scale sk (q . ck_j) + log2(sv): the weights that go into
// the second product are then p_j sv_j relative to the largest of them, and binary16 loses
// nothing to pages whose scales are far apart; the denominator takes each back by 1 / sv.
//
// 32 ragged sequences up to 4096 tokens, 32 heads of 128 (579 MB): 98.7 us, 5.9 TB/s (of 64, 289 MB: 68.0 us,
// 4.3 TB/s); one of 131072 tokens, 64 over 8 heads (269 MB): 54.9 us, 4.9 TB/s, of which the join of 57 shares a
// head takes about 6.
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv8_device.cuh"

namespace dptq {

constexpr int kDecWarps = 4, kDecThreads = 32 * kDecWarps;
constexpr int kDecKeys = 32;        // keys of a step
// Fewest steps that a CTA is started for: one a warp (one sequence, 8 heads, with 4 / 8 steps, us: of 512 tokens
// 9.5 / 10.1, of 2048 12.8 / 10.9, of 8192 13.5 / 16.6).  Most partial results joined at once (57 of one sequence of 131072 tokens in two levels: 54.9 us;
// in one: 59.3 us), and of a group, or groups: sqrt of a grid of 1024 CTAs at most.
constexpr int kDecMinSteps = 4, kDecJoin = 12, kDecJoinMost = 32;

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Four codes of two keys to four pairs (key a, key b).
__device__ __forceinline__ void widen_pairs(uint32_t a, uint32_t b, uint32_t (&r)[4]) {
  const uint32_t lo = __byte_perm(a, b, 0x5140) ^ 0x80808080u, hi = __byte_perm(a, b, 0x7362) ^ 0x80808080u;
  r[0] = less_1152(__byte_perm(lo, 0x64646464u, 0x4140));
  r[1] = less_1152(__byte_perm(lo, 0x64646464u, 0x4342));
  r[2] = less_1152(__byte_perm(hi, 0x64646464u, 0x4140));
  r[3] = less_1152(__byte_perm(hi, 0x64646464u, 0x4342));
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

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {   // of binary16, two of a row in each lane
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <int D, int RT>   // RT: tiles of 8 rows (1 or 2)
__global__ void __launch_bounds__(kDecThreads, RT == 1 ? kDecodeCtas8 : kDecodeCtas16)
kv8_decode_kernel(const Kv8AttendArgs A) {
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

  pdl_launch_dependents();
  pdl_wait();

  // ---- this CTA's share
  long long total = 0;
  int some = 0;   // sequences with steps
  bool none = false;   // a sequence of rows without a key
  int mine = 0, ahead = 0;   // this thread's sequence of the last 128: its steps, those before it
  for (int s0 = 0; s0 < c.seqs; s0 += kDecThreads) {
    Seq q;
    int n = 0, all;
    if (s0 + tid < c.seqs && load_seq(c, s0 + tid, q, blockIdx.x == 0)) {
      n = seq_steps(q, A.window, A.sinks).count;
      none |= n == 0 && q.n > 0;
    }
    ahead = block_scan(n, red, all);
    mine = n;
    total += all;
    some += __syncthreads_count(n > 0);
  }
  total *= c.kv_heads;
  long long ctas = (total + kDecMinSteps - 1) / kDecMinSteps;
  if (ctas > gridDim.x) ctas = gridDim.x;
  const int extra = total >= (long long)kDecExtraFrom * ctas ? kDecExtra : 0;
  total += (long long)extra * some * c.kv_heads;
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
      found[0] = s;
      found[1] = (int)((begin - at) / n);
      found[2] = (int)((begin - at) % n);
    }
    __syncthreads();
  };
  if (c.seqs <= kDecThreads && (extra == 0 || some == c.seqs)) {   // from the sums at hand
    find(tid, mine > 0 ? mine + extra : 0, ((long long)ahead + (long long)extra * tid) * c.kv_heads);
  } else {
    long long before = 0;
    for (int s0 = 0; s0 < c.seqs; s0 += kDecThreads) {
      Seq q;
      int n = 0, all;
      if (s0 + tid < c.seqs && load_seq(c, s0 + tid, q, false)) n = seq_steps(q, A.window, A.sinks).count;
      n += n > 0 ? extra : 0;
      find(s0 + tid, n, before + (long long)block_scan(n, red, all) * c.kv_heads);
      before += (long long)all * c.kv_heads;
      if (before > begin) break;
    }
  }
  int s = found[0], head = found[1], v0 = found[2];   // (v: steps with the extra ones)

  Seq q;
  load_seq(c, s, q, false);
  Steps st = seq_steps(q, A.window, A.sinks);
  for (long long it = begin; it < end;) {
    const int vs = st.count + extra, v1 = (int)(end - it < vs - v0 ? v0 + (end - it) : vs);
    const int i0 = v0 > extra ? v0 - extra : 0, i1 = v1 - extra;
    if (i1 > i0) {
      const int rows = q.n * A.group;

      // ---- this share's rows of q, in the order of the dims that the keys' bytes have
      uint32_t qf[RT][D / 16][2];
      int pos[RT][2];   // positions of the two rows whose logits this lane holds
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        // (lanes without a row read the first one: a load in a branch would wait for its own data)
        const int row = g + 8 * r < rows ? g + 8 * r : 0, tok = row / A.group, hh = row - tok * A.group;
        const __half* src = A.q + (size_t)(q.tok0 + tok) * A.q_stride + (size_t)(head * A.group + hh) * D;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint2 v = ld_plain(reinterpret_cast<const uint2*>(src + D / 4 * t + 4 * k));
          qf[r][k][0] = v.x;
          qf[r][k][1] = v.y;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int mine = 8 * r + 2 * t + e;
          pos[r][e] = mine < rows ? q.start + mine / A.group : -1;
        }
      }
      // weighted values of two rows, dims VB g + 2 j and the next
      float o[RT][VB / 2][4], m[RT][2], l[RT][2];
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        m[r][0] = m[r][1] = -INFINITY;
        l[r][0] = l[r][1] = 0.f;
#pragma unroll
        for (int j = 0; j < VB / 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[r][j][e] = 0.f;
      }

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
        // logits of 16 keys and 8 rows: keys g, g + 8, rows 2 t, 2 t + 1
        float x[2][RT][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[h][r][e] = 0.f;
#pragma unroll
          for (int ch = 0; ch < D / 64; ++ch) {
            const uint4 k0 = *reinterpret_cast<const uint4*>(sk + swz((16 * h + g) * D + D / 4 * t + 16 * ch));
            const uint4 k1 = *reinterpret_cast<const uint4*>(sk + swz((16 * h + 8 + g) * D + D / 4 * t + 16 * ch));
            const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint32_t a0, a1, a2, a3;
              widen4(w0[k], a0, a2);
              widen4(w1[k], a1, a3);
#pragma unroll
              for (int r = 0; r < RT; ++r) mma_16816(x[h][r], a0, a1, a2, a3, qf[r][4 * ch + k][0], qf[r][4 * ch + k][1]);
            }
          }
        }
        // every row sees every key of the step
        const bool all = held0 && held1 && key + kDecKeys - 1 <= q.start &&
                         (A.window == 0 || key > q.len - 1 - A.window || key + kDecKeys <= A.sinks);
        float inv[2], top[RT][2];
#pragma unroll
        for (int r = 0; r < RT; ++r) top[r][0] = m[r][0], top[r][1] = m[r][1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {   // per 16 keys one factor and one addend
          const float v = fmaxf(h ? scl.w : scl.z, 0x1p-40f);   // (below, 127 sv is no binary16 any more)
          const bool finite = isfinite(h ? scl.y : scl.x) && isfinite(h ? scl.w : scl.z);
          // (what is not seen is masked below: such a page stays with the rows that see it)
          const float fa = (h ? scl.y : scl.x) * (A.scale * 1.4426950408889634f), fb = finite ? __log2f(v) : NAN;
          inv[h] = __frcp_rn(v);
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[h][r][e] = fmaf(x[h][r][e], fa, fb);
        }
        if (!all) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (!((h ? held1 : held0) &&
                      kv8_sees(pos[r][e & 1], key + 16 * h + g + 8 * (e >> 1), A.window, A.sinks)))
                  x[h][r][e] = -INFINITY;
        }
        bool grown = false;
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float v = fmaxf(fmaxf(x[0][r][e], x[0][r][e + 2]), fmaxf(x[1][r][e], x[1][r][e + 2]));
            grown |= v > m[r][e];
            top[r][e] = fmaxf(v, m[r][e]);
          }
        if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
              for (int w = 4; w < 32; w <<= 1) top[r][e] = fmaxf(top[r][e], __shfl_xor_sync(0xffffffffu, top[r][e], w));
              const float f = top[r][e] == m[r][e] ? 1.f : exp2_fast(m[r][e] - top[r][e]);
              m[r][e] = top[r][e];
              l[r][e] *= f;
#pragma unroll
              for (int j = 0; j < VB / 2; ++j) o[r][j][e] *= f, o[r][j][e + 2] *= f;
            }
        }
        uint32_t pf[2][RT][2];   // B fragments of the weights, per 16 keys
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const float m0 = m[r][0] == -INFINITY ? 0.f : m[r][0], m1 = m[r][1] == -INFINITY ? 0.f : m[r][1];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float p0 = exp2_fast(x[h][r][0] - m0), p1 = exp2_fast(x[h][r][1] - m1);
            const float p2 = exp2_fast(x[h][r][2] - m0), p3 = exp2_fast(x[h][r][3] - m1);
            l[r][0] = fmaf(p0 + p2, inv[h], l[r][0]);
            l[r][1] = fmaf(p1 + p3, inv[h], l[r][1]);
            pf[h][r][0] = transpose8x8(pack_half2(p0, p1));
            pf[h][r][1] = transpose8x8(pack_half2(p2, p3));
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t vw[4][VB / 4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {   // keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
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
            uint32_t a[4], b[4];
            widen_pairs(vw[0][w], vw[1][w], a);
            widen_pairs(vw[2][w], vw[3][w], b);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
              mma_16816(o[r][2 * w], a[0], a[1], b[0], b[1], pf[h][r][0], pf[h][r][1]);
              mma_16816(o[r][2 * w + 1], a[2], a[3], b[2], b[3], pf[h][r][0], pf[h][r][1]);
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
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = 8 * r + 2 * t + e;
#pragma unroll
          for (int w = 4; w < 32; w <<= 1) l[r][e] += __shfl_xor_sync(0xffffffffu, l[r][e], w);
          float* dst = reinterpret_cast<float*>(&ring) + row * D + VB * g;
#pragma unroll
          for (int j = 0; j < VB / 2; ++j) *reinterpret_cast<float2*>(dst + 2 * j) = make_float2(o[r][j][e], o[r][j][e + 2]);
          if (g == 0) {
            s_m[warp][row] = m[r][e];
            s_l[warp][row] = l[r][e];
          }
        }
      __syncthreads();
      const bool whole = i0 == 0 && i1 == st.count;
      const long long seg0 = it - v0 + extra;   // the (sequence, head)'s steps: seg0 .. seg0 + count - 1
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
    }

    // ---- on to the next (sequence, head)
    it += v1 - v0;
    v0 = 0;
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
  return launch_after(fn, num_sms * (RT == 1 ? kDecodeCtas8 : kDecodeCtas16), kDecThreads, smem, s, 1, a);
}

cudaError_t launch_kv8_decode(const Kv8AttendArgs& a, int num_sms, cudaStream_t s) {
  const bool one = a.c.max_tokens * a.group <= 8;
  if (a.c.head_dim == 64) return one ? launch_decode<64, 1>(a, num_sms, s) : launch_decode<64, 2>(a, num_sms, s);
  return one ? launch_decode<128, 1>(a, num_sms, s) : launch_decode<128, 2>(a, num_sms, s);
}

}  // namespace dptq
