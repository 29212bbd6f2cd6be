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

#include "kv_decode.cuh"

namespace dptq {

constexpr int kDecKeys = 32;        // keys of a step
// Fewest steps that a CTA is started for: one a warp (one sequence, 8 heads, with 4 / 8 steps, us: of 512 tokens
// 9.5 / 10.1, of 2048 12.8 / 10.9, of 8192 13.5 / 16.6).  Most partial results joined at once (57 of one sequence of 131072 tokens in two levels: 54.9 us;
// in one: 59.3 us).
constexpr int kDecMinSteps = 4, kDecJoin = 12;
// Four codes of two keys to four pairs (key a, key b).
__device__ __forceinline__ void widen_pairs(uint32_t a, uint32_t b, uint32_t (&r)[4]) {
  const uint32_t lo = __byte_perm(a, b, 0x5140) ^ 0x80808080u, hi = __byte_perm(a, b, 0x7362) ^ 0x80808080u;
  r[0] = less_1152(__byte_perm(lo, 0x64646464u, 0x4140));
  r[1] = less_1152(__byte_perm(lo, 0x64646464u, 0x4342));
  r[2] = less_1152(__byte_perm(hi, 0x64646464u, 0x4140));
  r[3] = less_1152(__byte_perm(hi, 0x64646464u, 0x4342));
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
// Where byte `at` (a multiple of 8) of a half of a step stands.
__device__ __forceinline__ uint32_t swz(uint32_t at) { return at ^ (((at >> 7) & 7u) << 4); }

template <int D, int RT>   // RT: tiles of 8 rows (1 or 2)
__global__ void __launch_bounds__(kDecThreads, RT == 1 ? kDecodeCtas8 : kDecodeCtas16)
kv8_decode_kernel(const Kv8AttendArgs A) {
  constexpr int VB = D / 8;                       // bytes of a V row for one lane; n-tiles of the second product
  constexpr int R = 8 * RT;
  constexpr int NS = Ring<D>::kStages, H = Ring<D>::kHalf;
  extern __shared__ __align__(128) uint8_t sm[];
  __shared__ JoinShared<R> S;
  Ring<D>* rings = reinterpret_cast<Ring<D>*>(sm);   // (each warp's becomes its weighted values [R][D] at a share's end)
  const Kv8Args& c = A.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int P = 1 << c.log2_page;
  Ring<D>& ring = rings[warp];

  pdl_launch_dependents();
  pdl_wait();

  decode_shares<D, R, kDecKeys, kDecMinSteps, kDecJoin, false>(c, A, S, sm, sizeof(Ring<D>), [&](const Seq& q, int s, const Steps& st, int head, int i0, int i1) {
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
          S.m[warp][row] = m[r][e];
          S.l[warp][row] = l[r][e];
        }
      }
  });
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
