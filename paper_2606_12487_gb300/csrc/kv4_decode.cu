// kv4_decode.cu -- attention of a few rows (at most 16 for each sequence and KV head) over the
// paged 4-bit cache: decode steps and a few speculative tokens.
//
// The call is a stream over the visible codes and scales (a byte for two values, read once), so bytes bound it, and
// almost as closely the codes' way into the tensor cores: a step of 64 keys is about 1100 instructions of a warp.  Work is cut into equal
// shares of steps (kv_decode.cuh); inside a CTA the warps take every fourth step, each with a ring of steps of its
// own in shared memory, filled by asynchronous 16-byte copies (no barrier between warps).
//
// A warp multiplies with 16 x 8 x 16 register MMAs, codes first (keys x rows of q, then dims x rows):
//   * logits: the A fragment of key g takes any order of the dims as long as q has the same, so a lane takes
//     D / 4 consecutive dims of its keys, and the pairs (0, 4), (1, 5), .. that a word widens to;
//   * values: the A fragment of dim g takes any order of the dims across its tiles, so a lane takes D / 8
//     consecutive dims of four keys; the 16-bit halves of two keys' words make pairs (key, key).
// Each 32-byte part of a 128-byte line stands at its place xor the line's number mod 4, so that neither
// read meets a bank twice.
//
// Softmax in base 2 on x_j = log2(e) scale sk (q . ck_j) + log2(sv): codes are the exact operands, scales
// stay in fp32, and the weights that go into the second product are p_j sv_j relative to 2^-15 of the largest of
// them: binary16 holds 29 binades of those at full precision.  They are rounded to it, 2^-11 of each (both operands of an MMA
// have one type); the denominator, in fp32, takes each unrounded one back by 1 / sv.  The rms error of outputs is 2.21e-4 of
// them instead of the 2.08e-4 of rounding the exact ones.
//
// Both operands are the codes themselves.  (K's nibbles as code + 8, one instruction less a pair, a row's sum starting at -8 times the sum of
// its q: errors go by 8 sum |q| then, which a channel of q far above the others, over keys with the code 0 there, brings into the
// logits, for 121 instead of 122 us at the first size below, and 161 instead of 159 with two rows each of 64 sequences of 8000.  V's: what
// cancels is 8 times the sum of the weights, and outputs next to zero do not survive it.)
//
// 64 ragged sequences up to 16384 tokens, 64 over 8 heads of 128 (590 MB): 122.5 us, 4.8 TB/s (its copies alone take 98 us, its
// instructions alone 113); 32 up to 4096, 32 heads (298 MB): 72 us, of 64 51 us; one of 131072 tokens, 8 heads (138 MB): 41 us;
// one of 512: 9 us.
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv4_device.cuh"
#include "kv_decode.cuh"

namespace dptq {

// A warp's ring: steps of 16 NG keys, K codes, then V codes, and what goes with a step.
template <int D, int NG>
struct alignas(128) Ring4 {
  static constexpr int kKeys = 16 * NG, kHalf = kKeys * D / 2;   // bytes of K (and of V)
  static constexpr int kStages = 8192 / kHalf;                   // 16 KB a warp
  uint8_t kv[kStages][2 * kHalf];
  uint16_t scale[kStages][2][kKeys];
  float4 factor[kKeys];      // of a step's keys: x = a S + b; 1 / sv
  uint32_t held[kStages];    // bit h: the page of keys 16 h .. is there
};
// (a page that is not there reads page 0: its keys are masked)
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// Where byte `at` of a half of a step stands: 32-byte parts of the lines of 8 rows.
template <int D>
__device__ __forceinline__ uint32_t swz32(uint32_t at) {
  return at ^ (((at >> 7) & (D / 32 - 1u)) << 5);
}
__device__ __forceinline__ uint32_t bits(const __half2& h) { return *reinterpret_cast<const uint32_t*>(&h); }

__device__ __forceinline__ float log2_fast(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Keys of a step, in 16s.  Four, with three CTAs an SM, 64 ragged sequences: 122 us; two: 139, and with four CTAs of shorter rings an
// SM 139.  Two rows of each of 64 sequences of 8000, four / two: 159 / 178 us.
constexpr int kNG = 4;
// A power of two, a step a warp; and results of as many CTAs are joined at once: four sequences of 4000 tokens, 8 heads, 15.1 us (shares
// without regard to heads, of 12 at once: 23.9), one of 8192 15.3 (19.0), one of 2048 11.7 (11.3), 16 up to 8000 over 4 heads 26.5 (29.4).
constexpr int kDec4MinSteps = 4, kDec4Join = 20;
constexpr float kDecUnit = 15.f;   // weights are relative to 2^-15 of the largest

template <int D, int RT, int NG>   // RT: tiles of 8 rows (1 or 2)
__global__ void __launch_bounds__(kDecThreads, RT == 1 ? kDecode4Ctas8 : kDecodeCtas16)
kv4_decode_kernel(const Kv4AttendArgs A) {
  using Ring = Ring4<D, NG>;
  constexpr int KW = D / 32, VW = D / 64, VB = D / 8;   // words of a K and V row, and dims of a V row, for a lane
  constexpr int R = 8 * RT, NS = Ring::kStages, H = Ring::kHalf, kKeys = Ring::kKeys;
  extern __shared__ __align__(128) uint8_t sm[];
  __shared__ JoinShared<R> S;
  const Kv8Args& c = A.k.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int P = 1 << c.log2_page;
  Ring& ring = reinterpret_cast<Ring*>(sm)[warp];   // (becomes the warp's weighted values [R][D] at a share's end)

  // Where a lane's copies go, and its reads of K and V come from, within a step (8 and 16 keys on, the swizzle is the same).
  const uint32_t to_lane = smem_u32(ring.kv[0]) + swz32<D>(16 * lane), k_lane = swz32<D>(g * (D / 2) + D / 8 * t);
  const uint32_t v_lane[2] = {swz32<D>(2 * t * (D / 2) + D / 16 * g), swz32<D>((2 * t + 1) * (D / 2) + D / 16 * g)};
  // (scales: lanes 2 h and 2 h + 1 copy K's of the step's keys 16 h .., the next 2 NG lanes V's)
  const uint32_t to_scale = smem_u32(ring.scale[0][lane / (2 * NG) & 1]) + 16 * (lane % (2 * NG));
  const uint8_t *k_from = A.k.codes[0] + 16 * lane, *v_from = A.k.codes[1] + 16 * lane;
  const uint8_t* s_from = reinterpret_cast<const uint8_t*>(lane / (2 * NG) ? A.k.scales[1] : A.k.scales[0]) + 16 * (lane & 1);
  const Nibbles nib;
  const float unit = A.scale * 1.4426950408889634f;

  pdl_launch_dependents();
  pdl_wait();

  decode_shares<D, R, kKeys, kDec4MinSteps, kDec4Join, true>(c, A, S, sm, sizeof(Ring), [&](const Seq& q, int s, const Steps& st, int head, int i0, int i1) {
    const int rows = q.n * A.group;
    // ---- this share's rows of q, in the order of the dims that a widened word has
    uint32_t qf[RT][D / 16][2];
    int pos[RT][2];   // positions of the two rows whose logits this lane holds
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      // (lanes without a row read the first one: a load in a branch would wait for its own data)
      const int row = g + 8 * r < rows ? g + 8 * r : 0, tok = row / A.group, hh = row - tok * A.group;
      const __half* src = A.q + (size_t)(q.tok0 + tok) * A.q_stride + (size_t)(head * A.group + hh) * D + D / 4 * t;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const uint4 v = ld_plain(reinterpret_cast<const uint4*>(src) + w);
        // nibbles (0, 4), (2, 6) and (1, 5), (3, 7) together
        qf[r][2 * w][0] = __byte_perm(v.x, v.z, 0x5410);
        qf[r][2 * w][1] = __byte_perm(v.y, v.w, 0x5410);
        qf[r][2 * w + 1][0] = __byte_perm(v.x, v.z, 0x7632);
        qf[r][2 * w + 1][1] = __byte_perm(v.y, v.w, 0x7632);
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
    auto key_of = [&](int i) { return i < st.sink ? i * kKeys : st.from + (i - st.sink) * kKeys; };
    // Lane h: the page of the step's keys 16 h .., or -1 (pages that no row sees are not looked up)
    auto page_of = [&](int i) {
      if (i >= i1 || lane >= NG) return -1;
      const int k = key_of(i) + 16 * lane;
      const bool seen = k < q.len && (A.window == 0 || k + 15 > (q.start > 0 ? q.start : 0) - A.window || k < A.sinks);
      return seen ? load_page(c, s, k >> c.log2_page) : -1;
    };
    // copies step i into its stage; always one group, so that the waits can count
    auto issue = [&](int i, int stage, int page) {
      if (i < i1) {
        const int in = key_of(i) & (P - 1);
        const uint32_t held = __ballot_sync(0xffffffffu, page >= 0);
        const int from = max(page, 0);
        auto row_of = [&](int h) {   // of the cache, of the step's key 16 h (fewer than 2^32, checked on the host)
          return ((unsigned)__shfl_sync(0xffffffffu, from, h) * c.kv_heads + head) * P + ((in + 16 * h) & (P - 1));
        };
        const uint32_t dst = to_lane + stage * (2 * H);
#pragma unroll
        for (int h = 0; h < NG; ++h) {
          const unsigned row = row_of(h);
          const uint8_t *ks = k_from + (unsigned long long)row * (D / 2), *vs = v_from + (unsigned long long)row * (D / 2);
#pragma unroll
          for (int u = 0; u < D / 64; ++u) {
            copy16(dst + 8 * D * h + 512 * u, ks + 512 * u);
            copy16(dst + H + 8 * D * h + 512 * u, vs + 512 * u);
          }
        }
        const unsigned row = row_of((lane >> 1) % NG);
        if (lane < 4 * NG) copy16(to_scale + stage * (4 * kKeys), s_from + (unsigned long long)row * 2);
        if (lane == 0) ring.held[stage] = held;
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };

    int i = i0 + warp, stage = 0;
#pragma unroll
    for (int k = 0; k < NS; ++k) issue(i + k * kDecWarps, k, page_of(i + k * kDecWarps));
    for (; i < i1; i += kDecWarps) {
      const int page = page_of(i + NS * kDecWarps);   // (used after this step)
      asm volatile("cp.async.wait_group %0;" ::"n"(NS - 1) : "memory");
      __syncwarp();
      const uint8_t* ck = ring.kv[stage];
      const uint8_t* cv = ck + H;
      const uint32_t held = ring.held[stage];
      const int key = key_of(i);
      // a key's factor and addend, made by a lane for all
#pragma unroll
      for (int k = lane; k < kKeys; k += 32) {
        const uint32_t sk = ring.scale[stage][0][k], sv = ring.scale[stage][1][k];
        const float v = fmaxf(bf16_float(sv), 0x1p-40f);   // (zeros, which add nothing)
        // (NaN for a scale that is no number; what is not seen is masked below, so it stays with the rows that see it)
        ring.factor[k] = make_float4(bf16_float(sk) * unit, kv4_bad(max(sk, sv)) ? NAN : log2_fast(v), rcp_fast(v), 0.f);
      }
      // logits of 16 keys and 8 rows: keys g, g + 8, rows 2 t, 2 t + 1
      float x[NG][RT][4];
#pragma unroll
      for (int h = 0; h < NG; ++h) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[h][r][e] = 0.f;
        uint32_t w0[KW], w1[KW];
        const uint8_t* p0 = ck + k_lane + 8 * D * h;
        const uint8_t* p1 = p0 + 4 * D;
        if constexpr (D == 128) {
          const uint4 a = *reinterpret_cast<const uint4*>(p0), b = *reinterpret_cast<const uint4*>(p1);
          w0[0] = a.x, w0[1] = a.y, w0[2] = a.z, w0[3] = a.w;
          w1[0] = b.x, w1[1] = b.y, w1[2] = b.z, w1[3] = b.w;
        } else {
          const uint2 a = *reinterpret_cast<const uint2*>(p0), b = *reinterpret_cast<const uint2*>(p1);
          w0[0] = a.x, w0[1] = a.y;
          w1[0] = b.x, w1[1] = b.y;
        }
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          __half2 a[4], b[4];
          nib.codes(w0[w], a);
          nib.codes(w1[w], b);
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int k = 0; k < 2; ++k)
              mma_16816(x[h][r], bits(a[k]), bits(b[k]), bits(a[k + 2]), bits(b[k + 2]), qf[r][2 * w + k][0], qf[r][2 * w + k][1]);
        }
      }
      __syncwarp();
#pragma unroll
      for (int h = 0; h < NG; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float2 f = *reinterpret_cast<const float2*>(&ring.factor[16 * h + g + 8 * e]);
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            x[h][r][2 * e] = fmaf(x[h][r][2 * e], f.x, f.y);
            x[h][r][2 * e + 1] = fmaf(x[h][r][2 * e + 1], f.x, f.y);
          }
        }
      // every row sees every key of the step
      const bool all = held == (1u << NG) - 1 && key + kKeys - 1 <= q.start &&
                       (A.window == 0 || key > q.len - 1 - A.window || key + kKeys <= A.sinks);
      if (!all) {
#pragma unroll
        for (int h = 0; h < NG; ++h)
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!((held >> h & 1u) && kv8_sees(pos[r][e & 1], key + 16 * h + g + 8 * (e >> 1), A.window, A.sinks)))
                x[h][r][e] = -INFINITY;
      }
      float top[RT][2];
      bool grown = false;
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float v = -INFINITY;
#pragma unroll
          for (int h = 0; h < NG; ++h) v = max3(v, x[h][r][e], x[h][r][e + 2]);
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
      uint32_t pf[NG][RT][2];   // B fragments of the weights, per 16 keys
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        // (rounded up: a weight above 2^15 may be none that binary16 holds)
        const float m0 = m[r][0] == -INFINITY ? 0.f : __fsub_ru(m[r][0], kDecUnit), m1 = m[r][1] == -INFINITY ? 0.f : __fsub_ru(m[r][1], kDecUnit);
#pragma unroll
        for (int h = 0; h < NG; ++h) {
          const float p0 = exp2_fast(x[h][r][0] - m0), p1 = exp2_fast(x[h][r][1] - m1);
          const float p2 = exp2_fast(x[h][r][2] - m0), p3 = exp2_fast(x[h][r][3] - m1);
          const float i0 = ring.factor[16 * h + g].z, i1 = ring.factor[16 * h + g + 8].z;
          l[r][0] = fmaf(p0, i0, fmaf(p2, i1, l[r][0]));
          l[r][1] = fmaf(p1, i0, fmaf(p3, i1, l[r][1]));
          pf[h][r][0] = transpose8x8(pack_half2(p0, p1));
          pf[h][r][1] = transpose8x8(pack_half2(p2, p3));
        }
      }
#pragma unroll
      for (int h = 0; h < NG; ++h) {
        uint32_t vw[4][VW];
#pragma unroll
        for (int u = 0; u < 4; ++u) {   // keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
          const uint8_t* p = cv + v_lane[u & 1] + 8 * D * h + 4 * D * (u >> 1);
          if constexpr (D == 128) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            vw[u][0] = v.x, vw[u][1] = v.y;
          } else {
            vw[u][0] = *reinterpret_cast<const uint32_t*>(p);
          }
        }
#pragma unroll
        for (int w = 0; w < VW; ++w)
#pragma unroll
          for (int k = 0; k < 2; ++k) {   // dims 8 w + 4 k .. of the lane's
            __half2 a[4], b[4];
            nib.codes(__byte_perm(vw[0][w], vw[1][w], k ? 0x7632 : 0x5410), a);
            nib.codes(__byte_perm(vw[2][w], vw[3][w], k ? 0x7632 : 0x5410), b);
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
              for (int j = 0; j < 2; ++j)
                mma_16816(o[r][4 * w + 2 * k + j], bits(a[2 * j]), bits(a[2 * j + 1]), bits(b[2 * j]), bits(b[2 * j + 1]),
                          pf[h][r][0], pf[h][r][1]);
          }
      }
      __syncwarp();
      issue(i + NS * kDecWarps, stage, page);
      stage = stage + 1 == NS ? 0 : stage + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();

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
static cudaError_t launch_decode4(const Kv4AttendArgs& a, int num_sms, cudaStream_t s) {
  const auto fn = kv4_decode_kernel<D, RT, kNG>;
  const size_t smem = sizeof(Ring4<D, kNG>) * kDecWarps;
  const cudaError_t e = ensure_max_dyn_smem(fn);
  if (e != cudaSuccess) return e;
  static_assert(kDecode4Ctas8 * 256 <= kDecJoinMost * kDecJoinMost, "groups of a join");   // (up to 256 SMs)
  if (num_sms > 256) return cudaErrorInvalidValue;
  return launch_after(fn, num_sms * (RT == 1 ? kDecode4Ctas8 : kDecodeCtas16), kDecThreads, smem, s, 1, a);
}

cudaError_t launch_kv4_decode(const Kv4AttendArgs& a, int num_sms, cudaStream_t s) {
  const bool one = a.k.c.max_tokens * a.group <= 8;
  if (a.k.c.head_dim == 64) return one ? launch_decode4<64, 1>(a, num_sms, s) : launch_decode4<64, 2>(a, num_sms, s);
  return one ? launch_decode4<128, 1>(a, num_sms, s) : launch_decode4<128, 2>(a, num_sms, s);
}

}  // namespace dptq
