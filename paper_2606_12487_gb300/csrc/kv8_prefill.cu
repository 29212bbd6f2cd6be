// kv8_prefill.cu -- attention of many rows (prompts, chunks of prompts, more than 16 rows of a
// sequence and KV head) over the paged int8 cache, on the 5th-generation tensor cores.
//
// The rows of a KV head (a token's query heads side by side, then the next token's) are cut
// into tiles of 256; a CTA takes two row tiles of 128 so that one's softmax runs while the
// tensor cores work for the other, and both share every widened K and V tile of 128 keys:
//   S = q ck^T   128 x 128 x D   both operands in shared memory, S in tensor memory
//   O += P cv    128 x D x 128   P in tensor memory (over half of S), cv in shared memory
// The codes enter the MMAs as they are (int8 is exact in binary16); scales and the softmax in
// base 2 are as in the decode kernel: x_j = log2(e) scale sk S_j + log2(sv), weights p_j sv_j
// relative to the row's maximum, the denominator taken back by 1 / sv, per 16 keys of a page.
// O is rescaled only where a row's maximum has grown by more than 2^8 (binary16 holds the
// weights that stay relative to the old one).
//
// Warp roles: 0-3 and 4-7 softmax and output of the row tiles, a row a thread; 8-11 widen K and
// V tiles (global to registers a tile ahead, then to shared memory in the 128-byte swizzle);
// 12 issues the MMAs.
//
// Many rows (kPairRows): pairs of CTAs, each widening half of every tile (PAIR below).  Few row
// tiles are split along the keys: each CTA leaves its rows' sums, and a second launch joins
// them.
//
// What bounds it, at a prompt of 8192 tokens, 64 over 8 heads of 128 (1.1 TFLOP, 811 us, 1356
// TFLOP/s, 71 % of the measured bf16 rate): the chain of a row tile from S over its softmax
// (about 2400 cycles, two tiles taking turns) back to the next S.  Without the softmax's
// waits the MMAs and the widening take 605 us (pairs; 720 us for CTAs alone, which are short of
// shared-memory bandwidth: q, K and V tiles are read at its full rate by the MMAs).  The same prompt with
// heads of 64, which take no pairs: 705 us; 256 rows behind 16000 tokens, 8 over one head, split along
// the keys, with the join: 38 us.  The roles' code has to stay short: they fetch it from one
// instruction cache (rolled loops and rare code apart: 1041 -> 904 and 878 -> 817 us).
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv8_device.cuh"

namespace dptq {

constexpr int kConvWarps = 4, kMmaWarp = 8 + kConvWarps, kPreThreads = 32 * (kMmaWarp + 4);
constexpr int kTileRows = 128, kTileKeys = 128, kPreStages = 2, kMeta = 4;
constexpr int kNoEntry = (int)0x80000000;

struct KeyMeta {     // of 16 keys
  float a, b, inv;   // x = a S + b; 1 / sv
  float pad;
};
struct PreShared {
  KeyMeta meta[kMeta][kTileKeys / 16];
  uint64_t kfull[kPreStages], kempty[kPreStages], vfull[kPreStages], vempty[kPreStages];
  uint64_t mfull[kMeta];   // meta is there (filled and read within a CTA)
  uint64_t qfull[2], sfull[2], pfull[2][2], ofull[2], drain;   // pfull: the two halves of a tile's keys
  uint64_t phalf[2];   // the first half's product is complete
  uint32_t tmem;
  int abort;
};

// D[tmem] (+)= A B^T, binary16 operands, fp32 accumulators: A in shared memory or tensor memory.
// PAIR: 128 rows of A and D and half of B's columns in each CTA of a pair.
template <bool PAIR>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Instruction descriptor: binary16 operands, fp32 accumulators, m rows (128, or 256 of a pair);
// b_mn: B's columns (N) are contiguous instead of its K.
__host__ __device__ constexpr uint32_t idesc_f16(int m, int n, bool b_mn) {
  return (1u << 4) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// B with contiguous N in the 128-byte swizzle: atoms of 64 n x 8 k, 1024 bytes apart along k,
// `n_stride` bytes apart along n.
__device__ __forceinline__ uint64_t sdesc_mn128(uint32_t saddr, uint32_t n_stride) {
  return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)(n_stride >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* r) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
        "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]),
        "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]),
        "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(taddr));
}
// Waits for the tensor-memory loads under way; `r`'s values exist from here on.
__device__ __forceinline__ void tmem_ld_arrived(float (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]), "+f"(r[8]),
                 "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]), "+f"(r[16]),
                 "+f"(r[17]), "+f"(r[18]), "+f"(r[19]), "+f"(r[20]), "+f"(r[21]), "+f"(r[22]), "+f"(r[23]), "+f"(r[24]),
                 "+f"(r[25]), "+f"(r[26]), "+f"(r[27]), "+f"(r[28]), "+f"(r[29]), "+f"(r[30]), "+f"(r[31])::"memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
template <int N>
__device__ __forceinline__ void reg_more() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void reg_less() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// mbar_wait_warp in few instructions (its clock starts at the first poll that finds nothing): the
// roles' loops together have to stay in the instruction cache.  With everything unrolled the
// MMA warp spent more time on fetching its code than on issuing it.  The bound is in cycles: a poll
// may be suspended for any time, so that a number of polls bounds nothing.
template <class Arrived>
__device__ __forceinline__ bool wait_near(Arrived arrived, volatile int* abort_flag, int* err, int code, long long limit) {
  for (long long t0 = 0; !__all_sync(0xffffffffu, arrived());) {
    const long long now = clock64();
    if (t0 == 0) t0 = now;
    __nanosleep(20);
    if (__any_sync(0xffffffffu, *abort_flag != 0 || now - t0 > limit)) {
      *abort_flag = 1;
      atomicCAS(err, 0, code);
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool mbar_wait_near(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* err,
                                               int code, long long limit) {
  return wait_near([&] { return mbar_try_wait(bar, parity); }, abort_flag, err, code, limit);
}
// What the arrivals released at cluster scope is seen (mbar_arrive_remote_release).
__device__ __forceinline__ bool mbar_wait_near_cluster(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* err,
                                                       int code, long long limit) {
  return wait_near([&] { return mbar_try_wait_cluster(bar, parity); }, abort_flag, err, code, limit);
}
// Two barriers, whose answers come back together.
__device__ __forceinline__ bool mbar_wait2_near(uint64_t* b0, uint32_t p0, uint64_t* b1, uint32_t p1,
                                                volatile int* abort_flag, int* err, int code, long long limit) {
  return wait_near(
      [&] {
        const bool r0 = mbar_try_wait(b0, p0), r1 = mbar_try_wait(b1, p1);
        return r0 && r1;
      },
      abort_flag, err, code, limit);
}

// The 128-key tiles that a CTA's rows see: `sink` tiles from key 0, then tiles from key `from`.
struct Tiles {
  int sink, from, count;
  __device__ __forceinline__ int key(int j) const { return j < sink ? j * kTileKeys : from + (j - sink) * kTileKeys; }
};
__device__ __forceinline__ Tiles row_tiles(int p_lo, int p_hi, int window, int sinks) {   // positions of the rows
  Tiles r{0, 0, 0};
  if (p_hi < 0) return r;
  if (window > 0) {
    const int first = (p_lo > 0 ? p_lo : 0) - window + 1;
    if (first >= kTileKeys) {
      r.from = first & ~(kTileKeys - 1);
      r.sink = sinks < r.from ? (sinks + kTileKeys - 1) / kTileKeys : r.from / kTileKeys;
    }
  }
  r.count = r.sink + (p_hi + 1 - r.from + kTileKeys - 1) / kTileKeys;
  return r;
}

// The n lowest bits (n of any size).
__device__ __forceinline__ uint32_t low_bits(int n) {
  return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1;
}

// The addend b of a page with a scale that is infinite or NaN.  It is finite, so that a masked S = -inf still gives
// x = -inf (+inf would give NaN to rows that do not see the page); a row that sees such a key ends
// with it as its maximum, and no other row gets near it: those rows' results are NaN.
constexpr float kNoNumber = 3.402823466e38f;
__device__ __forceinline__ float one_over_sum(float m, float l) {
  return m >= kNoNumber ? __int_as_float(0x7FFFFFFF) : l == 0.f ? 0.f : __frcp_rn(l);
}

// Writes -inf over the scores of the keys that this thread's row does not see, in tensor memory: the
// few tiles that need it pay for the pass, and the code that every tile runs stays short (with
// the masks in its middle, 929 instead of 855 us for a prompt of 8192 tokens, 64 over 8 heads).
__device__ __forceinline__ void mask_scores(uint32_t tS, int pos, int key, int window, int sinks) {
#pragma unroll 1
  for (int k = 0; k < kTileKeys; k += 16) {
    uint32_t v[16];
    tmem_ld16(tS + k, v);
    uint32_t bits = low_bits(pos - key - k + 1);   // bit e: the row sees key k + e
    if (window > 0) bits &= ~low_bits(pos - window + 1 - key - k) | low_bits(sinks - key - k);
    tmem_ld_wait();
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = bits >> e & 1u ? v[e] : 0xFF800000u;
    tmem_st16(tS + k, v);
  }
  tmem_st_wait();
}

template <int D, bool PAIR>
struct PreLayout {
  static constexpr int kHalf = 128 * 128;                          // 64 dims x 128 rows
  static constexpr int kQTile = D / 64 * kHalf;                    // a row tile of q
  static constexpr int kTile = PAIR ? kQTile / 2 : kQTile;         // this CTA's part of a widened tile:
  static constexpr int kKHalf = PAIR ? kHalf / 2 : kHalf;          // K: 64 dims x its keys; V: its dims x 128 keys
  static constexpr int kQ = 0, kK = 2 * kQTile, kV = kK + kPreStages * kTile, kEnd = kV + kPreStages * kTile;
  static constexpr int kBytes = kEnd + (int)sizeof(PreShared) + 1024;   // (1024: alignment)
};

// SPLIT: this CTA's part of the keys goes to the scratch, for kv8_join_kernel.
// PAIR: two CTAs of a cluster work on 512 rows, 256 each; the tensor cores of both take K and V
// tiles of which each CTA widens and holds one half (of K's keys, of V's dims).  That halves the
// widening, its stores and what the MMAs read of K and V from shared memory, which is what a
// CTA alone is short of.  The first CTA issues the MMAs.  What the second one stores for them reaches
// its barriers in three ways: q, once, released at cluster scope; K and V on the second CTA's own
// barriers, from which its MMA warp, which has no loads under way, passes them on released at cluster
// scope; P, stores to tensor memory, as mbar_arrive_remote says.
template <int D, bool SPLIT, bool PAIR>
__global__ void __launch_bounds__(kPreThreads, 1) kv8_prefill_kernel(const Kv8AttendArgs A, int nsplit) {
  static_assert(!PAIR || (D == 128 && !SPLIT), "a pair's halves of V are 64 dims; few rows take no pairs");
  using L = PreLayout<D, PAIR>;
  constexpr int kCtas = PAIR ? 2 : 1, kRows = kCtas * 2 * kTileRows;   // rows of a CTA or pair
  extern __shared__ uint8_t raw[];
  uint8_t* sm = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  PreShared& S = *reinterpret_cast<PreShared*>(sm + L::kEnd);
  const Kv8Args& c = A.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int head = blockIdx.x / kCtas, rank = PAIR ? blockIdx.x & 1 : 0, seq = blockIdx.y;
  const int split = SPLIT ? blockIdx.z % nsplit : 0, zt = SPLIT ? blockIdx.z / nsplit : blockIdx.z;
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(c, seq, q, tid == 0 && blockIdx.z == 0 && head == 0)) return;
  const int rows = q.n * A.group;
  const int tile = (rows + kRows - 1) / kRows - 1 - zt;   // the last rows, with the most keys, first
  if (tile < 0) return;
  const int row0 = tile * kRows, nrows = rows - row0 < kRows ? rows - row0 : kRows;
  const int halves = nrows > kCtas * kTileRows ? 2 : 1;   // row tiles (of a pair: 256 rows)
  const int p_first = q.start + row0 / A.group, p_last = q.start + (row0 + nrows - 1) / A.group;
  const Tiles all = row_tiles(p_first, p_last, A.window, A.sinks);
  const int j0 = SPLIT ? (int)((long long)all.count * split / nsplit) : 0;
  const int nt = (SPLIT ? (int)((long long)all.count * (split + 1) / nsplit) : all.count) - j0;

  if (tid == 0) {
    for (int i = 0; i < kPreStages; ++i) {
      mbar_init(&S.kfull[i], (A.shortfall == 1) + kConvWarps + (PAIR && rank == 0 ? 1 : 0));   // (and the second CTA's MMA warp)
      mbar_init(&S.vfull[i], kConvWarps + (PAIR && rank == 0 ? 1 : 0));
      mbar_init(&S.kempty[i], 1);
      mbar_init(&S.vempty[i], 1);
    }
    for (int i = 0; i < kMeta; ++i) mbar_init(&S.mfull[i], 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&S.qfull[t], kCtas * kTileRows / 32);
      mbar_init(&S.pfull[t][0], kCtas * kTileRows / 32);
      mbar_init(&S.pfull[t][1], (A.shortfall == 2) + kCtas * kTileRows / 32);
      mbar_init(&S.sfull[t], 1);
      mbar_init(&S.phalf[t], 1);
      mbar_init(&S.ofull[t], (A.shortfall == 3) + 1);
    }
    mbar_init(&S.drain, 1);
    S.abort = 0;
    fence_mbar_init();
  }
  if (warp == kMmaWarp) tmem_alloc<PAIR>(&S.tmem, 512);
  tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) {   // the other CTA's barriers are initialized
    cluster_arrive();
    cluster_wait();
  }
  tc_fence_after();
  // Arrives for this warp on a barrier of the CTA that issues the MMAs; stored: for its stores to
  // shared memory.
  auto tell_first = [&](uint64_t* bar, bool stored) {
    __syncwarp();
    if (lane == 0) {
      if (!PAIR || rank == 0)
        mbar_arrive(bar);
      else if (stored)
        mbar_arrive_remote_release(cluster_map(smem_u32(bar), 0));
      else
        mbar_arrive_remote(cluster_map(smem_u32(bar), 0));
    }
  };
  const uint32_t tm = S.tmem;   // S of the row tiles at columns 0 and 128, O at 256 and 384
  volatile int* abort_flag = &S.abort;

  if (warp < 8) {
    // ------------------------------------------------------------------ softmax, a row a thread
    reg_more<160>();
    const int t = warp >> 2, r = tid & (kTileRows - 1), row = row0 + (t * kCtas + rank) * kTileRows + r;
    const bool mine = row < row0 + nrows;
    const int tok = row / A.group, hh = row - tok * A.group;
    const int pos = mine ? q.start + tok : -1;
    const uint32_t tlane = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tm + tlane + t * 128, tO = tm + tlane + 256 + t * 128;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    if (t < halves && nt > 0) {
      {   // the warp's rows of q, whole rows at a time, negated for a negative scale
        constexpr int kLanes = D / 8, kSide = 32 / kLanes;   // 16-byte chunks of a row; rows side by side
        const uint32_t flip = A.scale < 0.f ? 0x80008000u : 0u;
        // (rows past the last one read the tile's first row: a load in a branch would wait for its own
        // data, and nobody looks at their result)
        const int from_row = mine ? row : row0, from_tok = from_row / A.group;
        const long long at = (long long)(q.tok0 + from_tok) * A.q_stride +
                             (long long)(head * A.group + from_row - from_tok * A.group) * D;
        const int ch = lane % kLanes;
        uint8_t* dst = sm + L::kQ + t * L::kQTile + (ch >> 3) * L::kHalf;
#pragma unroll
        for (int i = 0; i < 32 / kSide; ++i) {
          const int from = kSide * i + lane / kLanes, rr = (warp & 3) * 32 + from;
          const long long src = __shfl_sync(0xffffffffu, at, from);
          uint4 v = ld_plain(reinterpret_cast<const uint4*>(A.q + src) + ch);
          v.x ^= flip, v.y ^= flip, v.z ^= flip, v.w ^= flip;
          *reinterpret_cast<uint4*>(dst + rr * 128 + (((ch & 7) ^ (rr & 7)) << 4)) = v;
        }
        fence_proxy_async_smem();
        tell_first(&S.qfull[t], true);
      }
      // positions of this row tile's rows
      const int r_lo = (t * kCtas + rank) * kTileRows;
      const int r_hi = r_lo + kTileRows - 1 < nrows - 1 ? r_lo + kTileRows - 1 : nrows - 1;
      const int p_lo = q.start + (row0 + r_lo) / A.group, p_hi = q.start + (row0 + r_hi) / A.group;
      for (int j = 0; j < nt && ok; ++j) {
        ok = mbar_wait2_near(&S.mfull[j % kMeta], (j / kMeta) & 1, &S.sfull[t], j & 1, abort_flag, c.err,
                             kDevTimeoutTmemFull, A.wait_cycles);
        if (!ok) break;
        tc_fence_after();
        const int key = all.key(j0 + j);
        const bool seen = key + kTileKeys - 1 <= p_lo &&
                          (A.window == 0 || key > p_hi - A.window || key + kTileKeys <= A.sinks);
        const KeyMeta* meta = S.meta[j % kMeta];
        if (!seen) mask_scores(tS, pos, key, A.window, A.sinks);
        // Halves of 64 keys, the second one first: its weights take the place of its S, and their
        // product begins while the first half is worked on.  The weights are relative to a maximum
        // that may lag by 2^8 (binary16 holds them), so they are made before the half's own maximum
        // is known; where that is larger still, what is relative to the old one is rescaled and
        // the half made again.
        float xa[32], xb[32];
        uint32_t p[32];
        // A quarter's weights, packed, their sum, and its largest x: h its place in the tile.
        auto quarter = [&](float (&x)[32], int h, uint32_t* w, float& s, float& top) {
          const KeyMeta* mh = meta + 2 * h;
          const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            const float a0 = mh[g].a, b0 = mh[g].b;
            const uint64_t a = f2_pack(a0, a0), b = f2_pack(b0 - base, b0 - base);
            uint64_t sum = 0;
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
              float y0, y1;
              f2_unpack(f2_fma(f2_pack(x[16 * g + k], x[16 * g + k + 1]), a, b), y0, y1);
              y0 = exp2_fast(y0);
              y1 = exp2_fast(y1);
              sum = k ? f2_add(sum, f2_pack(y0, y1)) : f2_pack(y0, y1);
              w[8 * g + k / 2] = pack_half2(y0, y1);
            }
            float s0, s1;
            f2_unpack(sum, s0, s1);
            s = fmaf(s0 + s1, mh[g].inv, s);
            float v[5];
#pragma unroll
            for (int k = 0; k < 5; ++k) v[k] = max3(x[16 * g + 3 * k], x[16 * g + 3 * k + 1], x[16 * g + 3 * k + 2]);
            const float u = fmaxf(max3(v[0], v[1], v[2]), max3(v[3], v[4], x[16 * g + 15]));
            top = fmaxf(top, fmaf(u, a0, b0));
          }
        };
        if (j == 0) {   // the first maximum, so that the first half is not made for nothing
#pragma unroll 1
          for (int h = 0; h < 4; ++h) {
            tmem_ld32(tS + 32 * h, xa);
            tmem_ld_arrived(xa);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              float v = xa[16 * g];
#pragma unroll
              for (int k = 1; k < 15; k += 2) v = max3(v, xa[16 * g + k], xa[16 * g + k + 1]);
              m = fmaxf(m, fmaf(fmaxf(v, xa[16 * g + 15]), meta[2 * h + g].a, meta[2 * h + g].b));
            }
          }
        }
        tmem_ld32(tS + 64, xa);
        int n = 0;
#pragma unroll 1
        for (;;) {   // (once, but for maxima that grow: that code stands apart from what every tile runs)
          float top;
#pragma unroll 1
          for (; n < 2; ++n) {
            const int h = 2 - 2 * n;
            float s = 0.f;
            top = -INFINITY;
            tmem_ld_arrived(xa);
            tmem_ld32(tS + 32 * h + 32, xb);   // (under the first quarter's work)
            quarter(xa, h, p, s, top);
            tmem_ld_arrived(xb);
            quarter(xb, h + 1, p + 16, s, top);
            if (__any_sync(0xffffffffu, top > m + 8.f)) break;
            l += s;
            tmem_st32(tS + 64 + 32 * n, p);
            if (n == 0) tmem_ld32(tS, xa);
            tmem_st_wait();
            tc_fence_before();
            tell_first(&S.pfull[t][n], false);
          }
          if (n == 2) break;
          const float mn = fmaxf(m, top), f = mn == m ? 1.f : exp2_fast(m - mn);   // (m = -inf: no key yet)
          m = mn;
          l *= f;
          // O: PV of tile j - 1 came before S of tile j, which is here; of tile j, the first half's
          // product may be under way.
          if (n == 1) {
            ok = mbar_wait_near(&S.phalf[t], j & 1, abort_flag, c.err, kDevTimeoutTmemFull, A.wait_cycles);
            if (!ok) break;
            tc_fence_after();
          }
          if (j > 0 || n == 1) {
#pragma unroll 1
            for (int k = 0; k < D; k += 16) {
              uint32_t o[16];
              tmem_ld16(tO + k, o);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
              tmem_st16(tO + k, o);
            }
          }
          tmem_ld32(tS + 64 * (1 - n), xa);
        }
      }
      if (ok) ok = mbar_wait_near(&S.ofull[t], 0, abort_flag, c.err, kDevTimeoutTmemFull, A.wait_cycles);
      tc_fence_after();
    }
    // ---- output
    if (ok && t < halves) {
      const float inv = one_over_sum(m, l);
      __half* dst = A.out + (size_t)(q.tok0 + tok) * A.out_stride + (size_t)(head * A.group + hh) * D;
      float* part = nullptr;
      if constexpr (SPLIT) {
        part = A.ws + ((((size_t)seq * (gridDim.z / nsplit) + tile) * gridDim.x + head) * nsplit + split) *
                          (2 * kTileRows * (D + 2));
        if (mine) {
          part[2 * kTileRows * D + t * kTileRows + r] = m;
          part[2 * kTileRows * (D + 1) + t * kTileRows + r] = l;
        }
        part += (size_t)(t * kTileRows + r) * D;
      }
#pragma unroll
      for (int k = 0; k < D; k += 32) {
        float o[32];
        if (nt > 0) {
          tmem_ld32(tO + k, o);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
        if (mine) {
          if constexpr (SPLIT) {
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<float4*>(part + k + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          } else {
#pragma unroll
            for (int e = 0; e < 32; e += 8)
              *reinterpret_cast<uint4*>(dst + k + e) =
                  make_uint4(pack_half2(o[e] * inv, o[e + 1] * inv), pack_half2(o[e + 2] * inv, o[e + 3] * inv),
                             pack_half2(o[e + 4] * inv, o[e + 5] * inv), pack_half2(o[e + 6] * inv, o[e + 7] * inv));
          }
        }
      }
    }
    tc_fence_before();
  } else if (warp < kMmaWarp) {
    // ------------------------------------------------------------------ K and V, widened
    reg_less<112>();
    const int w = warp - 8, kr = lane >> 2, col = lane & 3;
    // A warp takes 64 dims of 8 keys at a time, kUnits times: blocks kb0 + kWays i of dims 64 sub ..;
    // of a pair's tile, K: its 8 blocks of keys; V: its 64 dims.
    constexpr int kUnits = (PAIR ? 8 : 16) * (D / 64) / kConvWarps;
    constexpr int kWaysK = D == 128 ? kConvWarps / 2 : kConvWarps, kWaysV = PAIR ? kConvWarps : kWaysK;
    const int subk = D == 128 ? w & 1 : 0, kbk = (PAIR ? 8 * rank : 0) + (D == 128 ? w >> 1 : w);
    const int subv = PAIR ? rank : subk, kbv = PAIR ? w : kbk;
    const int P1 = (1 << c.log2_page) - 1;
    // whether any row sees one of the 16 keys from `k` on (pages that none does are not looked up)
    auto group_seen = [&](int k) {
      return k <= p_last && (A.window == 0 || k + 15 > (p_first > 0 ? p_first : 0) - A.window || k < A.sinks);
    };
    // Lane g: the table's entry for the tile's keys 16 g .. (-1: not needed), asked for two tiles
    // ahead; it is checked when it has come.
    auto entry_of = [&](int j) {
      const int k = (j < nt ? all.key(j0 + j) : 0) + 16 * lane;
      const bool on = j < nt && lane < kTileKeys / 16 && group_seen(k);
      return on ? ld_plain(c.table + (long long)seq * c.table_stride + (k >> c.log2_page)) : kNoEntry;
    };
    auto checked = [&](int b) {
      if (b == kNoEntry) return -1;
      if (b >= 0 && b < c.num_blocks) return b;
      atomicCAS(c.bad, 0, kDevBadPage);
      return -1;
    };
    // (a page that is not there reads page 0: its keys have b = -inf below, and any codes do)
    auto load = [&](int j, int kv, int pages, uint4 (&v)[kUnits]) {
      const int key = all.key(j0 + j), kb0 = kv ? kbv : kbk, ways = kv ? kWaysV : kWaysK, sub = kv ? subv : subk;
      const int8_t* codes = kv ? c.codes[1] : c.codes[0];
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int kb = kb0 + ways * i, b = max(__shfl_sync(0xffffffffu, pages, kb >> 1), 0);
        const size_t at = ((((size_t)b * c.kv_heads + head) << c.log2_page) + ((key + 8 * kb) & P1) + kr) * D;
        v[i] = ld_plain(reinterpret_cast<const uint4*>(codes + at + 64 * sub + 16 * col));
      }
    };
    auto scale_of = [&](int kv, int pages) {   // (written to the tile's KeyMeta by one warp)
      return w == 0 && pages >= 0 ? ld_plain((kv ? c.scales[1] : c.scales[0]) + (size_t)pages * c.kv_heads + head) : 0.f;
    };
    auto store = [&](uint8_t* dst, int kv, const uint4 (&v)[kUnits]) {
      const int place = kv ? (PAIR ? 0 : subv * L::kHalf) + 8 * kbv * 128
                           : subk * L::kKHalf + 8 * (kbk - (PAIR ? 8 * rank : 0)) * 128;
      dst += place + kr * 128;
      const int step = 8 * 128 * (kv ? kWaysV : kWaysK);
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        uint8_t* p = dst + step * i;
        uint4 lo, hi;
        widen4(v[i].x, lo.x, lo.y);
        widen4(v[i].y, lo.z, lo.w);
        widen4(v[i].z, hi.x, hi.y);
        widen4(v[i].w, hi.z, hi.w);
        *reinterpret_cast<uint4*>(p + (((2 * col) ^ kr) << 4)) = lo;
        *reinterpret_cast<uint4*>(p + (((2 * col + 1) ^ kr) << 4)) = hi;
      }
      fence_proxy_async_smem();
    };
    // Units in order K 0, V 0, K 1, V 1, ..., each loaded while the one before it is widened.
    uint4 cur[kUnits], nxt[kUnits];
    const int entry0 = entry_of(0), entry1 = entry_of(1);
    int entry = entry_of(2), pages = checked(entry0), next = checked(entry1);
    if (nt > 0) load(0, 0, pages, nxt);
    float sk = scale_of(0, pages), sv = scale_of(1, pages);
#pragma unroll 1
    for (int u = 0; u < 2 * nt; ++u) {
      const int j = u >> 1, kv = u & 1, st = j % kPreStages, par = (j / kPreStages + 1) & 1;
#pragma unroll
      for (int i = 0; i < kUnits; ++i) cur[i] = nxt[i];
      if (u + 1 < 2 * nt) load((u + 1) >> 1, kv ^ 1, kv ? next : pages, nxt);
      if (!mbar_wait_near(kv ? &S.vempty[st] : &S.kempty[st], par, abort_flag, c.err, kDevTimeoutEmpty, A.wait_cycles))
        break;
      if (kv == 0) {
        if (w == 0 && lane < kTileKeys / 16) {
          const float s = fmaxf(sv, 0x1p-40f);   // (below, 127 sv is no binary16 any more)
          const bool finite = isfinite(sk) && isfinite(sv);
          // a > 0 and b < inf, so that a masked S = -inf gives x = -inf
          S.meta[j % kMeta][lane] = {finite ? fmaxf(sk * (fabsf(A.scale) * 1.4426950408889634f), 1e-37f) : 1e-37f,
                                     pages < 0 ? -INFINITY : finite ? __log2f(s) : kNoNumber, __frcp_rn(s), 0.f};
        }
        sk = scale_of(0, next);
        sv = scale_of(1, next);
      }
      store(sm + (kv ? L::kV : L::kK) + st * L::kTile, kv, cur);
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(kv ? &S.vfull[st] : &S.kfull[st]);
        // (here, and not where the scales are stored: 840 instead of 808 us for the long prompt)
        if (w == 0 && kv == 0) mbar_arrive(&S.mfull[j % kMeta]);
      }
      if (kv) {
        pages = next;
        next = checked(entry);
        entry = entry_of(j + 3);
      }
    }
  } else {
    reg_less<80>();
    if (warp == kMmaWarp && nt > 0 && rank == 0) {
      // ------------------------------------------------------------------ MMAs
      constexpr uint32_t kIdS = idesc_f16(kCtas * kTileRows, kTileKeys, false), kIdO = idesc_f16(kCtas * kTileRows, D, true);
      const auto commit = [](uint64_t* bar) { PAIR ? mma_commit_pair(bar) : mma_commit(bar); };   // (in both CTAs)
      const bool leader = elect_one();
      auto wait = [&](uint64_t* bar, int par, int code) {
        const bool ok = mbar_wait_near(bar, (uint32_t)par & 1u, abort_flag, c.err, code, A.wait_cycles);
        tc_fence_after();
        return ok;
      };
      auto wait_stored = [&](uint64_t* bar, int par, int code) {   // (for both CTAs' shared memory)
        const bool ok = PAIR ? mbar_wait_near_cluster(bar, (uint32_t)par & 1u, abort_flag, c.err, code, A.wait_cycles)
                             : mbar_wait_near(bar, (uint32_t)par & 1u, abort_flag, c.err, code, A.wait_cycles);
        tc_fence_after();
        return ok;
      };
      const uint64_t q0 = sdesc_sw128(smem_u32(sm + L::kQ)), k0 = sdesc_sw128(smem_u32(sm + L::kK));
      const uint64_t v0 = sdesc_mn128(smem_u32(sm + L::kV), L::kHalf);
      auto mma_s = [&](int t, int st) {
#pragma unroll 1
        for (int h = 0; h < D / 64; ++h) {
          const uint64_t a = q0 + ((t * L::kQTile + h * L::kHalf) >> 4), b = k0 + ((st * L::kTile + h * L::kKHalf) >> 4);
#pragma unroll
          for (int k = 0; k < 4; ++k) mma_f16<PAIR>(tm + t * 128, a + 2 * k, b + 2 * k, kIdS, h > 0 || k > 0);
        }
      };
      auto mma_o = [&](int t, int st, int n, bool first) {   // n = 0: the second half of the keys
        const uint32_t a = tm + t * 128 + 64 + 32 * n;
        const uint64_t b = v0 + ((st * L::kTile + 8192 * (1 - n)) >> 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) mma_f16_ts<PAIR>(tm + 256 + t * 128, a + 8 * k, b + 128 * k, kIdO, !first || k > 0);
      };
      bool ok = wait_stored(&S.kfull[0], 0, kDevTimeoutConv);
      for (int t = 0; t < halves && ok; ++t) {
        ok = wait_stored(&S.qfull[t], 0, kDevTimeoutFull);
        if (ok && leader) {
          mma_s(t, 0);
          commit(&S.sfull[t]);
          if (t == halves - 1 && nt > kPreStages) commit(&S.kempty[0]);
        }
        __syncwarp();
      }
#pragma unroll 1
      for (int j = 0; j < nt && ok; ++j) {
        const int st = j % kPreStages, s1 = (j + 1) % kPreStages;
        const bool more = j + 1 < nt;
        ok = wait_stored(&S.vfull[st], j / kPreStages, kDevTimeoutConv);
#pragma unroll 1
        for (int t = 0; t < halves && ok; ++t) {
          ok = wait(&S.pfull[t][0], j, kDevTimeoutTmemEmpty);
          if (ok && leader) {
            mma_o(t, st, 0, j == 0);
            commit(&S.phalf[t]);
          }
          __syncwarp();
          if (ok && more && t == 0) ok = wait_stored(&S.kfull[s1], (j + 1) / kPreStages, kDevTimeoutConv);
          if (ok) ok = wait(&S.pfull[t][1], j, kDevTimeoutTmemEmpty);
          if (ok && leader) {
            mma_o(t, st, 1, false);
            if (more) {
              mma_s(t, s1);
              commit(&S.sfull[t]);
            } else {
              commit(&S.ofull[t]);
            }
            if (t == halves - 1) {
              // (a slot that no tile follows in is waited for by nobody)
              if (j + kPreStages < nt) commit(&S.vempty[st]);
              if (j + 1 + kPreStages < nt) commit(&S.kempty[s1]);
            }
          }
          __syncwarp();
        }
      }
      if (leader) commit(&S.drain);
      __syncwarp();
    } else if (PAIR && warp == kMmaWarp) {
      // ------------------------------------------------------------------ the second CTA's units, passed on
#pragma unroll 1
      for (int u = 0; u < 2 * nt; ++u) {   // K 0, V 0, K 1, V 1, ..., as they are widened
        const int j = u >> 1, st = j % kPreStages;
        uint64_t* bar = u & 1 ? &S.vfull[st] : &S.kfull[st];
        if (!mbar_wait_near(bar, (j / kPreStages) & 1, abort_flag, c.err, kDevTimeoutConv, A.wait_cycles)) break;
        if (lane == 0) mbar_arrive_remote_release(cluster_map(smem_u32(bar), 0));
        __syncwarp();
      }
    }
    if (warp == kMmaWarp && nt > 0) {
      // The MMAs and their arrivals (in both CTAs) end before tensor memory is freed and the CTA
      // leaves, whichever warp's wait gave up: also the last ones', which only the softmax waits for.
      // (the full bound, whatever the caller's is)
      int no_abort = 0;
      mbar_wait_warp(&S.drain, 0, &no_abort, c.err, kDevTimeoutDrain);
    }
  }
  __syncthreads();
  if constexpr (PAIR) {   // neither CTA leaves, or frees what the other's MMAs read, before both are done
    cluster_arrive_relaxed();
    cluster_wait();
  }
  tc_fence_after();
  if (warp == kMmaWarp) {
    tmem_relinquish<PAIR>();
    tmem_dealloc<PAIR>(tm, 512);
  }
}

// Joins the parts of the keys: a warp a row.
template <int D>
__global__ void __launch_bounds__(256) kv8_join_kernel(const Kv8AttendArgs A, int nsplit, int tiles) {
  const int row = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31, head = blockIdx.y, seq = blockIdx.z;
  pdl_launch_dependents();
  pdl_wait();
  Seq q;
  if (!load_seq(A.c, seq, q, false) || row >= q.n * A.group) return;
  const int tile = row / (2 * kTileRows), r = row % (2 * kTileRows);
  constexpr size_t kPart = 2 * kTileRows * (D + 2);
  const float* part = A.ws + (((size_t)seq * tiles + tile) * gridDim.y + head) * nsplit * kPart;
  float M = -INFINITY;
  for (int i = lane; i < nsplit; i += 32) M = fmaxf(M, __ldcg(part + i * kPart + 2 * kTileRows * D + r));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  const float base = M == -INFINITY ? 0.f : M;
  constexpr int E = D / 32;
  float l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 4
  for (int i = 0; i < nsplit; ++i) {
    const float* p = part + i * kPart;
    const float f = exp2_fast(__ldcg(p + 2 * kTileRows * D + r) - base);
    l = fmaf(f, __ldcg(p + 2 * kTileRows * (D + 1) + r), l);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(f, __ldcg(p + (size_t)r * D + E * lane + e), o[e]);
  }
  const float inv = one_over_sum(M, l);
  const int tok = row / A.group, hh = row - tok * A.group;
  __half* dst = A.out + (size_t)(q.tok0 + tok) * A.out_stride + (size_t)(head * A.group + hh) * D + E * lane;
#pragma unroll
  for (int e = 0; e < E; e += 2) *reinterpret_cast<__half2*>(dst + e) = __floats2half2_rn(o[e] * inv, o[e + 1] * inv);
}

// Rows of a sequence and KV head from which pairs of CTAs take them.  Pairs / CTAs alone, us, 64 over 8
// heads: 16 sequences x 64 new tokens behind 4000: 119 / 133; 16 x 256: 369 / 405; 4 x 1024: 382 / 429;
// 1 x 2048 behind 8000: 471 / 549; 2 x 4096: 364 / 391; 1 x 8192: 811 / 898; 32 over 8 heads, 8 x 512 behind up to
// 4000: 173 / 187.  Pairs lose where sequences of one or two pair tiles round up into another wave (16 x
// about 100 behind 4000: 220 / 200) and where rows without a context see few tiles each (4 x 1024: 85 / 81;
// 32 heads, 8 x 512: 61 / 46): long sums, which pairs serve, weigh more than the start of short ones.
constexpr int kPairRows = 512;

template <int D>
static cudaError_t launch_prefill(const Kv8AttendArgs& a, int num_sms, cudaStream_t s) {
  const int tiles = ceil_div((long long)a.c.max_tokens * a.group, 2 * kTileRows);
  const long long ctas = (long long)tiles * a.c.kv_heads * a.c.seqs;
  if (tiles > 65535) return cudaErrorInvalidValue;
  // Grids that leave half of the SMs without a CTA are split along the keys, but not below
  // two tiles of 128 keys a CTA.
  const long long key_tiles = ceil_div(a.window > 0 && a.window + a.sinks < a.c.max_len - a.c.max_tokens
                                           ? (long long)a.window + a.sinks + a.c.max_tokens
                                           : a.c.max_len,
                                       kTileKeys);
  long long nsplit = num_sms / ctas;
  if (nsplit > key_tiles / 2) nsplit = key_tiles / 2;
  if constexpr (D == 128) {
    if (nsplit <= 1 && (long long)a.c.max_tokens * a.group >= kPairRows) {
      const auto pair = kv8_prefill_kernel<D, false, true>;
      const cudaError_t e = ensure_max_dyn_smem(pair);
      if (e != cudaSuccess) return e;
      const int tiles4 = ceil_div((long long)a.c.max_tokens * a.group, 4 * kTileRows);
      return launch_after(pair, dim3(2 * a.c.kv_heads, a.c.seqs, tiles4), kPreThreads, PreLayout<D, true>::kBytes, s, 2,
                          a, 1);
    }
  }
  constexpr int smem = PreLayout<D, false>::kBytes;
  const auto fn = nsplit > 1 ? kv8_prefill_kernel<D, true, false> : kv8_prefill_kernel<D, false, false>;
  const cudaError_t e = ensure_max_dyn_smem(fn);
  if (e != cudaSuccess) return e;
  if (nsplit <= 1) return launch_after(fn, dim3(a.c.kv_heads, a.c.seqs, tiles), kPreThreads, smem, s, 1, a, 1);
  const cudaError_t e2 =
      launch_after(fn, dim3(a.c.kv_heads, a.c.seqs, (unsigned)(tiles * nsplit)), kPreThreads, smem, s, 1, a, (int)nsplit);
  if (e2 != cudaSuccess) return e2;
  const int rows = a.c.max_tokens * a.group;
  return launch_after(kv8_join_kernel<D>, dim3(ceil_div(rows, 8), a.c.kv_heads, a.c.seqs), 256, 0, s, 1, a, (int)nsplit,
                      tiles);
}

cudaError_t launch_kv8_prefill(const Kv8AttendArgs& a, int num_sms, cudaStream_t s) {
  return a.c.head_dim == 64 ? launch_prefill<64>(a, num_sms, s) : launch_prefill<128>(a, num_sms, s);
}

}  // namespace dptq
