// kv_prefill.cuh -- what the prompt kernels of both paged caches share: the binary16 MMAs of the 5th-generation tensor
// cores with fp32 accumulators in tensor memory, tiles of keys and their masks, the layout of shared memory.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv8_device.cuh"

namespace dptq {

constexpr int kConvWarps = 4, kMmaWarp = 8 + kConvWarps, kPreThreads = 32 * (kMmaWarp + 4);
constexpr int kTileRows = 128, kTileKeys = 128, kPreStages = 2, kMeta = 4;
constexpr int kNoEntry = (int)0x80000000;

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
template <int N>
__device__ __forceinline__ void reg_more() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void reg_less() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
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

// Writes -inf over the scores of the keys that this thread's row does not see (gone: bit g, of the tile's keys 16 g ..,
// none does), in tensor memory: the few tiles that need it pay for the pass, and the code that every tile runs stays short
// (with the masks in its middle, 929 instead of 855 us for a prompt of 8192 tokens, 64 over 8 heads, int8 cache).
__device__ __forceinline__ void mask_scores(uint32_t tS, int pos, int key, int window, int sinks,
                                            uint32_t gone = 0) {
#pragma unroll 1
  for (int k = 0; k < kTileKeys; k += 16) {
    uint32_t v[16];
    tmem_ld16(tS + k, v);
    uint32_t bits = low_bits(pos - key - k + 1);   // bit e: the row sees key k + e
    if (window > 0) bits &= ~low_bits(pos - window + 1 - key - k) | low_bits(sinks - key - k);
    if (gone >> (k / 16) & 1u) bits = 0;
    tmem_ld_wait();
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = bits >> e & 1u ? v[e] : 0xFF800000u;
    tmem_st16(tS + k, v);
  }
  tmem_st_wait();
}

// kShared: bytes of what stands behind the tiles.
template <int D, bool PAIR, int kShared>
struct PreLayout {
  static constexpr int kHalf = 128 * 128;                          // 64 dims x 128 rows
  static constexpr int kQTile = D / 64 * kHalf;                    // a row tile of q
  static constexpr int kTile = PAIR ? kQTile / 2 : kQTile;         // this CTA's part of a widened tile:
  static constexpr int kKHalf = PAIR ? kHalf / 2 : kHalf;          // K: 64 dims x its keys; V: its dims x 128 keys
  static constexpr int kQ = 0, kK = 2 * kQTile, kV = kK + kPreStages * kTile, kEnd = kV + kPreStages * kTile;
  static constexpr int kBytes = kEnd + kShared + 1024;   // (1024: alignment)
};

}  // namespace dptq
