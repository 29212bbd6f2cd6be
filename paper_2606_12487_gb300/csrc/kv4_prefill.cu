// kv4_prefill.cu -- attention of many rows (prompts, chunks of prompts, more than 16 rows of a
// sequence and KV head) over the paged 4-bit cache, on the 5th-generation tensor cores.
//
// The rows of a KV head (a token's query heads side by side, then the next token's) are cut
// into tiles of 256; a CTA takes two row tiles of 128 so that one's softmax runs while the
// tensor cores work for the other, and both share every widened K and V tile of 128 keys:
//   S = q k^T   128 x 128 x D   both operands in shared memory, S in tensor memory
//   O += P v    128 x D x 128   P in tensor memory (over half of S), v in shared memory
// A bfloat16 scale times a code is a binary16 number, so tiles are widened to the cached values themselves and the
// softmax knows nothing of scales: weights 2^(log2(e) scale (S - m) + 7) relative to the row's maximum m, which
// may lag by 2^8 (O is rescaled only where it has grown by more): binary16 holds 2^15, and 21 binades
// below the largest weight at full precision.  The weights are rounded to it, 2^-11 of each, since both operands of an MMA have
// V's type (fp32 ones would take tf32 MMAs, at half the rate, and twice P's room); sums are of the unrounded ones.  The rms error
// of outputs is 2.23e-4 of them instead of the 2.08e-4 of rounding the exact ones.
//
// Warp roles: 0-3 and 4-7 softmax and output of the row tiles, a row a thread; 8-11 widen K and
// V tiles (global to registers a tile ahead, then to shared memory in the 128-byte swizzle);
// 12 issues the MMAs.  Many rows (kPairRows): pairs of CTAs, each widening half of every tile (PAIR below).
//
// A task is the 256 rows (512 of a pair) of one (sequence, KV head).  Tasks that would leave SMs without work in the
// last wave are split along the keys (Cut): each CTA leaves its rows' sums, and a second launch joins them.
//
// What bounds it, at a prompt of 8192 tokens, 64 over 8 heads of 128 (1.1 TFLOP, 836 us, 1315 TFLOP/s, 68 % of the measured bf16 rate):
// the chain of a row tile from S over its softmax back to the next S, in which widening and softmax share the issue slots: of the
// 846 us of an earlier form, 735 were left without the softmax's work, 691 without both (all barriers kept), 848 without the
// exponentials alone.  512 rows behind 16000 tokens: 220 us; three chunks up to 500 behind up to 12000, window 4096: 182 us.
//
// The order of the dims: a word of eight nibbles widens to the pairs (0, 4), (1, 5), (2, 6), (3, 7).  q is stored in
// that order too, and the output's registers are written from it.
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_fp16.h>

#include "kv4_device.cuh"
#include "kv_prefill.cuh"

namespace dptq {

constexpr float kUnit = 7.f;   // weights are relative to 2^-7 of the largest
// Rows whose largest score is more than that, in powers of two, are made from S - m, apart from the others: log2(e) scale S + (7 - m) in
// one fma is off by a step of m, 2^-10 here and 2 at 2^25, where weights would be too large whatever m is.  (All rows that
// way: 849 instead of 827 us for a prompt of 8192 tokens, 64 over 8 heads.)
constexpr float kFar = 16384.f;
// log2(e) |scale|, above 0 so that a masked score of -inf stays, and finite so that the largest score's difference to itself is 0.
__device__ __forceinline__ float kv4_unit(float scale) {
  return fminf(fmaxf(fabsf(scale) * 1.4426950408889634f, 1e-37f), 1e37f);
}

// Where the rows of a CTA or pair go: slot of the scratch for a part of a task's keys, -1 for whole tasks.
struct Out {
  int tok0, row0, nrows, head, slot;
};
struct Pre4Shared {
  uint64_t kfull[kPreStages], kempty[kPreStages], vfull[kPreStages], vempty[kPreStages];
  uint64_t mfull[kMeta];   // `gone` is there (filled and read within a CTA)
  uint64_t qfull[2], sfull[2], pfull[2][2], ofull[2], drain;   // pfull: the two halves of a tile's keys
  uint64_t phalf[2];   // the first half's product is complete
  uint32_t gone[kMeta];   // bit g: no page for the tile's keys 16 g ..
  Out out;
  uint32_t tmem;
  int abort;
};

// Waits for barriers (a warp together) in few instructions, bounded in cycles: a poll may be suspended for any time, so that a number
// of polls bounds nothing.
template <class Arrived>
__device__ __forceinline__ bool wait_bounded(Arrived arrived, volatile int* abort_flag, int* err, int code, long long limit) {
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
__device__ __forceinline__ bool wait_one(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* err, int code,
                                         long long limit) {
  return wait_bounded([&] { return mbar_try_wait(bar, parity); }, abort_flag, err, code, limit);
}
// What the arrivals released at cluster scope is seen (mbar_arrive_remote_release).
__device__ __forceinline__ bool wait_cluster(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* err, int code,
                                             long long limit) {
  return wait_bounded([&] { return mbar_try_wait_cluster(bar, parity); }, abort_flag, err, code, limit);
}
// Two barriers, whose answers come back together.
__device__ __forceinline__ bool wait_two(uint64_t* b0, uint32_t p0, uint64_t* b1, uint32_t p1, volatile int* abort_flag,
                                         int* err, int code, long long limit) {
  return wait_bounded(
      [&] {
        const bool r0 = mbar_try_wait(b0, p0), r1 = mbar_try_wait(b1, p1);
        return r0 && r1;
      },
      abort_flag, err, code, limit);
}

// How the device cuts a call: all tasks, and those from `whole` on in `parts` parts of their keys each.
struct Cut {
  int tasks, whole, parts;
};
// Whole waves of tasks stay whole.  The r tasks behind them, where they are fewer than the P that run at a time, are cut
// into floor(P / r) parts, or, from P / 2 to 2 P / 3, into three (two shorter waves); most: the host's bound, 1 for calls whose last wave is
// a small part of them.
__device__ __forceinline__ Cut cut_tasks(int tasks, int P, int most) {
  Cut r{tasks, tasks, 1};
  if (most < 2) return r;
  const int left = tasks % P;
  if (left == 0) return r;
  int parts = P / left;
  if (parts < 2 && 3 * left <= 2 * P) parts = 3;
  if (parts > most) parts = most;
  if (parts > 1) r.whole = tasks - left, r.parts = parts;
  return r;
}
// A task: a sequence, a KV head, and the number of its row tile counted from the sequence's last one, which sees the most
// keys; tasks are taken in the order of that number, so that long ones come first, then of sequences and heads.
struct Task {
  int seq, head, from_last;
};
constexpr int kFewSeqs = 32;   // sequences that a warp knows the tiles of
// The part `index` of a call of at most kFewSeqs sequences: its task, which of the task's parts it is, and how the call is
// cut; false past the last one.  Every warp finds it by itself.  All results come out of shuffles and votes: the compiler
// then knows that they are the same in a warp, and loops that it takes to be divergent would cost a prompt of 8192 tokens
// 160 us.
__device__ __forceinline__ bool find_task(const Kv8Args& c, int group, int rows, int index, int P, int most, bool tells, Cut& cut,
                                          Task& task, int& part) {
  const int lane = threadIdx.x & 31;
  Seq q;
  const int mine = lane < c.seqs && load_seq(c, lane, q, tells) ? (q.n * group + rows - 1) / rows : 0;
  cut = cut_tasks(__reduce_add_sync(0xffffffffu, mine) * c.kv_heads, P, most);
  int u = index;
  part = 0;
  if (u >= cut.whole) {
    u = cut.whole + (index - cut.whole) / cut.parts;
    part = (index - cut.whole) % cut.parts;
  }
  if (u >= cut.tasks) return false;
  task.head = u % c.kv_heads;
  const int tile = u / c.kv_heads;
  // the largest z of which min(tiles, z) over all sequences make at most `tile`
  int z = 0;
  for (int step = 1 << (31 - __clz(__reduce_max_sync(0xffffffffu, mine))); step > 0; step >>= 1)
    if (__reduce_add_sync(0xffffffffu, min(mine, z + step)) <= tile) z += step;
  const uint32_t there = __ballot_sync(0xffffffffu, mine > z);
  const int k = tile - __reduce_add_sync(0xffffffffu, min(mine, z));
  task.from_last = z;
  task.seq = __ffs(__ballot_sync(0xffffffffu, (there >> lane & 1u) && __popc(there & ((1u << lane) - 1)) == k)) - 1;
  return true;
}

// PAIR: two CTAs of a cluster work on 512 rows, 256 each; the tensor cores of both take K and V
// tiles of which each CTA widens and holds one half (of K's keys, of V's dims).  That halves the
// widening, its stores and what the MMAs read of K and V from shared memory, which is what a
// CTA alone is short of.  The first CTA issues the MMAs.  What the second one stores for them reaches
// its barriers in three ways: q, once, released at cluster scope; K and V on the second CTA's own
// barriers, from which its MMA warp, which has no loads under way, passes them on released at cluster
// scope; P, stores to tensor memory, as mbar_arrive_remote says.
// CUT: tasks may be cut (P, most: cut_tasks); otherwise the grid is KV heads x sequences x row tiles.
template <int D, bool PAIR, bool CUT>
__global__ void __launch_bounds__(kPreThreads, 1) kv4_prefill_kernel(const Kv4AttendArgs A, int P, int most) {
  static_assert(!PAIR || D == 128, "a pair's halves of V are 64 dims");
  using L = PreLayout<D, PAIR, (int)sizeof(Pre4Shared)>;
  constexpr int kCtas = PAIR ? 2 : 1, kRows = kCtas * 2 * kTileRows;   // rows of a CTA or pair
  extern __shared__ uint8_t raw[];
  uint8_t* sm = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
  Pre4Shared& S = *reinterpret_cast<Pre4Shared*>(sm + L::kEnd);
  const Kv8Args& c = A.k.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = PAIR ? blockIdx.x & 1 : 0;
  pdl_launch_dependents();
  pdl_wait();
  Cut cut{0, 0, 1};
  Task task;
  int part = 0;
  const int index = blockIdx.x / kCtas;
  if constexpr (CUT) {
    if (!find_task(c, A.group, kRows, index, P, most, blockIdx.x == 0 && warp == 0, cut, task, part)) return;
  } else {
    task = {(int)blockIdx.y, index, (int)blockIdx.z};
  }
  const int seq = task.seq, head = task.head;
  const bool split = CUT && index >= cut.whole;
  Seq q;
  if (!load_seq(c, seq, q, !CUT && tid == 0 && head == 0 && blockIdx.z == 0)) return;
  const int rows = q.n * A.group;
  const int tile = (rows + kRows - 1) / kRows - 1 - task.from_last;
  if (!CUT && tile < 0) return;
  const int row0 = tile * kRows, nrows = rows - row0 < kRows ? rows - row0 : kRows;
  const int halves = nrows > kCtas * kTileRows ? 2 : 1;   // row tiles (of a pair: 256 rows)
  const int p_first = q.start + row0 / A.group, p_last = q.start + (row0 + nrows - 1) / A.group;
  const Tiles all = row_tiles(p_first, p_last, A.window, A.sinks);
  // (at most 2^20 tiles and 256 parts)
  const int j0 = split ? (int)((unsigned)all.count * part / (unsigned)cut.parts) : 0;
  const int nt = (split ? (int)((unsigned)all.count * (part + 1) / (unsigned)cut.parts) : all.count) - j0;

  if (CUT && tid == 0) S.out = {q.tok0, row0, nrows, head, split ? index - cut.whole : -1};
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
    const int pos = mine ? q.start + row / A.group : -1;
    const uint32_t tlane = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tm + tlane + t * 128, tO = tm + tlane + 256 + t * 128;
    float m = -INFINITY, far_m = 0.f, l = 0.f;   // the largest score so far: m, or far_m where that is not 0 (m is then -inf)
    bool ok = true;
    const float unit = kv4_unit(A.scale);
    if (t < halves && nt > 0) {
      {   // the warp's rows of q, whole rows at a time, in the order of the dims that a widened word has, negated for a
          // negative scale
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
          v = make_uint4(__byte_perm(v.x, v.z, 0x5410) ^ flip, __byte_perm(v.x, v.z, 0x7632) ^ flip,
                         __byte_perm(v.y, v.w, 0x5410) ^ flip, __byte_perm(v.y, v.w, 0x7632) ^ flip);
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
        ok = wait_two(&S.mfull[j % kMeta], (j / kMeta) & 1, &S.sfull[t], j & 1, abort_flag, c.err,
                             kDevTimeoutTmemFull, A.wait_cycles);
        if (!ok) break;
        tc_fence_after();
        const int key = all.key(j0 + j);
        const bool seen = key + kTileKeys - 1 <= p_lo &&
                          (A.window == 0 || key > p_hi - A.window || key + kTileKeys <= A.sinks);
        const uint32_t gone = S.gone[j % kMeta];
        if (!seen || gone != 0) mask_scores(tS, pos, key, A.window, A.sinks, gone);
        // Halves of 64 keys, the second one first: its weights take the place of its S, and their
        // product begins while the first half is worked on.  The weights are relative to a maximum
        // that may lag by 2^8 (binary16 holds them), so they are made before the half's own maximum
        // is known; where that is larger still, what is relative to the old one is rescaled and
        // the half made again.
        float xa[32], xb[32];
        uint32_t p[32];
        // A quarter's weights, packed, and their sum.
        auto quarter = [&](float (&x)[32], uint32_t* w, float& s) {
          const float off = fmaf(m == -INFINITY ? 0.f : -m, unit, kUnit);
          const uint64_t a = f2_pack(unit, unit), b = f2_pack(off, off);
          uint64_t sum = 0;
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            float y0, y1;
            f2_unpack(f2_fma(f2_pack(x[k], x[k + 1]), a, b), y0, y1);
            y0 = exp2_fast(y0);
            y1 = exp2_fast(y1);
            sum = k ? f2_add(sum, f2_pack(y0, y1)) : f2_pack(y0, y1);
            w[k / 2] = pack_half2(y0, y1);
          }
          float s0, s1;
          f2_unpack(sum, s0, s1);
          s += s0 + s1;
        };
        auto largest = [&](float (&x)[32]) {
          float v[11];
#pragma unroll
          for (int k = 0; k < 10; ++k) v[k] = max3(x[3 * k], x[3 * k + 1], x[3 * k + 2]);
          v[10] = fmaxf(x[30], x[31]);
          return fmaxf(max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), max3(v[6], v[7], v[8])), fmaxf(v[9], v[10]));
        };
        auto far = [&](float v) { return fabsf(v) * unit > kFar && fabsf(v) < INFINITY; };
        // A half's weights are stored, and the next half's scores asked for.
        auto give = [&](int n) {
          tmem_st32(tS + 64 + 32 * n, p);
          if (n == 0) tmem_ld32(tS, xa);
          tmem_st_wait();
          tc_fence_before();
          tell_first(&S.pfull[t][n], false);
        };
        if (j == 0) {   // the first maximum, so that the first half is not made for nothing
#pragma unroll 1
          for (int h = 0; h < 4; ++h) {
            tmem_ld32(tS + 32 * h, xa);
            tmem_ld_arrived(xa);
            float v = xa[0];
#pragma unroll
            for (int k = 1; k < 31; k += 2) v = max3(v, xa[k], xa[k + 1]);
            m = fmaxf(m, fmaxf(v, xa[31]));
          }
          if (far(m)) m = -INFINITY;
        }
        tmem_ld32(tS + 64, xa);
        int n = 0;
#pragma unroll 1
        for (;;) {   // (once, but for maxima that grow: that code stands apart from what every tile runs)
          float top;
          bool more;
#pragma unroll 1
          for (; n < 2; ++n) {
            const int h = 2 - 2 * n;
            float s = 0.f;
            more = false;
            tmem_ld_arrived(xa);
            tmem_ld32(tS + 32 * h + 32, xb);   // (under the first quarter's work)
            quarter(xa, p, s);
            tmem_ld_arrived(xb);
            quarter(xb, p + 16, s);
            // The sum says whether a weight may be above 2^15: the scores' maximum is looked for only then, and where there is
            // no m.  (A sum above 2^15 has a weight above 2^8, so a score is above m; relative to the half's own maximum no
            // weight is above 2^7 but for the rounding that kFar bounds, and 64 of them make no such sum: a half is made
            // again once.)
            if (__any_sync(0xffffffffu, s > 32768.f || m == -INFINITY)) {
              top = fmaxf(largest(xa), largest(xb));
              more = s > 32768.f || (m == -INFINITY && top > m);
              if (__any_sync(0xffffffffu, more)) break;
            }
            l += s;
            give(n);
          }
          if (n == 2) break;
          // (a row whose own maximum may still lag keeps it: its result has nothing to do with the warp's other rows)
          const float was = far_m != 0.f ? far_m : m;   // (-inf: no key yet)
          const float now = far_m != 0.f ? fmaxf(far_m, top) : more ? top : m;
          const float f = now == was ? 1.f : exp2_fast((was - now) * unit);
          m = far(now) ? -INFINITY : now;
          far_m = far(now) ? now : 0.f;
          l *= f;
          // O: PV of tile j - 1 came before S of tile j, which is here; of tile j, the first half's
          // product may be under way.
          if (n == 1) {
            ok = wait_one(&S.phalf[t], j & 1, abort_flag, c.err, kDevTimeoutTmemFull, A.wait_cycles);
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
          if (!__any_sync(0xffffffffu, far_m != 0.f)) {
            tmem_ld32(tS + 64 * (1 - n), xa);
            continue;
          }
          // A warp with such rows makes its half here (x - 0 for the others: the weights and sums that they have anyway).
          float s = 0.f;
#pragma unroll
          for (int k = 0; k < 32; ++k) xa[k] -= far_m, xb[k] -= far_m;
          quarter(xa, p, s);
          quarter(xb, p + 16, s);
          l += s;
          give(n);
          if (++n == 2) break;
        }
      }
      if (ok) ok = wait_one(&S.ofull[t], 0, abort_flag, c.err, kDevTimeoutTmemFull, A.wait_cycles);
      tc_fence_after();
    }
    // ---- output (the accumulators of a chunk of 8 dims stand in the order 0 4 1 5 2 6 3 7); of a call that is cut, where it
    // goes comes from shared memory, since registers for it would be missing in the loop
    if (ok && t < halves) {
      Out w{q.tok0, row0, nrows, head, -1};
      if constexpr (CUT) {
        volatile const Out& v = S.out;
        w = {v.tok0, v.row0, v.nrows, v.head, v.slot};
      }
      const int at = (t * kCtas + rank) * kTileRows + r, row = w.row0 + at;
      const bool mine = at < w.nrows, sums_only = CUT && w.slot >= 0;
      float* sums = nullptr;
      if (sums_only) {   // weighted values [kRows][D], then maxima, then sums
        sums = A.ws + (size_t)w.slot * (kRows * (D + 2));
        if (mine) {
          sums[kRows * D + at] = far_m != 0.f ? far_m : m;
          sums[kRows * (D + 1) + at] = l;
        }
        sums += (size_t)at * D;
      }
      const float inv = l == 0.f ? 0.f : __frcp_rn(l);
      const int tok = row / A.group, hh = row - tok * A.group;
      __half* dst = A.out + (size_t)(w.tok0 + tok) * A.out_stride + (size_t)(w.head * A.group + hh) * D;
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
        if (mine && !sums_only) {
#pragma unroll
          for (int e = 0; e < 32; e += 8)
            *reinterpret_cast<uint4*>(dst + k + e) =
                make_uint4(pack_half2(o[e] * inv, o[e + 2] * inv), pack_half2(o[e + 4] * inv, o[e + 6] * inv),
                           pack_half2(o[e + 1] * inv, o[e + 3] * inv), pack_half2(o[e + 5] * inv, o[e + 7] * inv));
        }
        if (mine && sums_only) {
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            *reinterpret_cast<float4*>(sums + k + e) = make_float4(o[e], o[e + 2], o[e + 4], o[e + 6]);
            *reinterpret_cast<float4*>(sums + k + e + 4) = make_float4(o[e + 1], o[e + 3], o[e + 5], o[e + 7]);
          }
        }
      }
    }
    tc_fence_before();
  } else if (warp < kMmaWarp) {
    // ------------------------------------------------------------------ K and V, widened
    reg_less<112>();
    const int w = warp - 8;
    const Nibbles nib;
    // A warp takes rows of 16 bytes (32 dims) a lane, kUnits times 32 lanes of a tile: of K whole rows, and of a pair's
    // the CTA's half of the keys; of V all keys, and of a pair's the CTA's 64 dims of each.
    constexpr int kLanesK = D / 32, kLanesV = PAIR ? 2 : D / 32, kUnits = kLanesK * kTileKeys / 32 / kConvWarps / kCtas;
    static_assert(kLanesV * kTileKeys / 32 / kConvWarps == kUnits, "as many units of V");
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
    // Row (of K or V) of a lane in unit i: its key in the tile.
    auto key_in = [&](int i, int kv) {
      const int lanes = kv ? kLanesV : kLanesK;
      return (kv ? 0 : rank * (kTileKeys / kCtas)) + 32 / lanes * (w + kConvWarps * i) + lane / lanes;
    };
    // Codes of a unit of a tile, and its scales: what a warp holds while the one before is widened.  (A page that is not
    // there reads page 0: its keys are masked, and V values are finite whatever they are.)
    auto load = [&](int j, int kv, int pages, uint4 (&v)[kUnits], uint32_t (&sk)[kUnits], uint32_t (&sv)[kUnits]) {
      const int key = all.key(j0 + j), lanes = kv ? kLanesV : kLanesK;
      const uint8_t* codes = (kv ? A.k.codes[1] : A.k.codes[0]) + 16 * (lane % lanes) + (kv && PAIR ? 32 * rank : 0);
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int at = key_in(i, kv), b = max(__shfl_sync(0xffffffffu, pages, at >> 4), 0);
        const size_t row = (((size_t)b * c.kv_heads + head) << c.log2_page) + ((key + at) & P1);
        v[i] = ld_plain(reinterpret_cast<const uint4*>(codes + row * (D / 2)));
        sk[i] = ld_plain(A.k.scales[0] + row);
        sv[i] = ld_plain(A.k.scales[1] + row);
      }
    };
    auto store = [&](uint8_t* dst, int kv, const uint4 (&v)[kUnits], const uint32_t (&sk)[kUnits], const uint32_t (&sv)[kUnits]) {
      const int lanes = kv ? kLanesV : kLanesK, col = lane % lanes;
      // (rows of four lanes: dims 64 .. stand kHalf on, in the same banks, so their lanes take their words in
      // another order)
      const bool other = lanes == 4 && col >= 2;
      dst += other ? (kv ? L::kHalf : L::kKHalf) : 0;
      uint32_t sb[kUnits];
      bool odd = false;
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        // A scale that is no number makes its key's K values NaN, so that its scores are for the rows that see it, and its
        // V values 0, so that no other row meets it.
        const bool bad = kv4_bad(max(sk[i], sv[i]));
        sb[i] = kv ? (bad ? 0u : sv[i]) : (bad ? 0x7FC0u : sk[i]);
        odd |= kv4_odd(sb[i]);
      }
      const int chunk = 4 * (col & 1) + (other ? 2 : 0);
      auto place = [&](int i, int k) {   // of word k of unit i
        const int at = key_in(i, kv) - (kv ? 0 : rank * (kTileKeys / kCtas));
        return reinterpret_cast<uint4*>(dst + at * 128 + (((chunk ^ k) ^ (at & 7)) << 4));
      };
      if (!__any_sync(0xffffffffu, odd)) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
          const uint32_t x[4] = {other ? v[i].z : v[i].x, other ? v[i].w : v[i].y, other ? v[i].x : v[i].z, other ? v[i].y : v[i].w};
          const __half2 s2 = __float2half2_rn(bf16_float(sb[i]));
#pragma unroll
          for (int k = 0; k < 4; ++k) *place(i, k) = nib.values(x[k], s2);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
#pragma unroll 1
          for (int k = 0; k < 4; ++k) {
            const int from = other ? k ^ 2 : k;
            *place(i, k) = values_slow<true>(from == 0 ? v[i].x : from == 1 ? v[i].y : from == 2 ? v[i].z : v[i].w, bf16_float(sb[i]));
          }
        }
      }
      fence_proxy_async_smem();
    };
    // Units in order K 0, V 0, K 1, V 1, ..., each loaded while the one before it is widened.
    uint4 cur[kUnits], nxt[kUnits];
    uint32_t csk[kUnits], csv[kUnits], nsk[kUnits], nsv[kUnits];
    const int entry0 = entry_of(0), entry1 = entry_of(1);
    int entry = entry_of(2), pages = checked(entry0), next = checked(entry1);
    if (nt > 0) load(0, 0, pages, nxt, nsk, nsv);
#pragma unroll 1
    for (int u = 0; u < 2 * nt; ++u) {
      const int j = u >> 1, kv = u & 1, st = j % kPreStages, par = (j / kPreStages + 1) & 1;
#pragma unroll
      for (int i = 0; i < kUnits; ++i) cur[i] = nxt[i], csk[i] = nsk[i], csv[i] = nsv[i];
      if (u + 1 < 2 * nt) load((u + 1) >> 1, kv ^ 1, kv ? next : pages, nxt, nsk, nsv);
      if (!wait_one(kv ? &S.vempty[st] : &S.kempty[st], par, abort_flag, c.err, kDevTimeoutEmpty, A.wait_cycles))
        break;
      if (kv == 0 && w == 0) {
        const uint32_t gone = __ballot_sync(0xffffffffu, lane < kTileKeys / 16 && pages < 0);
        if (lane == 0) S.gone[j % kMeta] = gone;
      }
      store(sm + (kv ? L::kV : L::kK) + st * L::kTile, kv, cur, csk, csv);
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(kv ? &S.vfull[st] : &S.kfull[st]);
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
        const bool ok = wait_one(bar, (uint32_t)par & 1u, abort_flag, c.err, code, A.wait_cycles);
        tc_fence_after();
        return ok;
      };
      auto wait_stored = [&](uint64_t* bar, int par, int code) {   // (for both CTAs' shared memory)
        const bool ok = PAIR ? wait_cluster(bar, (uint32_t)par & 1u, abort_flag, c.err, code, A.wait_cycles)
                             : wait_one(bar, (uint32_t)par & 1u, abort_flag, c.err, code, A.wait_cycles);
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
        if (!wait_one(bar, (j / kPreStages) & 1, abort_flag, c.err, kDevTimeoutConv, A.wait_cycles)) break;
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

// Joins the parts of the keys of the tasks that were cut (blockIdx.y counts them): a warp a row.
constexpr int kJoinThreads = 256;
template <int D>
__global__ void __launch_bounds__(kJoinThreads) kv4_join_kernel(const Kv4AttendArgs A, int rows, int P, int most) {
  const int r = blockIdx.x * (kJoinThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  const Kv8Args& c = A.k.c;
  pdl_launch_dependents();
  pdl_wait();
  Cut cut;
  Task task;
  int part;
  if (!find_task(c, A.group, rows, 0, P, most, false, cut, task, part) || cut.whole + (int)blockIdx.y >= cut.tasks) return;
  find_task(c, A.group, rows, cut.whole + blockIdx.y * cut.parts, P, most, false, cut, task, part);
  Seq q;
  load_seq(c, task.seq, q, false);
  const int n = q.n * A.group, row = ((n + rows - 1) / rows - 1 - task.from_last) * rows + r;
  if (row >= n) return;
  const size_t pitch = (size_t)rows * (D + 2);
  const float* sums = A.ws + (size_t)blockIdx.y * cut.parts * pitch;
  float M = -INFINITY;
  for (int k = lane; k < cut.parts; k += 32) M = fmaxf(M, __ldcg(sums + k * pitch + (size_t)rows * D + r));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  const float base = M == -INFINITY ? 0.f : M, unit = kv4_unit(A.scale);
  constexpr int E = D / 32;
  float l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 4
  for (int k = 0; k < cut.parts; ++k) {
    const float* p = sums + k * pitch;
    const float f = exp2_fast((__ldcg(p + (size_t)rows * D + r) - base) * unit);
    l = fmaf(f, __ldcg(p + (size_t)rows * (D + 1) + r), l);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(f, __ldcg(p + (size_t)r * D + E * lane + e), o[e]);
  }
  const float inv = l == 0.f ? 0.f : __frcp_rn(l);
  const int tok = row / A.group, hh = row - tok * A.group;
  __half* dst = A.out + (size_t)(q.tok0 + tok) * A.out_stride + (size_t)(task.head * A.group + hh) * D + E * lane;
#pragma unroll
  for (int e = 0; e < E; e += 2) *reinterpret_cast<__half2*>(dst + e) = __floats2half2_rn(o[e] * inv, o[e + 1] * inv);
}

// Of so many keys of a sequence, those that its rows see.
static long long keys_seen(const Kv4AttendArgs& a, long long keys) {
  return a.window > 0 ? std::min(keys, (long long)a.window + a.sinks + a.k.c.max_tokens) : keys;
}
// Pairs of CTAs take sequences of so many rows (of a KV head) and, on average over the rows, so many keys.  Pairs / CTAs
// alone, us, 64 over 8 heads: 1 x 8192 836 / 876; 1 x 512 behind 16000 220 / 240; 1 x 2048 behind 8000 463 / 483; 16 x 100 behind
// 4000 213 / 191 (another wave); 1 x 1000 behind 100000 2558 / 2757; with fewer keys 32 heads, 8 x 512 64 / 46; 32 over 8, 3 x 2048 100 / 95.
constexpr int kPairRows = 512, kPairKeys = 2048;
// Calls of so many waves are not cut, since their tasks do not end together, and calls whose last tasks have fewer keys are
// not, since the join costs more than it saves.
// Cut / whole, us, 64 over 8 heads: 3 x 500 with a window of 4096 182 / 203; 16 x 100 behind 4000 213 / 229; 2048 behind 8000
// 463 / 485 (3.4 waves each); 2 x 3000 behind up to 9000, 32 over 4 (4.2 waves) 595 / 582; 300 behind 300, 40 heads, 44 / 20; 4 x 1683
// behind up to 873, 8 heads of 64, 50 / 38.
constexpr int kCutWaves = 4, kCutKeys = 20 * kTileKeys;

template <int D, bool PAIR>
static cudaError_t launch_prefill4(const Kv4AttendArgs& a, int num_sms, cudaStream_t s) {
  constexpr int kCtas = PAIR ? 2 : 1, kRows = kCtas * 2 * kTileRows;
  constexpr int smem = PreLayout<D, PAIR, (int)sizeof(Pre4Shared)>::kBytes;
  const Kv8Args& c = a.k.c;
  const long long P = std::max(num_sms / kCtas, 1), each = ceil_div((long long)c.max_tokens * a.group, kRows);
  // Most tasks that there can be: whole tiles of all rows, and each sequence's last one.
  const long long tasks = std::min((long long)c.tokens * a.group / kRows + c.seqs, each * c.seqs) * c.kv_heads;
  // The tasks that would be cut are the last ones, with the fewest keys: those of a call's context, or, where all tasks run
  // at once, up to all of its keys.  A part has two tiles of 128 keys at least.
  const long long keys = keys_seen(a, tasks < P ? c.max_len : c.max_len - c.max_tokens);
  // (P = 1: no task is ever left over)
  if (P < 2 || c.seqs > kFewSeqs || tasks >= kCutWaves * P || 3 * (tasks % P) > 2 * P || keys < kCutKeys) {
    const auto fn = kv4_prefill_kernel<D, PAIR, false>;
    const cudaError_t e = ensure_max_dyn_smem(fn);
    if (e != cudaSuccess) return e;
    if (each > 65535) return cudaErrorInvalidValue;
    return launch_after(fn, dim3((unsigned)(kCtas * c.kv_heads), c.seqs, (unsigned)each), kPreThreads, smem, s, kCtas, a, 0, 1);
  }
  const auto fn = kv4_prefill_kernel<D, PAIR, true>;
  cudaError_t e = ensure_max_dyn_smem(fn);
  if (e != cudaSuccess) return e;
  const int most = (int)(keys / (2 * kTileKeys));
  const long long parts = tasks < P ? std::max(P, std::min(3 * tasks, 2 * P)) : tasks + 4 * P / 3;
  e = launch_after(fn, dim3((unsigned)(kCtas * parts)), kPreThreads, smem, s, kCtas, a, (int)P, most);
  if (e != cudaSuccess) return e;
  return launch_after(kv4_join_kernel<D>, dim3(kRows / (kJoinThreads / 32), (unsigned)std::min(tasks, 2 * P / 3)), kJoinThreads, 0,
                      s, 1, a, kRows, (int)P, most);
}

cudaError_t launch_kv4_prefill(const Kv4AttendArgs& a, int num_sms, cudaStream_t s) {
  if (a.k.c.head_dim == 64) return launch_prefill4<64, false>(a, num_sms, s);
  const bool pairs = (long long)a.k.c.max_tokens * a.group >= kPairRows && keys_seen(a, a.k.c.max_len - a.k.c.max_tokens / 2) >= kPairKeys;
  return pairs ? launch_prefill4<128, true>(a, num_sms, s) : launch_prefill4<128, false>(a, num_sms, s);
}

}  // namespace dptq
