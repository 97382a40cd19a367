// Products of 16-bit operands on the 5th-generation tensor cores, as a frame that the operators fill in: a pair of
// CTAs on two SMs (tcgen05, cta_group::2) computes tiles of 256 x 256, or (Op::kPair = false) one CTA tiles of 128 x 128,
// with binary32 sums in tensor memory,
//     acc[i][j] = sum over k of A[i][k] * B[j][k],
// and an operator `Op` says which tiles there are, where their operands lie, and what becomes of the sums.
//
// k may run along the rows of an operand's tensor ("K-major") or down its columns (transposed operands, as both gradients
// of a product need): the boxes that are fetched and the MMA's descriptors say which, so no tensor is ever transposed in
// memory for a product.  A stage is 64 or 32 elements of k (Op::kK), 16 or 8 KB per operand, plane and CTA:
//   64  boxes of 64 rows by 64 columns, rows of 128 bytes in 128-byte swizzle, two one below the other (K-major) or side
//       by side
//   32  one box of 128 rows by 32 columns, rows of 64 bytes in 64-byte swizzle (K-major), or two of 32 rows by 64 columns
//       in 128-byte swizzle side by side
// Short stages keep more copies in flight in the same shared memory: one is worked on, the others are on their way.
// Operands may consist of two planes (value = high + low, see Op::kPlanes): a stage then holds both and feeds three
// products, high x high, high x low and low x high, so what is fetched from L2 per product is 2/3 of one plane's.
//   warp 0     one lane issues the copies (each CTA its half, counted on the leader's barrier)
//   warp 1     leader: one lane issues the MMAs
//   warps 4-   (Op::kWarps: eight or sixteen) read the accumulators, two or four warps per quarter of the lanes, which
//              share the columns
//   warps 2-3  for operators whose epilogue reads and writes 16-bit tiles (Op::kSlots > 0): one lane per half of the
//              columns fetches, and stores, 128 rows by 32 columns at a time through a ring of slots in shared memory.
//              An epilogue that did its own copies spent four fifths of its time waiting for them.
// Two sets of accumulators let the next tile's products run under the epilogue.
//
// Bounds: 256 x 256 tiles fetch 64 KB from L2 per 64 elements of k and pair, which is 512 cycles of MMA: 128 bytes per
// cycle and pair, within what L2 delivers; one CTA with 128 x 256 would need 1.5 times that.  Measured: the scores of 8192
// tokens over 30522 words, 1024 wide, with their losses 318 us, 1.6 PFLOP/s.
#pragma once

#include "ps_mma.cuh"

namespace psb {

constexpr int kTcMaxStages = 10;

constexpr int kTcMaxSlots = 4;
constexpr int kTcSideThreads = 64;                          // of a CTA, for work beside the tiles

struct TcControl {
  unsigned long long full[kTcMaxStages], empty[kTcMaxStages], acc_full[2], acc_empty[2];
  // slots of either half of the columns: holds what the epilogue reads, holds what it has written, may be used again
  unsigned long long staged[2][kTcMaxSlots], filled[2][kTcMaxSlots], freed[2][kTcMaxSlots];
  unsigned int tmem;
};
constexpr int kTcControl = 512;
static_assert(sizeof(TcControl) <= kTcControl, "control block");

constexpr int kTcPlane = 128 * 64;                          // bytes of 128 rows by 32 columns of 16 bits
constexpr int kTcSlot = 2 * kTcPlane;
constexpr int kTcVector = 1024;                             // two vectors of 128 floats

template <typename Op>
struct TcCfg {
  static constexpr int kThreads = 128 + 32 * Op::kWarps;
  static constexpr int kOperand = 128 * Op::kK * 2;         // a CTA's 128 rows of one plane of one operand
  static constexpr int kStage = 2 * Op::kPlanes * kOperand;
  static constexpr int kStages = Op::kStages;
  static constexpr int kSlotsAt = kStages * kStage, kVectorsAt = kSlotsAt + 2 * Op::kSlots * kTcSlot;
  // Vectors of a half's tiles, in turn.  A tile's are fetched when the slot of its first entry is free; with as many sets
  // as slots (counting tiles with entries) that entry's last user came after the set's.
  static constexpr int kSets = Op::kSlots == 1 ? 2 : Op::kSlots;
  static constexpr int kControlAt = kVectorsAt + 2 * kSets * kTcVector;
  static constexpr int kSmem = kControlAt + kTcControl;
  static_assert(kSmem <= 227 * 1024 && kStages <= kTcMaxStages && Op::kSlots <= kTcMaxSlots, "stages do not fit");
};

// One tile: its operands and how far k runs.
struct TcTile {
  const CUtensorMap* a;                  // the planes' maps follow one another
  const CUtensorMap* b;
  int a_mn, b_mn;                        // 1: k runs down the columns of the tensor
  int a_row, b_row;                      // first row of A and of B (their position in the other dimension)
  int a_k, b_k;                          // where k starts in either tensor
  int nk;                                // stages
  const unsigned int* ready;             // wait until *ready >= need before the first copy; nullptr: nothing to wait for
  unsigned int need;
};

// The MMA's view of an operand in shared memory.  Strides in units of 16 bytes: between boxes of 64 columns (only where k
// runs down them) and between groups of eight rows.
template <int K>
__device__ __forceinline__ unsigned long long tc_desc(unsigned int addr, int mn) {
  const unsigned long long at = (unsigned long long)((addr & 0x3ffffu) >> 4) | (1ull << 46);
  if (mn) return at | ((unsigned long long)(K * 128 / 16) << 16) | (64ull << 32) | (2ull << 61);
  return at | (1ull << 16) | (K == 64 ? (64ull << 32) | (2ull << 61) : (32ull << 32) | (4ull << 61));
}

template <bool PAIR>
__device__ __forceinline__ void tc_mma(unsigned int d, unsigned long long a, unsigned long long b, unsigned int idesc,
                                       bool accumulate) {
  if constexpr (PAIR)
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t"
        "}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((unsigned int)accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "setp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t"
        "}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((unsigned int)accumulate)
        : "memory");
}

template <bool PAIR>
__device__ __forceinline__ bool tc_wait(unsigned int bar, unsigned int parity, int* status) {    // the other CTA may arrive there
  if constexpr (PAIR) return pair_wait(bar, parity, status);
  else return mm_wait(bar, parity, status);
}
template <bool PAIR>
__device__ __forceinline__ void tc_commit(unsigned int bar) {
  if constexpr (PAIR) pair_commit(bar);
  else mm_commit(bar);
}

// This CTA's 128 rows of an operand, K elements of k.
template <bool PAIR, int K>
__device__ __forceinline__ void tc_fetch(unsigned int dst, const CUtensorMap* map, int mn, int row, int k, unsigned int bar) {
  auto box = [&](unsigned int at, int x, int y) {
    if constexpr (PAIR) pair_tma(at, map, x, y, bar);
    else mm_tma(at, map, x, y, bar);
  };
  if (mn) {
    box(dst, row, k);
    box(dst + K * 128, row + 64, k);
  } else {
    box(dst, k, row);
    if constexpr (K == 64) box(dst + 64 * 128, k, row + 64);
  }
}

// Waits for the tiles that a tile's operands come from; what other CTAs stored is then visible to copies of this thread.
__device__ __forceinline__ bool tc_wait_ready(const TcTile& t, int* status) {
  if (!t.ready) return true;
  unsigned int have;
  const long long t0 = clock64();
  while (true) {
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(have) : "l"(t.ready) : "memory");
    if (have >= t.need) break;
    if (clock64() - t0 > kMmWaitCycles) {
      atomicExch(status, 1);
      return false;
    }
  }
  asm volatile("fence.proxy.async;" ::: "memory");
  return true;
}

// A slot's planes have rows of 64 bytes in 64-byte swizzle, so that lanes that read or write a row each meet in no bank.
// The byte address of a row's 16-byte piece:
__device__ __forceinline__ unsigned int tc_piece_at(int row, int piece) {
  return (unsigned int)(row * 64 + ((piece ^ ((row >> 1) & 3)) << 4));
}

__device__ __forceinline__ void tc_store(const CUtensorMap* map, int x, int y, unsigned int src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src)
               : "memory");
}
__device__ __forceinline__ void tc_arrive(unsigned int bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// A warp's 32 x 32 values, a row per lane, become a column per lane: v[i] what lane i held for this lane's column.
__device__ __forceinline__ void tc_exchange(float (&v)[32], int lane) {
#pragma unroll
  for (int k = 16; k >= 1; k >>= 1) {
    const bool upper = (lane & k) != 0;
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if ((i & k) == 0) {
        const float got = __shfl_xor_sync(0xffffffffu, upper ? v[i] : v[i | k], k);
        v[i] = upper ? got : v[i];
        v[i | k] = upper ? v[i | k] : got;
      }
  }
}

// What an epilogue warp knows of its place, and its walk over the slots.
struct TcWarp {
  unsigned char* slots;                  // of the warp's half
  const float* vectors;                  // the same, of the current tile
  unsigned int staged, filled;           // barriers of slot 0
  int lane, row, col;                    // the warp's first row and column in the tile
  int* status;
  unsigned long long mark = 0;           // the epilogue's: when the tile before was done
};

// Op:
//   kPair; kWarps; kPlanes; kK; kStages; kType (0 fp16, 1 bf16); kSegment (0, or: after so many stages the sums are taken over into
//   registers); kSlots; Args with `int* status`
//   tiles(args, this CTA or pair, their number, first, end, stride); Item item(args, index), what the roles need to know of a tile, read one tile ahead; tile(args, item, TcTile*)
//   Epilogue(args, item, TcWarp&, cursor): begin() before the sums are there, columns(32 sums of this lane's row, their
//   place among the warp's columns), end()
//   kSide (without slots): warps 2 and 3 do side(args, thread, threads)
// and with slots
//   entries(args, item, rank, half), how many slots the half's columns pass through; load(args, item, rank, half, entry,
//   slot, vectors, barrier), which arrives; store(args, item, rank, half, entry, slot); done(args, item, rank)
template <typename Op>
__global__ void __cluster_dims__(Op::kPair ? 2 : 1, 1, 1) __launch_bounds__(TcCfg<Op>::kThreads, 1)
ps_tc_kernel(const __grid_constant__ typename Op::Args args) {
  using Cfg = TcCfg<Op>;
  // (no static shared memory beside it: the stages start where the swizzle needs them to, at a multiple of 1024)
  extern __shared__ __align__(1024) unsigned char stages[];
  TcControl& ctl = *reinterpret_cast<TcControl*>(stages + Cfg::kControlAt);
  const unsigned int base = mm_smem(stages);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  constexpr bool kPair = Op::kPair;
  constexpr int kCtas = kPair ? 2 : 1, kTile = kCtas * 128, kColumns = kTile / (Op::kWarps / 4);       // a tile's rows; a warp's columns
  unsigned int rank = 0;
  if constexpr (kPair) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));

  if (tid == 0) {
    for (int s = 0; s < Cfg::kStages; ++s) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.full[s])) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.empty[s])) : "memory");
    }
    for (int b = 0; b < 2; ++b) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.acc_full[b])) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(mm_smem(&ctl.acc_empty[b])), "n"(kCtas * Op::kWarps) : "memory");
    }
    for (int h = 0; h < 2; ++h)
      for (int b = 0; b < Op::kSlots; ++b) {
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.staged[h][b])) : "memory");
        asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(mm_smem(&ctl.filled[h][b])), "n"(Op::kWarps / 2) : "memory");
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.freed[h][b])) : "memory");
      }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if constexpr (kPair) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(mm_smem(&ctl.tmem)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 256;" ::"r"(mm_smem(&ctl.tmem)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if constexpr (kPair) mm_cluster_sync();                 // both CTAs' barriers and tensor memory exist
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const unsigned int tmem = ctl.tmem;
  mm_pdl();

  int first, tiles, stride;                               // this CTA's (pair's) tiles: first, first + stride, ... below `tiles`
  Op::tiles(args, (int)(blockIdx.x / kCtas), (int)(gridDim.x / kCtas), &first, &tiles, &stride);

  // Taking sums over into registers needs more of them than a third of the file per warpgroup: 128 x (40 + 2 x 232) is
  // what the 384 threads were launched with (168 each).
  if (warp < 4) {
    if constexpr (Op::kSegment > 0) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
  if (warp == 0) {
    if (mm_elect()) {
      MmCursor<Cfg::kStages> at;
      const unsigned int full = kPair ? pair_leader(mm_smem(&ctl.full[0])) : mm_smem(&ctl.full[0]);
      unsigned int issued = 0;
      bool ok = true;
      typename Op::Item next = Op::item(args, first, tiles);
      for (int index = first; ok && index < tiles; index += stride) {
        const typename Op::Item item = next;
        next = Op::item(args, index + stride, tiles);
        TcTile t;
        Op::tile(args, item, &t);
        if (!tc_wait_ready(t, args.status)) { ok = false; break; }
        const int row_a = t.a_row + (int)rank * 128, row_b = t.b_row + (int)rank * 128;
        for (int k = 0; k < t.nk; ++k, at.next(), ++issued) {
          if (!mm_wait(mm_smem(&ctl.empty[0]) + 8 * at.s, at.parity ^ 1u, args.status)) { ok = false; break; }
          unsigned int dst = base + at.s * Cfg::kStage;
          const unsigned int bar = full + 8 * at.s;
          // the leader arms its barrier with the bytes of both CTAs; the bytes themselves may come first
          if (rank == 0)
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(mm_smem(&ctl.full[0]) + 8 * at.s),
                         "n"(kCtas * Cfg::kStage)
                         : "memory");
#pragma unroll
          for (int p = 0; p < Op::kPlanes; ++p, dst += Cfg::kOperand) tc_fetch<kPair, Op::kK>(dst, t.a + p, t.a_mn, row_a, t.a_k + k * Op::kK, bar);
#pragma unroll
          for (int p = 0; p < Op::kPlanes; ++p, dst += Cfg::kOperand) tc_fetch<kPair, Op::kK>(dst, t.b + p, t.b_mn, row_b, t.b_k + k * Op::kK, bar);
        }
      }
      if (!ok && rank == 0)                               // an expired wait: let the copies in flight land
        for (unsigned int s = 0; s < (unsigned)Cfg::kStages && s < issued; ++s)
          mm_wait(mm_smem(&ctl.full[s]), ((issued - 1 - s) / Cfg::kStages) & 1u, args.status);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && mm_elect()) {
      MmCursor<Cfg::kStages> at;
      MmCursor<2> acc;
      bool ok = true;
      typename Op::Item next = Op::item(args, first, tiles);
      for (int index = first; ok && index < tiles; index += stride) {
        const typename Op::Item item = next;
        next = Op::item(args, index + stride, tiles);
        TcTile t;
        Op::tile(args, item, &t);
        const unsigned int idesc = (1u << 4) | ((unsigned)Op::kType << 7) | ((unsigned)Op::kType << 10) | ((unsigned)t.a_mn << 15) |
                                   ((unsigned)t.b_mn << 16) | ((unsigned)(kTile >> 3) << 17) | ((unsigned)(kTile >> 4) << 24);
        // 16 elements of k: 32 bytes along a row, or 16 rows of 128 bytes
        const unsigned int step_a = t.a_mn ? 128u : 2u, step_b = t.b_mn ? 128u : 2u;
        const int segment = Op::kSegment ? Op::kSegment : t.nk;
        for (int k0 = 0; ok && k0 < t.nk; k0 += segment, acc.next()) {
          if (!tc_wait<kPair>(mm_smem(&ctl.acc_empty[0]) + 8 * acc.s, acc.parity ^ 1u, args.status)) { ok = false; break; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const unsigned int d = tmem + acc.s * kTile;
          const int k1 = min(t.nk, k0 + segment);
          for (int k = k0; k < k1; ++k, at.next()) {
            if (!tc_wait<kPair>(mm_smem(&ctl.full[0]) + 8 * at.s, at.parity, args.status)) { ok = false; break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const unsigned long long da = tc_desc<Op::kK>(base + at.s * Cfg::kStage, t.a_mn);
            const unsigned long long db = tc_desc<Op::kK>(base + at.s * Cfg::kStage + Op::kPlanes * Cfg::kOperand, t.b_mn);
            bool more = k > k0;
            if constexpr (Op::kPlanes == 2) {             // the small products first, while the sums are small
#pragma unroll
              for (int i = 0; i < Op::kK / 16; ++i) {
                const unsigned long long a = da + i * step_a, b = db + i * step_b;
                tc_mma<kPair>(d, a, b + Cfg::kOperand / 16, idesc, more || i > 0);
                tc_mma<kPair>(d, a + Cfg::kOperand / 16, b, idesc, true);
              }
              more = true;
            }
#pragma unroll
            for (int i = 0; i < Op::kK / 16; ++i) tc_mma<kPair>(d, da + i * step_a, db + i * step_b, idesc, more || i > 0);
            tc_commit<kPair>(mm_smem(&ctl.empty[0]) + 8 * at.s);
          }
          tc_commit<kPair>(mm_smem(&ctl.acc_full[0]) + 8 * acc.s);
        }
      }
    }
    __syncwarp();
    } else if constexpr (Op::kSlots > 0) {
      if (mm_elect()) {
        MmCursor<Op::kSlots> at[2];
        const unsigned int slots = base + Cfg::kSlotsAt, vectors = base + Cfg::kVectorsAt;
        constexpr unsigned int kHalf = 8 * kTcMaxSlots;
        const unsigned int staged = mm_smem(&ctl.staged[0][0]), filled = mm_smem(&ctl.filled[0][0]), freed = mm_smem(&ctl.freed[0][0]);
        bool ok = true;
        int set[2] = {0, 0};
        typename Op::Item next = Op::item(args, first, tiles);
        for (int index = first; ok && index < tiles; index += stride) {
          const typename Op::Item item = next;
          next = Op::item(args, index + stride, tiles);
          const int entries[2] = {Op::entries(args, item, (int)rank, 0), Op::entries(args, item, (int)rank, 1)};
          if (warp == 2) {
            TcTile t;
            Op::tile(args, item, &t);
            if (!tc_wait_ready(t, args.status)) { ok = false; break; }       // (the copies below are waited for then)
            for (int e = 0; ok && e < max(entries[0], entries[1]); ++e)
#pragma unroll
              for (int h = 0; h < 2; ++h)
                if (e < entries[h]) {
                  if (!mm_wait(freed + h * kHalf + 8 * at[h].s, at[h].parity ^ 1u, args.status)) { ok = false; break; }
                  Op::load(args, item, (int)rank, h, e, slots + (h * Op::kSlots + at[h].s) * kTcSlot,
                           vectors + (h * Cfg::kSets + set[h]) * kTcVector, staged + h * kHalf + 8 * at[h].s);
                  at[h].next();
                }
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (entries[h] > 0 && ++set[h] == Cfg::kSets) set[h] = 0;
          } else {
            unsigned int last = 0;                        // the slot whose stores may not have read it yet
            for (int e = 0; ok && e < max(entries[0], entries[1]); ++e)
#pragma unroll
              for (int h = 0; h < 2; ++h)
                if (e < entries[h]) {
                  if (!mm_wait(filled + h * kHalf + 8 * at[h].s, at[h].parity, args.status)) { ok = false; break; }
                  Op::store(args, item, (int)rank, h, e, slots + (h * Op::kSlots + at[h].s) * kTcSlot);
                  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                  if (last) {
                    asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                    tc_arrive(last);
                  }
                  last = freed + h * kHalf + 8 * at[h].s;
                  at[h].next();
                }
            // all that the tile's epilogue has stored is there for copies of any CTA that sees the count
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            if (last) tc_arrive(last);
            if (ok) Op::done(args, item, (int)rank);
          }
        }
        // after an expired wait: copies into slots land before the CTA leaves (the slots that were asked for last)
        if (warp == 2 && !ok)
          for (int h = 0; h < 2; ++h)
            for (unsigned int s = 0; s < (unsigned)Op::kSlots; ++s)
              mm_wait(staged + h * kHalf + 8 * s, s < at[h].s ? at[h].parity : at[h].parity ^ 1u, args.status);
      }
      __syncwarp();
    } else if constexpr (Op::kSide) {
      Op::side(args, (int)blockIdx.x * kTcSideThreads + (warp - 2) * 32 + lane, (int)gridDim.x * kTcSideThreads);
      __syncwarp();
    }
  } else {
    if constexpr (Op::kSegment > 0) asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int quad = warp & 3, half = (warp - 4) >> 2;
    const unsigned int empty = kPair ? pair_leader(mm_smem(&ctl.acc_empty[0])) : mm_smem(&ctl.acc_empty[0]);
    MmCursor<2> acc;
    TcWarp w;
    w.slots = stages + Cfg::kSlotsAt + half * Op::kSlots * kTcSlot;
    w.staged = mm_smem(&ctl.staged[half][0]);
    w.filled = mm_smem(&ctl.filled[half][0]);
    w.lane = lane;
    w.row = (int)rank * 128 + quad * 32;
    w.col = half * kColumns;
    w.status = args.status;
    const unsigned int lanes = tmem + ((unsigned)(quad * 32) << 16) + half * kColumns;
    MmCursor<(Op::kSlots > 0 ? Op::kSlots : 1)> slot;
    int set = 0;
    typename Op::Item next = Op::item(args, first, tiles);
    for (int index = first; index < tiles; index += stride) {
      const typename Op::Item item = next;
      next = Op::item(args, index + stride, tiles);
      if constexpr (Op::kSlots > 0) {
        w.vectors = reinterpret_cast<const float*>(stages + Cfg::kVectorsAt + (half * Cfg::kSets + set) * kTcVector);
        if (Op::entries(args, item, (int)rank, half) > 0 && ++set == Cfg::kSets) set = 0;
      }
      typename Op::Epilogue e(args, item, w, slot);
      e.begin();
      if constexpr (Op::kSegment > 0) {
        // Binary32 sums of the tensor cores are cut off, not rounded: with every step they lose half a unit of their
        // last place, always towards zero.  Short stretches of k, added up here with rounding, keep that small.  The
        // total goes back to tensor memory, where the epilogue reads it a few columns at a time.
        float sum[kColumns];
#pragma unroll
        for (int i = 0; i < kColumns; ++i) sum[i] = 0.f;
        const int nk = Op::stages(args, item);
        bool ok = true;
        int k = 0;
        for (; ok && k + Op::kSegment < nk; k += Op::kSegment, acc.next()) {
          ok = __all_sync(0xffffffffu, mm_wait(mm_smem(&ctl.acc_full[0]) + 8 * acc.s, acc.parity, args.status));
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const unsigned int at = lanes + acc.s * kTile;
#pragma unroll
          for (int c = 0; c < kColumns; c += 16) {
            float v[16];
            mm_load<16>(at + c, v);
            if (c == kColumns - 16) {
              asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
              __syncwarp();
              if (lane == 0) pair_arrive(empty + 8 * acc.s);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[c + i] = __fadd_rn(sum[c + i], v[i]);
          }
        }
        if (!ok || !__all_sync(0xffffffffu, mm_wait(mm_smem(&ctl.acc_full[0]) + 8 * acc.s, acc.parity, args.status))) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (k > 0) {
          const unsigned int at = lanes + acc.s * kTile;
#pragma unroll
          for (int c = 0; c < kColumns; c += 16) {
            float v[16];
            mm_load<16>(at + c, v);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __fadd_rn(sum[c + i], v[i]);
            mm_store16(at + c, v);
          }
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        }
      } else {
        if (!__all_sync(0xffffffffu, mm_wait(mm_smem(&ctl.acc_full[0]) + 8 * acc.s, acc.parity, args.status))) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      }
      {
        const unsigned int at = lanes + acc.s * kTile;
#pragma unroll 1
        for (int c = 0; c < kColumns; c += 32) {
          float v[32];
          mm_load<32>(at + c, v);
          if (c == kColumns - 32) {                                  // all read: the next tile but one may have the accumulators
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) pair_arrive(empty + 8 * acc.s);
          }
          e.columns(v, c);
        }
        acc.next();
      }
      e.end();
    }
    __syncwarp();
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if constexpr (kPair) mm_cluster_sync();                 // neither CTA leaves while the other may signal it or read from it
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1) {
    if constexpr (kPair) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 256;" ::"r"(tmem) : "memory");
  }
}

}  // namespace psb
