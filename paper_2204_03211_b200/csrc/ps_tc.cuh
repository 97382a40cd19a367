// Products of 16-bit operands on the 5th-generation tensor cores, as a frame that the operators fill in: a pair of
// CTAs on two SMs (tcgen05, cta_group::2) computes tiles of 256 x 256 with binary32 sums in tensor memory,
//     acc[i][j] = sum over k of A[i][k] * B[j][k],
// and an operator `Op` says which tiles there are, where their operands lie, and what becomes of the sums.
//
// Operands are fetched as boxes of 64 rows by 64 columns (8 KB, rows of 128 bytes, 128-byte swizzle).  One box shape
// serves both orders: where k runs along a row of the tensor ("K-major") a stage takes two boxes one below the other,
// where it runs down the columns (transposed operands, as both gradients of a product need) two boxes side by side, and
// the MMA's descriptors say which.  So no tensor is ever transposed in memory for a product.
//
// A stage is 64 elements of k: 16 KB per operand and CTA.  Operands may consist of two planes (value = high + low, see
// Op::kPlanes): a stage then holds both and feeds three products, high x high, high x low and low x high, so what is
// fetched from L2 per product is 2/3 of one plane's.
//   warp 0     one lane issues the copies (each CTA its half, counted on the leader's barrier)
//   warp 1     leader: one lane issues the MMAs
//   warps 2-9  read the accumulators, two warps per quarter of the lanes, 128 columns each
// Two sets of accumulators (2 x 256 columns) let the next tile's products run under the epilogue.
//
// Bounds: 256 x 256 tiles fetch 64 KB from L2 per 64 elements of k and pair, which is 512 cycles of MMA: 128 bytes per
// cycle and pair, within what L2 delivers; one CTA with 128 x 256 would need 1.5 times that.
#pragma once

#include "ps_mma.cuh"

namespace psb {

constexpr int kTcThreads = 320;
constexpr int kTcTile = 256;                                // rows of A and of B in a tile
constexpr int kTcK = 64;                                    // elements of k in a stage
constexpr int kTcBox = 64 * 128;                            // bytes of a box
constexpr int kTcOperand = 2 * kTcBox;                      // a CTA's 128 rows of one plane of one operand
constexpr int kTcMaxStages = 6;

struct TcControl {
  unsigned long long full[kTcMaxStages], empty[kTcMaxStages], acc_full[2], acc_empty[2];
  unsigned int tmem;
};
constexpr int kTcControl = 256;
static_assert(sizeof(TcControl) <= kTcControl, "control block");

template <int PLANES>
struct TcCfg {
  static constexpr int kStage = 2 * PLANES * kTcOperand;
  static constexpr int kStages = PLANES == 2 ? 3 : 6;
  static constexpr int kSmem = kStages * kStage + kTcControl;
  static_assert(kSmem <= 227 * 1024 && kStages <= kTcMaxStages, "stages do not fit");
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

// Strides of the MMA's view of an operand in shared memory, in units of 16 bytes: between 64-row boxes (only where k runs
// down the columns) and between groups of eight rows of 128 bytes.
__device__ __forceinline__ unsigned long long tc_desc(unsigned int addr, int mn) {
  const unsigned long long lead = mn ? kTcBox / 16 : 1;
  return (unsigned long long)((addr & 0x3ffffu) >> 4) | (lead << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}

__device__ __forceinline__ void tc_mma(unsigned int d, unsigned long long a, unsigned long long b, unsigned int idesc,
                                       bool accumulate) {
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t"
      "}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((unsigned int)accumulate)
      : "memory");
}

// This CTA's 128 rows of an operand, 64 elements of k.
__device__ __forceinline__ void tc_fetch(unsigned int dst, const CUtensorMap* map, int mn, int row, int k, unsigned int bar) {
  pair_tma(dst, map, mn ? row : k, mn ? k : row, bar);
  pair_tma(dst + kTcBox, map, mn ? row + 64 : k, mn ? k : row + 64, bar);
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

// What a warp has stored of a tile is visible to copies of any CTA that sees the count (16 warps per tile).
__device__ __forceinline__ void tc_signal(unsigned int* count, int lane) {
  asm volatile("fence.proxy.async;" ::: "memory");
  __threadfence();
  __syncwarp();
  if (lane == 0) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(count) : "memory");
}

// Op: kPlanes; kType (0 fp16, 1 bf16); Args with `int* status`; tiles(args); tile(args, index, TcTile*);
// an Epilogue(args, index, rank) with begin(row in tile, first column in tile, lane), columns(32 sums of this lane's row,
// column in tile), end(lane).
template <typename Op>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kTcThreads, 1)
ps_tc_kernel(const __grid_constant__ typename Op::Args args) {
  using Cfg = TcCfg<Op::kPlanes>;
  // (no static shared memory beside it: the stages start where the swizzle needs them to, at a multiple of 1024)
  extern __shared__ __align__(1024) unsigned char stages[];
  TcControl& ctl = *reinterpret_cast<TcControl*>(stages + Cfg::kStages * Cfg::kStage);
  const unsigned int base = mm_smem(stages);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  unsigned int rank;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));

  if (tid == 0) {
    for (int s = 0; s < Cfg::kStages; ++s) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.full[s])) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.empty[s])) : "memory");
    }
    for (int b = 0; b < 2; ++b) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.acc_full[b])) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 16;" ::"r"(mm_smem(&ctl.acc_empty[b])) : "memory");   // 8 warps of each
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(mm_smem(&ctl.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  mm_cluster_sync();                                      // both CTAs' barriers and tensor memory exist
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const unsigned int tmem = ctl.tmem;
  mm_pdl();

  const int tiles = Op::tiles(args), stride = (int)(gridDim.x / 2), first = (int)(blockIdx.x / 2);

  if (warp == 0) {
    if (mm_elect()) {
      MmCursor<Cfg::kStages> at;
      const unsigned int full = pair_leader(mm_smem(&ctl.full[0]));
      unsigned int issued = 0;
      bool ok = true;
      for (int index = first; ok && index < tiles; index += stride) {
        TcTile t;
        Op::tile(args, index, &t);
        if (!tc_wait_ready(t, args.status)) { ok = false; break; }
        const int row_a = t.a_row + (int)rank * 128, row_b = t.b_row + (int)rank * 128;
        for (int k = 0; k < t.nk; ++k, at.next(), ++issued) {
          if (!mm_wait(mm_smem(&ctl.empty[0]) + 8 * at.s, at.parity ^ 1u, args.status)) { ok = false; break; }
          unsigned int dst = base + at.s * Cfg::kStage;
          const unsigned int bar = full + 8 * at.s;
          // the leader arms its barrier with the bytes of both CTAs; the bytes themselves may come first
          if (rank == 0)
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(mm_smem(&ctl.full[0]) + 8 * at.s),
                         "n"(2 * Cfg::kStage)
                         : "memory");
#pragma unroll
          for (int p = 0; p < Op::kPlanes; ++p, dst += kTcOperand) tc_fetch(dst, t.a + p, t.a_mn, row_a, t.a_k + k * kTcK, bar);
#pragma unroll
          for (int p = 0; p < Op::kPlanes; ++p, dst += kTcOperand) tc_fetch(dst, t.b + p, t.b_mn, row_b, t.b_k + k * kTcK, bar);
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
      for (int index = first; ok && index < tiles; index += stride, acc.next()) {
        TcTile t;
        Op::tile(args, index, &t);
        if (!pair_wait(mm_smem(&ctl.acc_empty[0]) + 8 * acc.s, acc.parity ^ 1u, args.status)) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const unsigned int d = tmem + acc.s * kTcTile;
        const unsigned int idesc = (1u << 4) | ((unsigned)Op::kType << 7) | ((unsigned)Op::kType << 10) | ((unsigned)t.a_mn << 15) |
                                   ((unsigned)t.b_mn << 16) | ((unsigned)(kTcTile >> 3) << 17) | ((unsigned)(kTcTile >> 4) << 24);
        // 16 elements of k: 32 bytes along a row, or 16 rows of 128 bytes
        const unsigned int step_a = t.a_mn ? 128u : 2u, step_b = t.b_mn ? 128u : 2u;
        for (int k = 0; k < t.nk; ++k, at.next()) {
          if (!pair_wait(mm_smem(&ctl.full[0]) + 8 * at.s, at.parity, args.status)) { ok = false; break; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const unsigned long long da = tc_desc(base + at.s * Cfg::kStage, t.a_mn);
          const unsigned long long db = tc_desc(base + at.s * Cfg::kStage + Op::kPlanes * kTcOperand, t.b_mn);
#pragma unroll
          for (int i = 0; i < kTcK / 16; ++i) {
            const unsigned long long a = da + i * step_a, b = db + i * step_b;
            tc_mma(d, a, b, idesc, k > 0 || i > 0);
            if constexpr (Op::kPlanes == 2) {
              tc_mma(d, a, b + kTcOperand / 16, idesc, true);
              tc_mma(d, a + kTcOperand / 16, b, idesc, true);
            }
          }
          pair_commit(mm_smem(&ctl.empty[0]) + 8 * at.s);
        }
        pair_commit(mm_smem(&ctl.acc_full[0]) + 8 * acc.s);
      }
    }
    __syncwarp();
  } else {
    const int quad = warp & 3, half = (warp - 2) >> 2;
    const unsigned int empty = pair_leader(mm_smem(&ctl.acc_empty[0]));
    MmCursor<2> acc;
    for (int index = first; index < tiles; index += stride, acc.next()) {
      typename Op::Epilogue e(args, index);
      e.begin((int)rank * 128 + quad * 32 + lane, half * 128, lane);
      if (!__all_sync(0xffffffffu, mm_wait(mm_smem(&ctl.acc_full[0]) + 8 * acc.s, acc.parity, args.status))) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const unsigned int at = tmem + ((unsigned)(quad * 32) << 16) + acc.s * kTcTile + half * 128;
#pragma unroll 1
      for (int c = 0; c < 128; c += 32) {
        float v[32];
        mm_load<32>(at + c, v);
        if (c == 96) {                                    // all read: the next tile but one may have the accumulators
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) pair_arrive(empty + 8 * acc.s);
        }
        e.columns(v, half * 128 + c);
      }
      e.end(lane);
    }
    __syncwarp();
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  mm_cluster_sync();                                      // neither CTA leaves while the other may signal it or read from it
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

}  // namespace psb
