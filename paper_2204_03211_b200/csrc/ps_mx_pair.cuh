// Product of two microscaled 4-bit operands, large form: a pair of CTAs on two SMs
// computes tiles of 256 rows of A by 256 rows of B (tcgen05 with cta_group::2).
//
// In the pair each CTA loads its half of either operand, 35 KB for every 512 cycles of
// MMA (51 KB with 128 x 256 on one CTA), and the tensor cores of both read both
// halves.  The leader (rank 0) issues the MMAs; both CTAs load their own halves with
// their completion counted on the leader's barrier, which expects the bytes of both
// (scales are copied by tensor map too, because only those copies can signal the other
// CTA's barrier; the other CTA never arrives there itself: a remote arrive with release
// semantics takes its thread 1400 cycles, nearly three stages).  Commits release the
// stages of both.
//   warp 0      one lane issues the copies of codes
//   warp 1      leader only: scales to tensor memory, MMAs
//   warp 10     one lane issues the copies of scales
//   warps 2-9   read the accumulators, two warps per quarter of the lanes, 128
//               columns each, then release them and store while the next tile runs
// 256 columns of accumulators and two sets of scales leave no room for a second set of
// accumulators, so the release after the read is what lets the next tile start.
//
// Measured: 8192 x 4096 x 4096 49 us (5.6 PFLOP/s; on one CTA with 128 x 256 79.9 us),
// 8192^3 178 us (6.2), 8192 x 4096 x 1024 20 us (3.5).  The tensor cores are busy 64 % of
// the first: of 10000 cycles per tile 8192 are MMA and 1350 the wait for the accumulators
// to be read; the rest is start, end and, under load, the power cap.  Short K is bound by
// the stores of the result (3500 cycles per tile); so are fp32 results (8192 x 4096 x 4096
// 61 us, 8192 x 4096 x 1024 31 us).
#pragma once

#include "ps_mx_gemm.cuh"

namespace psb {

constexpr int kPairThreads = 352;
constexpr int kPairTile = 256;                              // rows of A and of B in a tile
constexpr int kPairHalf = 128 * 128;                        // bytes of a CTA's half of one operand in a stage
constexpr int kPairBytesS = 3 * 2 * kMxAtom;                // scales: its own 128 rows of A, all 256 of B
constexpr int kPairStage = 2 * kPairHalf + kPairBytesS;
constexpr int kPairStages = 6;
constexpr int kPairSmem = kPairStages * kPairStage + 8 * kMmStaging + 256;      // stages, staging for stores, barriers
constexpr int kPairScaleCol = 256;                          // tensor memory: accumulators, then two sets of scales of 24 columns
static_assert(kPairStage % 1024 == 0 && kPairSmem <= kMmSmem, "stages do not fit");

struct PairControl {
  unsigned long long full[kPairStages], empty[kPairStages], acc_full, acc_empty;
  unsigned int tmem;
};
static_assert(sizeof(PairControl) <= 256, "control block");

// The address of this CTA's shared memory word in the pair's leader: the rank is one bit of a shared::cluster address.
__device__ __forceinline__ unsigned int pair_leader(unsigned int addr) {
  unsigned int r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}

// A copy of this CTA whose bytes are counted on `bar`, a barrier of either CTA of the pair.
__device__ __forceinline__ void pair_tma(unsigned int dst, const CUtensorMap* map, int x, int y, unsigned int bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          dst),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}

// mm_wait on a barrier that the other CTA arrives at.
__device__ __forceinline__ bool pair_try_wait(unsigned int bar, unsigned int parity) {
  unsigned int ok;
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool pair_wait(unsigned int bar, unsigned int parity, int* status) {
  if (pair_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!pair_try_wait(bar, parity)) {
    if (clock64() - t0 > kMmWaitCycles) {
      atomicExch(status, 1);
      return false;
    }
  }
  return true;
}

// Arrives on a barrier of either CTA.  (Release at CTA scope, the default: what is handed over is tensor memory, whose
// reads the tcgen05 fence before this orders.  At cluster scope the arrival waits for the warp's stores of the previous
// tile, over a thousand cycles.)
__device__ __forceinline__ void pair_arrive(unsigned int bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void pair_commit(unsigned int bar) {       // arrives on both CTAs' barrier at this offset
  asm volatile(
      "{\n\t"
      ".reg .b16 m;\n\t"
      "mov.b16 m, 3;\n\t"
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n\t"
      "}" ::"r"(bar)
      : "memory");
}

__device__ __forceinline__ void pair_copy_scales(unsigned int tmem, unsigned long long desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}

__device__ __forceinline__ void pair_mma(unsigned int d, unsigned long long a, unsigned long long b, unsigned int idesc,
                                         unsigned int sa, unsigned int sb, bool accumulate) {
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "setp.ne.u32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t"
      "}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned int)accumulate)
      : "memory");
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
ps_mx_matmul_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                         const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
                         const __grid_constant__ MmArgs args) {
  // (no static shared memory beside it: the stages start where the swizzle needs them to, at a multiple of 1024)
  extern __shared__ __align__(1024) unsigned char stages[];
  PairControl& ctl = *reinterpret_cast<PairControl*>(stages + kPairStages * kPairStage + 8 * kMmStaging);
  const unsigned int base = mm_smem(stages);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  unsigned int rank;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));

  if (tid == 0) {
    for (int s = 0; s < kPairStages; ++s) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 2;" ::"r"(mm_smem(&ctl.full[s])) : "memory");     // the leader's two producers
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.empty[s])) : "memory");
    }
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.acc_full)) : "memory");
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 16;" ::"r"(mm_smem(&ctl.acc_empty)) : "memory");    // 8 warps of each
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_sa) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_sb) : "memory");
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
  mx_pdl();

  const int tiles = args.tiles_p * args.tiles_q, stride = (int)(gridDim.x / 2);
  const int first = (int)(blockIdx.x / 2), nk = args.stages_k;

  if (warp == 0 || warp == 10) {
    if (mm_elect()) {
      MmCursor<kPairStages> at;
      const unsigned int full = pair_leader(mm_smem(&ctl.full[0]));
      unsigned int issued = 0;
      bool ok = true;
      for (int tile = first; ok && tile < tiles; tile += stride) {
        int tp, tq;
        mm_tile(args, tile, &tp, &tq);
        // the leader's producers arm its barrier with the bytes of both CTAs; the bytes themselves may come first
        if (warp == 0) {
          const int row_a = tp * kPairTile + (int)rank * 128, row_b = tq * kPairTile + (int)rank * 128;
          for (int k = 0; k < nk; ++k, at.next(), ++issued) {
            if (!mm_wait(mm_smem(&ctl.empty[0]) + 8 * at.s, at.parity ^ 1u, args.status)) { ok = false; break; }
            const unsigned int dst = base + at.s * kPairStage, bar = full + 8 * at.s;
            if (rank == 0)
              asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(mm_smem(&ctl.full[0]) + 8 * at.s),
                           "n"(4 * kPairHalf)
                           : "memory");
            pair_tma(dst, &map_a, k * 128, row_a, bar);
            pair_tma(dst + kPairHalf, &map_b, k * 128, row_b, bar);
          }
        } else {
          // atoms of scales: 128-row block times atoms per block, two per stage (blocks that do not exist read as zeros)
          const int at_a = (int)((tp * 2 + (int)rank) * args.atoms), at_b = (int)(tq * 2 * args.atoms);
          for (int k = 0; k < nk; ++k, at.next(), ++issued) {
            if (!mm_wait(mm_smem(&ctl.empty[0]) + 8 * at.s, at.parity ^ 1u, args.status)) { ok = false; break; }
            const unsigned int dst = base + at.s * kPairStage + 2 * kPairHalf, bar = full + 8 * at.s;
            if (rank == 0)
              asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(mm_smem(&ctl.full[0]) + 8 * at.s),
                           "n"(2 * kPairBytesS)
                           : "memory");
            pair_tma(dst, &map_sa, 0, at_a + 2 * k, bar);
            pair_tma(dst + 2 * kMxAtom, &map_sb, 0, at_b + 2 * k, bar);
            pair_tma(dst + 4 * kMxAtom, &map_sb, 0, at_b + (int)args.atoms + 2 * k, bar);
          }
        }
      }
      if (!ok && rank == 0)                               // an expired wait: let the copies in flight land
        for (unsigned int s = 0; s < (unsigned)kPairStages && s < issued; ++s)
          mm_wait(mm_smem(&ctl.full[s]), ((issued - 1 - s) / kPairStages) & 1u, args.status);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && mm_elect()) {
      MmCursor<kPairStages> at;
      constexpr unsigned int kIdesc = (1u << 7) | (1u << 10) | ((unsigned)(kPairTile >> 3) << 17) | (1u << 23) | (16u << 24);
      unsigned int set = 0, acc_parity = 1;
      bool ok = true;
      for (int tile = first; ok && tile < tiles; tile += stride, acc_parity ^= 1u) {
        if (!pair_wait(mm_smem(&ctl.acc_empty), acc_parity, args.status)) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (int k = 0; k < nk; ++k, at.next(), set ^= 32u) {
          if (!pair_wait(mm_smem(&ctl.full[0]) + 8 * at.s, at.parity, args.status)) { ok = false; break; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const unsigned long long da = mm_desc_codes(base + at.s * kPairStage);
          const unsigned long long ds = mm_desc_scales(base + at.s * kPairStage + 2 * kPairHalf);
          const unsigned int ta = tmem + kPairScaleCol + set, tb = ta + 8;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            pair_copy_scales(ta + j * 4, ds + j * (kMxAtom / 16));
            pair_copy_scales(tb + j * 8, ds + (2 + j) * (kMxAtom / 16));
            pair_copy_scales(tb + j * 8 + 4, ds + (4 + j) * (kMxAtom / 16));
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            pair_mma(tmem, da + 2 * i, da + kPairHalf / 16 + 2 * i, kIdesc | ((unsigned)(i & 1) << 30) | ((unsigned)(i & 1) << 5),
                     ta + (i >> 1) * 4, tb + (i >> 1) * 8, k > 0 || i > 0);
          pair_commit(mm_smem(&ctl.empty[0]) + 8 * at.s);
        }
        pair_commit(mm_smem(&ctl.acc_full));
      }
    }
    __syncwarp();
  } else {
    const int quad = warp & 3, half = (warp - 2) >> 2;
    unsigned char* staging = stages + kPairStages * kPairStage + (warp - 2) * kMmStaging;
    const unsigned int empty = pair_leader(mm_smem(&ctl.acc_empty));
    const unsigned int acc = tmem + ((unsigned)(quad * 32) << 16) + half * 128;
    unsigned int n = 0;
    for (int tile = first; tile < tiles; tile += stride, ++n) {
      if (!__all_sync(0xffffffffu, mm_wait(mm_smem(&ctl.acc_full), n & 1u, args.status))) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      float v[128];
      mm_load<128>(acc, v);
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) pair_arrive(empty);
      int tp, tq;
      mm_tile(args, tile, &tp, &tq);
      const long long m = (long long)tp * kPairTile + rank * 128 + quad * 32;
      const long long q = (long long)tq * kPairTile + half * 128;
      mm_store_rows<128>(args, staging, lane, m, q, args.rows_p, args.rows_q, v);
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
