// Product of two microscaled 4-bit operands, large form: a pair of CTAs on two SMs
// computes tiles of 256 rows of A by 256 rows of B (tcgen05 with cta_group::2).
//
// What bounds the one-CTA form on large operands is the traffic into shared memory:
// at 128 x 256 a tile takes in 51 KB for every 512 cycles of MMA.  In the pair each
// CTA loads its half of either operand, 35 KB for the same time, and the tensor cores
// of both read both halves.  The leader (rank 0) issues the MMAs; both CTAs load their
// own halves with their completion counted on the leader's barrier, which expects the
// bytes of both (scales are copied by tensor map too, because only those copies can
// signal the other CTA's barrier; the other CTA never arrives there itself: a remote
// arrive with release semantics takes its thread 1400 cycles, nearly three stages).
// Commits release the stages of both.
//   warp 0      one lane issues the copies of codes
//   warp 1      leader only: scales to tensor memory, MMAs
//   warp 10     one lane issues the copies of scales
//   warps 2-9   read the accumulators, two warps per quarter of the lanes, 128
//               columns each, then release them and store while the next tile runs
// 256 columns of accumulators and two sets of scales leave no room for a second set of
// accumulators, so the release after the read is what lets the next tile start.
#pragma once

#include "ps_mx_gemm.cuh"

namespace psb {

constexpr int kPairThreads = 352;
constexpr int kPairTile = 256;                              // rows of A and of B in a tile
constexpr int kPairHalf = 128 * 128;                        // bytes of a CTA's half of one operand in a stage
constexpr int kPairBytesS = 3 * 2 * kMxAtom;                // scales: its own 128 rows of A, all 256 of B
constexpr int kPairStage = 2 * kPairHalf + kPairBytesS;
constexpr int kPairStages = 6;
constexpr int kPairSmem = 1024 + kPairStages * kPairStage;
constexpr int kPairScaleCol = 256;                          // tensor memory: accumulators, then two sets of scales of 24 columns
static_assert(kPairStage % 1024 == 0 && kPairSmem <= kMmSmem - 1024, "stages do not fit");

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

__device__ __forceinline__ void pair_arrive(unsigned int bar) {       // an address of the cluster
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
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

// 32 columns, without waiting for them.
__device__ __forceinline__ void pair_load32(unsigned int tmem, float* v) {
  unsigned int* u = reinterpret_cast<unsigned int*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
        "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]),
        "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]),
        "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(tmem));
}

// A thread's 256 bits: one whole sector.
__device__ __forceinline__ void store256(void* p, const unsigned int (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// 32 accumulators of row m, columns n..n+31.
__device__ __forceinline__ void pair_store(const MmArgs& a, long long m, long long n, const float* v) {
  if (m >= a.rows_p) return;
  if (a.vec_ok > 1 && n + 32 <= a.rows_q) {
    unsigned int w[8];
    if (a.out_f32) {
      float* o = static_cast<float*>(a.c) + (size_t)m * (size_t)a.ldc + (size_t)n;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] = __float_as_uint(v[8 * i + q]);
        store256(o + 8 * i, w);
      }
    } else {
      unsigned short* o = static_cast<unsigned short*>(a.c) + (size_t)m * (size_t)a.ldc + (size_t)n;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] = mm_bf16x2(v[16 * i + 2 * q], v[16 * i + 2 * q + 1]);
        store256(o + 16 * i, w);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; i += 4)
      if (n + i < a.rows_q) mm_store4(a, m, n + i, a.rows_q, make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]));
  }
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
ps_mx_matmul_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                         const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb,
                         const __grid_constant__ MmArgs args) {
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) unsigned long long s_full[kPairStages], s_empty[kPairStages], s_acc_full, s_acc_empty;
  __shared__ unsigned int s_tmem;
  unsigned char* stages = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const unsigned int base = mm_smem(stages);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  unsigned int rank;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));

  if (tid == 0) {
    for (int s = 0; s < kPairStages; ++s) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 2;" ::"r"(mm_smem(&s_full[s])) : "memory");     // the leader's two producers
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&s_empty[s])) : "memory");
    }
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&s_acc_full)) : "memory");
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 16;" ::"r"(mm_smem(&s_acc_empty)) : "memory");    // 8 warps of each
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_sa) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_sb) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(mm_smem(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  mm_cluster_sync();                                      // both CTAs' barriers and tensor memory exist
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const unsigned int tmem = s_tmem;
  mx_pdl();

  const int tiles = args.tiles_p * args.tiles_q, stride = (int)(gridDim.x / 2);
  const int first = (int)(blockIdx.x / 2), nk = args.stages_k;

  if (warp == 0 || warp == 10) {
    if (mm_elect()) {
      MmCursor<kPairStages> at;
      const unsigned int full = pair_leader(mm_smem(&s_full[0]));
      unsigned int issued = 0;
      bool ok = true;
      for (int tile = first; ok && tile < tiles; tile += stride) {
        int tp, tq;
        mm_tile(args, tile, &tp, &tq);
        // the leader's producers arm its barrier with the bytes of both CTAs; the bytes themselves may come first
        if (warp == 0) {
          const int row_a = tp * kPairTile + (int)rank * 128, row_b = tq * kPairTile + (int)rank * 128;
          for (int k = 0; k < nk; ++k, at.next(), ++issued) {
            if (!mm_wait(mm_smem(&s_empty[0]) + 8 * at.s, at.parity ^ 1u, args.status)) { ok = false; break; }
            const unsigned int dst = base + at.s * kPairStage, bar = full + 8 * at.s;
            if (rank == 0)
              asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(mm_smem(&s_full[0]) + 8 * at.s),
                           "n"(4 * kPairHalf)
                           : "memory");
            pair_tma(dst, &map_a, k * 128, row_a, bar);
            pair_tma(dst + kPairHalf, &map_b, k * 128, row_b, bar);
          }
        } else {
          // atoms of scales: 128-row block times atoms per block, two per stage (blocks that do not exist read as zeros)
          const int at_a = (int)((tp * 2 + (int)rank) * args.atoms), at_b = (int)(tq * 2 * args.atoms);
          for (int k = 0; k < nk; ++k, at.next(), ++issued) {
            if (!mm_wait(mm_smem(&s_empty[0]) + 8 * at.s, at.parity ^ 1u, args.status)) { ok = false; break; }
            const unsigned int dst = base + at.s * kPairStage + 2 * kPairHalf, bar = full + 8 * at.s;
            if (rank == 0)
              asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(mm_smem(&s_full[0]) + 8 * at.s),
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
          mm_wait(mm_smem(&s_full[s]), ((issued - 1 - s) / kPairStages) & 1u, args.status);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0 && mm_elect()) {
      MmCursor<kPairStages> at;
      constexpr unsigned int kIdesc = (1u << 7) | (1u << 10) | ((unsigned)(kPairTile >> 3) << 17) | (1u << 23) | (16u << 24);
      unsigned int set = 0, acc_parity = 1;
      bool ok = true;
      for (int tile = first; ok && tile < tiles; tile += stride, acc_parity ^= 1u) {
        if (!pair_wait(mm_smem(&s_acc_empty), acc_parity, args.status)) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (int k = 0; k < nk; ++k, at.next(), set ^= 32u) {
          if (!pair_wait(mm_smem(&s_full[0]) + 8 * at.s, at.parity, args.status)) { ok = false; break; }
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
          pair_commit(mm_smem(&s_empty[0]) + 8 * at.s);
        }
        pair_commit(mm_smem(&s_acc_full));
      }
    }
    __syncwarp();
  } else {
    const int quad = warp & 3, half = (warp - 2) >> 2;
    const unsigned int empty = pair_leader(mm_smem(&s_acc_empty));
    const unsigned int acc = tmem + ((unsigned)(quad * 32) << 16) + half * 128;
    unsigned int n = 0;
    for (int tile = first; tile < tiles; tile += stride, ++n) {
      if (!__all_sync(0xffffffffu, mm_wait(mm_smem(&s_acc_full), n & 1u, args.status))) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      float v[128];
#pragma unroll
      for (int c = 0; c < 4; ++c) pair_load32(acc + c * 32, v + c * 32);
      asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) pair_arrive(empty);
      int tp, tq;
      mm_tile(args, tile, &tp, &tq);
      const long long m = (long long)tp * kPairTile + rank * 128 + quad * 32 + lane;
      const long long q = (long long)tq * kPairTile + half * 128;
#pragma unroll
      for (int c = 0; c < 4; ++c) pair_store(args, m, q + c * 32, v + c * 32);
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
