// Product of two microscaled 4-bit operands on the 5th-generation tensor cores:
//     C[m][n] = sum_k A[m][k] * B[n][k],   fp32 accumulation, fp32 or bf16 result.
//
// tcgen05.mma of kind mxf4 takes E2M1 operands from shared memory and one E8M0
// scale per 32 elements of either from tensor memory.  A CTA computes tiles of
// 128 rows of one operand ("P") by BN rows of the other ("Q"), 256 elements of K
// per pipeline stage: a stage is 128 and BN rows of 128 bytes (TMA, 128-byte
// swizzle) and their atoms of scales (plain bulk copies; the quantiser stores
// them in the order in which scale memory takes them).
//   warp 0     one lane issues the copies of codes
//   warp 1     one lane copies the scales to tensor memory and issues the MMAs
//   warps 2-5  read the accumulators and store the result
//   warp 6     one lane issues the copies of scales
// A stage is 512 cycles of MMA at most, and what a single lane issues for it is of
// that order (a ready barrier alone costs about 100): the lanes are elected, which
// lets their operands live in uniform registers, addresses advance by addition, and
// the copies are spread over two warps.
// Where one operand has few rows (single tokens) it is Q and the other, usually
// the weight, P, whichever of A and B that is: the MMA's 128 rows are then full
// and what is left is reading P once.  Such a product has few tiles, so the CTAs
// of a cluster share a tile's K and add their parts in rank order through
// distributed shared memory: no workspace, no atomics, the same result each time.
//
// Measured, the weight in L2 | weights of 300 MB in rotation, calls in a row: 1 x 4096 x 1024
// 3.3 | 3.9 us, 8 x 4096 x 4096 5.5 | 6.4, 37 x 30522 x 1024 5.9 | 6.7 (10 us alone with cold
// caches), 16 x 8192 x 8192 7.4 | 10.3, 1 x 28672 x 8192 21.7 | 23.8 (5.2 TB/s of the weight);
// 1000 x 256 x 300 3.8 us.  What is left of the shorter ones is latency: launch, the first
// copy, the MMAs of one tile, its store.
#pragma once

#include <cuda.h>

#include "ps_mx.cuh"

namespace psb {

constexpr int kMmThreads = 224;
constexpr int kMmP = 128;                       // rows of P in a tile
constexpr int kMmStageK = 256;                  // elements of K in a stage: 128 bytes of codes, 2 atoms of scales
constexpr int kMmMaxStages = 8;
constexpr int kMmSmem = 227 * 1024;
constexpr int kMmStaging = 2048;                // bytes of an epilogue warp's staging for stores

struct MmControl {
  unsigned long long full[kMmMaxStages], empty[kMmMaxStages], acc_full[2], acc_empty[2];
  unsigned int tmem;
};
constexpr int kMmControl = 256;
static_assert(sizeof(MmControl) <= kMmControl, "control block");

template <int BN>
struct MmCfg {
  static constexpr int kBytesP = kMmP * 128, kBytesQ = BN * 128;
  static constexpr int kBytesS = 2 * kMxAtom;                   // scales of one 128-row block in a stage
  static constexpr int kStage = kBytesP + kBytesQ + 2 * kBytesS;
  // Q of up to 64 rows: two CTAs share an SM, so that more tiles of P are on their way at once
  static constexpr int kCtas = BN <= 64 ? 2 : 1;
  static constexpr int kFit = ((kMmSmem + 1024) / kCtas - 1024 - kMmControl - 4 * kMmStaging) / kStage;
  static constexpr int kStages = kFit < kMmMaxStages ? kFit : kMmMaxStages;
  static constexpr int kAcc = 2;                                // accumulators: the second hides the epilogue
  static constexpr int kScaleCol = kAcc * BN;                   // tensor memory: accumulators, then two sets of scales
  static constexpr int kScaleSet = 16;
  static constexpr int kCols = kScaleCol + 2 * kScaleSet;
  static constexpr int kAlloc = kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
  static_assert(BN <= 128, "one block of scales per operand");
  static constexpr int kSmem = kStages * kStage + 4 * kMmStaging + kMmControl;
  static_assert(kStages >= 3 && kCols <= 512 && kStage % 1024 == 0, "tile does not fit");
};

struct MmArgs {
  const uint8_t* sp;                            // scales of P and Q
  const uint8_t* sq;
  void* c;
  long long ldc;
  long long rows_p, rows_q;
  long long atoms;                              // atoms of scales per 128 rows
  int stages_k;                                 // stages along K
  int tiles_p, tiles_q;
  int splits;                                   // CTAs (one cluster) per tile
  int swap;                                     // 1: P is B, so a lane's row is a column of C
  int out_f32;
  int vec_ok;                                   // rows of C allow 128-bit stores
  int* status;
};

constexpr long long kMmWaitCycles = 2000000000ll;     // about a second

__device__ __forceinline__ unsigned int mm_smem(const void* p) {
  return static_cast<unsigned int>(__cvta_generic_to_shared(p));
}

// One lane of the (converged) warp; the compiler knows that it is one.
__device__ __forceinline__ bool mm_elect() {
  unsigned int p;
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "}"
      : "=r"(p));
  return p != 0;
}

__device__ __forceinline__ bool mm_try_wait(unsigned int bar, unsigned int parity) {
  unsigned int ok;
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

// Bounded wait: false if the limit ran out (the status word then says so and the launch's results are undefined).
__device__ __forceinline__ bool mm_wait(unsigned int bar, unsigned int parity, int* status) {
  if (mm_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mm_try_wait(bar, parity)) {
    if (clock64() - t0 > kMmWaitCycles) {
      atomicExch(status, 1);
      return false;
    }
  }
  return true;
}

__device__ __forceinline__ void mm_tma(unsigned int dst, const CUtensorMap* map, int x, int y, unsigned int bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}

__device__ __forceinline__ void mm_bulk(unsigned int dst, const void* src, unsigned int bytes, unsigned int bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

__device__ __forceinline__ void mm_commit(unsigned int bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// The stage that comes next, and the parity of its barriers.
template <int STAGES>
struct MmCursor {
  unsigned int s = 0, parity = 0;
  __device__ __forceinline__ void next() {
    if (++s == STAGES) { s = 0; parity ^= 1u; }
  }
};

// Shared memory descriptors: rows of 128 bytes in 128-byte swizzle (8-row groups 1024 bytes apart), and an atom of
// scales, 32 rows of 16 bytes (8-row groups 128 bytes apart, no swizzle).
__device__ __forceinline__ unsigned long long mm_desc_codes(unsigned int addr) {
  return (unsigned long long)((addr & 0x3ffffu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ unsigned long long mm_desc_scales(unsigned int addr) {
  return (unsigned long long)((addr & 0x3ffffu) >> 4) | (1ull << 16) | (8ull << 32) | (1ull << 46);
}

__device__ __forceinline__ void mm_copy_scales(unsigned int tmem, unsigned long long desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}

__device__ __forceinline__ void mm_mma(unsigned int d, unsigned long long a, unsigned long long b, unsigned int idesc,
                                       unsigned int sa, unsigned int sb, bool accumulate) {
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "setp.ne.u32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t"
      "}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((unsigned int)accumulate)
      : "memory");
}

// 32 or 16 columns of this warp's 32 lanes, without waiting for them.
__device__ __forceinline__ void mm_load32(unsigned int tmem, float* v) {
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
__device__ __forceinline__ void mm_load16(unsigned int tmem, float* v) {
  unsigned int* u = reinterpret_cast<unsigned int*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
        "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(tmem));
}
template <int N>
__device__ __forceinline__ void mm_load(unsigned int tmem, float (&v)[N]) {
  if constexpr (N == 16) {
    mm_load16(tmem, v);
  } else {
#pragma unroll
    for (int c = 0; c < N; c += 32) mm_load32(tmem + c, v + c);
  }
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ unsigned int mm_bf16x2(float lo, float hi) {
  unsigned int r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ void mm_store1(const MmArgs& a, long long m, long long n, float v) {
  const size_t at = (size_t)m * (size_t)a.ldc + (size_t)n;
  if (a.out_f32) static_cast<float*>(a.c)[at] = v;
  else static_cast<unsigned short*>(a.c)[at] = (unsigned short)mm_bf16x2(v, 0.f);
}

// A warp's 32 rows (m0.. of C) of COLS columns (n..), row `lane` in this lane's v, through 2 KB of shared memory, 16 rows
// at a time: rows of up to 128 bytes in 16-byte pieces, permuted by the row so that neither side meets in a bank.
// Stored straight from the registers, a warp's store touches 32 lines, and that was what products of short K waited for
// (8192 x 4096 x 1024: 22.7 us, and 56 us where C's rows allow no wide stores, against 19.1 us).
template <int COLS, bool F32>
__device__ __forceinline__ void mm_store_rows_as(const MmArgs& a, unsigned char* buf, int lane, long long m0, long long n,
                                                 long long rows, long long cols, const float* v) {
  constexpr int kEs = F32 ? 4 : 2, kRow = COLS * kEs, kPieces = kRow / 16, kStep = 32 / kPieces;
  static_assert(kRow <= 128 && 16 * kRow <= kMmStaging && (kPieces & (kPieces - 1)) == 0, "staging row");
  const int live = (int)min(32ll, rows - m0);                 // rows of the warp inside C
  const int live_cols = (int)min((long long)COLS, cols - n);
  const bool wide = a.vec_ok && live_cols == COLS;
  const int each = lane / kPieces, piece = lane % kPieces;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r0 = h * 16;
    if ((lane >> 4) == h) {
      uint4* mine = reinterpret_cast<uint4*>(buf + (lane & 15) * kRow);
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        if constexpr (F32)
          mine[i ^ (lane & (kPieces - 1))] = make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                                                        __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
        else
          mine[i ^ (lane & (kPieces - 1))] =
              make_uint4(mm_bf16x2(v[8 * i], v[8 * i + 1]), mm_bf16x2(v[8 * i + 2], v[8 * i + 3]),
                         mm_bf16x2(v[8 * i + 4], v[8 * i + 5]), mm_bf16x2(v[8 * i + 6], v[8 * i + 7]));
      }
    }
    __syncwarp();
    if (wide) {
      unsigned char* o = static_cast<unsigned char*>(a.c) + ((size_t)(m0 + r0 + each) * (size_t)a.ldc + (size_t)n) * kEs + piece * 16;
#pragma unroll
      for (int r = 0; r < 16; r += kStep) {
        const int row = r + each;
        const uint4 q = *reinterpret_cast<const uint4*>(buf + row * kRow + ((piece ^ (row & (kPieces - 1))) << 4));
        if (r0 + row < live) *reinterpret_cast<uint4*>(o + (size_t)r * (size_t)a.ldc * kEs) = q;
      }
    } else {
#pragma unroll 4
      for (int r = 0; r < 16; ++r) {
        const size_t at = (size_t)(m0 + r0 + r) * (size_t)a.ldc + (size_t)n;
#pragma unroll
        for (int c0 = 0; c0 < COLS; c0 += 32) {
          const int c = c0 + lane;
          if (r0 + r < live && c < live_cols) {
            const unsigned char* e = buf + r * kRow + ((((c * kEs) >> 4) ^ (r & (kPieces - 1))) << 4) + ((c * kEs) & 15);
            if constexpr (F32) static_cast<float*>(a.c)[at + c] = *reinterpret_cast<const float*>(e);
            else static_cast<unsigned short*>(a.c)[at + c] = *reinterpret_cast<const unsigned short*>(e);
          }
        }
      }
    }
    __syncwarp();
  }
}

// N accumulators (a multiple of 32, or 16) per lane.
template <int N>
__device__ __forceinline__ void mm_store_rows(const MmArgs& a, unsigned char* buf, int lane, long long m0, long long n,
                                              long long rows, long long cols, const float* v) {
  if (m0 >= rows) return;
  if (a.out_f32) {
    constexpr int kCols = N < 32 ? N : 32;
#pragma unroll
    for (int c = 0; c < N; c += kCols)
      if (n + c < cols) mm_store_rows_as<kCols, true>(a, buf, lane, m0, n + c, rows, cols, v + c);
  } else {
    constexpr int kCols = N < 64 ? N : 64;
#pragma unroll
    for (int c = 0; c < N; c += kCols)
      if (n + c < cols) mm_store_rows_as<kCols, false>(a, buf, lane, m0, n + c, rows, cols, v + c);
  }
}

// Stores N consecutive accumulators (rows q.. of Q) of this lane's row p of P, where P is B: the warp's lanes are
// neighbours in C.
template <int N>
__device__ __forceinline__ void mm_store_swapped(const MmArgs& a, long long p, long long q, const float (&v)[N]) {
  if (p >= a.rows_p) return;
  const int live = (int)min((long long)N, a.rows_q - q);
  const size_t at = (size_t)q * (size_t)a.ldc + (size_t)p;
  if (a.out_f32) {
    float* o = static_cast<float*>(a.c) + at;
#pragma unroll
    for (int i = 0; i < N; ++i, o += a.ldc)
      if (i < live) *o = v[i];
  } else {
    unsigned short* o = static_cast<unsigned short*>(a.c) + at;
#pragma unroll
    for (int i = 0; i < N; ++i, o += a.ldc)
      if (i < live) *o = (unsigned short)mm_bf16x2(v[i], 0.f);
  }
}

// Tiles are walked in groups of 16 along P, so that the tiles in flight share rows of both operands in L2.
__device__ __forceinline__ void mm_tile(const MmArgs& a, int tile, int* tp, int* tq) {
  constexpr int kGroup = 16;
  const int per = kGroup * a.tiles_q, g = tile / per, in = tile - g * per;
  const int n = min(kGroup, a.tiles_p - g * kGroup);
  *tq = in / n;
  *tp = g * kGroup + in - *tq * n;
}

__device__ __forceinline__ void mm_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Four floats at `addr` of this CTA's layout, from the cluster's CTA `rank`.  (volatile: not to be moved across the
// cluster barriers)
__device__ __forceinline__ float4 mm_remote4(unsigned int addr, unsigned int rank) {
  float4 v;
  asm volatile("{\n\t"
      ".reg .b32 r;\n\t"
      "mapa.shared::cluster.u32 r, %4, %5;\n\t"
      "ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [r];\n\t"
      "}"
      : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
      : "r"(addr), "r"(rank));
  return v;
}

// The sum over the cluster's parts in rank order: all loads are in flight together.
template <int S>
__device__ __forceinline__ float4 mm_sum_parts(unsigned int addr) {
  float4 t[S];
#pragma unroll
  for (int r = 0; r < S; ++r) t[r] = mm_remote4(addr, (unsigned)r);
#pragma unroll
  for (int r = 1; r < S; ++r) {
    t[0].x = __fadd_rn(t[0].x, t[r].x);
    t[0].y = __fadd_rn(t[0].y, t[r].y);
    t[0].z = __fadd_rn(t[0].z, t[r].z);
    t[0].w = __fadd_rn(t[0].w, t[r].w);
  }
  return t[0];
}

// Stores four neighbours of C's row m, columns n..n+3 (n < limit).
__device__ __forceinline__ void mm_store4(const MmArgs& a, long long m, long long n, long long limit, float4 v) {
  if (a.vec_ok && n + 4 <= limit) {
    const size_t at = (size_t)m * (size_t)a.ldc + (size_t)n;
    if (a.out_f32) *reinterpret_cast<float4*>(static_cast<float*>(a.c) + at) = v;
    else *reinterpret_cast<uint2*>(static_cast<unsigned short*>(a.c) + at) = make_uint2(mm_bf16x2(v.x, v.y), mm_bf16x2(v.z, v.w));
  } else {
    mm_store1(a, m, n, v.x);
    if (n + 1 < limit) mm_store1(a, m, n + 1, v.y);
    if (n + 2 < limit) mm_store1(a, m, n + 2, v.z);
    if (n + 3 < limit) mm_store1(a, m, n + 3, v.w);
  }
}

template <int BN>
__global__ void __launch_bounds__(kMmThreads, MmCfg<BN>::kCtas)
ps_mx_matmul_kernel(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_q,
                    const __grid_constant__ MmArgs args) {
  using Cfg = MmCfg<BN>;
  // (no static shared memory beside it: the stages start where the swizzle needs them to, at a multiple of 1024)
  extern __shared__ __align__(1024) unsigned char stages[];
  MmControl& ctl = *reinterpret_cast<MmControl*>(stages + Cfg::kStages * Cfg::kStage + 4 * kMmStaging);
  const unsigned int base = mm_smem(stages);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

  if (tid == 0) {
    for (int s = 0; s < Cfg::kStages; ++s) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 2;" ::"r"(mm_smem(&ctl.full[s])) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.empty[s])) : "memory");
    }
    for (int b = 0; b < Cfg::kAcc; ++b) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.acc_full[b])) : "memory");
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 4;" ::"r"(mm_smem(&ctl.acc_empty[b])) : "memory");
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_p) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(mm_smem(&ctl.tmem)),
                 "r"(Cfg::kAlloc)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const unsigned int tmem = ctl.tmem;
  mx_pdl();

  const int tiles = args.tiles_p * args.tiles_q;
  const int rank = args.splits > 1 ? (int)(blockIdx.x % (unsigned)args.splits) : 0;
  const int first = args.splits > 1 ? (int)(blockIdx.x / (unsigned)args.splits) : (int)blockIdx.x;
  const int stride = args.splits > 1 ? tiles : (int)gridDim.x;      // a cluster computes one tile
  const int k0 = (int)((long long)args.stages_k * rank / args.splits);
  const int k1 = (int)((long long)args.stages_k * (rank + 1) / args.splits);

  if (warp == 0 || warp == 6) {
    // the two producers wait for a stage, arm its barrier with their own bytes and issue their copies
    if (mm_elect()) {
      MmCursor<Cfg::kStages> at;
      unsigned int issued = 0;
      bool ok = true;
      for (int tile = first; ok && tile < tiles; tile += stride) {
        int tp, tq;
        mm_tile(args, tile, &tp, &tq);
        if (warp == 0) {
          for (int k = k0; k < k1; ++k, at.next(), ++issued) {
            if (!mm_wait(mm_smem(&ctl.empty[0]) + 8 * at.s, at.parity ^ 1u, args.status)) { ok = false; break; }
            const unsigned int bar = mm_smem(&ctl.full[0]) + 8 * at.s, dst = base + at.s * Cfg::kStage;
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "n"(Cfg::kBytesP + Cfg::kBytesQ)
                         : "memory");
            mm_tma(dst, &map_p, k * 128, tp * kMmP, bar);
            mm_tma(dst + Cfg::kBytesP, &map_q, k * 128, tq * BN, bar);
          }
        } else {
          const uint8_t* sp = args.sp + ((size_t)tp * (size_t)args.atoms + 2 * (size_t)k0) * kMxAtom;
          const uint8_t* sq = args.sq + ((size_t)(tq * BN / 128) * (size_t)args.atoms + 2 * (size_t)k0) * kMxAtom;
          for (int k = k0; k < k1; ++k, at.next(), ++issued, sp += Cfg::kBytesS, sq += Cfg::kBytesS) {
            if (!mm_wait(mm_smem(&ctl.empty[0]) + 8 * at.s, at.parity ^ 1u, args.status)) { ok = false; break; }
            const unsigned int bar = mm_smem(&ctl.full[0]) + 8 * at.s;
            const unsigned int dst = base + at.s * Cfg::kStage + Cfg::kBytesP + Cfg::kBytesQ;
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "n"(2 * Cfg::kBytesS) : "memory");
            mm_bulk(dst, sp, Cfg::kBytesS, bar);
            mm_bulk(dst + Cfg::kBytesS, sq, Cfg::kBytesS, bar);
          }
        }
      }
      if (!ok)                                        // an expired wait: let the copies in flight land
        for (unsigned int s = 0; s < (unsigned)Cfg::kStages && s < issued; ++s)
          mm_wait(mm_smem(&ctl.full[s]), ((issued - 1 - s) / Cfg::kStages) & 1u, args.status);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (mm_elect()) {
      constexpr unsigned int kIdesc = (1u << 7) | (1u << 10) | ((unsigned)(BN >> 3) << 17) | (1u << 23) | (8u << 24);
      MmCursor<Cfg::kStages> at;
      MmCursor<Cfg::kAcc> acc;
      unsigned int set = 0;
      bool ok = true;
      for (int tile = first; ok && tile < tiles; tile += stride, acc.next()) {
        if (!mm_wait(mm_smem(&ctl.acc_empty[0]) + 8 * acc.s, acc.parity ^ 1u, args.status)) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const unsigned int d = tmem + acc.s * BN;
        int tile_p, tile_q;
        mm_tile(args, tile, &tile_p, &tile_q);
        const unsigned int sub = (unsigned)(tile_q * BN % 128) / 32;       // where the tile's rows start in their block of scales
        for (int k = k0; k < k1; ++k, at.next(), set ^= Cfg::kScaleSet) {
          if (!mm_wait(mm_smem(&ctl.full[0]) + 8 * at.s, at.parity, args.status)) { ok = false; break; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const unsigned long long dp = mm_desc_codes(base + at.s * Cfg::kStage);
          const unsigned long long ds = mm_desc_scales(base + at.s * Cfg::kStage + Cfg::kBytesP + Cfg::kBytesQ);
          const unsigned int tp = tmem + Cfg::kScaleCol + set, tq = tp + 8;
          // scales: atom j of P and of Q, four columns each (a descriptor counts in 16 bytes)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            mm_copy_scales(tp + j * 4, ds + j * (kMxAtom / 16));
            mm_copy_scales(tq + j * 4, ds + (Cfg::kBytesS + j * kMxAtom) / 16);
          }
          // four MMAs of 64 elements (32 bytes) each; an atom serves two, which name its lower or upper pair of scales
#pragma unroll
          for (int i = 0; i < 4; ++i)
            mm_mma(d, dp + 2 * i, dp + Cfg::kBytesP / 16 + 2 * i, kIdesc | ((unsigned)(i & 1) << 30) | ((unsigned)(i & 1) << 5),
                   tp + (i >> 1) * 4, tq + (i >> 1) * 4 + sub, k > k0 || i > 0);
          mm_commit(mm_smem(&ctl.empty[0]) + 8 * at.s);
        }
        mm_commit(mm_smem(&ctl.acc_full[0]) + 8 * acc.s);
      }
    }
    __syncwarp();
  } else {
    unsigned char* staging = stages + Cfg::kStages * Cfg::kStage + (warp - 2) * kMmStaging;
    const int quad = warp & 3;                        // the quarter of tensor memory's lanes this warp may read
    unsigned int n = 0;
    for (int tile = first; tile < tiles; tile += stride, ++n) {
      const unsigned int buf = n % Cfg::kAcc;
      if (!__all_sync(0xffffffffu, mm_wait(mm_smem(&ctl.acc_full[buf]), (n / Cfg::kAcc) & 1u, args.status))) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      int tp, tq;
      mm_tile(args, tile, &tp, &tq);
      const int row = quad * 32 + lane;
      const unsigned int acc = tmem + ((unsigned)(quad * 32) << 16) + buf * BN;
      constexpr int kStep = BN < 64 ? BN : 64;
#pragma unroll 1
      for (int c = 0; c < BN; c += kStep) {
        float v[kStep];
        mm_load<kStep>(acc + c, v);
        if (args.splits > 1) {
          // this CTA's part goes to its shared memory (the stages are no longer in use), in an order in which neither
          // these stores nor the reads below meet in a bank
          float* red = reinterpret_cast<float*>(stages);
#pragma unroll
          for (int i = 0; i < kStep; i += 4) {
            if (args.swap) {
#pragma unroll
              for (int q = 0; q < 4; ++q) red[(c + i + q) * kMmP + row] = v[i + q];
            } else {
              *reinterpret_cast<float4*>(red + row * (BN + 4) + c + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
            }
          }
        } else if (args.swap) {
          mm_store_swapped<kStep>(args, (long long)tp * kMmP + row, (long long)tq * BN + c, v);
        } else {
          mm_store_rows<kStep>(args, staging, lane, (long long)tp * kMmP + quad * 32, (long long)tq * BN + c, args.rows_p,
                               args.rows_q, v);
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0)
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(mm_smem(&ctl.acc_empty[buf])) : "memory");
    }
    __syncwarp();
  }

  if (args.splits > 1) {
    mm_cluster_sync();
    int tp, tq;
    mm_tile(args, first, &tp, &tq);
    // groups of four neighbours in C; every CTA takes an equal share of them
    const int total = kMmP * BN / 4, e0 = (int)((long long)total * rank / args.splits);
    const int e1 = (int)((long long)total * (rank + 1) / args.splits);
    for (int e = e0 + tid; e < e1; e += kMmThreads) {
      const int row = args.swap ? e % (kMmP / 4) * 4 : e / (BN / 4), col = args.swap ? e / (kMmP / 4) : e % (BN / 4) * 4;
      const long long p = (long long)tp * kMmP + row, q = (long long)tq * BN + col;
      if (p >= args.rows_p || q >= args.rows_q) continue;
      const unsigned int at = base + 4u * (unsigned)(args.swap ? col * kMmP + row : row * (BN + 4) + col);
      const float4 v = args.splits == 8 ? mm_sum_parts<8>(at) : args.splits == 4 ? mm_sum_parts<4>(at) : mm_sum_parts<2>(at);
      if (args.swap) mm_store4(args, q, p, args.rows_p, v);
      else mm_store4(args, p, q, args.rows_q, v);
    }
    mm_cluster_sync();                                // nobody leaves while its shared memory is being read
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(Cfg::kAlloc) : "memory");
}

}  // namespace psb
