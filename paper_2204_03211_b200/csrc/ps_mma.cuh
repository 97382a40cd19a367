// What the tensor-core kernels share: elected lanes, bounded waits on mbarriers, tensor-map copies, commits,
// descriptors, reads of tensor memory, and the forms of them for a pair of CTAs on two SMs (cta_group::2).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace psb {

// The stream's next launch may start its prologue; this one waits until the launches before it have completed.
__device__ __forceinline__ void mm_pdl() {
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

__device__ __forceinline__ void store_sector(void* p, const unsigned int* w) {       // 32 bytes, written once
  asm volatile("st.global.cs.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

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

// Shared memory descriptor: rows of 128 bytes in 128-byte swizzle (8-row groups 1024 bytes apart).
__device__ __forceinline__ unsigned long long mm_desc_codes(unsigned int addr) {
  return (unsigned long long)((addr & 0x3ffffu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}

// Instructions that are `.aligned` want all lanes of the warp at once.  What comes before them here are waits in which each
// lane spins by itself and branches that some lanes take: mm_load, mm_store16 and mm_cluster_sync bring the lanes together
// first.

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
__device__ __forceinline__ void mm_store16(unsigned int tmem, const float* v) {      // without waiting
  const unsigned int* u = reinterpret_cast<const unsigned int*>(v);
  __syncwarp();
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(tmem),
      "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
      "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15])
      : "memory");
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
  __syncwarp();
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

__device__ __forceinline__ void mm_cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

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

}  // namespace psb
