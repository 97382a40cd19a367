// A barrier over all CTAs of a cooperative launch, and the clipping factor.
#pragma once

#include <cuda_runtime.h>

namespace psb {

struct GridBarrier {                     // device memory, zero before the first launch that uses it
  unsigned int count, generation;
};

constexpr long long kGridWaitCycles = 4000000000ll;     // about two seconds

// Every thread of every CTA calls this.  False (in all threads of the CTA) if the other CTAs did not arrive within
// `limit` cycles; the launch is cooperative, so they are resident and do arrive.  The last CTA to arrive clears the
// count, calls `last` (one thread) and advances the generation, so launches of different sizes can use one barrier
// after the other.  It is the one CTA that never waits: what the next launch has to find in order is put in order
// there, whoever gave up waiting.
template <typename F>
__device__ __forceinline__ bool grid_barrier(GridBarrier* b, long long limit, F last) {
  __shared__ int s_ok;
  __syncthreads();
  if (threadIdx.x == 0) {
    bool ok = true;
    const unsigned int mine = *reinterpret_cast<volatile unsigned int*>(&b->generation);
    __threadfence();
    if (atomicAdd(&b->count, 1u) == gridDim.x - 1) {
      b->count = 0;
      last();
      __threadfence();
      atomicAdd(&b->generation, 1u);
    } else {
      const long long t0 = clock64();
      while (*reinterpret_cast<volatile unsigned int*>(&b->generation) == mine) {
        if (clock64() - t0 > limit) { ok = false; break; }
      }
    }
    __threadfence();
    s_ok = ok;
  }
  __syncthreads();
  return s_ok != 0;
}

// min(1, max_norm / (norm + 1e-6)): a NaN norm gives a NaN factor, an infinite one zero; an infinite max_norm
// asks for the norm alone.
__device__ __forceinline__ float clip_factor(float norm, float max_norm) {
  if (max_norm == __int_as_float(0x7f800000)) return 1.0f;
  const float f = __fdiv_rn(max_norm, __fadd_rn(norm, 1e-6f));
  return f >= 1.0f ? 1.0f : f;
}

}  // namespace psb
