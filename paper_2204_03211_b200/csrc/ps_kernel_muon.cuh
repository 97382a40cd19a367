// The first launch of a PS_MUON aggregate: per element
//     G = grad_scale * (g_0 + ... + g_{W-1})      (the shared chunk bodies: binary32, worker order)
//     v = momentum v + G,   u = G + momentum v
// with v in place and u in a buffer, from which the orthogonalisation (ps_ortho.cuh) makes the update.  A chunk's sums
// go through that buffer: the second walk over the chunk finds them in L1 and L2.  Bound by memory: W shards and v are
// read once, v and u written: six layers 512 wide (18.9 M elements) with eight workers in 141 us, 5.9 TB/s.
// Every chunk publishes its sums of squares, of G for the block's statistics and of u for
// the norm, both in binary64 and added up in a fixed order later.
#pragma once

#include "ps_kernel_ldg.cuh"

namespace psb {

template <bool BF16>
__device__ __noinline__ double muon_sum(unsigned int tid, const void* const* shards, int W, float gs, float* u, size_t begin,
                                        unsigned int count, bool vec_ok) {
  Hp h;
  h.gs = gs;
  double sq = 0.0;
  run_chunk<kSumOnly, BF16, kThreads>(tid, h, shards, W, u, nullptr, nullptr, begin, count, vec_ok, sq);
  return sq;
}

// (T->p is the block's place in the buffer)
__global__ void __launch_bounds__(kThreads, 4)
ps_aggregate_muon_kernel(unsigned char* __restrict__ table, const PsJobDev* __restrict__ jobs, PsStat* __restrict__ stats,
                         double* __restrict__ partials, double* __restrict__ u_partials) {
  PsTableHdr* hdr = reinterpret_cast<PsTableHdr*>(table);
  PsTaskDev* tasks = reinterpret_cast<PsTaskDev*>(table + hdr->tasks_off);
  const unsigned int* starts = reinterpret_cast<const unsigned int*>(table + hdr->starts_off);
  const void* const* ptrs = reinterpret_cast<const void* const*>(table + hdr->ptrs_off);
  const unsigned int n_tasks = hdr->n_tasks, total = hdr->total_chunks;
  const bool profile = hdr->profile != 0;
  __shared__ unsigned int s_idx[2];
  __shared__ unsigned int s_task;
  __shared__ double s_red[2][kThreads / 32];
  const unsigned int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  unsigned int cursor = 0;   // meaningful in warp 0
  int buf = 0;
  if (tid == 0) s_idx[0] = atomicAdd(&hdr->counter, 1u);
  __syncthreads();

  while (true) {
    const unsigned int idx = s_idx[buf];
    if (idx >= total) break;
    if (warp == 0) {
      cursor = find_task(starts, n_tasks, cursor, idx, lane);
      if (lane == 0) s_task = cursor;
    } else if (tid == kThreads - 1) {
      s_idx[buf ^ 1] = atomicAdd(&hdr->counter, 1u);   // the next claim overlaps this chunk
    }
    __syncthreads();

    const unsigned long long t_begin = (profile && tid == 0) ? global_ns() : 0ull;
    const unsigned int t = s_task;
    const PsTaskDev* T = tasks + t;
    const PsJobDev* J = jobs + T->job;
    const size_t begin = (size_t)(idx - T->first_chunk) * T->chunk_elems;
    const unsigned int count = (unsigned int)min((unsigned long long)T->chunk_elems, T->nelem - begin);
    const void* const* shards = ptrs + T->shard_row;
    double sq = J->grad_dtype ? muon_sum<true>(tid, shards, J->W, J->gs, T->p, begin, count, T->vec_ok != 0)
                              : muon_sum<false>(tid, shards, J->W, J->gs, T->p, begin, count, T->vec_ok != 0);
    __syncthreads();                           // the chunk's sums are there
    float *u = T->p + begin, *v = T->s0 + begin;
    const float mom = J->mom;
    double usq = 0.0;
    auto element = [&](float& g, float& m) {
      m = __fadd_rn(__fmul_rn(mom, m), g);
      g = __fadd_rn(g, __fmul_rn(mom, m));
      usq = fma((double)g, (double)g, usq);
    };
    const unsigned int nvec = count >> 2;
#pragma unroll 2
    for (unsigned int i = tid; i < nvec; i += kThreads) {
      float4 g = reinterpret_cast<const float4*>(u)[i], m = reinterpret_cast<const float4*>(v)[i];
      element(g.x, m.x);
      element(g.y, m.y);
      element(g.z, m.z);
      element(g.w, m.w);
      reinterpret_cast<float4*>(u)[i] = g;
      reinterpret_cast<float4*>(v)[i] = m;
    }
    for (unsigned int i = (nvec << 2) + tid; i < count; i += kThreads) {
      float g = u[i], m = v[i];
      element(g, m);
      u[i] = g;
      v[i] = m;
    }

    // the chunk's sums of squares: lanes, then warps, in a fixed order
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      sq += __shfl_down_sync(0xffffffffu, sq, o);
      usq += __shfl_down_sync(0xffffffffu, usq, o);
    }
    if (lane == 0) {
      s_red[0][warp] = sq;
      s_red[1][warp] = usq;
    }
    __syncthreads();
    if (warp == 0) {
      double a = s_red[0][0], b = s_red[1][0];
#pragma unroll
      for (int k = 1; k < kThreads / 32; ++k) {
        a += s_red[0][k];
        b += s_red[1][k];
      }
      if (lane == 0) {
        u_partials[idx] = b;
        if (profile) profile_chunk(tasks + t, t_begin, global_ns());
      }
      // (by a warp: one thread that adds up 64 chunks of a block takes 38 us)
      publish_part(tasks, t, idx, 1, a, stats, partials, lane);
    }
    buf ^= 1;
  }
}

}  // namespace psb
