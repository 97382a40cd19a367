// Aggregation with the gradients clipped by their global norm.
//
// The factor min(1, max_norm / (norm + 1e-6)) needs the sum of squares over all of
// a job's tensors before any element may be updated, so the work has two passes
// with a barrier over the whole grid between them, in one cooperative launch:
//   1  sum the W shards in worker order, scale, add up the squares, keep the sum
//   2  factor, optimizer step
// The sums are kept, not the shards read again: a sum costs 4 bytes written and 4
// read, the shards W times 4.  What fits stays in the CTA's shared memory and never
// leaves the SM; the rest goes to a buffer that pass 2 walks backwards, so that what
// pass 1 wrote last is found in L2.
//
// Every CTA works on the same elements in both passes: a contiguous range of the
// launch's tasks, cut by cost (bytes), not by count, so that jobs with many and with
// few workers share the device evenly; a task costs a fixed amount besides, so that
// a run of tiny tensors, whose time is latency, is spread over several CTAs.  The unit
// of the cut is 256 elements (whole rows for a task with row-sparse shards).  All sums are binary64 and added in an
// order fixed by the partition: per CTA and task ("segment"), then over CTAs.
#pragma once

#include "ps_grid.cuh"
#include "ps_kernel_ldg.cuh"

namespace psb {

constexpr int kClipMaxJobs = 64;         // jobs in one clipped launch
constexpr unsigned int kClipUnit = 256;
constexpr unsigned int kClipTaskCost = 8192;   // bytes a CTA streams in about a microsecond
constexpr unsigned int kClipCache = 12288;     // sums in shared memory: 48 KB for each of an SM's four CTAs

struct __align__(16) PsClipHdr {         // 64 bytes at the start of the table
  unsigned int n_tasks, n_jobs;
  unsigned int tasks_off, costs_off, ptrs_off, sparse_off;   // byte offsets from the table base
  float max_norm;
  unsigned int cache_elems;              // sums a CTA keeps in shared memory
  unsigned long long total_cost;
  unsigned long long _r0, _r1, _r2;
};

struct __align__(16) PsClipCost {        // one per task
  unsigned long long start;              // cost of all earlier tasks
  unsigned int unit;                     // cost of one unit
  unsigned int unit_elems;
  unsigned int job_slot;                 // which of the launch's jobs
  unsigned int units;
  unsigned long long spool;              // where the task's sums start in the buffer
};

// The partition.  CTA c of G owns the units whose cost position x satisfies lo(c) <= x < lo(c + 1).
__device__ __forceinline__ unsigned long long clip_lo(unsigned long long total, unsigned int c, unsigned int G) {
  return (total / G) * c + (total % G) * c / G;
}
// The CTA that owns cost position x: the largest c with lo(c) <= x.
__device__ __forceinline__ unsigned int clip_owner(unsigned long long total, unsigned long long x, unsigned int G) {
  unsigned int lo = 0, hi = G - 1;
  while (lo < hi) {
    const unsigned int mid = (lo + hi + 1) >> 1;
    if (clip_lo(total, mid, G) <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

struct ClipSegment {                     // a CTA's part of one task
  size_t begin;
  unsigned long long count;
};

__device__ __forceinline__ ClipSegment clip_segment(const PsClipCost& k, unsigned long long nelem, unsigned long long lo,
                                                    unsigned long long hi) {
  const unsigned long long units = k.units, end_cost = k.start + units * k.unit;
  const unsigned long long j0 = lo <= k.start ? 0 : lo >= end_cost ? units : (lo - k.start + k.unit - 1) / k.unit;
  const unsigned long long j1 = hi <= k.start ? 0 : hi >= end_cost ? units : (hi - k.start + k.unit - 1) / k.unit;
  ClipSegment s;
  s.begin = (size_t)(j0 * k.unit_elems);
  const unsigned long long end = min(nelem, j1 * k.unit_elems);
  s.count = end > s.begin ? end - s.begin : 0;
  return s;
}

// Pass 1 over elements [begin, begin + count) of a task; the sum of element e goes to G[e].
// (A function of its own, like pass 2: inlined into the walk over tasks, both spilled inside their loops.)
template <int NT>
__device__ __noinline__ double clip_sum(unsigned int tid, const PsJobDev* J, const PsTaskDev* T,
                                      const void* const* shards, const PsSparseDev* sparse, float* G, size_t begin,
                                      unsigned int count, const void** srcs) {
  Hp h;
  h.gs = J->gs;
  double sq = 0.0;
  const int W = J->W;
  if (T->row_len) {
    if (J->grad_dtype) chunk_rows<kSumOnly, true, NT>(tid, h, shards, sparse, W, G, nullptr, nullptr, begin, count, T->row_len, srcs, sq);
    else chunk_rows<kSumOnly, false, NT>(tid, h, shards, sparse, W, G, nullptr, nullptr, begin, count, T->row_len, srcs, sq);
  } else if (J->grad_dtype) {
    run_chunk<kSumOnly, true, NT>(tid, h, shards, W, G, nullptr, nullptr, begin, count, T->vec_ok != 0, sq);
  } else {
    run_chunk<kSumOnly, false, NT>(tid, h, shards, W, G, nullptr, nullptr, begin, count, T->vec_ok != 0, sq);
  }
  return sq;
}

// Pass 2 over the same elements.  begin is a multiple of 4 elements and G, like p and the state, 16-byte aligned there.
template <int OPT, int NT>
__device__ __noinline__ void clip_apply(unsigned int tid, const PsJobDev* J, const PsTaskDev* T, float factor, const float* G,
                                        size_t begin, unsigned int count) {
  const Hp h = load_hp(J, T);
  float *p = T->p, *s0 = T->s0, *s1 = T->s1;
  const unsigned int nvec = count >> 2;
  constexpr int U = 2;
  for (unsigned int i = tid; i < nvec; i += U * NT) {
    float4 g[U], pv[U], av[U], bv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u * NT >= nvec) break;
      const size_t e = begin + 4 * (size_t)(i + u * NT);
      g[u] = *reinterpret_cast<const float4*>(G + e);
      pv[u] = *reinterpret_cast<const float4*>(p + e);
      av[u] = *reinterpret_cast<const float4*>(s0 + e);
      bv[u] = OPT == 1 ? *reinterpret_cast<const float4*>(s1 + e) : make_float4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i + u * NT >= nvec) break;
      const size_t e = begin + 4 * (size_t)(i + u * NT);
      apply_elem<OPT>(h, __fmul_rn(g[u].x, factor), pv[u].x, av[u].x, bv[u].x);
      apply_elem<OPT>(h, __fmul_rn(g[u].y, factor), pv[u].y, av[u].y, bv[u].y);
      apply_elem<OPT>(h, __fmul_rn(g[u].z, factor), pv[u].z, av[u].z, bv[u].z);
      apply_elem<OPT>(h, __fmul_rn(g[u].w, factor), pv[u].w, av[u].w, bv[u].w);
      *reinterpret_cast<float4*>(p + e) = pv[u];
      *reinterpret_cast<float4*>(s0 + e) = av[u];
      if (OPT == 1) *reinterpret_cast<float4*>(s1 + e) = bv[u];
    }
  }
  for (unsigned int i = (nvec << 2) + tid; i < count; i += NT) {
    const size_t e = begin + i;
    float P = p[e], A = s0[e], B = OPT == 1 ? s1[e] : 0.f;
    apply_elem<OPT>(h, __fmul_rn(G[e], factor), P, A, B);
    p[e] = P;
    s0[e] = A;
    if (OPT == 1) s1[e] = B;
  }
}

// job_parts: n_jobs doubles per CTA; seg_parts and seg_at: per segment its sum of squares and the place of its sums
// in shared memory, in slot task + CTA (increasing along a CTA's tasks and from CTA to CTA, so no two segments share
// one).
__device__ __forceinline__ void clip_body(const unsigned char* table, const PsJobDev* jobs, PsStat* stats, double* seg_parts,
                                          double* job_parts, unsigned int* seg_at, float* spool, GridBarrier* bar,
                                          float* norms_out, int* status) {
  const PsClipHdr* hdr = reinterpret_cast<const PsClipHdr*>(table);
  const PsTaskDev* tasks = reinterpret_cast<const PsTaskDev*>(table + hdr->tasks_off);
  const PsClipCost* costs = reinterpret_cast<const PsClipCost*>(table + hdr->costs_off);
  const void* const* ptrs = reinterpret_cast<const void* const*>(table + hdr->ptrs_off);
  const PsSparseDev* sparse = reinterpret_cast<const PsSparseDev*>(table + hdr->sparse_off);
  const unsigned int n_tasks = hdr->n_tasks, n_jobs = hdr->n_jobs, G = gridDim.x, c = blockIdx.x;
  const unsigned long long total = hdr->total_cost;
  const unsigned int cache_elems = hdr->cache_elems;

  extern __shared__ float cache[];
  __shared__ double s_red[kThreads / 32], s_job[kClipMaxJobs];
  __shared__ float s_factor[kClipMaxJobs];
  __shared__ const void* s_rowsrc[kThreads / 32][32];
  const unsigned int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  const unsigned long long lo = clip_lo(total, c, G), hi = clip_lo(total, c + 1, G);
  // the first task with a unit at or after lo: the last one that starts at or before it
  unsigned int t0 = 0;
  {
    unsigned int a = 0, b = n_tasks - 1;
    while (a < b) {
      const unsigned int mid = (a + b + 1) >> 1;
      if (costs[mid].start <= lo) a = mid; else b = mid - 1;
    }
    t0 = a;
  }
  for (unsigned int j = tid; j < n_jobs; j += kThreads) s_job[j] = 0.0;
  __syncthreads();

  unsigned int used = 0, t1 = t0;        // elements of shared memory in use; one past the last task
  for (unsigned int t = t0; t < n_tasks && costs[t].start < hi; ++t) {
    t1 = t + 1;
    const PsTaskDev* T = tasks + t;
    const PsClipCost& k = costs[t];
    const ClipSegment s = clip_segment(k, T->nelem, lo, hi);
    double sq = 0.0;
    if (s.count) {
      // what still fits goes to shared memory (whole units, so that both parts start aligned)
      const unsigned int room = (cache_elems - used) / k.unit_elems * k.unit_elems;
      const unsigned int near = (unsigned int)min((unsigned long long)room, s.count);
      const void* const* shards = ptrs + T->shard_row;
      if (tid == 0) seg_at[t + c] = used;
      // the near part, then the rest in pieces (a body takes 32-bit counts)
      const unsigned int piece = (1u << 30) / k.unit_elems * k.unit_elems;
      for (unsigned long long off = 0; off < s.count;) {
        const bool here = off < near;
        const unsigned int n = here ? near : (unsigned int)min(s.count - off, (unsigned long long)piece);
        sq += clip_sum<kThreads>(tid, jobs + T->job, T, shards, sparse + T->sparse_row,
                                 here ? cache + used - s.begin : spool + k.spool, s.begin + (size_t)off, n, s_rowsrc[warp]);
        off += n;
      }
      used = min(cache_elems, used + ((near + 7) & ~7u));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sq += __shfl_down_sync(0xffffffffu, sq, o);
    if (lane == 0) s_red[warp] = sq;
    __syncthreads();
    if (tid == 0) {
      double v = s_red[0];
#pragma unroll
      for (int w = 1; w < kThreads / 32; ++w) v += s_red[w];
      __stcg(seg_parts + t + c, v);
      s_job[k.job_slot] += v;
    }
    __syncthreads();
  }
  for (unsigned int j = tid; j < n_jobs; j += kThreads) __stcg(job_parts + (size_t)c * n_jobs + j, s_job[j]);

  if (!grid_barrier(bar)) {
    if (tid == 0) atomicExch(status, 1);
    return;
  }

  // every CTA adds the same numbers in the same order: one warp per job
  for (unsigned int j = warp; j < n_jobs; j += kThreads / 32) {
    double v = 0.0;
    for (unsigned int q = lane; q < G; q += 32) v += __ldcg(job_parts + (size_t)q * n_jobs + j);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
    if (lane == 0) {
      const float norm = (float)sqrt(v);
      s_factor[j] = clip_factor(norm, hdr->max_norm);
      if (c == 0 && norms_out) norms_out[j] = norm;
    }
  }
  __syncthreads();

  for (unsigned int t = t1; t-- > t0;) {
    const PsTaskDev* T = tasks + t;
    const PsClipCost& k = costs[t];
    const ClipSegment s = clip_segment(k, T->nelem, lo, hi);
    if (!s.count) continue;
    const unsigned int at = seg_at[t + c];                        // (written by this CTA)
    const unsigned int room = (cache_elems - at) / k.unit_elems * k.unit_elems;
    const unsigned int near = (unsigned int)min((unsigned long long)room, s.count);
    const PsJobDev* J = jobs + T->job;
    const float factor = s_factor[k.job_slot];
    // backwards in steps (the latest sums are still in L2), what is in shared memory last
    constexpr unsigned int kStep = 1u << 15;
    for (unsigned long long left = s.count; left;) {
      const bool here = left <= near;
      const unsigned int n = here ? near : (unsigned int)((left - near - 1) % kStep + 1);
      left -= n;
      const float* sums = here ? cache + at - s.begin : spool + k.spool;
      if (J->opt) clip_apply<1, kThreads>(tid, J, T, factor, sums, s.begin + (size_t)left, n);
      else clip_apply<0, kThreads>(tid, J, T, factor, sums, s.begin + (size_t)left, n);
    }
  }

  // per-block statistics: the task's segments in CTA order, one warp per task
  for (unsigned int t = c * (kThreads / 32) + warp; t < n_tasks; t += G * (kThreads / 32)) {
    const PsTaskDev* T = tasks + t;
    const PsClipCost& k = costs[t];
    const unsigned int c0 = clip_owner(total, k.start, G);
    const unsigned int c1 = clip_owner(total, k.start + (unsigned long long)(k.units - 1) * k.unit, G);
    const double v = sum_partials_warp(seg_parts + t + c0, c1 - c0 + 1, lane);
    if (lane == 0) {
      PsStat st;
      st.sqnorm = v;
      st.step = T->step;
      st.busy_ns = st.t_first = st.t_last = st._r0 = 0;
      stats[T->stat_idx] = st;
    }
  }
}

// The table in device memory ...
__global__ void __launch_bounds__(kThreads, 4)
ps_aggregate_clip_kernel(const unsigned char* __restrict__ table, const PsJobDev* __restrict__ jobs, PsStat* __restrict__ stats,
                         double* seg_parts, double* job_parts, unsigned int* seg_at, float* spool, GridBarrier* bar,
                         float* norms_out, int* status, unsigned int* exit_ctr, unsigned long long* done_word, unsigned long long seq) {
  clip_body(table, jobs, stats, seg_parts, job_parts, seg_at, spool, bar, norms_out, status);
  signal_exit(exit_ctr, done_word, seq);
}

// ... or, where it fits, in the kernel's parameters: no upload.
__global__ void __launch_bounds__(kThreads, 4)
ps_aggregate_clip_inline_kernel(const __grid_constant__ PsInlineTable tbl, const PsJobDev* __restrict__ jobs,
                                PsStat* __restrict__ stats, double* seg_parts, double* job_parts, unsigned int* seg_at,
                                float* spool, GridBarrier* bar, float* norms_out, int* status, unsigned int* exit_ctr,
                                unsigned long long* done_word, unsigned long long seq) {
  clip_body(tbl.bytes, jobs, stats, seg_parts, job_parts, seg_at, spool, bar, norms_out, status);
  signal_exit(exit_ctr, done_word, seq);
}

}  // namespace psb
