// Aggregation with the gradients clipped by their global norm.
//
// The factor min(1, max_norm / (norm + 1e-6)) needs the sum of squares over all of
// a job's tensors before any element may be updated, so the work has two passes
// with a barrier over the whole grid between them, in one cooperative launch:
//   1  sum the W shards in worker order, scale, add up the squares, keep the sum
//   2  factor, optimizer step
// The sums are kept, not the shards read again, where that is less: a sum costs 4
// bytes written and 4 read, the shards once more W times their element.  The first
// chunk of every CTA stays in its shared memory if it fits; it is fixed by the CTA's
// index, so pass 2 finds it there.  All other chunks are claimed from a counter in
// both passes, which evens out what SMs and jobs of different weight take; their sums
// go to a buffer that pass 2 walks backwards, so that what pass 1 wrote last is found
// in L2.  Like the other aggregation kernels this one is bound by memory latency:
// without the L2 prefetches of the shared chunk bodies pass 1 took 2.3 times as long.
//
// Measured (pass 1, barrier and norm, pass 2): 36.5 M elements, W = 8 fp32, SGD 190, 17
// and 108 us, 340 us a call (6.0 TB/s of what it moves, 5.1 of the 48 bytes per element
// that no call can do without); 1.05 M elements, W = 4 fp32 4.3, 4.6 and 2.0 us, 17 us a
// call; 335 M elements, W = 4 bf16, Adam 2.4 ms (5.5 TB/s of 40 bytes per element).
//
// Every chunk publishes one binary64 sum of squares.  After the barrier each CTA
// adds a job's chunk sums in the same fixed order (tasks are sorted by job, so they
// are neighbours): the norm depends on neither the claims nor their timing.
#pragma once

#include "ps_grid.cuh"
#include "ps_kernel_ldg.cuh"

namespace psb {

constexpr int kClipMaxJobs = 64;               // jobs in one clipped launch
constexpr unsigned int kClipSlot = 12288;      // sums a CTA keeps: 48 KB for each of an SM's four CTAs
constexpr unsigned int kClipChunkMin = 8192, kClipChunkMax = 32768;   // elements of a claimed chunk
// Bytes of shards per element up to which they are read again, by optimizer.  Per element a kept sum costs 8 bytes of
// traffic, and pass 2 is lighter without the sum; 233 M elements, read again | kept, in us after seconds under load:
// SGD  4 bytes (W = 2, bf16) 1049 | 1138, 6 bytes 1188..1238 | 1220, 8 bytes 1334..1404 | 1297
// Adam 2 bytes (W = 1, bf16) 1440 | 1480, 4 bytes 1602..1670 | 1554, 6 bytes 1800 | 1646
constexpr unsigned int kClipRereadSgd = 4, kClipRereadAdam = 2;

struct __align__(16) PsClipHdr {               // 64 bytes at the start of the table
  unsigned int n_tasks, n_jobs, total_chunks;
  unsigned int profile;                        // 1: record per-task device time; the chunk sums are followed by two times each
  unsigned int tasks_off, starts_off, ptrs_off, sparse_off;    // byte offsets from the table base
  unsigned int jobs_off;                       // first chunk of every job, and the end: n_jobs + 1 entries
  float max_norm;
  long long wait_cycles;                       // limit of the wait for the other CTAs
  unsigned int _r[4];
};
static_assert(sizeof(PsClipHdr) == 64, "header");

struct ClipShared {                            // device memory of the service, zero before the first launch
  GridBarrier bar;
  unsigned int claim1, claim2;                 // chunks claimed beyond the fixed ones; cleared at the barrier
};

// ---- pass 1: sums of one chunk; the scaled sum of element begin + i goes to G[i] --------------------------

// (Functions of their own, like the optimizer step: inlined into the walk over chunks they spilled inside their loops.)
template <int OPT, bool BF16, int NT>
__device__ __noinline__ double clip_sum_vec(unsigned int tid, const void* const* shards, int W, float gs, float* G, size_t begin,
                                            unsigned int count) {
  Hp h;
  h.gs = gs;
  double sq = 0.0;
  run_chunk<OPT, BF16, NT>(tid, h, shards, W, G - begin, nullptr, nullptr, begin, count, true, sq);
  return sq;
}

template <int NT>
__device__ __noinline__ double clip_sum_other(unsigned int tid, const PsJobDev* J, const PsTaskDev* T, const void* const* shards,
                                              const PsSparseDev* sparse, float* G, size_t begin, unsigned int first,
                                              unsigned int count, const void** srcs) {
  Hp h;
  h.gs = J->gs;
  const int W = J->W;
  float* at = G - begin;                       // (the shared bodies index by element)
  double sq = 0.0;
  if (T->row_len) {
    if (J->grad_dtype) chunk_rows<kSumOnly, true, NT>(tid, h, shards, sparse, W, at, nullptr, nullptr, begin, count, T->row_len, srcs, sq);
    else chunk_rows<kSumOnly, false, NT>(tid, h, shards, sparse, W, at, nullptr, nullptr, begin, count, T->row_len, srcs, sq);
  } else if (J->grad_dtype) {
    chunk_scalar<kSumOnly, true, NT>(tid, h, shards, W, at, nullptr, nullptr, begin, first, count, sq);
  } else {
    chunk_scalar<kSumOnly, false, NT>(tid, h, shards, W, at, nullptr, nullptr, begin, first, count, sq);
  }
  return sq;
}

// ---- pass 2: optimizer step of one chunk ------------------------------------------------------------------

template <int OPT, int NT>
__device__ __noinline__ void clip_apply(unsigned int tid, const PsJobDev* J, const PsTaskDev* T, float factor, const float* G,
                                        size_t begin, unsigned int count) {
  const Hp h = load_hp(J, T);
  float *p = T->p + begin, *s0 = T->s0 + begin, *s1 = OPT == 1 ? T->s1 + begin : nullptr;
  const unsigned int nvec = count >> 2;
  const bool pf_lane = (tid & 7) == 0;         // 8 lanes x 16 bytes = one line
  for (unsigned int i = tid; i < nvec; i += NT) {
    float4 pv = reinterpret_cast<const float4*>(p)[i], av = reinterpret_cast<const float4*>(s0)[i];
    float4 bv = OPT == 1 ? reinterpret_cast<const float4*>(s1)[i] : make_float4(0, 0, 0, 0);
    const float4 g = reinterpret_cast<const float4*>(G)[i];
    if (pf_lane && i + 2 * NT < nvec) {        // two trips ahead, without a register
      prefetch_l2(p + 4 * (i + 2 * NT));
      prefetch_l2(s0 + 4 * (i + 2 * NT));
      if (OPT == 1) prefetch_l2(s1 + 4 * (i + 2 * NT));
    }
    apply_elem<OPT>(h, __fmul_rn(g.x, factor), pv.x, av.x, bv.x);
    apply_elem<OPT>(h, __fmul_rn(g.y, factor), pv.y, av.y, bv.y);
    apply_elem<OPT>(h, __fmul_rn(g.z, factor), pv.z, av.z, bv.z);
    apply_elem<OPT>(h, __fmul_rn(g.w, factor), pv.w, av.w, bv.w);
    reinterpret_cast<float4*>(p)[i] = pv;
    reinterpret_cast<float4*>(s0)[i] = av;
    if (OPT == 1) reinterpret_cast<float4*>(s1)[i] = bv;
  }
  for (unsigned int i = (nvec << 2) + tid; i < count; i += NT) {
    float P = p[i], A = s0[i], B = OPT == 1 ? s1[i] : 0.f;
    apply_elem<OPT>(h, __fmul_rn(G[i], factor), P, A, B);
    p[i] = P;
    s0[i] = A;
    if (OPT == 1) s1[i] = B;
  }
}

// The same from the shards.
template <int OPT, bool BF16, int NT>
__device__ __noinline__ void clip_apply_shards(unsigned int tid, const PsJobDev* J, const PsTaskDev* T, float factor,
                                               const void* const* shards, size_t begin, unsigned int count) {
  Hp h = load_hp(J, T);
  h.clip = factor;
  double sq = 0.0;
  run_chunk<kClipped + OPT, BF16, NT>(tid, h, shards, J->W, T->p, T->s0, T->s1, begin, count, true, sq);
}

// ---- the walk ---------------------------------------------------------------------------------------------

// The task that owns chunk idx, found by one warp: the last one whose first chunk is <= idx.
__device__ __forceinline__ unsigned int clip_find(const unsigned int* starts, unsigned int n, unsigned int idx, unsigned int lane) {
  unsigned int lo = 0;
  while (n > 1) {
    const unsigned int step = (n + 31) / 32, at = lane * step;
    const bool le = at < n && starts[lo + at] <= idx;
    const unsigned int k = 31 - __clz(__ballot_sync(0xffffffffu, le));    // (lane 0's probe always holds)
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

// Where the sum of a chunk's element 0 is kept.  Of a task whose shards are read again only the last few elements of a
// chunk are (from element `whole` on, fewer than eight): eight places per chunk.
__device__ __forceinline__ float* clip_place(const PsTaskDev* T, unsigned int idx, unsigned int count, bool kept, float* cache,
                                             float* spool) {
  if (kept) return cache;
  const unsigned int k = idx - T->first_chunk;
  if (!T->reread) return spool + T->spool + (size_t)k * T->chunk_elems;
  return spool + T->spool + 8 * (size_t)k - (count & ~7u);
}

// A job's chunk sums in a fixed order: thread t takes t, t + NT, ..., then the block adds its threads.
template <int NT>
__device__ __forceinline__ double clip_total(const double* parts, unsigned int n, unsigned int tid, double* red) {
  double v = 0.0;
#pragma unroll 8
  for (unsigned int k = tid; k < n; k += NT) v += parts[k];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((tid & 31) == 0) red[tid >> 5] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NT / 32; ++w) v += red[w];
  return v;
}

__device__ __forceinline__ void clip_body(const unsigned char* table, const PsJobDev* jobs, PsStat* stats, double* parts,
                                          float* spool, ClipShared* sh, float* norms_out, int* status) {
  const PsClipHdr* hdr = reinterpret_cast<const PsClipHdr*>(table);
  const PsTaskDev* tasks = reinterpret_cast<const PsTaskDev*>(table + hdr->tasks_off);
  const unsigned int* starts = reinterpret_cast<const unsigned int*>(table + hdr->starts_off);
  const unsigned int* job_first = reinterpret_cast<const unsigned int*>(table + hdr->jobs_off);
  const void* const* ptrs = reinterpret_cast<const void* const*>(table + hdr->ptrs_off);
  const PsSparseDev* sparse = reinterpret_cast<const PsSparseDev*>(table + hdr->sparse_off);
  const unsigned int n_tasks = hdr->n_tasks, n_jobs = hdr->n_jobs, total = hdr->total_chunks;
  const bool profile = hdr->profile != 0;
  unsigned long long* times = reinterpret_cast<unsigned long long*>(parts + total);      // pass 1: start and end of every chunk
  const unsigned int G = gridDim.x, c = blockIdx.x;          // (never more CTAs than chunks)

  extern __shared__ __align__(16) float cache[];       // kClipSlot sums, in vectors of four
  __shared__ double s_red[kThreads / 32];
  __shared__ float s_factor[kClipMaxJobs];
  __shared__ unsigned int s_idx, s_task;
  __shared__ const void* s_rowsrc[kThreads / 32][32];
  const unsigned int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (profile && tid == 0)                     // pass 2 adds to these
    for (unsigned int t = c; t < n_tasks; t += G) {
      PsStat* st = stats + tasks[t].stat_idx;
      st->busy_ns = st->t_last = 0;
      st->t_first = ~0ull;
    }
  for (unsigned int round = 0;; ++round) {
    __syncthreads();                           // the previous chunk's s_idx, s_task and s_red have been read
    if (warp == 0) {
      unsigned int idx = c;
      if (round > 0) {
        if (lane == 0) idx = min(total, G + atomicAdd(&sh->claim1, 1u));
        idx = __shfl_sync(0xffffffffu, idx, 0);
      }
      unsigned int t = 0;
      if (idx < total) t = clip_find(starts, n_tasks, idx, lane);
      if (lane == 0) { s_idx = idx; s_task = t; }
    }
    __syncthreads();
    const unsigned int idx = s_idx;
    if (idx >= total) break;
    if (profile && tid == 0) times[2 * (size_t)idx] = global_ns();
    const PsTaskDev* T = tasks + s_task;
    const PsJobDev* J = jobs + T->job;
    const size_t begin = (size_t)(idx - T->first_chunk) * T->chunk_elems;
    const unsigned int count = (unsigned int)min((unsigned long long)T->chunk_elems, T->nelem - begin);
    const bool kept = round == 0 && T->chunk_elems <= kClipSlot;
    float* G_at = clip_place(T, idx, count, kept, cache, spool);
    const void* const* shards = ptrs + T->shard_row;
    double sq = 0.0;
    unsigned int done = 0;
    if (T->vec_ok && !T->row_len) {
      const bool store = kept || !T->reread;
      if (J->grad_dtype) {
        done = count & ~7u;
        sq = store ? clip_sum_vec<kSumOnly, true, kThreads>(tid, shards, J->W, J->gs, G_at, begin, done)
                   : clip_sum_vec<kNormOnly, true, kThreads>(tid, shards, J->W, J->gs, G_at, begin, done);
      } else {
        done = store ? count & ~3u : count & ~7u;
        sq = store ? clip_sum_vec<kSumOnly, false, kThreads>(tid, shards, J->W, J->gs, G_at, begin, done)
                   : clip_sum_vec<kNormOnly, false, kThreads>(tid, shards, J->W, J->gs, G_at, begin, done);
      }
    }
    // (the last few elements, unaligned shards, row-sparse shards: these sums are always kept)
    if (done != count)
      sq += clip_sum_other<kThreads>(tid, J, T, shards, sparse + T->sparse_row, G_at, begin, done, count, s_rowsrc[warp]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sq += __shfl_down_sync(0xffffffffu, sq, o);
    if (lane == 0) s_red[warp] = sq;
    if (total <= G && (tid & 7) == 0) {    // a short launch: what pass 2 reads is on its way during the barrier
      for (unsigned int i = tid * 4; i < count; i += kThreads * 4) {
        prefetch_l2(T->p + begin + i);
        prefetch_l2(T->s0 + begin + i);
        if (J->opt) prefetch_l2(T->s1 + begin + i);
      }
    }
    __syncthreads();
    if (tid == 0) {
      double v = s_red[0];
#pragma unroll
      for (int w = 1; w < kThreads / 32; ++w) v += s_red[w];
      __stcg(parts + idx, v);
      if (profile) times[2 * (size_t)idx + 1] = global_ns();
    }
  }

  // (claim1 for the next launch, claim2 for pass 2: by the last CTA to arrive, so also where others gave up waiting)
  if (!grid_barrier(&sh->bar, hdr->wait_cycles, [sh] { sh->claim1 = sh->claim2 = 0; })) {
    if (tid == 0) atomicExch(status, 1);
    return;
  }
  for (unsigned int j = 0; j < n_jobs; ++j) {
    const double v = clip_total<kThreads>(parts + job_first[j], job_first[j + 1] - job_first[j], tid, s_red);
    if (tid == 0) {
      const float norm = (float)sqrt(v);
      s_factor[j] = clip_factor(norm, hdr->max_norm);
      if (c == 0 && norms_out) norms_out[j] = norm;
    }
  }

  // claimed chunks from the last one down, then the CTA's own
  for (bool own = false; !own;) {
    __syncthreads();
    if (warp == 0) {
      unsigned int k = total;
      if (total > G) {
        if (lane == 0) k = atomicAdd(&sh->claim2, 1u);
        k = __shfl_sync(0xffffffffu, k, 0);
      }
      const unsigned int idx = k < total - G ? total - 1 - k : c;
      const unsigned int t = clip_find(starts, n_tasks, idx, lane);
      if (lane == 0) { s_idx = idx; s_task = t; }
    }
    __syncthreads();
    const unsigned int idx = s_idx;
    own = idx < G;
    const unsigned long long t_begin = profile && tid == 0 ? global_ns() : 0ull;
    const PsTaskDev* T = tasks + s_task;
    const PsJobDev* J = jobs + T->job;
    const size_t begin = (size_t)(idx - T->first_chunk) * T->chunk_elems;
    const unsigned int count = (unsigned int)min((unsigned long long)T->chunk_elems, T->nelem - begin);
    const bool kept = own && T->chunk_elems <= kClipSlot;
    const float* G_at = clip_place(T, idx, count, kept, cache, spool);
    const float factor = s_factor[T->job_slot];
    unsigned int done = 0;
    if (T->reread && !kept) {
      const void* const* shards = ptrs + T->shard_row;
      done = count & ~7u;
      if (J->opt) clip_apply_shards<1, true, kThreads>(tid, J, T, factor, shards, begin, done);      // (bf16: two bytes at most)
      else if (J->grad_dtype) clip_apply_shards<0, true, kThreads>(tid, J, T, factor, shards, begin, done);
      else clip_apply_shards<0, false, kThreads>(tid, J, T, factor, shards, begin, done);
    }
    if (done != count) {
      if (J->opt) clip_apply<1, kThreads>(tid, J, T, factor, G_at + done, begin + done, count - done);
      else clip_apply<0, kThreads>(tid, J, T, factor, G_at + done, begin + done, count - done);
    }
    if (profile) {
      __syncthreads();
      if (tid == 0) {
        PsStat* st = stats + T->stat_idx;
        const unsigned long long t_end = global_ns(), first = __ldcg(times + 2 * (size_t)idx);
        atomicAdd(&st->busy_ns, t_end - t_begin + (__ldcg(times + 2 * (size_t)idx + 1) - first));
        atomicMin(&st->t_first, first);
        atomicMax(&st->t_last, t_end);
      }
    }
  }

  // per-block statistics: a task's chunk sums in a fixed order, one CTA per task
  for (unsigned int t = c; t < n_tasks; t += G) {
    const PsTaskDev* T = tasks + t;
    const double v = clip_total<kThreads>(parts + T->first_chunk, T->nchunks, tid, s_red);
    if (tid == 0) {
      PsStat* st = stats + T->stat_idx;
      st->sqnorm = v;
      st->step = T->step;
      if (!profile) st->busy_ns = st->t_first = st->t_last = 0;
    }
  }
}

// The table in device memory ...
__global__ void __launch_bounds__(kThreads, 4)
ps_aggregate_clip_kernel(const unsigned char* __restrict__ table, const PsJobDev* __restrict__ jobs, PsStat* __restrict__ stats,
                         double* parts, float* spool, ClipShared* sh, float* norms_out, int* status, unsigned int* exit_ctr,
                         unsigned long long* done_word, unsigned long long seq) {
  clip_body(table, jobs, stats, parts, spool, sh, norms_out, status);
  signal_exit(exit_ctr, done_word, seq);
}

// ... or, where it fits, in the kernel's parameters: no upload.
__global__ void __launch_bounds__(kThreads, 4)
ps_aggregate_clip_inline_kernel(const __grid_constant__ PsInlineTable tbl, const PsJobDev* __restrict__ jobs,
                                PsStat* __restrict__ stats, double* parts, float* spool, ClipShared* sh, float* norms_out,
                                int* status, unsigned int* exit_ctr, unsigned long long* done_word, unsigned long long seq) {
  clip_body(tbl.bytes, jobs, stats, parts, spool, sh, norms_out, status);
  signal_exit(exit_ctr, done_word, seq);
}

}  // namespace psb
