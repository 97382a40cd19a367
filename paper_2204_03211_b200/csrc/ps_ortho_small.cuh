// Orthogonalisation of small matrices (up to 128 by 2048): all five steps in shared memory.
//
// In the general form (ps_ortho.cuh) a product of a small matrix is one tile, and what takes time is handing it from one
// tile to the next through L2: 6 to 8 us, fifteen times.  Here a CTA keeps 128 rows by up to 256 columns of X (two
// halves, 128 KB) and A or B (two halves, 64 KB) in shared memory, in the swizzled layout in which the tensor cores take
// operands: X is an operand along its rows in X X^T and across them in B X, from the same bytes.  Wider matrices are cut
// into columns over a cluster of 2, 4 or 8 CTAs; only A is a sum over all of them, which they add up through each
// other's shared memory, a share of the rows each, in rank order.  One launch does it all: norm, scaling, steps, result.
//
// Sixteen warps read the sums (row = lane, 32 columns at a time); thread 0 issues the products.  Arithmetic as in
// ps_ortho.cuh, with the small products of a pair of halves first and the long sums of A in two parts, so that few of
// the tensor cores' cut-off additions meet large sums.
#pragma once

#include "ps_ortho.cuh"

namespace psb {

constexpr int kSoThreads = 512;
constexpr int kSoRows = 128, kSoCols = 256;              // of a CTA's part of X
constexpr int kSoCtas = 8;
constexpr int kSoBlock = kSoRows * 128;                  // bytes of 128 rows by 64 columns of one plane
constexpr int kSoX = 2 * (kSoCols / 64) * kSoBlock, kSoE = 4 * kSoBlock;

struct SoControl {
  unsigned long long bar;
  double norm[kSoCtas];
  double red[kSoThreads / 32];
  float d[kSoRows], fd[kSoRows];
  unsigned int tmem;
};
constexpr int kSoSmem = kSoX + kSoE + 2048;
static_assert(sizeof(SoControl) <= 2048 && kSoSmem <= 227 * 1024, "does not fit");

struct SoArgs {
  const NsMat* mats;
  int* status;
  int ctas;                                              // of a cluster: 1, 2, 4 or 8
};

// Byte offset of 16-byte piece `piece` (8 columns) of a row, in planes of 64-column blocks.
__device__ __forceinline__ unsigned int so_piece(int row, int piece) {
  return (unsigned int)((piece >> 3) * kSoBlock + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
}
// ... and of 4 floats of a row of 128, for sums that other CTAs read.
__device__ __forceinline__ unsigned int so_float4(int row, int quad) { return (unsigned int)(row * 512 + ((quad ^ (row & 7)) << 4)); }

__device__ __forceinline__ unsigned int so_peer(unsigned int addr, int rank) {
  unsigned int r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}

template <int PLANES>
__global__ void __launch_bounds__(kSoThreads, 1)
ps_ortho_small_kernel(const __grid_constant__ SoArgs args) {
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char *const xs = smem, *const es = smem + kSoX;
  SoControl& ctl = *reinterpret_cast<SoControl*>(smem + kSoX + kSoE);
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const int ctas = args.ctas, rank = ctas > 1 ? (int)(blockIdx.x % (unsigned)ctas) : 0;
  const NsMat& M = args.mats[blockIdx.x / (unsigned)ctas];
  const int m = M.m, n = M.n;
  // this CTA's columns: whole blocks of 64
  const int share = (((n + ctas - 1) / ctas) + 63) / 64 * 64;
  const int c0 = rank * share, cols = max(0, min(share, n - c0)), blocks = (cols + 63) / 64;
  const int mp = (m + 15) / 16 * 16, np = blocks * 64;

  if (tid == 0) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(mm_smem(&ctl.bar)) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 256;" ::"r"(mm_smem(&ctl.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (ctas > 1) mm_cluster_sync();                       // all of them run: their shared memory may be written
  mm_pdl();

  // ---- norm, and X0 as two planes (rows from m on and columns from `cols` on are zeros)
  const bool flip = M.flip != 0;
  auto source = [&](int r, int c) {                      // X[r][c0 + c]
    const size_t at = flip ? (size_t)(c0 + c) * (size_t)M.ld_src + (size_t)r : (size_t)r * (size_t)M.ld_src + (size_t)(c0 + c);
    return ns_source(M, at);
  };
  // lanes run along the source's rows
  const int fast = flip ? m : cols, slow = flip ? cols : m;
  double sq = 0.0;
  for (int s = warp; s < slow; s += kSoThreads / 32)
#pragma unroll 4
    for (int f = lane; f < fast; f += 32) {
      const double v = (double)(flip ? source(f, s) : source(s, f));
      sq = fma(v, v, sq);
    }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sq += __shfl_down_sync(0xffffffffu, sq, o);
  if (lane == 0) ctl.red[warp] = sq;
  for (int i = tid; i < 2 * blocks * (kSoBlock / 16); i += kSoThreads) reinterpret_cast<uint4*>(xs)[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  if (tid < ctas) {                                      // this CTA's sum, to every CTA of the cluster
    double v = ctl.red[0];
    for (int w = 1; w < kSoThreads / 32; ++w) v += ctl.red[w];
    if (ctas > 1)
      asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(so_peer(mm_smem(&ctl.norm[rank]), tid)), "d"(v) : "memory");
    else
      ctl.norm[0] = v;
  }
  if (ctas > 1) mm_cluster_sync();
  else __syncthreads();
  double total = ctl.norm[0];
  for (int k = 1; k < ctas; ++k) total += ctl.norm[k];
  const float scale = (float)((double)kNsScaleX / (sqrt(total) + kNsEps));
  const unsigned int lo_at = (unsigned int)(blocks * kSoBlock);     // the low plane follows the high one
  for (int s = warp; s < slow; s += kSoThreads / 32)
#pragma unroll 4
    for (int f = lane; f < fast; f += 32) {
      const int r = flip ? f : s, c = flip ? s : f;
      __half hi, lo;
      ns_split(source(r, c) * scale, hi, lo);
      unsigned char* p = xs + so_piece(r, c >> 3) + (c & 7) * 2;
      *reinterpret_cast<__half*>(p) = hi;
      *reinterpret_cast<__half*>(p + lo_at) = lo;
    }
  asm volatile("fence.proxy.async;" ::: "memory");
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const unsigned int tmem = ctl.tmem;
  const unsigned int xa = mm_smem(xs), ea = mm_smem(es), bar = mm_smem(&ctl.bar);
  const unsigned int mine = tmem + ((unsigned)((warp & 3) * 32) << 16);
  const int row = (warp & 3) * 32 + lane, part = warp >> 2;        // part: which 32 of 128 columns
  unsigned int parity = 0;

  // All products of one kind, by one thread: D (+)= A B^T over `steps` times 16 of k.  The strides of a step, and of every
  // fourth one where k runs along rows of 64 elements.
  auto products = [&](unsigned int d, unsigned int a, unsigned int a_lo, unsigned int b, unsigned int b_lo, bool b_mn, int k0, int k1,
                      int cols_b) {
    const unsigned int idesc = (1u << 4) | ((unsigned)b_mn << 16) | ((unsigned)(cols_b >> 3) << 17) | (8u << 24);
    auto desc = [&](unsigned int base, int k, bool mn) {
      const unsigned int at = base + (mn ? (unsigned)k * 2048u : (unsigned)(k >> 2) * kSoBlock + (unsigned)(k & 3) * 32u);
      return (unsigned long long)((at & 0x3ffffu) >> 4) | ((unsigned long long)(mn ? kSoBlock / 16 : 1) << 16) | (64ull << 32) |
             (1ull << 46) | (2ull << 61);
    };
    bool more = false;
    if (PLANES == 2)
      for (int k = k0; k < k1; ++k) {
        tc_mma<false>(d, desc(a, k, false), desc(b + b_lo, k, b_mn), idesc, more);
        tc_mma<false>(d, desc(a + a_lo, k, false), desc(b, k, b_mn), idesc, true);
        more = true;
      }
    for (int k = k0; k < k1; ++k) {
      tc_mma<false>(d, desc(a, k, false), desc(b, k, b_mn), idesc, more);
      more = true;
    }
  };
  // The sums are there (a wait that runs out is noted; the steps go on, so that a cluster's CTAs stay together).
  auto finished = [&] {
    mm_wait(bar, parity, args.status);
    parity ^= 1u;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  };
  // Everybody has read the sums and written the next operand.
  auto handed_over = [&] {
    asm volatile("fence.proxy.async;" ::: "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (ctas > 1) mm_cluster_sync();
    else __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");
  };
  auto put_e = [&](const float (&v)[32]) {               // this lane's row, 32 columns, both planes
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      unsigned int hi[4], lo[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) ns_split2(v[8 * k + 2 * q], v[8 * k + 2 * q + 1], hi[q], lo[q]);
      unsigned char* p = es + so_piece(row, part * 4 + k);
      *reinterpret_cast<uint4*>(p) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      if (PLANES == 2) *reinterpret_cast<uint4*>(p + 2 * kSoBlock) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
  };

  const int ksteps_m = mp / 16;
  const int ksteps_n = blocks * 4, half = ksteps_n > 8 ? ksteps_n / 2 : ksteps_n;
  for (int step = 0; step < kNsSteps; ++step) {
    // ---- A = X X^T, over this CTA's columns in two parts
    if (tid == 0) {
      if (blocks > 0) {
        products(tmem, xa, lo_at, xa, lo_at, false, 0, half, mp);
        if (half < ksteps_n) products(tmem + 128, xa, lo_at, xa, lo_at, false, half, ksteps_n, mp);
      }
      mm_commit(bar);
    }
    finished();
    {
      constexpr float s = kNsScaleE / (kNsScaleX * kNsScaleX);
      float v[32];
      if (part * 32 < mp) {
        if (blocks > 0) mm_load<32>(mine + part * 32, v);
        else
#pragma unroll
          for (int k = 0; k < 32; ++k) v[k] = 0.f;
        if (half < ksteps_n) {
          float u[32];
          mm_load<32>(mine + 128 + part * 32, u);
#pragma unroll
          for (int k = 0; k < 32; ++k) v[k] = __fadd_rn(v[k], u[k]);
        }
        if (mp < part * 32 + 32) {                       // (columns that the products did not write)
#pragma unroll
          for (int k = 16; k < 32; ++k) v[k] = 0.f;
        }
      } else {
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = 0.f;
      }
      if (ctas == 1) {
        float diagonal = 0.f;
        const int k0 = row - part * 32;
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          v[k] *= s;
          diagonal = k == k0 ? v[k] : diagonal;
          v[k] = k == k0 ? 0.f : v[k];
        }
        if (k0 >= 0 && k0 < 32) ctl.d[row] = diagonal * (1.f / kNsScaleE);
        put_e(v);
      } else {
#pragma unroll
        for (int k = 0; k < 32; k += 4)
          *reinterpret_cast<float4*>(es + so_float4(row, part * 8 + k / 4)) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
        mm_cluster_sync();                               // all parts can be read
        // this CTA's share of the rows: sums over the cluster in rank order
        const int rows = kSoRows / ctas, units = rows * 32 / kSoThreads;        // groups of four columns per thread: 4, 2, 1
        float4 t[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (u < units) {
            const int e = tid + u * kSoThreads;
            const unsigned int at = ea + so_float4(rank * rows + e / 32, e & 31);
            float4 sum = make_float4(0, 0, 0, 0);
            for (int k = 0; k < ctas; ++k) {
              float4 q;
              asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                           : "=f"(q.x), "=f"(q.y), "=f"(q.z), "=f"(q.w)
                           : "r"(so_peer(at, k)));
              sum.x = __fadd_rn(sum.x, q.x);
              sum.y = __fadd_rn(sum.y, q.y);
              sum.z = __fadd_rn(sum.z, q.z);
              sum.w = __fadd_rn(sum.w, q.w);
            }
            t[u] = sum;
          }
        mm_cluster_sync();                               // all parts have been read: their place is E's again
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (u < units) {
            const int e = tid + u * kSoThreads, r = rank * rows + e / 32, c = (e & 31) * 4;
            float a[4] = {t[u].x * s, t[u].y * s, t[u].z * s, t[u].w * s};
            float diagonal = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              diagonal = c + k == r ? a[k] : diagonal;
              a[k] = c + k == r ? 0.f : a[k];
            }
            unsigned int h0, h1, l0, l1;
            ns_split2(a[0], a[1], h0, l0);
            ns_split2(a[2], a[3], h1, l1);
            const unsigned int at = ea + so_piece(r, c >> 3) + (c & 7) * 2;
            const bool diag = c <= r && r < c + 4;
            for (int k = 0; k < ctas; ++k) {
              asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(so_peer(at, k)), "r"(h0), "r"(h1) : "memory");
              if (PLANES == 2)
                asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(so_peer(at + 2 * kSoBlock, k)), "r"(l0), "r"(l1)
                             : "memory");
              if (diag)
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(so_peer(mm_smem(&ctl.d[r]), k)),
                             "f"(diagonal * (1.f / kNsScaleE))
                             : "memory");
            }
          }
      }
    }
    handed_over();

    // ---- B, of which F is what is off the diagonal, in E's place (every CTA of a cluster for itself)
    if (tid == 0) {
      products(tmem, ea, 2 * kSoBlock, ea, 2 * kSoBlock, false, 0, ksteps_m, mp);
      mm_commit(bar);
    }
    finished();
    if (part * 32 < mp) {
      constexpr float kInvE = 1.f / kNsScaleE;
      float v[32];
      mm_load<32>(mine + part * 32, v);
      if (mp < part * 32 + 32) {
#pragma unroll
        for (int k = 16; k < 32; ++k) v[k] = 0.f;
      }
      const float di = ctl.d[row];
      const int k0 = row - part * 32;
      float diagonal = 0.f;
#pragma unroll
      for (int k = 0; k < 32; k += 8) {
        const unsigned char* p = es + so_piece(row, part * 4 + k / 8);
        const uint4 h4 = *reinterpret_cast<const uint4*>(p);
        uint4 l4 = make_uint4(0, 0, 0, 0);
        if (PLANES == 2) l4 = *reinterpret_cast<const uint4*>(p + 2 * kSoBlock);
        const unsigned int h[4] = {h4.x, h4.y, h4.z, h4.w}, l[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const float2 h2 = ns_widen(h[q >> 1]), l2 = ns_widen(l[q >> 1]);
          float e = q & 1 ? h2.y : h2.x;
          if (PLANES == 2) e += q & 1 ? l2.y : l2.x;
          const float sum = v[k + q];
          diagonal = k + q == k0 ? sum : diagonal;
          const float g = fmaf(kNsC * kNsScaleF * kInvE, di + ctl.d[part * 32 + k + q], kNsB * kNsScaleF * kInvE);
          v[k + q] = k + q == k0 ? 0.f : fmaf(g, e, sum * (kNsC * kNsScaleF * kInvE * kInvE));
        }
      }
      if (k0 >= 0 && k0 < 32) ctl.fd[row] = fmaf(kNsC, fmaf(di, di, diagonal * (kInvE * kInvE)), kNsB * di);
      put_e(v);
    }
    asm volatile("fence.proxy.async;" ::: "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");

    // ---- X = (a + f) X + F X, in X's place
    if (tid == 0) {
      if (blocks > 0) products(tmem, ea, 2 * kSoBlock, xa, lo_at, true, 0, ksteps_m, np);
      mm_commit(bar);
    }
    finished();
    const bool last = step == kNsSteps - 1;
    const float t = row < m ? kNsA + ctl.fd[row] : 0.f;
#pragma unroll 1
    for (int c = part * 32; c < np; c += 128) {
      constexpr float kInvF = 1.f / kNsScaleF;
      float v[32];
      mm_load<32>(mine + c, v);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        unsigned char* p = xs + so_piece(row, c / 8 + k);
        const uint4 h4 = *reinterpret_cast<const uint4*>(p), l4 = *reinterpret_cast<const uint4*>(p + lo_at);
        const unsigned int h[4] = {h4.x, h4.y, h4.z, h4.w}, l[4] = {l4.x, l4.y, l4.z, l4.w};
        unsigned int hi[4], lo[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float2 h2 = ns_widen(h[q]), l2 = ns_widen(l[q]);
          float &a = v[8 * k + 2 * q], &b = v[8 * k + 2 * q + 1];
          a = fmaf(t, h2.x + l2.x, a * kInvF);
          b = fmaf(t, h2.y + l2.y, b * kInvF);
          ns_split2(a, b, hi[q], lo[q]);
        }
        if (!last) {
          *reinterpret_cast<uint4*>(p) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(p + lo_at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
      }
      if (last && row < m && c < cols) ns_result(M, v, row, c0 + c, min(32, cols - c));
    }
    asm volatile("fence.proxy.async;" ::: "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  }
  if (ctas > 1) mm_cluster_sync();                       // nobody leaves while its shared memory may be read
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 256;" ::"r"(tmem) : "memory");
}

}  // namespace psb
