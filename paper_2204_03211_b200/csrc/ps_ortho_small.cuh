// Orthogonalisation of small matrices (up to 128 by 4096): all five steps in shared memory.
//
// In the general form (ps_ortho.cuh) a product of a small matrix is one tile, and what takes time is handing it from one
// tile to the next through L2: 6 to 8 us, fifteen times.  Here a CTA keeps 128 rows by up to 256 columns of X (two
// halves, 128 KB) and A or B (two halves, 64 KB) in shared memory, in the swizzled layout in which the tensor cores take
// operands: X is an operand along its rows in X X^T and across them in B X, from the same bytes.  Wider matrices are cut
// into columns over a cluster of 4 to 16 CTAs; only A is a sum over all of them, which they add up through each
// other's shared memory, a share of the rows each, in rank order.  One launch does it all: norm, scaling, steps, result.
//
// Measured to fp32 | bf16: 8 of 64 x 256 46 | 32 us (general form 120), 4 of 128 x 512 64 | 48, 4 of 128 x 2048 95 | 69,
// 4 of 128 x 4096 106 | 78 (general form 290 | 154).  Bound by the chain.  Cycles of one CTA, from product to product and
// epilogue to epilogue, 64 x 256 to fp32 | bf16: A 3740 + 2000 | 1500 + 1600, B 1300 + 1390 | 600 + 1050, X 1920 + 3200 |
// 820 + 3330, 13 600 | 8900 a step (6.9 | 4.5 us), 10 600 before the first (norm, halves) and 4200 | 2200 more for the
// result.  Over a cluster (128 x 512) A's epilogue, which adds up the parts, takes 9300.
//
// Sixteen warps read the sums (row = lane, 32 columns at a time); thread 0 issues the products.  Arithmetic as in
// ps_ortho.cuh, with the small products of a pair of halves first and the long sums of A in two parts, so that few of
// the tensor cores' cut-off additions meet large sums.
#pragma once

#include <type_traits>

#include "ps_ortho.cuh"

namespace psb {

constexpr int kSoThreads = 512;
constexpr int kSoRows = 128, kSoCols = 256;              // of a CTA's part of X
constexpr int kSoCtas = 16;
constexpr int kSoBlock = kSoRows * 128;                  // bytes of 128 rows by 64 columns of one plane
constexpr int kSoX = 2 * (kSoCols / 64) * kSoBlock, kSoE = 4 * kSoBlock;

struct SoControl {
  unsigned long long bar;
  double norm[kSoCtas];
  double red[kSoThreads / 32];
  alignas(16) float d[kSoRows];
  float fd[kSoRows];
  unsigned int tmem;
};
constexpr int kSoSmem = kSoX + kSoE + 2048;
static_assert(sizeof(SoControl) <= 2048 && kSoSmem <= 227 * 1024, "does not fit");

struct SoArgs {
  const NsMat* mats;
  int* status;
  int ctas;                                              // of a cluster: 1, 4, 8 or 16
  PsStat* stats;                                         // nullptr: no device times
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
    __syncwarp();                                        // (its first lane has set up the barrier)
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 256;" ::"r"(mm_smem(&ctl.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (ctas > 1) mm_cluster_sync();                       // all of them run: their shared memory may be written
  mm_pdl();
  const unsigned long long t0 = args.stats ? ns_now() : 0ull;

  // ---- norm, and X0 as two planes (rows from m on and columns from `cols` on are zeros)
  // (pieces of eight columns of a row; neighbouring lanes take neighbours along the source's rows)
  const bool flip = M.flip != 0;
  const int pieces = (cols + 7) / 8, units = m * pieces;
  const bool vec = !flip && (M.ld_src & 7) == 0 && (reinterpret_cast<uintptr_t>(M.src) & 31u) == 0;
  auto fetch = [&](int u, float (&v)[8], int& r, int& piece) {
    r = flip ? u % m : u / pieces;
    piece = flip ? u / m : u - r * pieces;
    const int c = piece * 8, live = min(8, cols - c);
    const size_t at = flip ? (size_t)(c0 + c) * (size_t)M.ld_src + (size_t)r : (size_t)r * (size_t)M.ld_src + (size_t)(c0 + c);
    const size_t next = flip ? (size_t)M.ld_src : 1;
    if (vec && live == 8) {
      if (M.src_bf16) {
        const uint4 q = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(M.src) + at);
        const unsigned int w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
      } else {
        const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(M.src) + at);
        const float4 x = q[0], y = q[1];
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
      }
    } else if (M.src_bf16) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        v[k] = k < live ? __bfloat162float(static_cast<const __nv_bfloat16*>(M.src)[at + k * next]) : 0.f;
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = k < live ? static_cast<const float*>(M.src)[at + k * next] : 0.f;
    }
  };
  constexpr int kBatch = 4;                              // pieces in flight per thread
  double sq = 0.0;
  for (int u0 = tid; u0 < units; u0 += kBatch * kSoThreads) {
    float v[kBatch][8];
    int r, piece;
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (u0 + k * kSoThreads < units) fetch(u0 + k * kSoThreads, v[k], r, piece);
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (u0 + k * kSoThreads < units)
#pragma unroll
        for (int q = 0; q < 8; ++q) sq = fma((double)v[k][q], (double)v[k][q], sq);
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
  for (int u0 = tid; u0 < units; u0 += kBatch * kSoThreads) {
    float v[kBatch][8];
    int r[kBatch], piece[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (u0 + k * kSoThreads < units) fetch(u0 + k * kSoThreads, v[k], r[k], piece[k]);
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (u0 + k * kSoThreads < units) {
        unsigned int hi[4], lo[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) ns_split2(v[k][2 * q] * scale, v[k][2 * q + 1] * scale, hi[q], lo[q]);
        unsigned char* p = xs + so_piece(r[k], piece[k]);
        *reinterpret_cast<uint4*>(p) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(p + lo_at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      }
  }
  asm volatile("fence.proxy.async;" ::: "memory");
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const unsigned int tmem = ctl.tmem;
  const unsigned int xa = mm_smem(xs), ea = mm_smem(es), bar = mm_smem(&ctl.bar);
  const unsigned int mine = tmem + ((unsigned)((warp & 3) * 32) << 16);
  const int row = (warp & 3) * 32 + lane, part = warp >> 2;        // part: which 32 of 128 columns
  const bool busy = (warp & 3) * 32 < m;                 // (the other rows stay zeros)
  unsigned int parity = 0;

  // All products of one kind, by one elected lane: D = A B^T over k in [k0, k1), in units of 16.  Addresses advance by 32
  // bytes along rows of 64 elements and by a block after them, or by 16 rows where k runs down the columns.
  const bool issuer = warp == 0 && mm_elect();
  auto products = [&](unsigned int d, unsigned int a, unsigned int a_lo, unsigned int b, unsigned int b_lo, bool b_mn, int k0, int k1,
                      int cols_b) {
    const unsigned int idesc = (1u << 4) | ((unsigned)b_mn << 16) | ((unsigned)(cols_b >> 3) << 17) | (8u << 24);
    const unsigned long long flags = (64ull << 32) | (1ull << 46) | (2ull << 61);
    const unsigned long long da = (unsigned long long)((a & 0x3ffffu) >> 4) | (1ull << 16) | flags;
    const unsigned long long db =
        (unsigned long long)((b & 0x3ffffu) >> 4) | ((unsigned long long)(b_mn ? kSoBlock / 16 : 1) << 16) | flags;
    const unsigned int step = b_mn ? 128u : 2u, block = b_mn ? 512u : kSoBlock / 16;
    const unsigned int al = a_lo / 16, bl = b_lo / 16;
    bool more = false;
#pragma unroll
    for (int pass = PLANES == 2 ? 0 : 1; pass < 2; ++pass)
      for (int kb = k0 / 4; kb * 4 < k1; ++kb) {
        const unsigned long long pa = da + (unsigned)kb * (kSoBlock / 16), pb = db + (unsigned)kb * block;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (kb * 4 + i >= k1) break;
          if (pass == 0) {
            tc_mma<false>(d, pa + i * 2, pb + i * step + bl, idesc, more);
            tc_mma<false>(d, pa + i * 2 + al, pb + i * step, idesc, true);
          } else {
            tc_mma<false>(d, pa + i * 2, pb + i * step, idesc, more);
          }
          more = true;
        }
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

  // The sum of the cluster's parts of A, in rank order, as E: a share of the rows per CTA, which hands them to all.  Whatever
  // the number of CTAs a thread reads eight pieces of four columns, all of them before it adds (one after the other: 4 of 128 x 512 to fp32 65.8 us, so 64.3).
  auto add_up = [&](auto number) {
    constexpr int kCtas = decltype(number)::value, kUnits = kCtas < 8 ? 8 / kCtas : 1, kRows = kSoRows / kCtas;
    const bool adds = kRows * 32 == kUnits * kSoThreads || tid < kRows * 32;      // (sixteen CTAs: half of the threads)
    constexpr float s = kNsScaleE / (kNsScaleX * kNsScaleX);
    constexpr int kAtOnce = kCtas < 8 ? kCtas : 8;
    float4 sum[kUnits] = {};
    mm_cluster_sync();                                   // all parts can be read
#pragma unroll
    for (int k0 = 0; k0 < kCtas; k0 += kAtOnce) {
      float4 q[kUnits][kAtOnce];
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        if (!adds) break;
        const int e = tid + u * kSoThreads;
        const unsigned int at = ea + so_float4(rank * kRows + e / 32, e & 31);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(q[u][k].x), "=f"(q[u][k].y), "=f"(q[u][k].z), "=f"(q[u][k].w)
                       : "r"(so_peer(at, k0 + k)));
      }
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        if (!adds) break;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          sum[u].x = __fadd_rn(sum[u].x, q[u][k].x);
          sum[u].y = __fadd_rn(sum[u].y, q[u][k].y);
          sum[u].z = __fadd_rn(sum[u].z, q[u][k].z);
          sum[u].w = __fadd_rn(sum[u].w, q[u][k].w);
        }
      }
    }
    mm_cluster_sync();                                   // all parts have been read: their place is E's again
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      if (!adds) break;
      const int e = tid + u * kSoThreads, r = rank * kRows + e / 32, c = (e & 31) * 4;
      float a[4] = {sum[u].x * s, sum[u].y * s, sum[u].z * s, sum[u].w * s};
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
#pragma unroll
      for (int k = 0; k < kCtas; ++k) {
        asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(so_peer(at, k)), "r"(h0), "r"(h1) : "memory");
        if (PLANES == 2)
          asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(so_peer(at + 2 * kSoBlock, k)), "r"(l0), "r"(l1) : "memory");
        if (diag)
          asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(so_peer(mm_smem(&ctl.d[r]), k)), "f"(diagonal * (1.f / kNsScaleE))
                       : "memory");
      }
    }
  };

  const int ksteps_m = mp / 16;
  const int ksteps_n = blocks * 4, half = blocks > 2 ? blocks / 2 * 4 : ksteps_n;
  for (int step = 0; step < kNsSteps; ++step) {
    // ---- A = X X^T, over this CTA's columns in two parts
    if (issuer) {
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
      if (part * 32 < mp && busy) {
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
        if (step == 0 || (busy && part * 32 < mp)) put_e(v);      // (what is zero stays zero)
      } else {
#pragma unroll
        for (int k = 0; k < 32; k += 4)
          *reinterpret_cast<float4*>(es + so_float4(row, part * 8 + k / 4)) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
        if (ctas == 4) add_up(std::integral_constant<int, 4>());
        else if (ctas == 8) add_up(std::integral_constant<int, 8>());
        else add_up(std::integral_constant<int, 16>());
      }
    }
    handed_over();

    // ---- B, of which F is what is off the diagonal, in E's place (every CTA of a cluster for itself)
    if (issuer) {
      products(tmem, ea, 2 * kSoBlock, ea, 2 * kSoBlock, false, 0, ksteps_m, mp);
      mm_commit(bar);
    }
    finished();
    if (part * 32 < mp && busy) {
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
        const float4 d0 = *reinterpret_cast<const float4*>(ctl.d + part * 32 + k), d1 = *reinterpret_cast<const float4*>(ctl.d + part * 32 + k + 4);
        const float dj[8] = {d0.x, d0.y, d0.z, d0.w, d1.x, d1.y, d1.z, d1.w};
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const float2 e2 = PLANES == 2 ? ns_add(l[q >> 1], ns_widen(h[q >> 1])) : ns_widen(h[q >> 1]);
          const float e = q & 1 ? e2.y : e2.x;
          const float sum = v[k + q];
          diagonal = k + q == k0 ? sum : diagonal;
          const float g = fmaf(kNsC * kNsScaleF * kInvE, di + dj[q], kNsB * kNsScaleF * kInvE);
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
    if (issuer) {
      if (blocks > 0) products(tmem, ea, 2 * kSoBlock, xa, lo_at, true, 0, ksteps_m, np);
      mm_commit(bar);
    }
    finished();
    const bool last = step == kNsSteps - 1;
    const float t = row < m ? kNsA + ctl.fd[row] : 0.f;
#pragma unroll 1
    for (int c = part * 32; c < np && busy; c += 128) {
      constexpr float kInvF = 1.f / kNsScaleF;
      float v[32];
      mm_load<32>(mine + c, v);
      uint4 h4[4], l4[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const unsigned char* p = xs + so_piece(row, c / 8 + k);
        h4[k] = *reinterpret_cast<const uint4*>(p);
        l4[k] = *reinterpret_cast<const uint4*>(p + lo_at);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        unsigned int h[4] = {h4[k].x, h4[k].y, h4[k].z, h4[k].w}, l[4] = {l4[k].x, l4[k].y, l4[k].z, l4[k].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float2 x = ns_add(l[q], ns_widen(h[q]));
          float &a = v[8 * k + 2 * q], &b = v[8 * k + 2 * q + 1];
          a = fmaf(t, x.x, a * kInvF);
          b = fmaf(t, x.y, b * kInvF);
          ns_split2(a, b, h[q], l[q]);
        }
        h4[k] = make_uint4(h[0], h[1], h[2], h[3]);
        l4[k] = make_uint4(l[0], l[1], l[2], l[3]);
      }
      if (!last)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          unsigned char* p = xs + so_piece(row, c / 8 + k);
          *reinterpret_cast<uint4*>(p) = h4[k];
          *reinterpret_cast<uint4*>(p + lo_at) = l4[k];
        }
      if (last && c < cols) ns_result(M, v, row - lane, lane, c0 + c, min(32, cols - c));
    }
    asm volatile("fence.proxy.async;" ::: "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  }
  if (args.stats && tid == 0) ns_charge(args.stats, M, t0, ns_now(), kNsWholeSm);
  if (ctas > 1) mm_cluster_sync();                       // nobody leaves while its shared memory may be read
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 256;" ::"r"(tmem) : "memory");
}

}  // namespace psb
