// Orthogonalisation of matrices by five Newton-Schulz steps, the heart of Muon's update:
//     X = G / (|G| + 1e-7)   (Frobenius norm),   five times:   A = X X^T,  B = b A + c A A,  X = a X + B X
// for m x n matrices with m <= n; taller ones are worked on as their transposes.
//
// Three products per step and 15 per matrix, each needing the one before it, for a list of matrices at once.  All of
// them run in ONE cooperative launch of the frame of ps_tc.cuh: every tile names the matrix and the product it belongs
// to, tiles are listed step by step, and a tile waits until its matrix's earlier products are done (one counter per
// matrix).  The host deals the tiles out, each to the CTA that has least to do so far, and every CTA works on its own in
// the order of all: the first unfinished tile of all is always the next one of its CTA, so every wait ends;
// there is no barrier over the grid, and one matrix's wait is another one's work.  A and B are symmetric: where the tiles
// outnumber the CTAs only those on and below the diagonal are computed, and stored twice.
//
// Measured: 24 of 1024 x 4096 to bf16 1.85 ms cool (1 PFLOP/s, tensor cores 65 % busy; X in two halves, 400 MB, comes from
// HBM for every product, 6.4 GB in all), 2.2 to 2.5 ms in a row under the power cap, to fp32 4.4 to 4.8 ms; 24 of 512 x 512 to bf16
// 165 us and 3 of 777 x 300 to fp32 187 us, bound by the latency of fifteen products in a row.
//
// Arithmetic.  Operands are fp16 (11 bits) scaled by powers of two, sums are binary32.
//  - The largest entries of A and B stand on their diagonals, and the last steps subtract them from a; they are
//    kept apart in binary32 and enter in the epilogues (A A = E E + (d_i + d_j) E + d^2, and (a + f_i) X + F X), where E
//    and F are what is off the diagonal.  One rounding of the whole B costs four times the error.
//  - X is kept as high + low halves (22 bits).  Directions that the gradient hardly has grow by a^5 = 485, and with
//    them whatever X was rounded to: with 11 bits a matrix of falling singular values comes out 2 % wrong.
//  - Results in bf16 take one product, of the high halves: 5e-4 to 1e-3 of the result's norm (its own rounding is
//    1.7e-3).  Results in binary32, and the service's update, also split E and F and take three (high x high, high x
//    low, low x high): what is left is the rounding of the tensor cores' sums.
// Scales: X by 2^15 (singular values, and so entries, are at most 1.21), E by 2^15 (at most 1.47), F by 2^14 (at most
// 2.9): the largest powers of two that overflow nothing, because small entries beside large ones lose bits at fp16's
// subnormal end.
#pragma once

#include <cuda_fp16.h>

#include "ps_ortho.h"
#include "ps_tc.cuh"

namespace psb {

constexpr int kNsSteps = 5;
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr double kNsEps = 1e-7;
constexpr float kNsScaleX = 32768.f, kNsScaleE = 32768.f, kNsScaleF = 16384.f;

constexpr int kNsMaps = 20, kNsTall = 8, kNsMirror = 16;

struct NsMat {                           // one matrix, in its working orientation: m <= n
  int m, n;
  int flip;                              // 1: source and result are the transposes
  int mirror;                            // 1: symmetric products compute the lower tiles and store them twice
  int out;                               // kNsOut*
  long long pitch_x, pitch_e;            // elements; multiples of 64
  __half* x[2][2];                       // two buffers of two planes: a step reads one and writes the other
  __half* e[2];                          // planes of what is off A's diagonal; the second where products are split
  __half* f[2];                          // and off B's
  float *d, *fd;                         // the diagonals
  // Two planes each: x[0], x[1], e, f by 64 x 64 (one product: operands) or x[0], x[1] by 32 x 64 (three: transposed
  // operands); x[0], x[1], e, f by 128 x 32 (kNsTall: the epilogues', and three products' operands); e, f by 32 x 32
  // (kNsMirror).
  const CUtensorMap* maps;
  const void* src;                       // rows x cols as the caller sees them
  long long ld_src;
  int src_bf16;
  int nparts;
  double* parts;                         // partial sums of squares
  void* dst;
  long long ld_dst;
  int wide;                              // rows of dst allow 256-bit accesses
  float decay, step;                     // kNsOutUpdate: dst = dst * decay - step * O
  int parts_s, parts_x;                  // what `done` counts in a symmetric product and in the last one
  unsigned int* done;                    // CTAs' finished parts of tiles (those that have rows of the matrix)
  unsigned int stat;                     // its record of device times
};

struct NsTile {                          // one tile of the list
  int mat;
  short step, product;                   // product 0: A, 1: B, 2: X
  int ti, tj;
};

struct NsArgs {
  int* status;
  const NsMat* mats;
  const NsTile* list;                    // CTA after CTA (or pair), each with its tiles in their common order
  const int* begin;                      // where each one's start, and the end
  PsStat* stats;                         // nullptr: no device times
};

// Adds the time since t0 to a matrix's record.  The unit is the time of one of four CTAs on an SM, as in the aggregates of
// other blocks, so that tasks of all kinds can be weighed against each other: a CTA that has an SM to itself counts four times.
constexpr unsigned int kNsWholeSm = 4;
__device__ __forceinline__ unsigned long long ns_now() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
__device__ __forceinline__ void ns_charge(PsStat* stats, const NsMat& M, unsigned long long t0, unsigned long long t1, unsigned int units) {
  atomicAdd(&stats[M.stat].busy_ns, (t1 - t0) * units);
  atomicMax(&stats[M.stat].t_last, t1);
}

// c + a and c - a for the lower and the upper of two fp16 numbers: mixed-precision additions widen as they add.
__device__ __forceinline__ float2 ns_add(unsigned int a, float2 c) {
  float2 r;
  asm("{\n\t"
      ".reg .b16 l, h;\n\t"
      "mov.b32 {l, h}, %2;\n\t"
      "add.rn.f32.f16 %0, l, %3;\n\t"
      "add.rn.f32.f16 %1, h, %4;\n\t"
      "}"
      : "=f"(r.x), "=f"(r.y)
      : "r"(a), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ float2 ns_sub(unsigned int a, float2 c) { return ns_add(a ^ 0x80008000u, c); }

// Two values as high and low halves: fp16 numbers whose sums they are (to 22 bits).
__device__ __forceinline__ void ns_split2(float a, float b, unsigned int& hi, unsigned int& lo) {
  const __half2 h = __floats2half2_rn(a, b);
  hi = *reinterpret_cast<const unsigned int*>(&h);
  const float2 r = ns_sub(hi, make_float2(a, b));
  const __half2 l = __floats2half2_rn(r.x, r.y);
  lo = *reinterpret_cast<const unsigned int*>(&l);
}
__device__ __forceinline__ void ns_split(float v, __half& hi, __half& lo) {
  hi = __float2half_rn(v);
  lo = __float2half_rn(v - __half2float(hi));
}
__device__ __forceinline__ float2 ns_widen(unsigned int u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }

// The last step's result, scaled: a warp's rows i0 ... and columns j ..., `cols` of them, a row per lane.  Where dst's rows
// allow it a lane stores along its row; else the warp's lanes store neighbours, down the columns of a dst that lies the
// other way, or along the rows after an exchange.
__device__ __forceinline__ void ns_result(const NsMat& M, float (&v)[32], int i0, int lane, int j, int cols) {
  constexpr float s = 1.f / kNsScaleX;
  const bool update = M.out == kNsOutUpdate;
  const float decay = M.decay, rate = M.step;
#pragma unroll
  for (int k = 0; k < 32; ++k) v[k] *= s;
  if (M.wide && cols >= 32) {
    if (i0 + lane >= M.m) return;
    const size_t at = (size_t)(i0 + lane) * (size_t)M.ld_dst + (size_t)j;
    if (M.out == kNsOutBf16) {
      __nv_bfloat16* p = static_cast<__nv_bfloat16*>(M.dst) + at;
      unsigned int u[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) u[k] = mm_bf16x2(v[2 * k], v[2 * k + 1]);
      store_sector(p, u);
      store_sector(p + 16, u + 8);
      return;
    }
    float* p = static_cast<float*>(M.dst) + at;
    if (update) {
#pragma unroll
      for (int k = 0; k < 32; k += 4) {
        const float4 q = *reinterpret_cast<const float4*>(p + k);
        v[k] = q.x * decay - rate * v[k];
        v[k + 1] = q.y * decay - rate * v[k + 1];
        v[k + 2] = q.z * decay - rate * v[k + 2];
        v[k + 3] = q.w * decay - rate * v[k + 3];
      }
    }
#pragma unroll
    for (int k = 0; k < 32; k += 8) store_sector(p + k, reinterpret_cast<const unsigned int*>(v) + k);
    return;
  }
  if (!M.flip) tc_exchange(v, lane);
  const int rows = min(32, M.m - i0), count = M.flip ? cols : rows;
  if (lane >= (M.flip ? rows : cols)) return;
  const size_t ld = (size_t)M.ld_dst, at = (M.flip ? (size_t)j * ld + (size_t)i0 : (size_t)i0 * ld + (size_t)j) + (size_t)lane;
  if (M.out == kNsOutBf16) {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(M.dst) + at;
#pragma unroll
    for (int k = 0; k < 32; ++k)
      if (k < count) p[k * ld] = __float2bfloat16_rn(v[k]);
    return;
  }
  float* p = static_cast<float*>(M.dst) + at;
  if (update) {                          // (sixteen loads before the first store: a round of two layers 36 wide 102 us, so 64)
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
      float q[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) q[k] = h + k < count ? p[(h + k) * ld] : 0.f;
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (h + k < count) p[(h + k) * ld] = q[k] * decay - rate * v[h + k];
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < 32; ++k)
    if (k < count) p[k * ld] = v[k];
}

template <int PLANES, bool PAIR>
struct NsOp {
  static constexpr bool kPair = PAIR, kSide = false;
  static constexpr int kWarps = 8;
  static constexpr int kPlanes = PLANES, kType = 0, kTile = PAIR ? 256 : 128, kColumns = kTile / 2;
  // Three products of a stage take three times as long as one, so they need short stages to have enough of them (long |
  // short: 24 x 1024 x 4096 to fp32 4.86 | 4.44 ms); a single one is slowed by 64-byte rows (to bf16 2.46 | 2.63 ms).
  static constexpr int kSlots = 2, kK = PLANES == 2 ? 32 : 64, kStages = 4;
  static constexpr int kSegment = PLANES == 1 ? 0 : PAIR ? 8 : 4;
  using Args = NsArgs;

  static __device__ __forceinline__ void tiles(const NsArgs& a, int mine, int, int* first, int* end, int* stride) {
    *first = a.begin[mine];
    *end = a.begin[mine + 1];
    *stride = 1;
  }

  using Item = NsTile;

  static __device__ __forceinline__ Item item(const NsArgs& a, int index, int tiles) { return a.list[max(0, min(index, tiles - 1))]; }

  static __device__ __forceinline__ int stages(const NsArgs& a, const NsTile& at) {
    const NsMat& M = a.mats[at.mat];
    return ((at.product == 0 ? M.n : M.m) + kK - 1) / kK;
  }

  // A tile waits for its matrix's earlier products.
  static __device__ __forceinline__ void tile(const NsArgs& a, const NsTile& at, TcTile* t) {
    const NsMat& M = a.mats[at.mat];
    t->ready = M.done;
    t->need = (unsigned)(at.step * (2 * M.parts_s + M.parts_x) + at.product * M.parts_s);
    t->a_row = at.ti * kTile;
    t->b_row = at.tj * kTile;
    t->a_k = t->b_k = 0;
    t->a_mn = 0;
    t->b_mn = at.product == 2;           // X's rows are k there
    const CUtensorMap *rows = M.maps + (kK == 32 ? kNsTall : 0), *x = rows + 2 * (at.step & 1), *e = rows + 4;
    t->a = at.product == 0 ? x : at.product == 1 ? e : e + 2;
    t->b = at.product == 0 ? x : at.product == 1 ? e : M.maps + 2 * (at.step & 1);
    t->nk = stages(a, at);
  }

  // ---- slots: 128 rows by 32 columns of E (product 1) or X (product 2) go in, of E, F or X come out.  Symmetric results
  // of tiles off the diagonal also go out mirrored: from the slot's second plane, or, where both planes are results,
  // from a slot of their own.

  static __device__ __forceinline__ int width(const NsMat& M, const NsTile& at) { return at.product == 2 ? M.n : M.m; }
  static __device__ __forceinline__ bool mirrored(const NsMat& M, const NsTile& at) { return M.mirror && at.product < 2 && at.ti != at.tj; }
  static __device__ __forceinline__ int per_chunk(const NsMat& M, const NsTile& at) { return PLANES == 2 && mirrored(M, at) ? 2 : 1; }

  static __device__ __forceinline__ int entries(const NsArgs& a, const NsTile& at, int rank, int half) {
    const NsMat& M = a.mats[at.mat];
    const int left = width(M, at) - (at.tj * kTile + half * kColumns);
    if (left <= 0 || at.ti * kTile + rank * 128 >= M.m) return 0;
    return min(kColumns / 32, (left + 31) / 32) * per_chunk(M, at);
  }

  static __device__ __forceinline__ void load(const NsArgs& a, const NsTile& at, int rank, int half, int entry, unsigned int slot,
                                              unsigned int vectors, unsigned int bar) {
    const NsMat& M = a.mats[at.mat];
    const int per = per_chunk(M, at), c = entry / per * 32, i0 = at.ti * kTile + rank * 128, j0 = at.tj * kTile + half * kColumns;
    if (at.product == 0 || entry % per) {                // nothing to read
      tc_arrive(bar);
      return;
    }
    const int planes = at.product == 1 ? PLANES : 2;
    const unsigned int first = entry == 0 ? (at.product == 1 ? 512 + 4 * kColumns : 512) : 0;
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(planes * kTcPlane + first) : "memory");
    if (entry == 0) {                                    // the diagonal at the rows, and at the columns
      mm_bulk(vectors, (at.product == 1 ? M.d : M.fd) + i0, 512, bar);
      if (at.product == 1) mm_bulk(vectors + 512, M.d + j0, 4 * kColumns, bar);
    }
    const CUtensorMap* map = M.maps + kNsTall + (at.product == 1 ? 4 : 2 * (at.step & 1));
    for (int p = 0; p < planes; ++p) mm_tma(slot + p * kTcPlane, map + p, j0 + c, i0, bar);
  }

  static __device__ __forceinline__ void store(const NsArgs& a, const NsTile& at, int rank, int half, int entry, unsigned int slot) {
    const NsMat& M = a.mats[at.mat];
    if (at.product == 2 && at.step == kNsSteps - 1) return;                  // (results go out from registers)
    const int per = per_chunk(M, at), c = entry / per * 32, i0 = at.ti * kTile + rank * 128, j = at.tj * kTile + half * kColumns + c;
    const bool direct = entry % per == 0, mirror = mirrored(M, at) && (PLANES == 1 || !direct);
    if (direct) {
      const CUtensorMap* map = M.maps + kNsTall + (at.product == 0 ? 4 : at.product == 1 ? 6 : 2 * ((at.step & 1) ^ 1));
      for (int p = 0; p < (at.product == 2 ? 2 : PLANES); ++p) tc_store(map + p, j, i0, slot + p * kTcPlane);
    }
    if (mirror) {
      const CUtensorMap* map = M.maps + kNsMirror + 2 * at.product;
      for (int p = 0; p < PLANES; ++p)
        for (int q = 0; q < 4; ++q)
          if (i0 + 32 * q < M.m) tc_store(map + p, i0 + 32 * q, j, slot + (PLANES == 1 ? kTcPlane : p * kTcPlane) + q * (kTcPlane / 4));
    }
  }

  static __device__ __forceinline__ void done(const NsArgs& a, const NsTile& at, int rank) {
    if (at.product == 2 && at.step == kNsSteps - 1) return;                  // (nobody waits for results)
    if (at.ti * kTile + rank * 128 >= a.mats[at.mat].m) return;              // (would count before the tile is done)
    asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(a.mats[at.mat].done) : "memory");
  }

  struct Epilogue {
    const NsTile& at;
    const NsMat& M;
    TcWarp& w;
    MmCursor<kSlots>& slot;
    int i, j0, width_;                   // this lane's row; the warp's first column, and where the columns end
    bool live, last;
    PsStat* const stats;

    __device__ __forceinline__ Epilogue(const NsArgs& a, const NsTile& item, TcWarp& warp, MmCursor<kSlots>& cursor)
        : at(item), M(a.mats[item.mat]), w(warp), slot(cursor), stats(a.stats) {}

    __device__ __forceinline__ void begin() {
      const int i0 = at.ti * kTile + w.row;
      i = i0 + w.lane;
      j0 = at.tj * kTile + w.col;
      width_ = width(M, at);
      live = (i0 & ~127) < M.m;                            // (as entries(): the CTA's rows hold something)
      if (stats && w.mark == 0) w.mark = ns_now();
      last = at.step == kNsSteps - 1;
    }

    __device__ __forceinline__ uint4* piece(int p, int k) {
      return reinterpret_cast<uint4*>(w.slots + slot.s * kTcSlot + p * kTcPlane + tc_piece_at((w.row & 127) + w.lane, k));
    }

    __device__ __forceinline__ void wait_staged() { mm_wait(w.staged + 8 * slot.s, slot.parity, w.status); }

    // The warp's part of the slot may go out.
    __device__ __forceinline__ void hand_over() {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (w.lane == 0) tc_arrive(w.filled + 8 * slot.s);
      slot.next();
    }

    // This lane's row of both planes: v as high and low halves.
    __device__ __forceinline__ void put(const float (&v)[32], bool low) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        unsigned int hi[4], lo[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) ns_split2(v[8 * k + 2 * q], v[8 * k + 2 * q + 1], hi[q], lo[q]);
        *piece(0, k) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        if (low) *piece(1, k) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      }
    }

    // The same down a column: the mirrored 32 x 32, high or low halves.
    __device__ __forceinline__ void put_mirrored(const float (&v)[32], int p, bool low) {
      unsigned char* base = w.slots + slot.s * kTcSlot + p * kTcPlane + ((w.row & 127) >> 5) * (kTcPlane / 4) + (w.lane & 7) * 2;
#pragma unroll
      for (int k = 0; k < 32; k += 2) {
        unsigned int hi, lo;
        ns_split2(v[k], v[k + 1], hi, lo);
        const unsigned int u = low ? lo : hi;
        *reinterpret_cast<unsigned short*>(base + tc_piece_at(k, w.lane >> 3)) = (unsigned short)(u & 0xffffu);
        *reinterpret_cast<unsigned short*>(base + tc_piece_at(k + 1, w.lane >> 3)) = (unsigned short)(u >> 16);
      }
    }

    // Off-diagonal entries of a symmetric matrix, already scaled, and where they mirror.
    __device__ __forceinline__ void put_symmetric(const float (&v)[32]) {
      put(v, PLANES == 2);
      if (PLANES == 1 && mirrored(M, at)) put_mirrored(v, 1, false);
      hand_over();
      if (PLANES == 2 && mirrored(M, at)) {
        wait_staged();
        put_mirrored(v, 0, false);
        put_mirrored(v, 1, true);
        hand_over();
      }
    }

    __device__ __forceinline__ void columns(float (&v)[32], int c) {
      const int j = j0 + c;
      if (!live || j >= width_) return;
      wait_staged();
      if (at.product == 0) gram(v, j);
      else if (at.product == 1) poly(v, j, c);
      else apply(v, j);
    }

    __device__ __forceinline__ void gram(float (&v)[32], int j) {
      constexpr float s = kNsScaleE / (kNsScaleX * kNsScaleX);
#pragma unroll
      for (int k = 0; k < 32; ++k) v[k] *= s;
      if (at.ti == at.tj) {
        const int k0 = i - j;
        float diagonal = 0.f;
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          diagonal = k == k0 ? v[k] : diagonal;
          v[k] = k == k0 ? 0.f : v[k];
        }
        if (k0 >= 0 && k0 < 32 && i < M.m) M.d[i] = diagonal * (1.f / kNsScaleE);
      }
      put_symmetric(v);
    }

    __device__ __forceinline__ void poly(float (&v)[32], int j, int c) {
      constexpr float kInvE = 1.f / kNsScaleE;
      const float di = w.vectors[(w.row & 127) + w.lane];
      const float* d = w.vectors + 128 + c;
      const int k0 = at.ti == at.tj ? i - j : -1;
      float diagonal = 0.f;
#pragma unroll
      for (int k = 0; k < 32; k += 8) {
        const uint4 h4 = *piece(0, k >> 3);
        uint4 l4 = make_uint4(0, 0, 0, 0);
        if constexpr (PLANES == 2) l4 = *piece(1, k >> 3);
        const float4 d0 = *reinterpret_cast<const float4*>(d + k), d1 = *reinterpret_cast<const float4*>(d + k + 4);
        const float dj[8] = {d0.x, d0.y, d0.z, d0.w, d1.x, d1.y, d1.z, d1.w};
        const unsigned int h[4] = {h4.x, h4.y, h4.z, h4.w}, l[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const float2 e2 = PLANES == 2 ? ns_add(l[q >> 1], ns_widen(h[q >> 1])) : ns_widen(h[q >> 1]);
          const float e = q & 1 ? e2.y : e2.x;
          // (b e + c (sum + (d_i + d_j) e)) in F's scale, e and sum in E's and its square
          const float sum = v[k + q];
          diagonal = k + q == k0 ? sum : diagonal;
          const float g = fmaf(kNsC * kNsScaleF * kInvE, di + dj[q], kNsB * kNsScaleF * kInvE);
          v[k + q] = k + q == k0 ? 0.f : fmaf(g, e, sum * (kNsC * kNsScaleF * kInvE * kInvE));
        }
      }
      if (k0 >= 0 && k0 < 32 && i < M.m) M.fd[i] = fmaf(kNsC, fmaf(di, di, diagonal * (kInvE * kInvE)), kNsB * di);
      if (mirrored(M, at)) __syncwarp();                    // all have read the slot before others' columns are written there
      put_symmetric(v);
    }

    __device__ __forceinline__ void apply(float (&v)[32], int j) {
      constexpr float kInvF = 1.f / kNsScaleF;
      const float t = kNsA + w.vectors[(w.row & 127) + w.lane];
#pragma unroll
      for (int k = 0; k < 32; k += 8) {
        const uint4 h4 = *piece(0, k >> 3), l4 = *piece(1, k >> 3);
        const unsigned int h[4] = {h4.x, h4.y, h4.z, h4.w}, l[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float2 x = ns_add(l[q], ns_widen(h[q]));
          v[k + 2 * q] = fmaf(t, x.x, v[k + 2 * q] * kInvF);
          v[k + 2 * q + 1] = fmaf(t, x.y, v[k + 2 * q + 1] * kInvF);
        }
      }
      if (!last) {
        put(v, true);                                    // (a lane overwrites what it has read itself)
        hand_over();
        return;
      }
      hand_over();
      if (i - w.lane < M.m) ns_result(M, v, i - w.lane, w.lane, j, min(32, M.n - j));
    }

    // (the CTA's time from tile to tile, waiting included, is the later one's)
    __device__ __forceinline__ void end() {
      if (stats && live && w.lane == 0 && w.col == 0 && (w.row & 127) == 0) {
        const unsigned long long now = ns_now();
        ns_charge(stats, M, w.mark, now, kNsWholeSm);
        w.mark = now;
      }
    }
  };
};

// ---- before the products: the norm, and X in its working form ---------------------------------------------

constexpr int kNsThreads = 256;
constexpr int kNsUnitRows = 64, kNsUnitCols = 256;       // of the source

__device__ __forceinline__ float ns_source(const NsMat& M, size_t at) {
  return M.src_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(M.src)[at]) : static_cast<const float*>(M.src)[at];
}

// Eight neighbours of a source row, `live` of them inside it (the rest zeros).  vec: 16-byte aligned pieces.
__device__ __forceinline__ void ns_fetch8(const NsMat& M, size_t at, int live, bool vec, float (&v)[8]) {
  if (vec && live >= 8) {
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
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < live ? ns_source(M, at + k) : 0.f;
  }
}
__device__ __forceinline__ bool ns_vec(const NsMat& M) {
  return (M.ld_src & 7) == 0 && (reinterpret_cast<uintptr_t>(M.src) & 15u) == 0;
}

__device__ __forceinline__ double ns_block_sum(double v) {
  __shared__ double red[kNsThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < kNsThreads / 32; ++w) v += red[w];
  return v;
}

// The unit's pieces of eight columns, four at a time in flight per thread: f(row, column, values).
template <typename F>
__device__ __forceinline__ void ns_each_piece(const NsMat& M, int r0, int c0, int rows, int cols, F f) {
  constexpr int kPieces = kNsUnitCols / 8, kBatch = 4, kRows = kNsThreads / kPieces;
  const bool vec = ns_vec(M);
  const int c = c0 + ((int)threadIdx.x % kPieces) * 8, first = (int)threadIdx.x / kPieces, live = cols - c;
  if (live <= 0) return;
#pragma unroll 1
  for (int r = first; r < kNsUnitRows; r += kBatch * kRows) {
    float v[kBatch][8];
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (r0 + r + k * kRows < rows) ns_fetch8(M, (size_t)(r0 + r + k * kRows) * (size_t)M.ld_src + (size_t)c, live, vec, v[k]);
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (r0 + r + k * kRows < rows) f(r0 + r + k * kRows, c, v[k]);
  }
}

// One unit's sum of squares, in binary64.
__global__ void __launch_bounds__(kNsThreads)
ps_ortho_norm_kernel(const NsMat* __restrict__ mats, const int2* __restrict__ units) {
  mm_pdl();
  const int2 u = units[blockIdx.x];                      // matrix, unit within it
  const NsMat& M = mats[u.x];
  const int rows = M.flip ? M.n : M.m, cols = M.flip ? M.m : M.n;
  const int across = (cols + kNsUnitCols - 1) / kNsUnitCols;
  double s = 0.0;
  ns_each_piece(M, u.y / across * kNsUnitRows, u.y % across * kNsUnitCols, rows, cols, [&](int, int, const float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 8; ++k) s = fma((double)v[k], (double)v[k], s);
  });
  s = ns_block_sum(s);
  if (threadIdx.x == 0) M.parts[u.y] = s;
}

// Eight values of a row of X as pieces of both planes; up to seven of them may lie behind the row's end, in its padding.
__device__ __forceinline__ void ns_put8(const NsMat& M, int r, int c, const float (&v)[8], float scale) {
  unsigned int hi[4], lo[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) ns_split2(v[2 * q] * scale, v[2 * q + 1] * scale, hi[q], lo[q]);
  const size_t o = (size_t)r * (size_t)M.pitch_x + (size_t)c;
  *reinterpret_cast<uint4*>(M.x[0][0] + o) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  *reinterpret_cast<uint4*>(M.x[0][1] + o) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}

// One unit of X, scaled, as two planes.
__global__ void __launch_bounds__(kNsThreads)
ps_ortho_prepare_kernel(const NsMat* __restrict__ mats, const int2* __restrict__ units, PsStat* __restrict__ stats) {
  __shared__ float tile[64][65];
  mm_pdl();
  const unsigned long long t0 = stats ? ns_now() : 0ull;
  const int2 u = units[blockIdx.x];
  const NsMat& M = mats[u.x];
  double total = 0.0;
  for (int k = (int)threadIdx.x; k < M.nparts; k += kNsThreads) total += M.parts[k];
  total = ns_block_sum(total);
  const float scale = (float)((double)kNsScaleX / (sqrt(total) + kNsEps));
  if (u.y == 0 && threadIdx.x == 0) *M.done = 0;
  const int rows = M.flip ? M.n : M.m, cols = M.flip ? M.m : M.n;
  const int across = (cols + kNsUnitCols - 1) / kNsUnitCols;
  const int r0 = u.y / across * kNsUnitRows, c0 = u.y % across * kNsUnitCols;
  if (!M.flip) {
    ns_each_piece(M, r0, c0, rows, cols, [&](int r, int c, const float (&v)[8]) { ns_put8(M, r, c, v, scale); });
    if (stats && threadIdx.x == 0) ns_charge(stats, M, t0, ns_now(), 1);
    return;
  }
  // transposed, 64 x 64 at a time: pieces along the source's rows in, along its columns out
  const bool vec = ns_vec(M);
  const int piece = (int)threadIdx.x & 7, line = (int)threadIdx.x >> 3;
  for (int part = 0; part < kNsUnitCols; part += 64) {
    const int c = c0 + part;
    if (c >= cols) break;                                // (the same for the whole CTA)
    float v[2][8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = r0 + line + 32 * k, live = min(8, cols - (c + piece * 8));
      if (r < rows && live > 0) ns_fetch8(M, (size_t)r * (size_t)M.ld_src + (size_t)(c + piece * 8), live, vec, v[k]);
      else
#pragma unroll
        for (int q = 0; q < 8; ++q) v[k][q] = 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int q = 0; q < 8; ++q) tile[line + 32 * k][piece * 8 + q] = v[k][q];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int x = line + 32 * k;                       // row of X in the tile
      if (c + x < cols && r0 + piece * 8 < rows) {
        float w[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] = tile[piece * 8 + q][x];
        ns_put8(M, c + x, r0 + piece * 8, w, scale);
      }
    }
  }
  if (stats && threadIdx.x == 0) ns_charge(stats, M, t0, ns_now(), 1);
}

}  // namespace psb
