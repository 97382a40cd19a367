// Softmax cross entropy of T tokens over V words without keeping the T x V scores, and its gradients:
//     s_tv = sum_d x_td w_vd,  lse_t = log sum_v exp(s_tv),  loss_t = lse_t - s_t,target(t)
//     d_tv = g_t (exp(s_tv - lse_t) - [v = target(t)]),  dx = d w,  dw = d^T x
//
// All four products run in the frame of ps_tc.cuh.  The losses' pass keeps of every 256 x 256 tile of scores one
// maximum and one sum of exponentials per row and warp (128 or 64 columns), which a small kernel joins.  The gradients' pass walks
// the vocabulary in pieces: the scores of a piece are computed again, turned into d (bf16) and stored; the next launch
// reads them twice, along the rows for dx and down the columns for dw, and computes the following piece's d beside it,
// so that what each launch ends with is covered by work that does not depend on it.  A piece of d takes up to
// 40 MB and so stays in L2 between its writing and its reading.
//
// Bound by the tensor cores, and in a row by power, where the width is 1024 and more: losses of 8192 x 30522 x 1024 in 318 to 331 us
// (1.55 to 1.6 PFLOP/s), both gradients in 1317 to 1340 us (three products of 2 T V D, 1.15 PFLOP/s); by the epilogues of the
// scores and the ends of launches below (2048 x 33278 x 512: 61 us, tensor cores 62 % busy, and 202 us, 34 to 54 %); by
// its launches where everything is small (37 x 500 x 64: 21 us for four).
//
// Roundings: products of bf16 values are exact and summed in binary32 by the tensor cores, whose additions cut off rather
// than round: losses and lse of 1024 wide x are off by 3.4e-7 of themselves (5e-8 with rounded additions), 512 wide by
// 1.7e-7.  Maxima, sums of exponentials, lse and losses are binary32.  What is
// stored of d is exp(s - lse) - [v = target], rounded to bf16 (it is an operand, and x and w are bf16, which one MMA wants
// of both): at most 2^-8 of each entry, of either sign, and none where it matters most, at the target of an unlikely word,
// whose -1 is exact.  The factor g_t stays out of it, because its own rounding would be the same for all of a token's
// entries (a mean over 7680 tokens came out 3.5e-3 wrong): scale enters in the epilogues, token_scale there for dx and in
// the copy of x for dw.
#pragma once

#include "ps_tc.cuh"

namespace psb {

constexpr int kXeTile = 256, kXeK = 64;

enum { kXeStats = 0, kXeProb = 1, kXeDx = 2, kXeDw = 3 };

struct XeSeg {                           // a launch's tiles of one kind, tiles_m x tiles_n (x slices)
  int kind, first, tiles_m, tiles_n;
  int v0;                                // first word of the piece
  int nk;                                // stages along k, over all slices
  int slices;                            // kXeDx, kXeDw: the words or tokens are shared out; each slice has sums of its own
  int buf;                               // which of the two pieces of d
  int start;                             // kXeDx: 1: the sums start here (else they are added to what is there)
  int finish;                            // kXeDx: 1: store dx itself
};
constexpr int kXeMaxSegs = 3;

// Copies a matrix of bf16 into rows of `pitch` elements (a multiple of eight; the rest zeros).  With targets the rows of
// ignored tokens become zeros, so that what padded places of a batch hold, NaN or not, does not reach the gradients, and
// the others are multiplied by their weight.
struct XeCopy {
  const unsigned short* src;             // nullptr: nothing to copy
  unsigned short* dst;
  long long rows, cols, ld, pitch;
  const void* targets;
  int target64;
  int wide;                              // rows of src allow 128-bit loads
  long long V;
  const float* weights;
};

__device__ __forceinline__ long long xe_target(const void* targets, int is64, long long t) {
  return is64 ? static_cast<const long long*>(targets)[t] : (long long)static_cast<const int*>(targets)[t];
}

// Eight elements at p, which lie at least eight from their row's start and sixteen from its end: two aligned loads and a
// shift by whole elements (element by element, w of 25600 x 1021 and both gradients for 128 tokens took 155 us, so 141).
__device__ __forceinline__ uint4 xe_shifted(const unsigned short* p) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  const uint4* base = reinterpret_cast<const uint4*>(at & ~(uintptr_t)15);
  const uint4 a = base[0], b = base[1];
  unsigned int u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int k = 0; k < 6; ++k) u[k] = at & 8 ? u[k + 2] : u[k];
#pragma unroll
  for (int k = 0; k < 5; ++k) u[k] = at & 4 ? u[k + 1] : u[k];
#pragma unroll
  for (int k = 0; k < 4; ++k) u[k] = at & 2 ? __funnelshift_r(u[k], u[k + 1], 16) : u[k];
  return make_uint4(u[0], u[1], u[2], u[3]);
}

// Pieces of eight elements first, first + stride, ...
__device__ __forceinline__ void xe_copy(const XeCopy& c, long long first, long long stride) {
  const unsigned int per = (unsigned int)(c.pitch / 8);
  const long long total = c.rows * per;
#pragma unroll 4
  for (long long i = first; i < total; i += stride) {
    const long long r = i / per, col = (i - r * per) * 8;
    uint4 q = make_uint4(0, 0, 0, 0);
    bool keep = true;
    if (c.targets) {
      const long long t = xe_target(c.targets, c.target64, r);
      keep = t >= 0 && t < c.V;
    }
    if (keep) {
      const unsigned short* p = c.src + (size_t)r * (size_t)c.ld + (size_t)col;
      if (c.wide && col + 8 <= c.cols) {
        q = *reinterpret_cast<const uint4*>(p);
      } else if (col >= 8 && col + 16 <= c.cols) {
        q = xe_shifted(p);
      } else {
        unsigned int u[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) u[k] = col + k < c.cols ? p[k] : 0;
        q = make_uint4(u[0] | u[1] << 16, u[2] | u[3] << 16, u[4] | u[5] << 16, u[6] | u[7] << 16);
      }
      if (c.weights) {
        const float g = c.weights[r];
        unsigned int u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = mm_bf16x2(__uint_as_float(u[k] << 16) * g, __uint_as_float(u[k] & 0xffff0000u) * g);
        q = make_uint4(u[0], u[1], u[2], u[3]);
      }
    }
    *reinterpret_cast<uint4*>(c.dst + (size_t)r * (size_t)c.pitch + (size_t)col) = q;
  }
}

struct XeArgs {
  CUtensorMap x, xm, w, d[2];            // xm: token_scale * x, the rows of ignored tokens zeroed
  int* status;
  int nseg, tiles;
  XeSeg seg[kXeMaxSegs];
  long long T, V, D;
  const void* targets;
  int target64;
  // losses' pass
  float2* parts;                         // (maximum, sum of exp(s - maximum)) per row and warp's columns, rows of nparts
  int nparts;
  float* score;                          // s_t,target(t)
  // gradients' pass
  const float* lse;
  const float* weights;                  // nullptr: 1
  float scale;
  __nv_bfloat16* d_out[2];               // T x piece
  int piece;
  float* dx_sums;                        // slices x T x pitch
  float* dw_sums;                        // slices x V x pitch, where there is more than one
  int pitch;                             // D, rounded up to a multiple of eight
  __nv_bfloat16* dx;
  void* dw;
  long long ld_dx, ld_dw;
  int dw_f32, dx_align, dw_align;        // align: bytes on whose multiples all rows start, at most 32
  XeCopy side;                           // done by warps that have nothing else to do: xm, needed from the next launch on
};

// Whether token t has a target, and g_t if it has.  An ignored one's row of dx is zeros by choice and not as a product:
// the sums of its zero entries with a row of w that holds an infinity are NaN.
__device__ __forceinline__ bool xe_factor(const void* targets, int is64, long long V, const float* weights, float scale, long long t,
                                          float* g) {
  const long long v = xe_target(targets, is64, t);
  if (v < 0 || v >= V) return false;
  *g = weights ? scale * weights[t] : scale;
  return true;
}

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float xe_exp2(float x) {      // (an argument that is far below zero gives zero)
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// A warp's 32 rows of 32 columns, a row per lane, as bf16 or binary32.  Rows from `rows` and columns from `cols` on are not
// there.  What all rows allow: 32-byte stores, 16-byte stores, or single elements.  Those are stored along the rows, after
// an exchange between the lanes: element by element down the columns every store touches 32 sectors (two tokens, 23680 x
// 952, loss and gradients: 270 us, so 77).
template <typename T>
__device__ __forceinline__ void xe_store(T* first, long long ld, float (&v)[32], int lane, int rows, int cols, int align) {
  static_assert(sizeof(T) == 2 || sizeof(T) == 4, "bf16 or binary32");
  constexpr int kWords = 8 * sizeof(T);                   // of 32 bits
  if (align >= 16 && cols >= 32) {
    if (lane >= rows) return;
    T* o = first + (size_t)lane * (size_t)ld;
    unsigned int u[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) u[i] = sizeof(T) == 4 ? __float_as_uint(v[i & 31]) : mm_bf16x2(v[(2 * i) & 31], v[(2 * i + 1) & 31]);
    if (align >= 32)
#pragma unroll
      for (int i = 0; i < kWords; i += 8) store_sector(reinterpret_cast<unsigned int*>(o) + i, u + i);
    else
#pragma unroll
      for (int i = 0; i < kWords; i += 4)
        *reinterpret_cast<uint4*>(reinterpret_cast<unsigned int*>(o) + i) = make_uint4(u[i], u[i + 1], u[i + 2], u[i + 3]);
    return;
  }
  tc_exchange(v, lane);
  if (lane >= cols) return;
#pragma unroll
  for (int i = 0; i < 32; ++i)
    if (i < rows) {
      if constexpr (sizeof(T) == 4) first[(size_t)i * (size_t)ld + lane] = v[i];
      else first[(size_t)i * (size_t)ld + lane] = __float2bfloat16_rn(v[i]);
    }
}

// Epilogue warps.  A tile's MMAs take 512 cycles per 64 elements of the width, the epilogue of a tile of scores 8800 with
// eight warps, which mostly wait for one another's results; sixteen are done sooner, but get in the way of the MMAs where
// those are what takes longest.  Eight | sixteen, us: losses of 4096 x 30000 x 128 120 | 100, losses and gradients of
// 3968 x 7658 x 512 188 | 169, losses of 1000 x 30522 x 1024 47.2 | 49.6.
constexpr long long kXeManyWarpsBelow = 768;
inline int xe_warps(long long D) { return D < kXeManyWarpsBelow ? 16 : 8; }

template <int WARPS>
struct XeOp {
  static constexpr bool kPair = true;
  static constexpr int kWarps = WARPS;
  static constexpr int kPlanes = 1, kType = 1, kK = kXeK, kStages = 6, kSlots = 0, kSegment = 0;
  static constexpr bool kSide = true;
  using Args = XeArgs;

  struct At { const XeSeg* seg; int m, n, slice; };
  using Item = int;

  static __device__ __forceinline__ At locate(const XeArgs& a, int index) {
    At at;
    int s = 0;
    while (s + 1 < a.nseg && index >= a.seg[s + 1].first) ++s;
    at.seg = &a.seg[s];
    int i = index - at.seg->first;
    const int per = at.seg->tiles_m * at.seg->tiles_n;
    at.slice = i / per;
    i -= at.slice * per;
    // groups of eight tiles along m: the tiles in flight share rows of both operands in L2
    constexpr int kGroup = 8;
    const int band = kGroup * at.seg->tiles_n, g = i / band, in = i - g * band;
    const int rows = min(kGroup, at.seg->tiles_m - g * kGroup);
    at.n = in / rows;
    at.m = g * kGroup + in - at.n * rows;
    return at;
  }

  static __device__ __forceinline__ void tiles(const XeArgs& a, int mine, int all, int* first, int* end, int* stride) {
    *first = mine;
    *end = a.tiles;
    *stride = all;
  }
  static __device__ __forceinline__ Item item(const XeArgs&, int index, int) { return index; }
  static __device__ __forceinline__ void side(const XeArgs& a, int thread, int threads) {
    if (a.side.src) xe_copy(a.side, thread, threads);
  }

  static __device__ __forceinline__ void tile(const XeArgs& a, int index, TcTile* t) {
    const At at = locate(a, index);
    const XeSeg& s = *at.seg;
    t->ready = nullptr;
    t->need = 0;
    t->a_row = at.m * kXeTile;
    t->b_row = at.n * kXeTile;
    t->a_k = t->b_k = 0;
    t->nk = s.nk;
    t->a_mn = t->b_mn = 0;
    if (s.kind <= kXeProb) {             // tokens x words, over the width
      t->a = &a.x;
      t->b = &a.w;
      t->b_row += s.v0;
      return;
    }
    // over (a slice of) the piece's words, or the tokens
    const int k0 = (int)((long long)s.nk * at.slice / s.slices), k1 = (int)((long long)s.nk * (at.slice + 1) / s.slices);
    t->nk = k1 - k0;
    t->a = &a.d[s.buf];
    t->b_mn = 1;
    t->a_k = t->b_k = k0 * kXeK;
    if (s.kind == kXeDx) {               // tokens x width
      t->b = &a.w;
      t->b_k += s.v0;
    } else {                             // words x width
      t->b = &a.xm;
      t->a_mn = 1;
    }
  }

  struct Epilogue {
    const XeArgs& a;
    const TcWarp& w;
    const At at;
    long long row, word;                 // this lane's row; the target (kXeStats, kXeProb: relative to the tile's first column)
    float m, s, g = 0.f;                 // g: kXeDx: the factor of the row's gradient
    bool counts = false;                 // the row's token has a target

    __device__ __forceinline__ Epilogue(const XeArgs& args, int index, const TcWarp& warp, MmCursor<1>&)
        : a(args), w(warp), at(locate(args, index)) {}

    __device__ __forceinline__ void begin() {
      const int kind = at.seg->kind;
      row = (long long)at.m * kXeTile + w.row + w.lane;
      if (kind == kXeDx && row < a.T) counts = xe_factor(a.targets, a.target64, a.V, a.weights, a.scale, row, &g);
      if (kind <= kXeProb) {
        word = -1;
        m = __int_as_float(0xff800000);
        s = 0.f;
        counts = false;
        if (row < a.T) {
          const long long v = xe_target(a.targets, a.target64, row);
          counts = v >= 0 && v < a.V;
          if (counts) word = v - (at.seg->v0 + (long long)at.n * kXeTile);
          if (kind == kXeProb && counts) m = a.lse[row];
        }
      }
    }

    __device__ __forceinline__ void columns(float (&v)[32], int c) {
      c += w.col;
      switch (at.seg->kind) {
        case kXeStats: stats(v, c); break;
        case kXeProb: prob(v, c); break;
        case kXeDx: dx(v, c); break;
        default: dw(v, c); break;
      }
    }

    __device__ __forceinline__ void stats(float (&v)[32], int c) {
      const long long left = a.V - ((long long)at.n * kXeTile + c);
      if (left < 32) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (i >= left) v[i] = __int_as_float(0xff800000);
      }
      const long long in = word - c;
      if (in >= 0 && in < 32) {
        float score = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) score = i == (int)in ? v[i] : score;
        a.score[row] = score;
      }
      float t[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = fmaxf(fmaxf(v[i], v[8 + i]), fmaxf(v[16 + i], v[24 + i]));
      const float top = fmaxf(m, fmaxf(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])), fmaxf(fmaxf(t[4], t[5]), fmaxf(t[6], t[7]))));
      if (top == __int_as_float(0xff800000)) {
        // nothing yet, unless there are NaNs, which a maximum passes over
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (v[i] != v[i]) s = v[i];
        return;
      }
      // (differences first: a product with log2(e) that is rounded before would cost |s| times the error)
      s *= xe_exp2((m - top) * kLog2e);
      m = top;
      float u[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 32; ++i) u[i & 3] += xe_exp2((v[i] - top) * kLog2e);
      s += (u[0] + u[1]) + (u[2] + u[3]);
    }

    __device__ __forceinline__ void prob(float (&v)[32], int c) {
      const long long v0 = (long long)at.n * kXeTile + c;             // column in the piece
      if (row >= a.T) return;
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = xe_exp2((v[i] - m) * kLog2e);
      const long long in = word - c;
      if (in >= 0 && in < 32) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          v[i] -= i == (int)in ? 1.f : 0.f;
      }
      // zeros past the vocabulary, and in the rows of ignored tokens whatever x holds there
      const long long live = counts ? a.V - (at.seg->v0 + v0) : 0;
      if (live < 32) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (i >= live) v[i] = 0.f;
      }
      unsigned int u[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) u[i] = mm_bf16x2(v[2 * i], v[2 * i + 1]);
      __nv_bfloat16* o = a.d_out[at.seg->buf] + (size_t)row * (size_t)a.piece + (size_t)v0;
      store_sector(o, u);
      store_sector(o + 16, u + 8);
    }

    __device__ __forceinline__ void dx(float (&v)[32], int c) {
      const long long col = (long long)at.n * kXeTile + c, row0 = row - w.lane;
      const int rows = (int)min(32ll, a.T - row0), cols = (int)min(32ll, a.D - col);
      if (rows <= 0 || cols <= 0) return;
      // (sums lie in rows of whole groups of eight; past D they are sums of zeros)
      float* sums = a.dx_sums + ((size_t)at.slice * (size_t)a.T + (size_t)row) * (size_t)a.pitch + (size_t)col;
      const int live = w.lane < rows ? cols : 0;
      if (!at.seg->start) {
#pragma unroll
        for (int i = 0; i < 32; i += 4)
          if (i < live) {
            const float4 q = __ldcg(reinterpret_cast<const float4*>(sums + i));
            v[i] += q.x;
            v[i + 1] += q.y;
            v[i + 2] += q.z;
            v[i + 3] += q.w;
          }
      }
      if (at.seg->finish) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = counts ? v[i] * g : 0.f;
        xe_store(a.dx + (size_t)row0 * (size_t)a.ld_dx + (size_t)col, a.ld_dx, v, w.lane, rows, cols, a.dx_align);
      } else {
#pragma unroll
        for (int i = 0; i < 32; i += 8)
          if (i < live) store_sector(sums + i, reinterpret_cast<const unsigned int*>(v) + i);
      }
    }

    __device__ __forceinline__ void dw(float (&v)[32], int c) {
      const long long col = (long long)at.n * kXeTile + c, out = at.seg->v0 + row - w.lane;
      const int rows = (int)min(32ll, a.V - out), cols = (int)min(32ll, a.D - col);
      if (rows <= 0 || cols <= 0) return;
      if (at.seg->slices > 1) {
        float* sums = a.dw_sums + ((size_t)at.slice * (size_t)a.V + (size_t)out + w.lane) * (size_t)a.pitch + (size_t)col;
#pragma unroll
        for (int i = 0; i < 32; i += 8)
          if (i < cols && w.lane < rows) store_sector(sums + i, reinterpret_cast<const unsigned int*>(v) + i);
        return;
      }
      const size_t o = (size_t)out * (size_t)a.ld_dw + (size_t)col;
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] *= a.scale;
      if (a.dw_f32) xe_store(static_cast<float*>(a.dw) + o, a.ld_dw, v, w.lane, rows, cols, a.dw_align);
      else xe_store(static_cast<__nv_bfloat16*>(a.dw) + o, a.ld_dw, v, w.lane, rows, cols, a.dw_align);
    }

    __device__ __forceinline__ void end() {
      if (at.seg->kind == kXeStats && row < a.T) {
        constexpr int kColumns = kXeTile / (WARPS / 4);
        const long long part = (long long)at.n * (kXeTile / kColumns) + w.col / kColumns;
        if (part < a.nparts) a.parts[(size_t)row * (size_t)a.nparts + (size_t)part] = make_float2(m, s);
      }
    }
  };
};

// Joins a row's parts: one warp per row.  Ignored rows get zeros.
constexpr int kXeJoinThreads = 128;
__global__ void __launch_bounds__(kXeJoinThreads)
ps_xent_join_kernel(const float2* __restrict__ parts, int nparts, const float* __restrict__ score, const void* __restrict__ targets,
                    int target64, long long T, long long V, float* __restrict__ loss, float* __restrict__ lse) {
  mm_pdl();
  const long long row = (long long)blockIdx.x * (kXeJoinThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (row >= T) return;
  const long long target = xe_target(targets, target64, row);
  const bool counts = target >= 0 && target < V;
  const float2* p = parts + (size_t)row * (size_t)nparts;
  float m = __int_as_float(0xff800000), s = 0.f;
  if (counts)
    for (int i = lane; i < nparts; i += 4 * 32) {
      float2 q[4];                                        // (loads before what depends on them)
#pragma unroll
      for (int k = 0; k < 4; ++k) q[k] = i + 32 * k < nparts ? p[i + 32 * k] : make_float2(__int_as_float(0xff800000), 0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float top = fmaxf(m, q[k].x);
        if (top == __int_as_float(0xff800000)) {
          s += q[k].y;                                    // (zeros, or NaN)
        } else {
          s = s * xe_exp2((m - top) * kLog2e) + q[k].y * xe_exp2((q[k].x - top) * kLog2e);
          m = top;
        }
      }
    }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m2 = __shfl_down_sync(0xffffffffu, m, o), s2 = __shfl_down_sync(0xffffffffu, s, o);
    const float top = fmaxf(m, m2);
    if (top == __int_as_float(0xff800000)) {
      s += s2;
    } else {
      s = s * xe_exp2((m - top) * kLog2e) + s2 * xe_exp2((m2 - top) * kLog2e);
      m = top;
    }
  }
  if (lane == 0) {
    const float l = counts ? m + logf(s) : 0.f;
    if (lse) lse[row] = l;
    if (loss) loss[row] = counts ? l - score[row] : 0.f;
  }
}

constexpr int kXeCopyThreads = 256;
__global__ void __launch_bounds__(kXeCopyThreads)
ps_xent_copy_kernel(const __grid_constant__ XeCopy x, const __grid_constant__ XeCopy w) {
  mm_pdl();
  const long long first = (long long)blockIdx.x * kXeCopyThreads + threadIdx.x, stride = (long long)gridDim.x * kXeCopyThreads;
  if (x.src) xe_copy(x, first, stride);
  if (w.src) xe_copy(w, first, stride);
}

// One gradient as the sum over its slices, in order: four columns of a row per thread.  dx's rows have factors of their
// own (targets not NULL).
struct XeSum {
  const float* sums;                     // slices x rows x pitch
  int slices, pitch;
  long long rows, cols, ld;
  void* out;
  int f32, wide;                         // wide: rows allow stores of four
  float scale;
  const void* targets;
  int target64;
  long long V;
  const float* weights;
};

__global__ void __launch_bounds__(kXeCopyThreads)
ps_xent_slices_kernel(const __grid_constant__ XeSum q) {
  mm_pdl();
  const unsigned int per = (unsigned int)q.pitch / 4;
  const size_t n = (size_t)q.rows * (size_t)q.pitch;
  const long long units = q.rows * per, stride = (long long)gridDim.x * kXeCopyThreads;
  for (long long i = (long long)blockIdx.x * kXeCopyThreads + threadIdx.x; i < units; i += stride) {
    const long long r = i / per, c = (i - r * per) * 4;
    if (c >= q.cols) continue;
    float g = q.scale;
    const bool counts = !q.targets || xe_factor(q.targets, q.target64, q.V, q.weights, q.scale, r, &g);
    const float* p = q.sums + (size_t)r * (size_t)q.pitch + (size_t)c;
    float4 v = *reinterpret_cast<const float4*>(p);
#pragma unroll 8
    for (int k = 1; k < q.slices; ++k) {
      const float4 t = *reinterpret_cast<const float4*>(p + (size_t)k * n);
      v.x += t.x;
      v.y += t.y;
      v.z += t.z;
      v.w += t.w;
    }
    if (!counts) {
      v = make_float4(0.f, 0.f, 0.f, 0.f);
      g = 1.f;
    }
    const float e[4] = {v.x * g, v.y * g, v.z * g, v.w * g};
    const size_t o = (size_t)r * (size_t)q.ld + (size_t)c;
    if (q.f32) {
      float* out = static_cast<float*>(q.out) + o;
      if (q.wide) *reinterpret_cast<float4*>(out) = make_float4(e[0], e[1], e[2], e[3]);
      else
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c + k < q.cols) out[k] = e[k];
    } else {
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(q.out) + o;
      if (q.wide) *reinterpret_cast<uint2*>(out) = make_uint2(mm_bf16x2(e[0], e[1]), mm_bf16x2(e[2], e[3]));
      else
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c + k < q.cols) out[k] = __float2bfloat16_rn(e[k]);
    }
  }
}

}  // namespace psb
