// Softmax cross entropy of T tokens over V words without keeping the T x V scores, and its gradients:
//     s_tv = sum_d x_td w_vd,  lse_t = log sum_v exp(s_tv),  loss_t = lse_t - s_t,target(t)
//     d_tv = g_t (exp(s_tv - lse_t) - [v = target(t)]),  dx = d w,  dw = d^T x
//
// All four products run in the frame of ps_tc.cuh.  The losses' pass keeps of every 256 x 256 tile of scores one
// maximum and one sum of exponentials per row and 128 columns, which a small kernel joins.  The gradients' pass walks
// the vocabulary in pieces: the scores of a piece are computed again, turned into d (bf16) and stored; the next launch
// reads them twice, along the rows for dx and down the columns for dw, and computes the following piece's d beside it,
// so that what each launch ends with is covered by work that does not depend on it.  A piece of d takes about 32 MB
// and so stays in L2 between its writing and its reading.
//
// Roundings: products of bf16 values are exact and summed in binary32; maxima, sums, lse and losses are binary32.  What is
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
  int slices;                            // kXeDx: the piece's words are shared out; each slice has sums of its own
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
  float2* parts;                         // (maximum, sum of exp(s - maximum)) per row and 128 columns, rows of nparts
  int nparts;
  float* score;                          // s_t,target(t)
  // gradients' pass
  const float* lse;
  const float* weights;                  // nullptr: 1
  float scale;
  __nv_bfloat16* d_out[2];               // T x piece
  int piece;
  float* dx_sums;                        // slices x T x D
  __nv_bfloat16* dx;
  void* dw;
  long long ld_dx, ld_dw;
  int dw_f32, dx_wide, dw_wide;          // wide: rows allow 256-bit stores
  XeCopy side;                           // done by warps that have nothing else to do: xm, needed from the next launch on
};

// g_t; zero for an ignored token, whatever token_scale holds there.
__device__ __forceinline__ float xe_factor(const void* targets, int is64, long long V, const float* weights, float scale, long long t) {
  const long long v = xe_target(targets, is64, t);
  if (v < 0 || v >= V) return 0.f;
  return weights ? scale * weights[t] : scale;
}

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float xe_exp2(float x) {      // (an argument that is far below zero gives zero)
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// 32 values of one row as bf16 or binary32, `live` of them inside the row.
__device__ __forceinline__ void xe_store_bf16(__nv_bfloat16* o, const float* v, int live, bool wide) {
  if (wide && live >= 32) {
    unsigned int u[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = mm_bf16x2(v[2 * i], v[2 * i + 1]);
    store_sector(o, u);
    store_sector(o + 16, u + 8);
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (i < live) o[i] = __float2bfloat16_rn(v[i]);
  }
}
__device__ __forceinline__ void xe_store_f32(float* o, const float* v, int live, bool wide) {
  if (wide && live >= 32) {
#pragma unroll
    for (int i = 0; i < 32; i += 8) store_sector(o + i, reinterpret_cast<const unsigned int*>(v) + i);
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (i < live) o[i] = v[i];
  }
}

struct XeOp {
  static constexpr bool kPair = true;
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
    } else if (s.kind == kXeDx) {        // tokens x width, over (a slice of) the piece's words
      const int k0 = (int)((long long)s.nk * at.slice / s.slices), k1 = (int)((long long)s.nk * (at.slice + 1) / s.slices);
      t->a = &a.d[s.buf];
      t->b = &a.w;
      t->b_mn = 1;
      t->a_k = k0 * kXeK;
      t->b_k = s.v0 + k0 * kXeK;
      t->nk = k1 - k0;
    } else {                             // words x width, over the tokens
      t->a = &a.d[s.buf];
      t->b = &a.xm;
      t->a_mn = t->b_mn = 1;
    }
  }

  struct Epilogue {
    const XeArgs& a;
    const TcWarp& w;
    const At at;
    long long row, word;                 // this lane's row; the target (kXeStats, kXeProb: relative to the tile's first column)
    float m, s, g;                       // g: kXeDx: the factor of the row's gradient
    bool counts;                         // the row's token has a target

    __device__ __forceinline__ Epilogue(const XeArgs& args, int index, const TcWarp& warp, MmCursor<1>&)
        : a(args), w(warp), at(locate(args, index)) {}

    __device__ __forceinline__ void begin() {
      const int kind = at.seg->kind;
      row = (long long)at.m * kXeTile + w.row + w.lane;
      g = a.scale;
      if (kind == kXeDx && row < a.T) g = factor(a, row);
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

    static __device__ __forceinline__ float factor(const XeArgs& a, long long row) {
      return xe_factor(a.targets, a.target64, a.V, a.weights, a.scale, row);
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
      xe_store_bf16(a.d_out[at.seg->buf] + (size_t)row * (size_t)a.piece + (size_t)v0, v, 32, true);
    }

    __device__ __forceinline__ void dx(float (&v)[32], int c) {
      const long long col = (long long)at.n * kXeTile + c;
      const int live = (int)min(32ll, a.D - col);
      if (row >= a.T || live <= 0) return;
      float* sums = a.dx_sums + ((size_t)at.slice * (size_t)a.T + (size_t)row) * (size_t)a.D + (size_t)col;
      const bool wide = (a.D & 7) == 0;
      if (!at.seg->start) {
        if (wide && live >= 32) {
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 q = __ldcg(reinterpret_cast<const float4*>(sums + i));
            v[i] += q.x;
            v[i + 1] += q.y;
            v[i + 2] += q.z;
            v[i + 3] += q.w;
          }
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (i < live) v[i] += __ldcg(sums + i);
        }
      }
      if (at.seg->finish) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= g;
        xe_store_bf16(a.dx + (size_t)row * (size_t)a.ld_dx + (size_t)col, v, live, a.dx_wide != 0);
      } else {
        xe_store_f32(sums, v, live, wide);
      }
    }

    __device__ __forceinline__ void dw(float (&v)[32], int c) {
      const long long col = (long long)at.n * kXeTile + c, out = at.seg->v0 + row;
      const int live = (int)min(32ll, a.D - col);
      if (out >= a.V || live <= 0) return;
      const size_t o = (size_t)out * (size_t)a.ld_dw + (size_t)col;
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] *= a.scale;
      if (a.dw_f32) xe_store_f32(static_cast<float*>(a.dw) + o, v, live, a.dw_wide != 0);
      else xe_store_bf16(static_cast<__nv_bfloat16*>(a.dw) + o, v, live, a.dw_wide != 0);
    }

    __device__ __forceinline__ void end() {
      if (at.seg->kind == kXeStats && row < a.T) {
        const long long part = (long long)at.n * 2 + (w.col >> 7);
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
    for (int i = lane; i < nparts; i += 32) {
      const float2 q = p[i];
      const float top = fmaxf(m, q.x);
      if (top == __int_as_float(0xff800000)) {
        s += q.y;                                         // (zeros, or NaN)
      } else {
        s = s * xe_exp2((m - top) * kLog2e) + q.y * xe_exp2((q.x - top) * kLog2e);
        m = top;
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
ps_xent_copy_kernel(const __grid_constant__ XeCopy c) {
  mm_pdl();
  xe_copy(c, (long long)blockIdx.x * kXeCopyThreads + threadIdx.x, (long long)gridDim.x * kXeCopyThreads);
}

// dx = sum over the slices, in order: a CTA per row, four columns per thread where rows allow it.
__global__ void __launch_bounds__(kXeCopyThreads)
ps_xent_slices_kernel(const float* __restrict__ sums, int slices, long long T, long long D, const void* __restrict__ targets,
                      int target64, long long V, const float* __restrict__ weights, float scale, __nv_bfloat16* __restrict__ dx,
                      long long ld, int wide) {
  mm_pdl();
  const size_t n = (size_t)T * (size_t)D;
  for (long long r = blockIdx.x; r < T; r += gridDim.x) {
    const float g = xe_factor(targets, target64, V, weights, scale, r);
    const float* p = sums + (size_t)r * (size_t)D;
    __nv_bfloat16* o = dx + (size_t)r * (size_t)ld;
    if (wide) {
      for (long long c = 4 * threadIdx.x; c < D; c += 4 * kXeCopyThreads) {
        float4 v = *reinterpret_cast<const float4*>(p + c);
#pragma unroll 8
        for (int k = 1; k < slices; ++k) {
          const float4 q = *reinterpret_cast<const float4*>(p + (size_t)k * n + c);
          v.x += q.x;
          v.y += q.y;
          v.z += q.z;
          v.w += q.w;
        }
        *reinterpret_cast<uint2*>(o + c) = make_uint2(mm_bf16x2(v.x * g, v.y * g), mm_bf16x2(v.z * g, v.w * g));
      }
    } else {
      for (long long c = threadIdx.x; c < D; c += kXeCopyThreads) {
        float v = p[c];
#pragma unroll 8
        for (int k = 1; k < slices; ++k) v += p[(size_t)k * n + c];
        o[c] = __float2bfloat16_rn(v * g);
      }
    }
  }
}

}  // namespace psb
