// Global gradient norm over many tensors and clipping, on the worker's side of
// the boundary (declarations and contracts: include/ps_b200.h).
//
//     norm = sqrt(sum over all tensors of x*x),  dst = src * min(1, max_norm / (norm + 1e-6))
//
// One cooperative launch: every CTA adds the squares of its part, the grid meets at
// a barrier, every CTA adds the same per-CTA sums in the same order and scales its
// part.  The floor is one read and one write of every element; what the second pass
// reads again comes from L2 as far as that reaches, because it walks the part
// backwards.  Parts are contiguous ranges of the tensors laid end to end in units
// of 2048 elements, so every SM gets the same amount; which tensor a part starts in
// is worked out when the list is made.
//
// Short lists (up to 256 units, half a million elements in large tensors) run on one
// cluster of sixteen CTAs that keep their elements in registers between the passes: its
// barrier is the hardware's, and a launch that is not cooperative overlaps its start and
// the look at the list with the end of the stream's previous one.  Calls in a row take
// 3.6 us on 1024 elements and on 65536, 5.0 on 262144, 7.6 on 524288; a cooperative
// launch with one unit per CTA in registers took 6.0, 6.4, 7.2 and 8.2 us (with sums in
// binary32, where this took 4.7 and 7.0 on the larger two).  Above that sixteen SMs move
// too little.
//
// Squares are added in binary64, where each is exact: added eight at a time in binary32,
// the roundings of equal elements all point the same way, and the norm depended on how
// its tensors are aligned.  That costs 3 % on the small list below, 7 to 10 % on a
// quarter and half a million elements, up to 1 % on long lists.
//
// Measured, the 335 M elements of a 24-layer model: fp32 into bf16 544 us (10 bytes per
// element in two passes, 6.2 TB/s), fp32 into fp32 678 us (5.9), bf16 into bf16 353 us
// (5.7), the norm alone 202 us of fp32 (6.6 TB/s) and 109 of bf16 (6.1); 8.4 M fp32 into
// fp32 17 us, mostly out of L2 (22.6 us with eight lists in rotation); 170 K elements in
// 37 tensors 4.26 us a call, which is launch, two dependent trips to L2 and the cluster's
// barriers.  Tensors that are not aligned to eight elements: 1416 us for the first of
// these, 1375 for bf16, 11.3 us for 524288 elements.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "ps_grid.cuh"
#include "ps_math.cuh"
#include "ps_op.h"

namespace psb {

constexpr int kClipThreads = 512;
constexpr unsigned int kNormUnit = 2048;            // elements
constexpr uint32_t kClipMagic = 0x50534332u;        // "PSC2"

struct __align__(16) ClipTensor {
  const void* src;
  void* dst;
  unsigned long long nelem;
  unsigned long long first_unit;                    // units of all earlier tensors
  unsigned int src_bf16, dst_bf16, vec_ok, _pad;
};

// Eight consecutive elements, as loaded and as binary32.
template <bool BF16>
struct Raw8 {
  uint4 q[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void* src, size_t e) {
    const char* p = static_cast<const char*>(src) + e * (BF16 ? 2 : 4);
    if constexpr (BF16)
      q[0] = *reinterpret_cast<const uint4*>(p);
    else                                             // a thread's 256 bits: one whole sector
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(q[0].x), "=r"(q[0].y), "=r"(q[0].z), "=r"(q[0].w), "=r"(q[1].x), "=r"(q[1].y), "=r"(q[1].z), "=r"(q[1].w)
                   : "l"(p));
  }
  __device__ __forceinline__ void widen(float (&v)[8]) const {
    if constexpr (BF16) {
      widen8(q[0], v);
    } else {
      const float4 x = as_f4(q[0]), y = as_f4(q[1]);
      v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    }
  }
};

__device__ __forceinline__ void load8(const ClipTensor& t, size_t e, float (&v)[8]) {
  if (t.src_bf16) {
    Raw8<true> r;
    r.load(t.src, e);
    r.widen(v);
  } else {
    Raw8<false> r;
    r.load(t.src, e);
    r.widen(v);
  }
}

__device__ __forceinline__ float load1(const ClipTensor& t, size_t e) {
  return t.src_bf16 ? __uint_as_float((unsigned int)static_cast<const unsigned short*>(t.src)[e] << 16)
                    : static_cast<const float*>(t.src)[e];
}

__device__ __forceinline__ unsigned int round_bf16x2(float lo, float hi) {
  unsigned int r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <bool BF16>
__device__ __forceinline__ void store8_as(void* dst, size_t e, const float (&v)[8]) {
  if constexpr (BF16) {
    __stcs(reinterpret_cast<uint4*>(static_cast<unsigned short*>(dst) + e),
           make_uint4(round_bf16x2(v[0], v[1]), round_bf16x2(v[2], v[3]), round_bf16x2(v[4], v[5]), round_bf16x2(v[6], v[7])));
  } else {
    asm volatile("st.global.cs.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(static_cast<float*>(dst) + e),
                 "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])),
                 "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7]))
                 : "memory");
  }
}
__device__ __forceinline__ void store8(const ClipTensor& t, size_t e, const float (&v)[8]) {
  if (t.dst_bf16) store8_as<true>(t.dst, e, v);
  else store8_as<false>(t.dst, e, v);
}

__device__ __forceinline__ void store1(const ClipTensor& t, size_t e, float v) {
  if (t.dst_bf16) static_cast<unsigned short*>(t.dst)[e] = (unsigned short)round_bf16x2(v, 0.f);
  else static_cast<float*>(t.dst)[e] = v;
}

// |x| in binary64, where its square is exact, without a conversion, which issues at a fraction of the rate of an
// addition: exponent and mantissa are shifted into place, which is |x| times 2^-896, subnormals and zeros included, and
// scaled.  Infinities and NaNs become numbers from 2^128 on, which no finite x reaches.
__device__ __forceinline__ double widened(float x) {
  const unsigned int u = __float_as_uint(x);
  return __hiloint2double((int)((u & 0x7fffffffu) >> 3), (int)(u << 29)) * 0x1p896;
}
constexpr double kNotFinite = 0x1p256;            // a sum of their squares below it holds neither

// Adds eight squares to four sums: binary64 throughout, the chains of dependent additions short.  Every fourth element
// takes the conversion after all, which keeps both routes' units busy (bf16, 335 M elements, the norm alone: all by
// conversion 112 us, none 109.4, every fourth 109.1).
__device__ __forceinline__ void add_squares(const float (&v)[8], double (&acc)[4]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double d = (i & 3) == 3 ? (double)v[i] : widened(v[i]);
    acc[i & 3] = fma(d, d, acc[i & 3]);
  }
}
__device__ __forceinline__ double sum4(const double (&a)[4]) { return (a[0] + a[1]) + (a[2] + a[3]); }
// The same in binary32: what a sum that is not below kNotFinite stands for, infinity or NaN.
__device__ __forceinline__ void add_squares32(const float (&v)[8], float& sq) {
#pragma unroll
  for (int i = 0; i < 8; ++i) sq = __fmaf_rn(v[i], v[i], sq);
}

// Squares of elements [b, whole) of one type, whole vectors; the loads of U vectors are in flight before the first is
// used.
template <bool BF16, int U>
__device__ __forceinline__ double squares(const void* src, size_t b, size_t whole) {
  constexpr size_t kStep = kClipThreads * 8;
  double acc[4] = {0.0, 0.0, 0.0, 0.0};
  size_t i = b + threadIdx.x * 8;
  float v[8];
  for (; i + (U - 1) * kStep < whole; i += U * kStep) {
    Raw8<BF16> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u].load(src, i + u * kStep);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u].widen(v);
      add_squares(v, acc);
    }
  }
  for (; i < whole; i += kStep) {
    Raw8<BF16> r;
    r.load(src, i);
    r.widen(v);
    add_squares(v, acc);
  }
  const double sq = sum4(acc);
  if (sq < kNotFinite) return sq;
  float s = 0.f;
  for (i = b + threadIdx.x * 8; i < whole; i += kStep) {
    Raw8<BF16> r;
    r.load(src, i);
    r.widen(v);
    add_squares32(v, s);
  }
  return (double)s;
}

// The same elements times f, from the last one down.
template <bool SRC_BF16, bool DST_BF16, int U>
__device__ __forceinline__ void scale(const void* src, void* dst, size_t b, size_t whole, float f) {
  constexpr size_t kStep = kClipThreads * 8;
  if (whole <= b) return;
  const long long first = (long long)b + threadIdx.x * 8;
  long long i = first + (long long)((whole - b - 1) / kStep * kStep);
  if (i >= (long long)whole) i -= kStep;
  float v[8];
  for (; i - (long long)((U - 1) * kStep) >= first; i -= (long long)(U * kStep)) {
    Raw8<SRC_BF16> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u].load(src, (size_t)i - u * kStep);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u].widen(v);
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = __fmul_rn(v[q], f);
      store8_as<DST_BF16>(dst, (size_t)i - u * kStep, v);
    }
  }
  for (; i >= first; i -= (long long)kStep) {
    Raw8<SRC_BF16> r;
    r.load(src, (size_t)i);
    r.widen(v);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = __fmul_rn(v[q], f);
    store8_as<DST_BF16>(dst, (size_t)i, v);
  }
}

struct ClipArgs {
  const ClipTensor* tensors;
  const unsigned int* first;                        // the tensor that holds the first unit of every CTA, and of the end;
                                                    // short lists: of every unit
  unsigned int n;
  float max_norm;
  unsigned long long units;
  double* parts;                                    // one per CTA
  GridBarrier* bar;
  float* norm_out;
  int* status;
};

// Visits the CTA's part, units [u0, u1), tensor by tensor, forwards or backwards; t0 and t1 hold its first and last unit.
template <typename F>
__device__ __forceinline__ void each_part(const ClipArgs& a, unsigned long long u0, unsigned long long u1, unsigned int t0,
                                          unsigned int t1, bool backwards, F f) {
  for (unsigned int k = t0; k <= t1; ++k) {
    const ClipTensor T = a.tensors[backwards ? t1 - (k - t0) : k];
    const unsigned long long b = max(u0, T.first_unit) - T.first_unit;
    const unsigned long long e = min(T.nelem, (u1 - T.first_unit) * kNormUnit);
    f(T, (size_t)(b * kNormUnit), (size_t)e);
  }
}

// The factor, the same in every CTA: adds this CTA's squares to the others'.  False if the others did not arrive.
__device__ __forceinline__ bool clip_join(const ClipArgs& a, double sq, float* s_factor, double* s_red) {
  const unsigned int tid = threadIdx.x, G = gridDim.x, c = blockIdx.x;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sq += __shfl_down_sync(0xffffffffu, sq, o);
  if ((tid & 31) == 0) s_red[tid >> 5] = sq;
  __syncthreads();
  if (tid == 0) {
    double v = s_red[0];
#pragma unroll
    for (int w = 1; w < kClipThreads / 32; ++w) v += s_red[w];
    __stcg(a.parts + c, v);
  }
  if (!grid_barrier(a.bar, kGridWaitCycles, [] {})) {
    if (tid == 0) atomicExch(a.status, 1);
    return false;
  }
  if (tid < 32) {
    double v = 0.0;
#pragma unroll 4
    for (unsigned int q = tid; q < G; q += 32) v += a.parts[q];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
    if (tid == 0) {
      const float norm = (float)sqrt(v);
      *s_factor = clip_factor(norm, a.max_norm);
      if (c == 0 && a.norm_out) *a.norm_out = norm;
    }
  }
  __syncthreads();
  return true;
}

// ------------------------------------------------------------------ short lists

constexpr int kShortCtas = 16, kShortThreads = 1024, kUnitThreads = kNormUnit / 8;
constexpr unsigned int kShortStride = kShortCtas * (kShortThreads / kUnitThreads);      // units at a time
constexpr unsigned int kShortUnits = 4 * kShortStride;

// A unit: its elements [b, e) of a tensor and where its whole vectors end.
struct ClipUnit {
  ClipTensor t;
  size_t b, e, whole;
};

// Four units at a time per CTA.  A thread keeps eight elements of each of its units, a vector and one of the tail or
// eight single ones, from one pass to the other; the loads of all its units are independent of one another.
template <int kRounds>
__global__ void __cluster_dims__(kShortCtas, 1, 1) __launch_bounds__(kShortThreads, 1)
ps_clip_short_kernel(const __grid_constant__ ClipArgs a) {
  const unsigned int tid = threadIdx.x, lane = tid % kUnitThreads;
  const unsigned int mine = (tid / kUnitThreads) * kShortCtas + blockIdx.x;      // (the first units go to different CTAs)
  __shared__ double s_red[kShortThreads / 32], s_part;
  __shared__ float s_factor;
  __shared__ bool s_again;
  __shared__ ClipUnit s_unit[kShortThreads / kUnitThreads][kRounds];
  pdl_launch_dependents();
  if (lane < kRounds && mine + lane * kShortStride < a.units) {                  // (the list does not change)
    ClipUnit& k = s_unit[tid / kUnitThreads][lane];
    const unsigned int u = mine + lane * kShortStride;
    const ClipTensor t = a.tensors[a.first[u]];
    k.t = t;
    k.b = (size_t)(u - t.first_unit) * kNormUnit;
    k.e = (size_t)min(t.nelem, (unsigned long long)(k.b + kNormUnit));
    k.whole = t.vec_ok ? k.b + ((k.e - k.b) & ~(size_t)7) : k.b;
  }
  __syncthreads();
  pdl_wait();
  float v[kRounds][8], tail[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[r][k] = 0.f;
    tail[r] = 0.f;
    const unsigned int u = mine + r * kShortStride;
    if (u < a.units) {
      const ClipUnit& k = s_unit[tid / kUnitThreads][r];
      if (k.t.vec_ok) {
        if (k.b + lane * 8 < k.whole) load8(k.t, k.b + lane * 8, v[r]);
        if (k.whole + lane < k.e) tail[r] = load1(k.t, k.whole + lane);
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const size_t i = k.b + lane + q * kUnitThreads;
          if (i < k.e) v[r][q] = load1(k.t, i);
        }
      }
    }
  }
  double acc[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    if (mine + r * kShortStride < a.units) {
      add_squares(v[r], acc);
      const double d = widened(tail[r]);
      acc[r] = fma(d, d, acc[r]);
    }
  }
  double sq = sum4(acc);
  for (bool again = false;; again = true) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sq += __shfl_down_sync(0xffffffffu, sq, o);
    if ((tid & 31) == 0) s_red[tid >> 5] = sq;
    __syncthreads();
    if (tid < 32) {
      double w = s_red[tid];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) w += __shfl_down_sync(0xffffffffu, w, o);
      if (tid == 0) s_part = w;
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (tid == 0) {
      double total = 0.0;
      const unsigned int at = static_cast<unsigned int>(__cvta_generic_to_shared(&s_part));
#pragma unroll
      for (int c = 0; c < kShortCtas; ++c) {
        double w;
        asm volatile(
            "{\n\t"
            ".reg .b32 r;\n\t"
            "mapa.shared::cluster.u32 r, %1, %2;\n\t"
            "ld.shared::cluster.f64 %0, [r];\n\t"
            "}"
            : "=d"(w)
            : "r"(at), "r"(c));
        total += w;
      }
      const float norm = (float)sqrt(total);
      s_factor = clip_factor(norm, a.max_norm);
      s_again = !again && !(total < kNotFinite);
      if (blockIdx.x == 0 && a.norm_out) *a.norm_out = norm;
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // (nobody leaves while its part is being read)
    __syncthreads();
    if (!s_again) break;
    // an infinity or a NaN, in whichever CTA: all of them have the same total and add up once more, to tell which
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      add_squares32(v[r], s);
      s = __fmaf_rn(tail[r], tail[r], s);
    }
    sq = (double)s;
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  const float f = s_factor;
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const unsigned int u = mine + r * kShortStride;
    if (u < a.units) {
      const ClipUnit& k = s_unit[tid / kUnitThreads][r];
      if (f != 1.0f || k.t.src != k.t.dst) {
#pragma unroll
        for (int q = 0; q < 8; ++q) v[r][q] = __fmul_rn(v[r][q], f);
        if (k.t.vec_ok) {
          if (k.b + lane * 8 < k.whole) store8(k.t, k.b + lane * 8, v[r]);
          if (k.whole + lane < k.e) store1(k.t, k.whole + lane, __fmul_rn(tail[r], f));
        } else {
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const size_t i = k.b + lane + q * kUnitThreads;
            if (i < k.e) store1(k.t, i, v[r][q]);
          }
        }
      }
    }
  }
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__global__ void __launch_bounds__(kClipThreads, 2)
ps_clip_kernel(const __grid_constant__ ClipArgs a) {
  const unsigned int tid = threadIdx.x, G = gridDim.x, c = blockIdx.x;
  __shared__ double s_red[kClipThreads / 32];
  __shared__ float s_factor;
  const unsigned long long u0 = a.units * c / G, u1 = a.units * (c + 1) / G;
  // (the next CTA's first tensor is this one's last, or the one after it)
  const unsigned int t0 = a.first[c], tn = a.first[c + 1], t1 = tn < a.n && a.tensors[tn].first_unit < u1 ? tn : tn - 1;
  double sq = 0.0;
  each_part(a, u0, u1, t0, t1, false, [&](const ClipTensor& T, size_t b, size_t e) {
    if (T.vec_ok) {
      const size_t whole = b + ((e - b) & ~(size_t)7);
      sq += T.src_bf16 ? squares<true, 6>(T.src, b, whole) : squares<false, 3>(T.src, b, whole);
      b = whole;
    }
    for (size_t i = b + tid; i < e; i += kClipThreads) {
      const double v = load1(T, i);
      sq = fma(v, v, sq);
    }
  });
  if (!clip_join(a, sq, &s_factor, s_red)) return;
  const float f = s_factor;
  each_part(a, u0, u1, t0, t1, true, [&](const ClipTensor& T, size_t b, size_t e) {
    // nothing to do for a tensor that is clipped in place by a factor of one
    if (f == 1.0f && T.src == T.dst) return;
    size_t whole = b;
    if (T.vec_ok) whole = b + ((e - b) & ~(size_t)7);
    for (size_t i = whole + tid; i < e; i += kClipThreads) store1(T, i, __fmul_rn(load1(T, i), f));
    if (T.src_bf16) {
      if (T.dst_bf16) scale<true, true, 4>(T.src, T.dst, b, whole, f);
      else scale<true, false, 4>(T.src, T.dst, b, whole, f);
    } else {
      if (T.dst_bf16) scale<false, true, 3>(T.src, T.dst, b, whole, f);
      else scale<false, false, 3>(T.src, T.dst, b, whole, f);
    }
  });
}

}  // namespace psb

using namespace psb;

struct ps_clip {
  uint32_t magic = kClipMagic;
  int device = 0;
  int grid = 0;
  void (*cluster)(ClipArgs) = nullptr;               // a short list's kernel
  unsigned int n = 0;
  unsigned long long units = 0;
  // one allocation: tensors, first tensors, per-CTA sums, barrier, status word
  unsigned char* mem = nullptr;
  size_t first_off = 0, parts_off = 0, bar_off = 0, status_off = 0;
};

namespace {
bool alive(const ps_clip* c) { return c && c->magic == kClipMagic; }
}  // namespace

extern "C" {

int ps_clip_create(ps_clip** out, int device, int n, const void* const* srcs, int src_dtype, void* const* dsts, int dst_dtype,
                   const size_t* nelems) {
  if (!out) return PS_ERR_BAD_ARG;
  *out = nullptr;
  if (device < 0 || n < 0 || (n > 0 && (!srcs || !dsts || !nelems))) return PS_ERR_BAD_ARG;
  if ((src_dtype != PS_F32 && src_dtype != PS_BF16) || (dst_dtype != PS_F32 && dst_dtype != PS_BF16)) return PS_ERR_BAD_ARG;
  const uintptr_t ses = src_dtype == PS_BF16 ? 2 : 4, des = dst_dtype == PS_BF16 ? 2 : 4;
  std::vector<ClipTensor> ts;
  unsigned long long units = 0;
  try {
    ts.reserve((size_t)n);
    for (int i = 0; i < n; ++i) {
      if (nelems[i] == 0) continue;                  // an empty tensor adds nothing
      if (!srcs[i] || !dsts[i] || nelems[i] > ((size_t)1 << 40)) return PS_ERR_BAD_ARG;
      const uintptr_t s = reinterpret_cast<uintptr_t>(srcs[i]), d = reinterpret_cast<uintptr_t>(dsts[i]);
      if ((s & (ses - 1)) || (d & (des - 1))) return PS_ERR_ALIGN;
      // in place means the same elements: a destination that starts inside another tensor's memory is the caller's error,
      // one that starts at its own source with another element size would overwrite what is still to be read
      if (s == d && src_dtype != dst_dtype) return PS_ERR_BAD_ARG;
      ClipTensor t;
      std::memset(&t, 0, sizeof t);
      t.src = srcs[i];
      t.dst = dsts[i];
      t.nelem = nelems[i];
      t.first_unit = units;
      t.src_bf16 = src_dtype == PS_BF16;
      t.dst_bf16 = dst_dtype == PS_BF16;
      t.vec_ok = (s & (8 * ses - 1)) == 0 && (d & (8 * des - 1)) == 0;      // vectors of eight
      units += (nelems[i] + kNormUnit - 1) / kNormUnit;
      ts.push_back(t);
    }
  } catch (...) {
    return PS_ERR_NOMEM;
  }
  DeviceScope on(device);
  cudaError_t e = on.error;
  if (e != cudaSuccess) return op_cuda_error("cudaSetDevice", e);
  OpDevice d;
  int rc = op_device(&d);
  if (rc) return rc;
  int per_sm = 0;
  e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, ps_clip_kernel, kClipThreads, 0);
  if (e != cudaSuccess) return op_cuda_error("ps_clip_create", e);
  int clusters = 0;
  const auto short_kernel = units <= 2 * kShortStride ? ps_clip_short_kernel<2> : ps_clip_short_kernel<4>;
  if (units <= kShortUnits) {
    // a cluster of sixteen has to be allowed, and finds room where a GPU's SMs are not divided up
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)kShortCtas);
    cfg.blockDim = dim3((unsigned)kShortThreads);
    e = cudaFuncSetAttribute(short_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&clusters, short_kernel, &cfg);
    if (e != cudaSuccess) return op_cuda_error("ps_clip_create", e);
  }
  ps_clip* c = new (std::nothrow) ps_clip();
  if (!c) return PS_ERR_NOMEM;
  c->device = device;
  c->n = (unsigned int)ts.size();
  c->units = units;
  c->grid = (int)std::max<unsigned long long>(1, std::min<unsigned long long>(units, (unsigned long long)d.num_sms * std::max(1, per_sm)));
  if (clusters > 0) c->cluster = short_kernel;
  if (c->cluster) c->grid = (int)std::max<unsigned long long>(1, units);      // (entries of `first`: one per unit)
  c->first_off = (ts.size() * sizeof(ClipTensor) + 255) / 256 * 256;
  c->parts_off = c->first_off + (((size_t)c->grid + 1) * sizeof(unsigned int) + 255) / 256 * 256;
  c->bar_off = c->parts_off + ((size_t)c->grid * sizeof(double) + 255) / 256 * 256;
  c->status_off = c->bar_off + sizeof(GridBarrier);
  const size_t total = c->status_off + sizeof(int);
  std::vector<unsigned int> first;
  try {
    unsigned int t = 0;
    for (int k = 0; k <= c->grid; ++k) {
      const unsigned long long u = units * (unsigned long long)k / (unsigned long long)c->grid;
      while (t < c->n && u >= ts[t].first_unit + (ts[t].nelem + kNormUnit - 1) / kNormUnit) ++t;
      first.push_back(t);
    }
  } catch (...) {
    delete c;
    return PS_ERR_NOMEM;
  }
  void* mem = nullptr;
  e = cudaMalloc(&mem, total);
  if (e == cudaSuccess) e = cudaMemset(mem, 0, total);
  if (e == cudaSuccess && !ts.empty()) e = cudaMemcpy(mem, ts.data(), ts.size() * sizeof(ClipTensor), cudaMemcpyHostToDevice);
  if (e == cudaSuccess)
    e = cudaMemcpy(static_cast<unsigned char*>(mem) + c->first_off, first.data(), first.size() * sizeof(unsigned int),
                   cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);   // before other streams use it
  if (e != cudaSuccess) {
    if (mem) cudaFree(mem);
    delete c;
    return op_cuda_error("ps_clip_create", e);
  }
  c->mem = static_cast<unsigned char*>(mem);
  *out = c;
  return PS_OK;
}

int ps_clip_run(ps_clip* c, float max_norm, float* norm_out, void* stream_) {
  if (!alive(c)) return PS_ERR_BAD_HANDLE;
  if (!(max_norm > 0.0f)) return PS_ERR_BAD_ARG;
  if (reinterpret_cast<uintptr_t>(norm_out) & 3u) return PS_ERR_ALIGN;
  DeviceScope on(c->device);
  cudaError_t e = on.error;
  if (e != cudaSuccess) return op_cuda_error("cudaSetDevice", e);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  if (c->n == 0) {
    if (norm_out) e = cudaMemsetAsync(norm_out, 0, sizeof(float), stream);
    return e == cudaSuccess ? PS_OK : op_cuda_error("ps_clip_run", e);
  }
  ClipArgs a;
  a.tensors = reinterpret_cast<const ClipTensor*>(c->mem);
  a.first = reinterpret_cast<const unsigned int*>(c->mem + c->first_off);
  a.n = c->n;
  a.max_norm = max_norm;
  a.units = c->units;
  a.parts = reinterpret_cast<double*>(c->mem + c->parts_off);
  a.bar = reinterpret_cast<GridBarrier*>(c->mem + c->bar_off);
  a.norm_out = norm_out;
  a.status = reinterpret_cast<int*>(c->mem + c->status_off);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(c->cluster ? (unsigned)kShortCtas : (unsigned)c->grid);
  cfg.blockDim = dim3(c->cluster ? (unsigned)kShortThreads : (unsigned)kClipThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  if (c->cluster) {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
  } else {
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, c->cluster ? c->cluster : ps_clip_kernel, a);
  return e == cudaSuccess ? PS_OK : op_cuda_error("ps_clip_run", e);
}

int ps_clip_status(ps_clip* c, int* status_out) {
  if (!alive(c)) return PS_ERR_BAD_HANDLE;
  if (!status_out) return PS_ERR_BAD_ARG;
  DeviceScope on(c->device);
  cudaError_t e = on.error;
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(status_out, c->mem + c->status_off, sizeof(int), cudaMemcpyDeviceToHost);
  return e == cudaSuccess ? PS_OK : op_cuda_error("ps_clip_status", e);
}

int ps_clip_destroy(ps_clip* c) {
  if (!alive(c)) return PS_ERR_BAD_HANDLE;
  DeviceScope on(c->device);
  cudaError_t e = on.error;
  if (e == cudaSuccess) e = cudaFree(c->mem);        // waits for launches that still use it
  c->magic = 0;
  delete c;
  return e == cudaSuccess ? PS_OK : op_cuda_error("ps_clip_destroy", e);
}

}  // extern "C"
