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
// of 2048 elements, so every SM gets the same amount.
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

// Eight consecutive elements as binary32.
__device__ __forceinline__ void load8(const ClipTensor& t, size_t e, float (&v)[8]) {
  if (t.src_bf16) {
    widen8(*reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(t.src) + e), v);
  } else {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(t.src) + e);
    const float4 a = p[0], b = p[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
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

__device__ __forceinline__ void store8(const ClipTensor& t, size_t e, const float (&v)[8]) {
  if (t.dst_bf16) {
    __stcs(reinterpret_cast<uint4*>(static_cast<unsigned short*>(t.dst) + e),
           make_uint4(round_bf16x2(v[0], v[1]), round_bf16x2(v[2], v[3]), round_bf16x2(v[4], v[5]), round_bf16x2(v[6], v[7])));
  } else {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(t.dst) + e);
    __stcs(p, make_float4(v[0], v[1], v[2], v[3]));
    __stcs(p + 1, make_float4(v[4], v[5], v[6], v[7]));
  }
}

__device__ __forceinline__ void store1(const ClipTensor& t, size_t e, float v) {
  if (t.dst_bf16) static_cast<unsigned short*>(t.dst)[e] = (unsigned short)round_bf16x2(v, 0.f);
  else static_cast<float*>(t.dst)[e] = v;
}

// Sum of eight squares: in binary32 where neither overflow nor underflow can reach it (at most eight roundings, about
// 3e-7 of one eighth-of-a-vector's share), else in binary64.  A conversion to binary64 issues at an eighth of the
// rate of an addition, and one per element was what bounded the pass on bf16 gradients.
__device__ __forceinline__ double squares8(const float (&v)[8]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s = __fmaf_rn(v[i], v[i], s);
  if (s > 1e-20f && s < 1e30f) return (double)s;
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) d = fma((double)v[i], (double)v[i], d);
  return d;
}

struct ClipArgs {
  const ClipTensor* tensors;
  unsigned int n;
  float max_norm;
  unsigned long long units;
  double* parts;                                    // one per CTA
  GridBarrier* bar;
  float* norm_out;
  int* status;
};

// Visits the CTA's part of every tensor it touches, forwards or backwards.
template <typename F>
__device__ __forceinline__ void each_part(const ClipArgs& a, unsigned long long u0, unsigned long long u1, bool backwards, F f) {
  if (u0 >= u1) return;
  const unsigned long long at = backwards ? u1 - 1 : u0;
  unsigned int lo = 0, hi = a.n - 1;                // the tensor that holds unit `at`: the last that starts at or before it
  while (lo < hi) {
    const unsigned int mid = (lo + hi + 1) >> 1;
    if (a.tensors[mid].first_unit <= at) lo = mid; else hi = mid - 1;
  }
  for (unsigned int t = lo;;) {
    const ClipTensor T = a.tensors[t];
    const unsigned long long b = max(u0, T.first_unit) - T.first_unit;
    const unsigned long long e = min(T.nelem, (u1 - T.first_unit) * kNormUnit);
    if (e > b * kNormUnit) f(T, (size_t)(b * kNormUnit), (size_t)e);
    if (backwards) {
      if (t == 0 || T.first_unit <= u0) break;
      --t;
    } else {
      if (++t >= a.n || a.tensors[t].first_unit >= u1) break;
    }
  }
}

__global__ void __launch_bounds__(kClipThreads, 2)
ps_clip_kernel(const __grid_constant__ ClipArgs a) {
  const unsigned int tid = threadIdx.x, G = gridDim.x, c = blockIdx.x;
  const unsigned long long u0 = a.units * c / G, u1 = a.units * (c + 1) / G;
  __shared__ double s_red[kClipThreads / 32];
  __shared__ float s_factor;
  double sq = 0.0;
  each_part(a, u0, u1, false, [&](const ClipTensor& T, size_t b, size_t e) {
    if (T.vec_ok) {
      const size_t whole = b + ((e - b) & ~(size_t)7);
#pragma unroll 4
      for (size_t i = b + tid * 8; i < whole; i += kClipThreads * 8) {
        float v[8];
        load8(T, i, v);
        sq += squares8(v);
      }
      b = whole;
    }
    for (size_t i = b + tid; i < e; i += kClipThreads) {
      const double v = load1(T, i);
      sq = fma(v, v, sq);
    }
  });
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sq += __shfl_down_sync(0xffffffffu, sq, o);
  if ((tid & 31) == 0) s_red[tid >> 5] = sq;
  __syncthreads();
  if (tid == 0) {
    double v = s_red[0];
    for (int w = 1; w < kClipThreads / 32; ++w) v += s_red[w];
    __stcg(a.parts + c, v);
  }
  if (!grid_barrier(a.bar)) {
    if (tid == 0) atomicExch(a.status, 1);
    return;
  }
  if (tid < 32) {
    double v = 0.0;
    for (unsigned int q = tid; q < G; q += 32) v += __ldcg(a.parts + q);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
    if (tid == 0) {
      const float norm = (float)sqrt(v);
      s_factor = clip_factor(norm, a.max_norm);
      if (c == 0 && a.norm_out) *a.norm_out = norm;
    }
  }
  __syncthreads();
  const float f = s_factor;
  each_part(a, u0, u1, true, [&](const ClipTensor& T, size_t b, size_t e) {
    // nothing to do for a tensor that is clipped in place by a factor of one
    if (f == 1.0f && T.src == T.dst) return;
    size_t whole = b;
    if (T.vec_ok) whole = b + ((e - b) & ~(size_t)7);
    for (size_t i = whole + tid; i < e; i += kClipThreads) store1(T, i, __fmul_rn(load1(T, i), f));
    const long long trips = ((long long)(whole - b) + kClipThreads * 8 - 1) / (kClipThreads * 8);
#pragma unroll 4
    for (long long k = trips - 1; k >= 0; --k) {
      const size_t i = b + (size_t)k * (kClipThreads * 8) + tid * 8;
      if (i < whole) {
        float v[8];
        load8(T, i, v);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = __fmul_rn(v[q], f);
        store8(T, i, v);
      }
    }
  });
}

}  // namespace psb

using namespace psb;

struct ps_clip {
  uint32_t magic = kClipMagic;
  int device = 0;
  int grid = 0;
  unsigned int n = 0;
  unsigned long long units = 0;
  // one allocation: tensors, per-CTA sums, barrier, status word
  unsigned char* mem = nullptr;
  size_t parts_off = 0, bar_off = 0, status_off = 0;
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
      t.vec_ok = ((s | d) & 15u) == 0;
      units += (nelems[i] + kNormUnit - 1) / kNormUnit;
      ts.push_back(t);
    }
  } catch (...) {
    return PS_ERR_NOMEM;
  }
  cudaError_t e = cudaSetDevice(device);
  if (e != cudaSuccess) return op_cuda_error("cudaSetDevice", e);
  OpDevice d;
  int rc = op_device(&d);
  if (rc) return rc;
  int per_sm = 0;
  e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, ps_clip_kernel, kClipThreads, 0);
  if (e != cudaSuccess) return op_cuda_error("ps_clip_create", e);
  ps_clip* c = new (std::nothrow) ps_clip();
  if (!c) return PS_ERR_NOMEM;
  c->device = device;
  c->n = (unsigned int)ts.size();
  c->units = units;
  c->grid = (int)std::max<unsigned long long>(1, std::min<unsigned long long>(units, (unsigned long long)d.num_sms * std::max(1, per_sm)));
  const size_t tbytes = (ts.size() * sizeof(ClipTensor) + 255) / 256 * 256;
  c->parts_off = tbytes;
  c->bar_off = tbytes + ((size_t)c->grid * sizeof(double) + 255) / 256 * 256;
  c->status_off = c->bar_off + sizeof(GridBarrier);
  const size_t total = c->status_off + sizeof(int);
  void* mem = nullptr;
  e = cudaMalloc(&mem, total);
  if (e == cudaSuccess) e = cudaMemset(mem, 0, total);
  if (e == cudaSuccess && !ts.empty()) e = cudaMemcpy(mem, ts.data(), ts.size() * sizeof(ClipTensor), cudaMemcpyHostToDevice);
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
  cudaError_t e = cudaSetDevice(c->device);
  if (e != cudaSuccess) return op_cuda_error("cudaSetDevice", e);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  if (c->n == 0) {
    if (norm_out) e = cudaMemsetAsync(norm_out, 0, sizeof(float), stream);
    return e == cudaSuccess ? PS_OK : op_cuda_error("ps_clip_run", e);
  }
  ClipArgs a;
  a.tensors = reinterpret_cast<const ClipTensor*>(c->mem);
  a.n = c->n;
  a.max_norm = max_norm;
  a.units = c->units;
  a.parts = reinterpret_cast<double*>(c->mem + c->parts_off);
  a.bar = reinterpret_cast<GridBarrier*>(c->mem + c->bar_off);
  a.norm_out = norm_out;
  a.status = reinterpret_cast<int*>(c->mem + c->status_off);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)c->grid);
  cfg.blockDim = dim3((unsigned)kClipThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, ps_clip_kernel, a);
  return e == cudaSuccess ? PS_OK : op_cuda_error("ps_clip_run", e);
}

int ps_clip_status(ps_clip* c, int* status_out) {
  if (!alive(c)) return PS_ERR_BAD_HANDLE;
  if (!status_out) return PS_ERR_BAD_ARG;
  cudaError_t e = cudaSetDevice(c->device);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(status_out, c->mem + c->status_off, sizeof(int), cudaMemcpyDeviceToHost);
  return e == cudaSuccess ? PS_OK : op_cuda_error("ps_clip_status", e);
}

int ps_clip_destroy(ps_clip* c) {
  if (!alive(c)) return PS_ERR_BAD_HANDLE;
  cudaError_t e = cudaSetDevice(c->device);
  if (e == cudaSuccess) e = cudaFree(c->mem);        // waits for launches that still use it
  c->magic = 0;
  delete c;
  return e == cudaSuccess ? PS_OK : op_cuda_error("ps_clip_destroy", e);
}

}  // extern "C"
