// Microscaled 4-bit floating point: layout of an operand, quantisation along the
// rows and along the columns, and the way back.
//
// A block is 32 consecutive elements of one row.  Its scale is the power of two
// 2^(floor(log2 amax) - 2), held as a biased exponent byte, so the block's
// largest magnitude lands in [4, 8) and E2M1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and
// their negatives; rounding to nearest, ties to the even code, saturating at 6)
// holds the quotients.  Scaling by a power of two is exact in binary32, so the
// only rounding is the one to E2M1.  A block of zeros, and one whose scale would
// fall below 2^-127, has the scale 2^-127; a block that holds an infinity or a
// NaN has the scale byte 0xFF (its codes mean nothing) and reads back as NaN in all
// 32 places.
//
// Codes: two per byte, the lower nibble first, rows of ceil(cols/32)*16 bytes
// (padding elements are +0).  Scales: 512-byte atoms of 128 rows x 4 blocks, byte
// (row % 32)*16 + (row % 128)/32*4 + block % 4 — the order in which the tensor
// cores' scale memory takes them, so the product copies atoms without touching
// them.  Atoms of 128 rows follow one another along the columns, their number
// padded to an even one, because the product walks 256 columns at a time; scales
// that stand for no block are zero.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace psb {

constexpr int kMxBlock = 32;                 // elements that share a scale
constexpr int kMxTile = 128;                 // rows and columns of a quantiser tile: one atom of scales each way
constexpr int kMxAtom = 512;                 // bytes of an atom

__host__ __device__ inline long long mx_pitch(long long cols) { return (cols + 31) / 32 * 16; }
__host__ __device__ inline long long mx_atoms(long long cols) { return (cols + 255) / 256 * 2; }   // per 128 rows
__host__ __device__ inline size_t mx_scale_at(long long row, long long block, long long atoms) {
  return (size_t)((row >> 7) * atoms + (block >> 2)) * kMxAtom + (size_t)((row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3));
}

struct MxOut {                               // one direction of a quantisation; codes == nullptr: not wanted
  uint8_t* codes;
  uint8_t* scales;
};

// ------------------------------------------------------------------ arithmetic

// Scale byte of a block from the exponent field of its largest magnitude (binary32 and bf16 have the same).
__device__ __forceinline__ unsigned int mx_scale_byte(unsigned int e) {
  return e >= 255u ? 255u : e > 2u ? e - 2u : 0u;
}

// 1 / scale.  (For a block that is not finite this is not a power of two: its codes mean nothing, its scale is NaN.)
__device__ __forceinline__ float mx_inverse(unsigned int sb) { return __uint_as_float((254u - sb) << 23); }

// Eight values, already divided by their scale, as eight nibbles (v[0] lowest).
__device__ __forceinline__ unsigned int mx_pack8(const float (&v)[8]) {
  unsigned int r;
  asm("{\n\t"
      ".reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t"
      "}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}

__device__ __forceinline__ unsigned int mul_bf16x2(unsigned int a, unsigned int b) {
  unsigned int r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Eight bf16 values as codes.  The division by the scale is done on pairs: it is exact, or the quotient is below
// 2^-126 and far below the smallest code's half.  inv: 1 / scale of the values' block(s), twice.
__device__ __forceinline__ unsigned int mx_codes8(const unsigned int (&w)[4], unsigned int inv) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned int q = mul_bf16x2(w[i], inv);
    v[2 * i] = __uint_as_float(q << 16);
    v[2 * i + 1] = __uint_as_float(q & 0xffff0000u);
  }
  return mx_pack8(v);
}

__device__ __forceinline__ unsigned int mx_codes8(const float (&x)[8], float inv) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(x[i], inv);
  return mx_pack8(v);
}

// Largest magnitude, NaN if there is one; the result's sign bit means nothing.
__device__ __forceinline__ float max_abs(float a, float b) {
  float r;
  asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ unsigned int max_abs_bf16x2(unsigned int a, unsigned int b) {
  unsigned int r;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

__device__ __forceinline__ void mx_pdl() {
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ---------------------------------------------------------------- quantisation
//
// One CTA per 128 x 128 tile, i.e. one atom of scales in each direction.  Eight
// elements per thread and step are read (128-bit loads where the row allows it);
// along the rows a block then sits in four neighbouring lanes, whose maximum two
// shuffles give, and is converted straight from registers.  For the columns the
// tile goes through shared memory once: a thread takes one block of 32 rows of one
// column (two columns of bf16, packed), so both directions cost one read of x.
// The four row blocks of a column sit in one warp and are stored as 64 bytes; their
// shared memory reads would meet in the same banks (a stride of 32 rows is a
// multiple of 32 banks whatever the pitch), so the column index is permuted by the
// row block.

constexpr int kQuantThreads = 256;

template <bool BF16>
struct MxIn;
template <>
struct MxIn<false> { using T = float; };
template <>
struct MxIn<true> { using T = unsigned short; };

template <bool BF16>
__device__ __forceinline__ float mx_widen(typename MxIn<BF16>::T v) {
  if constexpr (BF16) return __uint_as_float((unsigned int)v << 16);
  else return v;
}

// Word of the tile in shared memory that holds column word c of row r.
template <int WORDS>
__device__ __forceinline__ int tile_word(int r, int c) { return r * WORDS + (c ^ (((r >> 5) & 3) << 3)); }

template <bool BF16, bool ROWS, bool COLS>
__global__ void __launch_bounds__(kQuantThreads)
ps_mx_quantize_kernel(const typename MxIn<BF16>::T* __restrict__ x, long long rows, long long cols, long long ld,
                      int vec_ok, unsigned int col_tiles, MxOut out, MxOut out_t) {
  using T = typename MxIn<BF16>::T;
  constexpr int kWords = BF16 ? 64 : 128;                     // 32-bit words of a tile row
  extern __shared__ unsigned int tile[];                      // COLS: 128 rows of kWords
  __shared__ __align__(16) unsigned char s_row[kMxAtom], s_col[kMxAtom];
  const int tid = threadIdx.x;
  const long long rt = blockIdx.x / col_tiles, ct = blockIdx.x % col_tiles;
  const long long r0 = rt * kMxTile, c0 = ct * kMxTile;
  if (tid < kMxAtom / 4) {
    if (ROWS) reinterpret_cast<unsigned int*>(s_row)[tid] = 0u;
    if (COLS) reinterpret_cast<unsigned int*>(s_col)[tid] = 0u;
  }
  __syncthreads();
  mx_pdl();

  // 16 lanes cover a row of the tile, 16 rows per step
  const int g = tid & 15, rr = tid >> 4;
  const long long c = c0 + g * 8;
#pragma unroll 4
  for (int step = 0; step < 8; ++step) {
    const int tr = step * 16 + rr;
    const long long r = r0 + tr;
    float v[8];
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (r < rows && c < cols) {
      const T* p = x + (size_t)r * (size_t)ld + (size_t)c;
      if (vec_ok && c + 8 <= cols) {
        if constexpr (BF16) {
          raw = *reinterpret_cast<const uint4*>(p);
        } else {
          const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
          v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
      } else {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = c + i < cols ? p[i] : T(0);
        if constexpr (BF16) {
          raw = make_uint4(t[0] | (unsigned int)t[1] << 16, t[2] | (unsigned int)t[3] << 16,
                           t[4] | (unsigned int)t[5] << 16, t[6] | (unsigned int)t[7] << 16);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = t[i];
        }
      }
    } else if constexpr (!BF16) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
    if constexpr (COLS) {
      if constexpr (BF16) {
        *reinterpret_cast<uint4*>(tile + tile_word<kWords>(tr, g * 4)) = raw;
      } else {
        *reinterpret_cast<float4*>(tile + tile_word<kWords>(tr, g * 8)) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(tile + tile_word<kWords>(tr, g * 8 + 4)) = make_float4(v[4], v[5], v[6], v[7]);
      }
    }
    if constexpr (ROWS) {
      unsigned int sb, q;
      if constexpr (BF16) {
        const unsigned int w[4] = {raw.x, raw.y, raw.z, raw.w};
        unsigned int m = max_abs_bf16x2(max_abs_bf16x2(w[0], w[1]), max_abs_bf16x2(w[2], w[3]));
        m = max_abs_bf16x2(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max_abs_bf16x2(m, __shfl_xor_sync(0xffffffffu, m, 2));
        m = max_abs_bf16x2(m, m >> 16);
        sb = mx_scale_byte((m >> 7) & 0xffu);
        q = mx_codes8(w, ((254u - sb) << 7) * 0x10001u);
      } else {
        float m = max_abs(max_abs(max_abs(v[0], v[1]), max_abs(v[2], v[3])), max_abs(max_abs(v[4], v[5]), max_abs(v[6], v[7])));
        m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, 2));
        sb = mx_scale_byte((__float_as_uint(m) >> 23) & 0xffu);
        q = mx_codes8(v, mx_inverse(sb));
      }
      if (r < rows && (c & ~31ll) < cols) {
        *reinterpret_cast<unsigned int*>(out.codes + (size_t)r * (size_t)mx_pitch(cols) + (size_t)(c >> 1)) = q;
        if ((g & 3) == 0) s_row[(tr & 31) * 16 + (tr >> 5) * 4 + (g >> 2)] = (unsigned char)sb;
      }
    }
  }
  __syncthreads();
  if constexpr (COLS) {
    // thread: row block rb of one column (fp32) or of a pair of columns (bf16)
    const int rb = (tid >> 3) & 3;
    const bool any = r0 + rb * 32 < rows;
    if constexpr (BF16) {
      const int cw = (tid & 7) + (tid >> 5) * 8;              // word = pair of columns
      unsigned int w[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) w[i] = tile[tile_word<kWords>(rb * 32 + i, cw)];
      unsigned int m = max_abs_bf16x2(w[0], w[1]);
#pragma unroll
      for (int i = 2; i < 32; ++i) m = max_abs_bf16x2(m, w[i]);
      const unsigned int sb[2] = {mx_scale_byte((m >> 7) & 0xffu), mx_scale_byte((m >> 23) & 0xffu)};
      const unsigned int inv = (((254u - sb[0]) << 7) & 0xffffu) | ((254u - sb[1]) << 23);
#pragma unroll
      for (int i = 0; i < 32; ++i) w[i] = mul_bf16x2(w[i], inv);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int tc = 2 * cw + h;
        uint4 q;
        unsigned int* qp = reinterpret_cast<unsigned int*>(&q);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i)
            v[i] = __uint_as_float(h ? w[k * 8 + i] & 0xffff0000u : w[k * 8 + i] << 16);
          qp[k] = mx_pack8(v);
        }
        if (any && c0 + tc < cols) {
          *reinterpret_cast<uint4*>(out_t.codes + (size_t)(c0 + tc) * (size_t)mx_pitch(rows) +
                                    (size_t)(r0 / 2 + rb * 16)) = q;
          s_col[(tc & 31) * 16 + (tc >> 5) * 4 + rb] = (unsigned char)sb[h];
        }
      }
    } else {
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        const int tc = (tid & 7) + (tid >> 5) * 8 + h * 64;
        float v[32], m = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          v[i] = __uint_as_float(tile[tile_word<kWords>(rb * 32 + i, tc)]);
          m = max_abs(m, v[i]);
        }
        const unsigned int sb = mx_scale_byte((__float_as_uint(m) >> 23) & 0xffu);
        const float inv = mx_inverse(sb);
        uint4 q;
        unsigned int* qp = reinterpret_cast<unsigned int*>(&q);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float u[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] = v[k * 8 + i];
          qp[k] = mx_codes8(u, inv);
        }
        if (any && c0 + tc < cols) {
          *reinterpret_cast<uint4*>(out_t.codes + (size_t)(c0 + tc) * (size_t)mx_pitch(rows) +
                                    (size_t)(r0 / 2 + rb * 16)) = q;
          s_col[(tc & 31) * 16 + (tc >> 5) * 4 + rb] = (unsigned char)sb;
        }
      }
    }
    __syncthreads();
  }
  // the atoms; tiles past the end exist to write the padding atoms' zeros
  if (tid < kMxAtom / 16) {
    if (ROWS && r0 < rows && ct < mx_atoms(cols))
      reinterpret_cast<uint4*>(out.scales + (size_t)(rt * mx_atoms(cols) + ct) * kMxAtom)[tid] =
          reinterpret_cast<const uint4*>(s_row)[tid];
    if (COLS && c0 < cols && rt < mx_atoms(rows))
      reinterpret_cast<uint4*>(out_t.scales + (size_t)(ct * mx_atoms(rows) + rt) * kMxAtom)[tid] =
          reinterpret_cast<const uint4*>(s_col)[tid];
  }
}

// -------------------------------------------------------------- dequantisation
//
// A lane takes four bytes of codes (eight elements), a warp 256 columns of a row, so
// that loads and stores are contiguous; a CTA takes 32 rows of such a strip.  A
// nibble s eem placed as sign, exponent field 0..3 and top mantissa bit of a bf16
// is its value times 2^-126, subnormals included: two
// exact multiplications (2^126, the scale) give the result without a conversion
// instruction, which issue at a fraction of the rate.

// Nibbles 2j and 2j+1 of w as a pair of bf16 values, unscaled.
__device__ __forceinline__ unsigned int mx_pair(unsigned int w, int j) {
  const unsigned int t = w >> (8 * j);
  const unsigned int n = (t & 0xfu) | ((t & 0xf0u) << 12);
  return mul_bf16x2(((n & 0x00070007u) << 6) | ((n & 0x00080008u) << 12), 0x7e807e80u);
}

// The scale as a bf16 pair: 2^-127 is a subnormal, 0xFF is NaN.
__device__ __forceinline__ unsigned int mx_scale_pair(unsigned int sb) {
  const unsigned int h = sb == 255u ? 0x7fc0u : sb == 0u ? 0x0040u : sb << 7;
  return h | h << 16;
}

constexpr int kDequantThreads = 256, kDequantCols = 256, kDequantRows = 32;

template <bool OUT_BF16>
__global__ void __launch_bounds__(kDequantThreads)
ps_mx_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, long long rows,
                        long long cols, void* __restrict__ out, long long ld, int vec_ok, unsigned int col_tiles) {
  mx_pdl();
  constexpr int kSteps = kDequantRows / (kDequantThreads / 32);
  const long long r0 = (long long)(blockIdx.x / col_tiles) * kDequantRows + (threadIdx.x >> 5);
  const long long c = (long long)(blockIdx.x % col_tiles) * kDequantCols + (threadIdx.x & 31) * 8;
  if (c >= cols) return;
  const size_t pitch = (size_t)mx_pitch(cols);
  unsigned int w[kSteps], sb[kSteps];
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    const long long r = r0 + k * (kDequantThreads / 32);
    if (r < rows) {
      w[k] = __ldcs(reinterpret_cast<const unsigned int*>(codes + (size_t)r * pitch + (size_t)(c >> 1)));
      sb[k] = scales[mx_scale_at(r, c >> 5, mx_atoms(cols))];
    }
  }
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    const long long r = r0 + k * (kDequantThreads / 32);
    if (r >= rows) break;
    const unsigned int s = mx_scale_pair(sb[k]);
    unsigned int v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = mul_bf16x2(mx_pair(w[k], j), s);
    if constexpr (OUT_BF16) {
      unsigned short* o = static_cast<unsigned short*>(out) + (size_t)r * (size_t)ld + (size_t)c;
      if (vec_ok && c + 8 <= cols) {
        *reinterpret_cast<uint4*>(o) = make_uint4(v[0], v[1], v[2], v[3]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < cols) o[i] = (unsigned short)(i & 1 ? v[i >> 1] >> 16 : v[i >> 1] & 0xffffu);
      }
    } else {
      float* o = static_cast<float*>(out) + (size_t)r * (size_t)ld + (size_t)c;
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
      if (vec_ok && c + 8 <= cols) {
        *reinterpret_cast<float4*>(o) = make_float4(f[0], f[1], f[2], f[3]);
        *reinterpret_cast<float4*>(o + 4) = make_float4(f[4], f[5], f[6], f[7]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c + i < cols) o[i] = f[i];
      }
    }
  }
}

}  // namespace psb
