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

#include "ps_mma.cuh"

namespace psb {

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

// The products of two pairs of bf16 values, in binary32: a mixed-precision fma unpacks and multiplies at once.  It adds
// -0, which keeps the sign of a zero.  (A product of pairs, then unpacked, made both directions 22.0 instead of 20.4 us
// for 8192 x 4096.)
__device__ __forceinline__ void mx_divide(unsigned int w, unsigned int inv, float* lo, float* hi) {
  asm("{\n\t"
      ".reg .b16 a0, a1, s0, s1;\n\t"
      "mov.b32 {a0, a1}, %2;\n\t"
      "mov.b32 {s0, s1}, %3;\n\t"
      "fma.rn.f32.bf16 %0, a0, s0, %4;\n\t"
      "fma.rn.f32.bf16 %1, a1, s1, %4;\n\t"
      "}"
      : "=f"(*lo), "=f"(*hi)
      : "r"(w), "r"(inv), "f"(-0.0f));
}

// Eight bf16 values as codes.  inv: 1 / scale of the values' block, twice.
__device__ __forceinline__ unsigned int mx_codes8(const unsigned int (&w)[4], unsigned int inv) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) mx_divide(w[i], inv, &v[2 * i], &v[2 * i + 1]);
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

// ---------------------------------------------------------------- quantisation
//
// One CTA per 128 x 128 tile, i.e. one atom of scales in each direction.  The tile
// goes to shared memory with asynchronous 16-byte copies, all of them in flight at
// once (read through registers, with a few loads in flight per thread, the kernel
// waited for memory: 35 us for 8192 x 4096 bf16 both ways against 22.5 then); both
// directions then cost one read of x.  Along the rows a block sits in two
// neighbouring lanes (one shuffle gives its maximum); along the columns a thread
// takes one block of 32 rows of one column (a pair of columns of bf16) and reads it
// twice, for the maximum and for the codes, which halves its registers.  The four
// row blocks of a column sit in one warp and are stored as 64 bytes; their shared
// memory reads would meet in the same banks (a stride of 32 rows is a multiple of 32
// banks whatever the pitch), so the column index is permuted by the row block.
//
// Measured on 8192 x 4096 bf16, three matrices in rotation: rows 14.6 us (5.8 TB/s of
// values and codes), columns 15.3 us, both 20.1 us (5.1 TB/s); fp32 25.4, 26.2 and 32.2 us
// (5.3 TB/s).  Both at once keep 67 % of the issue slots busy, and the largest stall is
// the wait for the tile.  Five CTAs per SM: with six the column pass spills (21.6 us).
// Rows that are not 16-byte aligned go through registers, element by element: 8191 x 4095
// both ways 35 us from bf16, 65 us from fp32.

constexpr int kQuantThreads = 256;

template <bool BF16>
struct MxIn;
template <>
struct MxIn<false> { using T = float; };
template <>
struct MxIn<true> { using T = unsigned short; };

// Word of the tile in shared memory that holds column word c of row r.
template <int WORDS>
__device__ __forceinline__ int tile_word(int r, int c) { return r * WORDS + (c ^ (((r >> 5) & 3) << 3)); }

__device__ __forceinline__ void copy16(unsigned int dst, const void* src, unsigned int bytes) {   // the rest is zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

template <bool BF16, bool ROWS, bool COLS>
__global__ void __launch_bounds__(kQuantThreads, BF16 ? 5 : 3)
ps_mx_quantize_kernel(const typename MxIn<BF16>::T* __restrict__ x, int rows, int cols, long long ld, int vec_ok,
                      unsigned int col_tiles, MxOut out, MxOut out_t) {
  using T = typename MxIn<BF16>::T;
  constexpr int kWords = BF16 ? 64 : 128;                     // 32-bit words of a tile row
  constexpr int kPiece = 16 / sizeof(T);                      // elements of a copy
  constexpr int kPieces = kMxTile / kPiece;                   // copies of a tile row
  extern __shared__ __align__(16) unsigned int tile[];        // 128 rows of kWords
  __shared__ __align__(16) unsigned char s_row[kMxAtom], s_col[kMxAtom];
  const int tid = threadIdx.x;
  const int rt = (int)(blockIdx.x / col_tiles), ct = (int)(blockIdx.x % col_tiles);
  const int r0 = rt * kMxTile, c0 = ct * kMxTile;            // (rows and columns stay below 2^30)
  const unsigned int pitch = (unsigned int)mx_pitch(cols), pitch_t = (unsigned int)mx_pitch(rows);
  if (tid < kMxAtom / 4) {
    if (ROWS) reinterpret_cast<unsigned int*>(s_row)[tid] = 0u;
    if (COLS) reinterpret_cast<unsigned int*>(s_col)[tid] = 0u;
  }
  mm_pdl();

  {
    constexpr int kStepRows = kQuantThreads / kPieces;
    const int g = tid % kPieces, rr = tid / kPieces;
    const int c = c0 + g * kPiece;
    const int left = cols - c;                                // elements of this thread's pieces inside the matrix
    const unsigned int n = left <= 0 ? 0u : left < kPiece ? (unsigned int)left : (unsigned int)kPiece;
    const T* p = x + (size_t)(r0 + rr) * (size_t)ld + (size_t)c;
#pragma unroll
    for (int step = 0; step < kMxTile / kStepRows; ++step) {
      const int tr = step * kStepRows + rr;
      unsigned int* w = tile + tile_word<kWords>(tr, g * 4);
      const unsigned int k = r0 + tr < rows ? n : 0u;
      if (vec_ok) {
        copy16((unsigned int)__cvta_generic_to_shared(w), k ? p : x, k * (unsigned int)sizeof(T));
      } else {
        T t[kPiece];
#pragma unroll
        for (int i = 0; i < kPiece; ++i) t[i] = (unsigned int)i < k ? p[i] : T(0);
        if constexpr (BF16)
          *reinterpret_cast<uint4*>(w) = make_uint4(t[0] | (unsigned int)t[1] << 16, t[2] | (unsigned int)t[3] << 16,
                                                    t[4] | (unsigned int)t[5] << 16, t[6] | (unsigned int)t[7] << 16);
        else
          *reinterpret_cast<float4*>(w) = make_float4(t[0], t[1], t[2], t[3]);
      }
      p += (size_t)kStepRows * (size_t)ld;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  }
  __syncthreads();

  if constexpr (ROWS) {
    // 8 lanes of 16 elements cover a row of the tile, 32 rows per step; two neighbouring lanes hold a block
    const int g = tid & 7, rr = tid >> 3;
    const int c = c0 + g * 16, first = g >> 2;                // which half a lane reads first: eight lanes then meet in no bank
    uint8_t* codes = out.codes + (size_t)(r0 + rr) * pitch + (size_t)(c >> 1);
#pragma unroll 2
    for (int step = 0; step < 4; ++step) {
      const int tr = step * 32 + rr;
      unsigned int sb, q[2];
      if constexpr (BF16) {
        // (8 words: the permutation moves them together)
        const uint4* p = reinterpret_cast<const uint4*>(tile + tile_word<kWords>(tr, g * 8));
        const uint4 u0 = p[first], u1 = p[first ^ 1];
        const unsigned int w0[4] = {u0.x, u0.y, u0.z, u0.w}, w1[4] = {u1.x, u1.y, u1.z, u1.w};
        unsigned int m = max_abs_bf16x2(max_abs_bf16x2(max_abs_bf16x2(w0[0], w0[1]), max_abs_bf16x2(w0[2], w0[3])),
                                        max_abs_bf16x2(max_abs_bf16x2(w1[0], w1[1]), max_abs_bf16x2(w1[2], w1[3])));
        m = max_abs_bf16x2(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max_abs_bf16x2(m, m >> 16);
        sb = mx_scale_byte((m >> 7) & 0xffu);
        const unsigned int inv = ((254u - sb) << 7) * 0x10001u;
        q[0] = mx_codes8(w0, inv);
        q[1] = mx_codes8(w1, inv);
      } else {
        // (halves of 8 elements, which the permutation moves apart, two 16-byte pieces each, in an order that also
        // depends on the lane: the codes of the two pieces change places below)
        const float4* p0 = reinterpret_cast<const float4*>(tile + tile_word<kWords>(tr, g * 16 + first * 8));
        const float4* p1 = reinterpret_cast<const float4*>(tile + tile_word<kWords>(tr, g * 16 + (first ^ 1) * 8));
        const int piece = (g >> 1) & 1;
        const float4 a = p0[piece], b = p0[piece ^ 1], d = p1[piece], e = p1[piece ^ 1];
        const float v0[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, v1[8] = {d.x, d.y, d.z, d.w, e.x, e.y, e.z, e.w};
        float m = max_abs(v0[0], v1[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) m = max_abs(m, max_abs(v0[i], v1[i]));
        m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, 1));
        sb = mx_scale_byte((__float_as_uint(m) >> 23) & 0xffu);
        const float inv = mx_inverse(sb);
        q[0] = mx_codes8(v0, inv);
        q[1] = mx_codes8(v1, inv);
        q[0] = __funnelshift_l(q[0], q[0], 16 * piece);
        q[1] = __funnelshift_l(q[1], q[1], 16 * piece);
      }
      if (r0 + tr < rows && (c & ~31) < cols) {
        *reinterpret_cast<uint2*>(codes) = first ? make_uint2(q[1], q[0]) : make_uint2(q[0], q[1]);
        if ((g & 1) == 0) s_row[(tr & 31) * 16 + (tr >> 5) * 4 + (g >> 1)] = (unsigned char)sb;
      }
      codes += 32 * (size_t)pitch;
    }
  }
  if constexpr (COLS) {
    // thread: row block rb of one column (fp32) or of a pair of columns (bf16)
    const int rb = (tid >> 3) & 3;
    const bool any = r0 + rb * 32 < rows;
    uint8_t* codes = out_t.codes + (r0 / 2 + rb * 16);
    if constexpr (BF16) {
      const int cw = (tid & 7) + (tid >> 5) * 8;              // word = pair of columns
      const unsigned int* w = tile + tile_word<kWords>(rb * 32, cw);    // (the permutation is the same in all 32 rows)
      unsigned int m = 0u;
#pragma unroll
      for (int i = 0; i < 32; ++i) m = max_abs_bf16x2(m, w[i * kWords]);
      const unsigned int sb[2] = {mx_scale_byte((m >> 7) & 0xffu), mx_scale_byte((m >> 23) & 0xffu)};
      const unsigned int inv = (((254u - sb[0]) << 7) & 0xffffu) | ((254u - sb[1]) << 23);
      unsigned int lo[4], hi[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float a[8], b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          mx_divide(w[(k * 8 + i) * kWords], inv, &a[i], &b[i]);
        }
        lo[k] = mx_pack8(a);
        hi[k] = mx_pack8(b);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int tc = 2 * cw + h;
        if (any && c0 + tc < cols) {
          *reinterpret_cast<uint4*>(codes + (size_t)(c0 + tc) * pitch_t) =
              h ? make_uint4(hi[0], hi[1], hi[2], hi[3]) : make_uint4(lo[0], lo[1], lo[2], lo[3]);
          s_col[(tc & 31) * 16 + (tc >> 5) * 4 + rb] = (unsigned char)sb[h];
        }
      }
    } else {
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        const int tc = (tid & 7) + (tid >> 5) * 8 + h * 64;
        const float* w = reinterpret_cast<const float*>(tile) + tile_word<kWords>(rb * 32, tc);
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) m = max_abs(m, w[i * kWords]);
        const unsigned int sb = mx_scale_byte((__float_as_uint(m) >> 23) & 0xffu);
        const float inv = mx_inverse(sb);
        unsigned int q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float u[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) u[i] = w[(k * 8 + i) * kWords];
          q[k] = mx_codes8(u, inv);
        }
        if (any && c0 + tc < cols) {
          *reinterpret_cast<uint4*>(codes + (size_t)(c0 + tc) * pitch_t) = make_uint4(q[0], q[1], q[2], q[3]);
          s_col[(tc & 31) * 16 + (tc >> 5) * 4 + rb] = (unsigned char)sb;
        }
      }
    }
  }
  __syncthreads();
  // the atoms; tiles past the end exist to write the padding atoms' zeros
  if (tid < kMxAtom / 16) {
    if (ROWS && r0 < rows && ct < mx_atoms(cols))
      reinterpret_cast<uint4*>(out.scales + (size_t)((long long)rt * mx_atoms(cols) + ct) * kMxAtom)[tid] =
          reinterpret_cast<const uint4*>(s_row)[tid];
    if (COLS && c0 < cols && rt < mx_atoms(rows))
      reinterpret_cast<uint4*>(out_t.scales + (size_t)((long long)ct * mx_atoms(rows) + rt) * kMxAtom)[tid] =
          reinterpret_cast<const uint4*>(s_col)[tid];
  }
}

// -------------------------------------------------------------- dequantisation
//
// A lane takes eight bytes of codes (sixteen elements, half a block), a warp 512
// columns of a row, so that a lane stores whole sectors; a CTA takes 32 rows of such a
// strip.  A nibble s eem placed as sign, exponent field 0..3 and top mantissa bit of a
// bf16 is its value times 2^-126, subnormals included: two exact multiplications
// (2^126, the scale) give the result without conversion instructions, which issue at a
// fraction of the rate.  8192 x 4096 to bf16, three matrices in rotation: 14.8 us, 5.7 TB/s
// of codes and values; one again and again, out of L2 in part, 12.0 us (with eight elements
// per lane and 128-bit stores 15.3 us).  Rows that allow no wide stores are written element
// by element: 8191 x 4095 takes 197 us to bf16, 152 us to fp32.

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

constexpr int kDequantThreads = 256, kDequantCols = 512, kDequantRows = 32;

template <bool OUT_BF16>
__global__ void __launch_bounds__(kDequantThreads)
ps_mx_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, long long rows,
                        long long cols, void* __restrict__ out, long long ld, int vec_ok, unsigned int col_tiles) {
  mm_pdl();
  constexpr int kSteps = kDequantRows / (kDequantThreads / 32);
  const long long r0 = (long long)(blockIdx.x / col_tiles) * kDequantRows + (threadIdx.x >> 5);
  const long long c = (long long)(blockIdx.x % col_tiles) * kDequantCols + (threadIdx.x & 31) * 16;
  if (c >= cols) return;
  const size_t pitch = (size_t)mx_pitch(cols);
  uint2 w[kSteps];
  unsigned int sb[kSteps];
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    const long long r = r0 + k * (kDequantThreads / 32);
    if (r < rows) {
      w[k] = __ldcs(reinterpret_cast<const uint2*>(codes + (size_t)r * pitch + (size_t)(c >> 1)));
      sb[k] = scales[mx_scale_at(r, c >> 5, mx_atoms(cols))];
    }
  }
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    const long long r = r0 + k * (kDequantThreads / 32);
    if (r >= rows) break;
    const unsigned int s = mx_scale_pair(sb[k]);
    unsigned int v[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = mul_bf16x2(mx_pair(w[k].x, j), s);
      v[4 + j] = mul_bf16x2(mx_pair(w[k].y, j), s);
    }
    if constexpr (OUT_BF16) {
      unsigned short* o = static_cast<unsigned short*>(out) + (size_t)r * (size_t)ld + (size_t)c;
      if (vec_ok == 2 && c + 16 <= cols) {
        store_sector(o, v);
      } else if (vec_ok && c + 16 <= cols) {
        reinterpret_cast<uint4*>(o)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<uint4*>(o)[1] = make_uint4(v[4], v[5], v[6], v[7]);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (c + i < cols) o[i] = (unsigned short)(i & 1 ? v[i >> 1] >> 16 : v[i >> 1] & 0xffffu);
      }
    } else {
      float* o = static_cast<float*>(out) + (size_t)r * (size_t)ld + (size_t)c;
      unsigned int f[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16;
      if (vec_ok == 2 && c + 16 <= cols) {
        store_sector(o, f);
        store_sector(o + 8, f + 8);
      } else if (vec_ok && c + 16 <= cols) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          reinterpret_cast<uint4*>(o)[i] = make_uint4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (c + i < cols) o[i] = __uint_as_float(f[i]);
      }
    }
  }
}

}  // namespace psb
