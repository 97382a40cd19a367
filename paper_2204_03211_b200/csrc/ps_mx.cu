// Host side of the 4-bit operators (declarations and contracts: include/ps_b200.h).
#include <algorithm>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <string>

#include "ps_mx_pair.cuh"
#include "ps_op.h"

namespace psb {

static thread_local std::string g_op_err;

int op_cuda_error(const char* what, cudaError_t e) {
  try {
    g_op_err = std::string(what) + ": " + cudaGetErrorString(e);
  } catch (...) {
  }
  cudaGetLastError();
  return e == cudaErrorMemoryAllocation ? PS_ERR_NOMEM : PS_ERR_CUDA;
}

constexpr int kOpMaxDevices = 64;
static std::mutex g_op_mu;
static OpDevice g_op_dev[kOpMaxDevices];

int op_device(OpDevice* out) {
  int id = -1;
  cudaError_t e = cudaGetDevice(&id);
  if (e != cudaSuccess) return op_cuda_error("cudaGetDevice", e);
  if (id < 0 || id >= kOpMaxDevices) return PS_ERR_BAD_ARG;
  std::lock_guard<std::mutex> lk(g_op_mu);
  OpDevice& d = g_op_dev[id];
  if (d.id < 0) {
    e = cudaDeviceGetAttribute(&d.num_sms, cudaDevAttrMultiProcessorCount, id);
    if (e != cudaSuccess) return op_cuda_error("cudaDeviceGetAttribute", e);
    d.id = id;
  }
  *out = d;
  return PS_OK;
}

namespace {

static __device__ int g_mx_status;

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Per device: the address of the status word, and that the product kernels may use their shared memory.
struct MxDevice {
  bool ready = false;
  int* status = nullptr;
};
MxDevice g_mx_dev[kOpMaxDevices];
EncodeTiled g_encode = nullptr;

template <int BN>
cudaError_t allow_smem() {
  return cudaFuncSetAttribute(ps_mx_matmul_kernel<BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, MmCfg<BN>::kSmem);
}

int mx_device(const OpDevice& d, int** status) {
  std::lock_guard<std::mutex> lk(g_op_mu);
  MxDevice& m = g_mx_dev[d.id];
  if (!m.ready) {
    void* p = nullptr;
    cudaError_t e = cudaGetSymbolAddress(&p, g_mx_status);
    if (e == cudaSuccess) e = allow_smem<16>();
    if (e == cudaSuccess) e = allow_smem<64>();
    if (e == cudaSuccess) e = allow_smem<128>();
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(ps_mx_matmul_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem);
    if (e == cudaSuccess && !g_encode) {
      void* fn = nullptr;
      cudaDriverEntryPointQueryResult q;
      e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
      if (e == cudaSuccess && (q != cudaDriverEntryPointSuccess || !fn)) e = cudaErrorNotSupported;
      if (e == cudaSuccess) g_encode = reinterpret_cast<EncodeTiled>(fn);
    }
    if (e != cudaSuccess) return op_cuda_error("preparing the 4-bit product", e);
    m.status = static_cast<int*>(p);
    m.ready = true;
  }
  *status = m.status;
  return PS_OK;
}

bool bad_dtype(int t) { return t != PS_F32 && t != PS_BF16; }
size_t esize(int t) { return t == PS_BF16 ? 2 : 4; }
bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

constexpr long long kMxMaxDim = 1ll << 30;       // rows and columns of an operand (TMA coordinates are 32-bit)

int check_operand(const ps_mx* q) {
  if (!q || q->rows < 0 || q->cols < 1 || q->rows >= kMxMaxDim || q->cols >= kMxMaxDim) return PS_ERR_BAD_ARG;
  if (q->rows > 0 && (!q->codes || !q->scales)) return PS_ERR_BAD_ARG;
  if (misaligned(q->codes, 16) || misaligned(q->scales, 16)) return PS_ERR_ALIGN;
  return PS_OK;
}

// A launch that may overlap its prologue with the tail of the stream's previous one (it waits for that launch to
// complete before it touches memory), optionally in clusters.
template <typename... KArgs, typename... Args>
int launch(const char* what, void (*kernel)(KArgs...), unsigned int grid, int block, size_t smem, int cluster,
           cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
  return e == cudaSuccess ? PS_OK : op_cuda_error(what, e);
}

template <bool BF16, bool ROWS, bool COLS>
int quantize(const void* x, long long rows, long long cols, long long ld, MxOut out, MxOut out_t, cudaStream_t stream) {
  using T = typename MxIn<BF16>::T;
  // the tiles that hold data, plus one row or column of tiles where a padding atom has to be written
  const long long nc = ROWS ? mx_atoms(cols) : (cols + 127) / 128, nr = COLS ? mx_atoms(rows) : (rows + 127) / 128;
  if (nc * nr > 0x7fffffffll) return PS_ERR_TOO_LARGE;
  const int vec_ok = !misaligned(x, 16) && (ld * (long long)sizeof(T)) % 16 == 0;
  const size_t smem = (size_t)kMxTile * kMxTile * sizeof(T);
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(ps_mx_quantize_kernel<BF16, ROWS, COLS>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return op_cuda_error("cudaFuncSetAttribute", e);
  }
  return launch("quantise", ps_mx_quantize_kernel<BF16, ROWS, COLS>, (unsigned)(nc * nr), kQuantThreads, smem, 1, stream,
                static_cast<const T*>(x), (int)rows, (int)cols, ld, vec_ok, (unsigned)nc, out, out_t);
}

bool make_map(CUtensorMap* m, const ps_mx* q, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)mx_pitch(q->cols), (cuuint64_t)q->rows};
  const cuuint64_t strides[1] = {(cuuint64_t)mx_pitch(q->cols)};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, step[2] = {1, 1};
  return g_encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, q->codes, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Atoms of scales, two (a stage's) at a time.
bool make_scale_map(CUtensorMap* m, const ps_mx* q) {
  const cuuint64_t dims[2] = {kMxAtom / 4, (cuuint64_t)((q->rows + 127) / 128 * mx_atoms(q->cols))};
  const cuuint64_t strides[1] = {kMxAtom};
  const cuuint32_t box[2] = {kMxAtom / 4, 2}, step[2] = {1, 1};
  return g_encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, q->scales, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int matmul_pair(const ps_mx* a, const ps_mx* b, MmArgs args, const OpDevice& d, cudaStream_t stream) {
  CUtensorMap ma, mb, msa, msb;
  if (!make_map(&ma, a, 128) || !make_map(&mb, b, 128) || !make_scale_map(&msa, a) || !make_scale_map(&msb, b))
    return op_cuda_error("tensor map", cudaErrorInvalidValue);
  const long long tp = (a->rows + kPairTile - 1) / kPairTile, tq = (b->rows + kPairTile - 1) / kPairTile;
  if (tp * tq > 0x3fffffffll || std::max(tp, tq) * 2 * args.atoms > 0x7fffffffll) return PS_ERR_TOO_LARGE;
  args.tiles_p = (int)tp;
  args.tiles_q = (int)tq;
  const unsigned int grid = 2u * (unsigned)std::min<long long>(tp * tq, d.num_sms / 2);
  return launch("4-bit product", ps_mx_matmul_pair_kernel, grid, kPairThreads, kPairSmem, 1, stream, ma, mb, msa, msb, args);
}

template <int BN>
int matmul(const ps_mx* p, const ps_mx* q, MmArgs args, const OpDevice& d, cudaStream_t stream) {
  using Cfg = MmCfg<BN>;
  CUtensorMap mp, mq;
  if (!make_map(&mp, p, kMmP) || !make_map(&mq, q, BN)) return op_cuda_error("tensor map", cudaErrorInvalidValue);
  const long long tp = (p->rows + kMmP - 1) / kMmP, tq = (q->rows + BN - 1) / BN;
  if (tp * tq > 0x3fffffffll) return PS_ERR_TOO_LARGE;
  args.tiles_p = (int)tp;
  args.tiles_q = (int)tq;
  const int tiles = (int)(tp * tq);
  // few tiles: 2, 4 or 8 CTAs share a tile's K while that many CTAs fit and each keeps four stages; with fewer the sum
  // of the parts costs more than it saves (1 x 4096 x 1024: 5.2 us as 4 x 1 stage, 3.8 us unsplit; 1 x 1024 x 4096:
  // 4.7 us as 4 x 4 stages, 5.3 us as 2 x 8)
  args.splits = 1;
  const int room = d.num_sms * Cfg::kCtas;
  while (args.splits < 8 && tiles * args.splits * 2 <= room && args.splits * 8 <= args.stages_k) args.splits *= 2;
  const unsigned int grid = args.splits > 1 ? (unsigned)(tiles * args.splits) : (unsigned)std::min(tiles, room);
  return launch("4-bit product", ps_mx_matmul_kernel<BN>, grid, kMmThreads, Cfg::kSmem, args.splits, stream, mp, mq, args);
}

}  // namespace
}  // namespace psb

using namespace psb;

extern "C" {

const char* ps_op_last_error(void) { return g_op_err.c_str(); }

int ps_mx_sizes(long long rows, long long cols, size_t* code_bytes_out, size_t* scale_bytes_out) {
  if (rows < 0 || cols < 1 || rows >= kMxMaxDim || cols >= kMxMaxDim) return PS_ERR_BAD_ARG;
  if (code_bytes_out) *code_bytes_out = (size_t)rows * (size_t)mx_pitch(cols);
  if (scale_bytes_out) *scale_bytes_out = (size_t)((rows + 127) / 128) * (size_t)mx_atoms(cols) * kMxAtom;
  return PS_OK;
}

int ps_mx_quantize(const void* x, int dtype, long long rows, long long cols, long long ld, const ps_mx* q,
                   const ps_mx* qt, void* stream_) {
  if (bad_dtype(dtype) || (!q && !qt) || rows < 0 || cols < 1 || ld < cols) return PS_ERR_BAD_ARG;
  if (rows > 0 && !x) return PS_ERR_BAD_ARG;
  if (misaligned(x, esize(dtype))) return PS_ERR_ALIGN;
  // (the transposed operand of a matrix without rows would have no columns: its description still has to match)
  if (rows == 0) return !q || (q->rows == 0 && q->cols == cols) ? PS_OK : PS_ERR_BAD_ARG;
  int rc = q ? check_operand(q) : PS_OK;
  if (!rc && qt) rc = check_operand(qt);
  if (rc) return rc;
  if (q && (q->rows != rows || q->cols != cols)) return PS_ERR_BAD_ARG;
  if (qt && (qt->rows != cols || qt->cols != rows)) return PS_ERR_BAD_ARG;
  const MxOut o = {q ? static_cast<uint8_t*>(q->codes) : nullptr, q ? static_cast<uint8_t*>(q->scales) : nullptr};
  const MxOut t = {qt ? static_cast<uint8_t*>(qt->codes) : nullptr, qt ? static_cast<uint8_t*>(qt->scales) : nullptr};
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  if (dtype == PS_BF16) {
    if (q && qt) return quantize<true, true, true>(x, rows, cols, ld, o, t, stream);
    if (q) return quantize<true, true, false>(x, rows, cols, ld, o, t, stream);
    return quantize<true, false, true>(x, rows, cols, ld, o, t, stream);
  }
  if (q && qt) return quantize<false, true, true>(x, rows, cols, ld, o, t, stream);
  if (q) return quantize<false, true, false>(x, rows, cols, ld, o, t, stream);
  return quantize<false, false, true>(x, rows, cols, ld, o, t, stream);
}

int ps_mx_dequantize(const ps_mx* q, int dtype, void* out, long long ld, void* stream_) {
  int rc = check_operand(q);
  if (rc) return rc;
  if (bad_dtype(dtype) || ld < q->cols) return PS_ERR_BAD_ARG;
  if (q->rows == 0) return PS_OK;
  if (!out) return PS_ERR_BAD_ARG;
  if (misaligned(out, esize(dtype))) return PS_ERR_ALIGN;
  const long long nc = (q->cols + kDequantCols - 1) / kDequantCols, nr = (q->rows + kDequantRows - 1) / kDequantRows;
  if (nc * nr > 0x7fffffffll) return PS_ERR_TOO_LARGE;
  // 2: rows that allow 256-bit stores, 1: 128-bit ones
  const long long row = ld * (long long)esize(dtype);
  const int vec_ok = !misaligned(out, 32) && row % 32 == 0 ? 2 : !misaligned(out, 16) && row % 16 == 0;
  const uint8_t *codes = static_cast<const uint8_t*>(q->codes), *scales = static_cast<const uint8_t*>(q->scales);
  return launch("dequantise", dtype == PS_BF16 ? ps_mx_dequantize_kernel<true> : ps_mx_dequantize_kernel<false>,
                (unsigned)(nc * nr), kDequantThreads, 0, 1, static_cast<cudaStream_t>(stream_), codes, scales, q->rows,
                q->cols, out, ld, vec_ok, (unsigned)nc);
}

int ps_mx_matmul(const ps_mx* a, const ps_mx* b, int dtype, void* c, long long ldc, void* stream_) {
  int rc = check_operand(a);
  if (!rc) rc = check_operand(b);
  if (rc) return rc;
  if (bad_dtype(dtype) || a->cols != b->cols || ldc < b->rows) return PS_ERR_BAD_ARG;
  if (a->rows == 0 || b->rows == 0) return PS_OK;
  if (!c) return PS_ERR_BAD_ARG;
  if (misaligned(c, esize(dtype))) return PS_ERR_ALIGN;
  OpDevice d;
  rc = op_device(&d);
  if (rc) return rc;
  MmArgs args;
  std::memset(&args, 0, sizeof args);
  rc = mx_device(d, &args.status);
  if (rc) return rc;
  const bool thin = std::min(a->rows, b->rows) <= 64;
  args.swap = thin && a->rows < b->rows;
  const ps_mx *p = args.swap ? b : a, *q = args.swap ? a : b;
  args.sp = static_cast<const uint8_t*>(p->scales);
  args.sq = static_cast<const uint8_t*>(q->scales);
  args.c = c;
  args.ldc = ldc;
  args.rows_p = p->rows;
  args.rows_q = q->rows;
  args.atoms = mx_atoms(a->cols);
  args.stages_k = (int)((a->cols + kMmStageK - 1) / kMmStageK);
  args.out_f32 = dtype == PS_F32;
  args.vec_ok = !misaligned(c, 16) && (ldc * (long long)esize(dtype)) % 16 == 0;
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  if (thin && q->rows <= 16) return matmul<16>(p, q, args, d, stream);
  if (thin) return matmul<64>(p, q, args, d, stream);
  // Up to one 128 x 128 tile per SM those tiles are taken, beyond that the pairs', which read each operand less often;
  // where 128 x 128 would leave half of the SMs idle, 128 x 64, two CTAs on an SM.  Pairs | 128 x 128 | 128 x 64 in us:
  // 2048 x 2048 x 4096 10.7 | 11.5 | 14.7, 1536 x 2048 x 4096 10.3 | 11.1 | 13.2, 1024 x 2048 x 4096 9.8 | 7.6 | 8.9,
  // 1024 x 1024 x 4096 9.4 | 10.2 | 9.5, 1024 x 1024 x 512 5.2 | 4.6 | 4.4, 256 x 1024 x 512 5.1 | 4.5 | 3.8
  const long long tiles = ((p->rows + 127) / 128) * ((q->rows + 127) / 128);
  if (tiles > d.num_sms) return matmul_pair(p, q, args, d, stream);
  if (tiles <= d.num_sms / 2) return matmul<64>(p, q, args, d, stream);
  return matmul<128>(p, q, args, d, stream);
}

int ps_mx_status(int* status_out) {
  if (!status_out) return PS_ERR_BAD_ARG;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(status_out, g_mx_status, sizeof(int));
  return e == cudaSuccess ? PS_OK : op_cuda_error("ps_mx_status", e);
}

}  // extern "C"
