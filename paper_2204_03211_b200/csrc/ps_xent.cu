// Host side of the cross entropy over a vocabulary (declarations and contracts: include/ps_b200.h).
#include <algorithm>
#include <cstdint>
#include <cstring>
#include <mutex>

#include "ps_op.h"
#include "ps_xent.cuh"

namespace psb {
namespace {

static __device__ int g_xent_status;

constexpr int kXeMaxDevices = 64;
// (A tile sums over the tokens, the width or a piece of the words: 0.3 s for the longest, where bounded waits are a second.
// TMA coordinates are 32-bit.)
constexpr long long kXeMaxTokens = 1ll << 26, kXeMaxWidth = 1ll << 24, kXeMaxWords = 1ll << 30;

struct XeDevice {
  bool ready = false;
  int* status = nullptr;
};
std::mutex g_xent_mu;
XeDevice g_xent_dev[kXeMaxDevices];

int xent_device(const OpDevice& d, int** status) {
  std::lock_guard<std::mutex> lk(g_xent_mu);
  XeDevice& x = g_xent_dev[d.id];
  if (!x.ready) {
    void* p = nullptr;
    cudaError_t e = cudaGetSymbolAddress(&p, g_xent_status);
    for (const auto kernel : {ps_tc_kernel<XeOp<8>>, ps_tc_kernel<XeOp<16>>})
      if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, TcCfg<XeOp<8>>::kSmem);
    if (e != cudaSuccess) return op_cuda_error("preparing the cross entropy", e);
    x.status = static_cast<int*>(p);
    x.ready = true;
  }
  *status = x.status;
  return PS_OK;
}

bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }
size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// How the gradients' pass is cut, and where everything lies in the workspace.  It depends on the sizes alone, so that
// ps_xent_sizes and the calls agree whatever device they run on.
struct XePlan {
  long long nparts, pitch, piece, pieces;
  int slices, dw_slices;                 // of dx, per piece; of dw
  size_t parts, score, xm, d[2], sums, dw_sums, x, w, end, end_unaligned;
};

// A piece of d: as many words as make 5 x 2^22 entries (40 MB), whole tiles, at least one.
constexpr long long kXePieceEntries = 5ll << 22;
constexpr int kXePairs = 74;             // CTA pairs that the cuts are made for
constexpr int kXeMaxSlices = 64, kXeMinStages = 16;
constexpr long long kXeSliceRows = 1ll << 14;    // slices x tokens, where there is more than one slice
constexpr long long kXeDwSliceRows = 1ll << 12;  // slices x words, the same for dw

XePlan xent_plan(long long T, long long V, long long D) {
  XePlan p;
  p.nparts = ceil_div(V, kXeTile / (xe_warps(D) / 4));
  p.pitch = ceil_div(D, 8) * 8;
  const long long all = ceil_div(V, kXeTile) * kXeTile;
  // (equal pieces: a short last one would leave the launches around it half empty)
  const long long most_words = std::min(all, std::max<long long>(1, kXePieceEntries / std::max(1ll, T) / kXeTile) * kXeTile);
  p.piece = ceil_div(ceil_div(V, ceil_div(V, most_words)), kXeTile) * kXeTile;
  p.pieces = ceil_div(V, p.piece);
  // dx has few tiles, each as long as the piece has words: its words are shared out to slices until one is no longer
  // than half of what a pair computes in a launch
  const long long tm = ceil_div(T, kXeTile), td = ceil_div(D, kXeTile), tv = p.piece / kXeTile, nk = p.piece / kXeK;
  const long long total = tm * tv * ceil_div(D, kXeK) + tm * td * nk + tv * td * ceil_div(T, kXeK);
  const long long longest = std::max<long long>(kXeMinStages, total / kXePairs / 2);
  const long long most_slices = std::min<long long>(kXeMaxSlices, std::max(1ll, kXeSliceRows / std::max(1ll, T)));
  p.slices = (int)std::min(most_slices, std::max(1ll, ceil_div(nk, longest)));
  // Few words: dw has few tiles, as long as there are tokens, which are shared out in the same way (6144 x 256 x 272, loss
  // and gradients: 58 us with one slice, 41 with six)
  const long long most_dw = std::min<long long>(kXeMaxSlices, std::max(1ll, kXeDwSliceRows / V));
  p.dw_slices = p.pieces == 1 ? (int)std::min(most_dw, std::max(1ll, ceil_div(ceil_div(T, kXeK), longest))) : 1;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += round256(bytes);
    return here;
  };
  p.xm = take((size_t)T * (size_t)p.pitch * 2);
  const size_t shared = at;              // the losses' pass is done with its part before the gradients' pass begins
  p.parts = take((size_t)T * (size_t)p.nparts * sizeof(float2));
  p.score = take((size_t)T * sizeof(float));
  const size_t forward = at;
  at = shared;
  for (int b = 0; b < 2; ++b) p.d[b] = take(b < p.pieces ? (size_t)T * (size_t)p.piece * 2 : 0);
  p.sums = take(p.slices > 1 || p.pieces > 1 ? (size_t)p.slices * (size_t)T * (size_t)p.pitch * sizeof(float) : 0);
  p.dw_sums = take(p.dw_slices > 1 ? (size_t)p.dw_slices * (size_t)V * (size_t)p.pitch * sizeof(float) : 0);
  at = std::max(at, forward);
  p.end = at;
  p.x = take((size_t)T * (size_t)p.pitch * 2);
  p.w = take((size_t)V * (size_t)p.pitch * 2);
  p.end_unaligned = at;
  return p;
}

// What any call of at most T tokens needs (a smaller batch is cut into larger pieces and more slices).
size_t xent_bytes(long long T, long long V, long long D, bool unaligned) {
  const size_t pitch = (size_t)ceil_div(D, 8) * 8, all = (size_t)ceil_div(V, kXeTile) * kXeTile, t = (size_t)T;
  const size_t x = (unaligned ? 2 : 1) * round256(t * pitch * 2), w = unaligned ? round256((size_t)V * pitch * 2) : 0;
  const size_t parts = round256(t * (size_t)ceil_div(V, 64) * sizeof(float2)) + round256(t * sizeof(float));
  const size_t piece = std::max(std::min(t * all, (size_t)kXePieceEntries), t * kXeTile);
  const size_t rows = std::max(t, std::min(t * kXeMaxSlices, (size_t)kXeSliceRows));
  const size_t dw_rows = 2 * V <= kXeDwSliceRows ? (size_t)std::min(V * kXeMaxSlices, kXeDwSliceRows) : 0;
  return std::max<size_t>(256, x + w + std::max(parts, 2 * round256(piece * 2) + round256(rows * pitch * sizeof(float)) +
                                                           round256(dw_rows * pitch * sizeof(float))));
}

bool make_map(EncodeTiled encode, CUtensorMap* m, const void* p, long long rows, long long cols, long long ld) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {64, 64}, step[2] = {1, 1};
  return encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct XeCall {
  const ps_xent* q;
  XePlan plan;
  OpDevice dev;
  cudaStream_t stream;
  char* ws;
  bool copy_x, copy_w;                   // rows that no tensor map can walk are copied first
  XeArgs args;
};

int row_alignment(const void* p, long long bytes) {
  const uintptr_t bits = reinterpret_cast<uintptr_t>(p) | (uintptr_t)bytes;
  return bits % 32 == 0 ? 32 : bits % 16 == 0 ? 16 : 1;
}

bool rows_aligned(const void* p, long long ld) { return !misaligned(p, 16) && ld % 8 == 0; }

int check(const ps_xent* q, XeCall* c) {
  if (!q || q->tokens < 0 || q->vocab < 1 || q->dim < 1 || q->tokens > kXeMaxTokens || q->vocab > kXeMaxWords ||
      q->dim > kXeMaxWidth || q->ldx < q->dim || q->ldw < q->dim || (q->target_bits != 32 && q->target_bits != 64))
    return PS_ERR_BAD_ARG;
  if (!q->w || !q->workspace || (q->tokens > 0 && (!q->x || !q->targets))) return PS_ERR_BAD_ARG;
  if (misaligned(q->x, 2) || misaligned(q->w, 2) || misaligned(q->targets, q->target_bits / 8) || misaligned(q->workspace, 256))
    return PS_ERR_ALIGN;
  if (ceil_div(q->tokens, kXeTile) * ceil_div(q->vocab, kXeTile) > 0x3fffffffll ||
      ceil_div(q->vocab, kXeTile) * ceil_div(q->dim, kXeTile) > 0x3fffffffll)
    return PS_ERR_TOO_LARGE;
  c->q = q;
  c->plan = xent_plan(q->tokens, q->vocab, q->dim);
  c->copy_w = !rows_aligned(q->w, q->ldw);
  c->copy_x = q->tokens > 0 && !rows_aligned(q->x, q->ldx);
  if (q->workspace_bytes < (c->copy_w || c->copy_x ? c->plan.end_unaligned : c->plan.end)) return PS_ERR_NOMEM;
  return PS_OK;
}

XeCopy copy_of(const XeCall& c, const void* src, long long rows, long long ld, size_t to, bool mask, const float* weights) {
  return XeCopy{static_cast<const unsigned short*>(src), reinterpret_cast<unsigned short*>(c.ws + to), rows, c.q->dim, ld, c.plan.pitch,
                mask ? c.q->targets : nullptr, c.q->target_bits == 64 ? 1 : 0, rows_aligned(src, ld) ? 1 : 0, c.q->vocab, weights};
}

// Rows that no tensor map can walk, into the workspace.
int copy_rows(const XeCall& c) {
  const ps_xent* q = c.q;
  XeCopy x = XeCopy(), w = XeCopy();
  if (c.copy_x) x = copy_of(c, q->x, q->tokens, q->ldx, c.plan.x, false, nullptr);
  if (c.copy_w) w = copy_of(c, q->w, q->vocab, q->ldw, c.plan.w, false, nullptr);
  const long long units = std::max(x.rows, w.rows) * (c.plan.pitch / 8);
  const unsigned grid = (unsigned)std::min<long long>(ceil_div(units, kXeCopyThreads), (long long)c.dev.num_sms * 8);
  return op_launch("cross entropy", ps_xent_copy_kernel, grid, kXeCopyThreads, 0, 1, c.stream, x, w);
}

// What both passes set up.
int begin(XeCall* c, void* stream, bool backward) {
  const ps_xent* q = c->q;
  const XePlan& p = c->plan;
  c->stream = static_cast<cudaStream_t>(stream);
  c->ws = static_cast<char*>(q->workspace);
  int rc = op_device(&c->dev);
  if (rc) return rc;
  std::memset(&c->args, 0, sizeof c->args);
  XeArgs& a = c->args;
  rc = xent_device(c->dev, &a.status);
  if (rc) return rc;
  EncodeTiled encode;
  rc = op_encoder(&encode);
  if (rc) return rc;
  a.T = q->tokens;
  a.V = q->vocab;
  a.D = q->dim;
  a.targets = q->targets;
  a.target64 = q->target_bits == 64;
  bool ok = c->copy_x ? make_map(encode, &a.x, c->ws + p.x, a.T, a.D, p.pitch) : make_map(encode, &a.x, q->x, a.T, a.D, q->ldx);
  ok = ok && (c->copy_w ? make_map(encode, &a.w, c->ws + p.w, a.V, a.D, p.pitch) : make_map(encode, &a.w, q->w, a.V, a.D, q->ldw));
  if (backward) {
    ok = ok && make_map(encode, &a.xm, c->ws + p.xm, a.T, a.D, p.pitch);
    for (int b = 0; b < 2 && b < p.pieces; ++b) ok = ok && make_map(encode, &a.d[b], c->ws + p.d[b], a.T, p.piece, p.piece);
  }
  if (!ok) return op_cuda_error("tensor map", cudaErrorInvalidValue);
  return c->copy_x || c->copy_w ? copy_rows(*c) : PS_OK;
}

int add_slices(const XeCall& c, const XeSum& q) {
  const unsigned grid = (unsigned)std::min<long long>(ceil_div(q.rows * (q.pitch / 4), kXeCopyThreads), (long long)c.dev.num_sms * 16);
  return op_launch("cross entropy", ps_xent_slices_kernel, grid, kXeCopyThreads, 0, 1, c.stream, q);
}

// Launches the segments of c->args, the longest tiles first.
int launch_segments(XeCall* c) {
  XeArgs& a = c->args;
  std::stable_sort(a.seg, a.seg + a.nseg, [](const XeSeg& p, const XeSeg& q) { return p.nk / p.slices > q.nk / q.slices; });
  long long tiles = 0;
  for (int i = 0; i < a.nseg; ++i) {
    a.seg[i].first = (int)tiles;
    tiles += (long long)a.seg[i].tiles_m * a.seg[i].tiles_n * a.seg[i].slices;
  }
  if (tiles > 0x3fffffffll) return PS_ERR_TOO_LARGE;
  a.tiles = (int)tiles;
  // (pairs beyond the tiles only copy, four pieces per thread: 192 x 305 x 1256, loss and gradients: 72 us with the two pairs of its tiles, 39
  // with 59)
  const long long copies = a.side.src ? ceil_div(a.side.rows * (a.side.pitch / 8), kTcSideThreads * 2 * 4) : 0;
  const unsigned grid = 2u * (unsigned)std::min<long long>(std::max(tiles, copies), c->dev.num_sms / 2);
  const bool many = xe_warps(a.D) == 16;
  return op_launch("cross entropy", many ? ps_tc_kernel<XeOp<16>> : ps_tc_kernel<XeOp<8>>, grid,
                   many ? TcCfg<XeOp<16>>::kThreads : TcCfg<XeOp<8>>::kThreads, TcCfg<XeOp<8>>::kSmem, 1, c->stream, a);
}

}  // namespace
}  // namespace psb

using namespace psb;

extern "C" {

int ps_xent_sizes(long long tokens, long long vocab, long long dim, size_t* bytes_out, size_t* bytes_unaligned_out) {
  if (tokens < 0 || vocab < 1 || dim < 1 || tokens > kXeMaxTokens || vocab > kXeMaxWords || dim > kXeMaxWidth) return PS_ERR_BAD_ARG;
  if (bytes_out) *bytes_out = xent_bytes(tokens, vocab, dim, false);
  if (bytes_unaligned_out) *bytes_unaligned_out = xent_bytes(tokens, vocab, dim, true);
  return PS_OK;
}

int ps_xent_forward(const ps_xent* q, float* loss, float* lse, void* stream) {
  XeCall c;
  int rc = check(q, &c);
  if (rc) return rc;
  if (q->tokens == 0) return PS_OK;
  if (!loss && !lse) return PS_ERR_BAD_ARG;
  if (misaligned(loss, 4) || misaligned(lse, 4)) return PS_ERR_ALIGN;
  rc = begin(&c, stream, false);
  if (rc) return rc;
  XeArgs& a = c.args;
  a.parts = reinterpret_cast<float2*>(c.ws + c.plan.parts);
  a.nparts = (int)c.plan.nparts;
  a.score = reinterpret_cast<float*>(c.ws + c.plan.score);
  a.nseg = 1;
  a.seg[0] = XeSeg{kXeStats, 0, (int)ceil_div(a.T, kXeTile), (int)ceil_div(a.V, kXeTile), 0, (int)ceil_div(a.D, kXeK), 1, 0, 0, 0};
  rc = launch_segments(&c);
  if (rc) return rc;
  return op_launch("cross entropy", ps_xent_join_kernel, (unsigned)ceil_div(a.T, kXeJoinThreads / 32), kXeJoinThreads, 0, 1,
                   c.stream, (const float2*)a.parts, a.nparts, (const float*)a.score, a.targets, a.target64, a.T, a.V, loss, lse);
}

int ps_xent_backward(const ps_xent* q, const float* lse, float scale, const float* token_scale, void* dx, long long lddx,
                     void* dw, int dw_dtype, long long lddw, void* stream) {
  XeCall c;
  int rc = check(q, &c);
  if (rc) return rc;
  if ((!dx && !dw) || (dw_dtype != PS_F32 && dw_dtype != PS_BF16) || (dx && lddx < q->dim) || (dw && lddw < q->dim))
    return PS_ERR_BAD_ARG;
  if (q->tokens > 0 && !lse) return PS_ERR_BAD_ARG;
  const size_t es = dw_dtype == PS_F32 ? 4 : 2;
  if (misaligned(lse, 4) || misaligned(token_scale, 4) || misaligned(dx, 2) || misaligned(dw, es)) return PS_ERR_ALIGN;
  if (q->tokens == 0) {                  // a sum over nothing
    if (!dw) return PS_OK;
    const cudaError_t e = cudaMemset2DAsync(dw, (size_t)lddw * es, 0, (size_t)q->dim * es, (size_t)q->vocab,
                                            static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? PS_OK : op_cuda_error("ps_xent_backward", e);
  }
  rc = begin(&c, stream, true);
  if (rc) return rc;
  XeArgs& a = c.args;
  const XePlan& p = c.plan;
  a.lse = lse;
  a.weights = token_scale;
  a.scale = scale;
  for (int b = 0; b < 2; ++b) a.d_out[b] = reinterpret_cast<__nv_bfloat16*>(c.ws + p.d[b]);
  a.piece = (int)p.piece;
  a.dx_sums = reinterpret_cast<float*>(c.ws + p.sums);
  a.dx = static_cast<__nv_bfloat16*>(dx);
  a.dw = dw;
  a.ld_dx = lddx;
  a.ld_dw = lddw;
  a.dw_f32 = dw_dtype == PS_F32;
  a.dx_align = row_alignment(dx, lddx * 2);
  a.dw_align = row_alignment(dw, lddw * (long long)es);
  a.pitch = (int)p.pitch;
  a.dw_sums = reinterpret_cast<float*>(c.ws + p.dw_sums);
  const int tm = (int)ceil_div(a.T, kXeTile), td = (int)ceil_div(a.D, kXeTile);
  int filled = 0;                        // slices of dx's sums that hold something
  const int dw_slices = std::min<int>(p.dw_slices, (int)ceil_div(a.T, kXeK));
  for (long long k = 0; k <= p.pieces; ++k) {
    a.nseg = 0;
    a.side = XeCopy();
    if (k == 0 && dw) a.side = copy_of(c, q->x, q->tokens, q->ldx, p.xm, true, token_scale);
    if (k < p.pieces) {
      const long long v0 = k * p.piece, words = std::min(p.piece, a.V - v0);
      a.seg[a.nseg++] = XeSeg{kXeProb, 0, tm, (int)ceil_div(words, kXeTile), (int)v0, (int)ceil_div(a.D, kXeK), 1, (int)(k & 1), 0, 0};
    }
    if (k > 0) {
      const long long v0 = (k - 1) * p.piece, words = std::min(p.piece, a.V - v0);
      const int nk = (int)ceil_div(words, kXeK), buf = (int)((k - 1) & 1);
      if (dx) {
        const int slices = std::min(p.slices, nk);       // (the last piece may be short; earlier ones filled all)
        a.seg[a.nseg++] = XeSeg{kXeDx, 0, tm, td, (int)v0, nk, slices, buf, k == 1, k == p.pieces && p.slices == 1};
        filled = std::max(filled, slices);
      }
      if (dw) a.seg[a.nseg++] = XeSeg{kXeDw, 0, (int)ceil_div(words, kXeTile), td, (int)v0, (int)ceil_div(a.T, kXeK), dw_slices, buf, 0, 0};
    }
    rc = launch_segments(&c);
    if (rc) return rc;
  }
  if (dx && p.slices > 1)
    rc = add_slices(c, XeSum{a.dx_sums, filled, a.pitch, a.T, a.D, lddx, dx, 0, !misaligned(dx, 8) && a.D % 4 == 0 && lddx % 4 == 0, scale,
                             a.targets, a.target64, a.V, token_scale});
  if (!rc && dw && dw_slices > 1)
    rc = add_slices(c, XeSum{a.dw_sums, dw_slices, a.pitch, a.V, a.D, lddw, dw, a.dw_f32,
                             !misaligned(dw, 4 * es) && a.D % 4 == 0 && lddw % 4 == 0, scale, nullptr, 0, 0, nullptr});
  return rc;
}

int ps_xent_status(int* status_out) {
  if (!status_out) return PS_ERR_BAD_ARG;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(status_out, g_xent_status, sizeof(int));
  return e == cudaSuccess ? PS_OK : op_cuda_error("ps_xent_status", e);
}

}  // extern "C"
