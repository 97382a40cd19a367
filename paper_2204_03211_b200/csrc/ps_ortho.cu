// Host side of the orthogonalisation (declarations and contracts: include/ps_b200.h).
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <functional>
#include <mutex>
#include <new>
#include <utility>

#include "ps_ortho.h"
#include "ps_ortho_small.cuh"

namespace psb {
namespace {

constexpr int kNsMaxDevices = 64;
constexpr long long kNsMaxDim = 1ll << 24;       // (a tile of the longest product takes 0.3 s, bounded waits a second)
constexpr long long kNsMaxTiles = 1ll << 26;     // tiles and units of a list

struct NsDevice {
  bool ready = false;
  int room[2][2];                        // by split and pair: tiles that are worked on together
};
std::mutex g_ns_mu;
NsDevice g_ns_dev[kNsMaxDevices];

// The four kernels: two planes or one, pairs of CTAs or single ones.
struct NsKernel {
  void (*fn)(NsArgs);
  int smem, ctas;
};
template <int PLANES, bool PAIR>
NsKernel kernel_as() {
  return {ps_tc_kernel<NsOp<PLANES, PAIR>>, TcCfg<NsOp<PLANES, PAIR>>::kSmem, PAIR ? 2 : 1};
}
NsKernel kernel_of(bool split, bool pair) {
  return split ? (pair ? kernel_as<2, true>() : kernel_as<2, false>()) : (pair ? kernel_as<1, true>() : kernel_as<1, false>());
}

int ns_device(bool split, bool pair, int* room) {
  OpDevice d;
  int rc = op_device(&d);
  if (rc) return rc;
  std::lock_guard<std::mutex> lk(g_ns_mu);
  NsDevice& n = g_ns_dev[d.id];
  if (!n.ready) {
    for (int s = 0; s < 2; ++s)
      for (int p = 0; p < 2; ++p) {
        const NsKernel k = kernel_of(s, p);
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)k.ctas);
        cfg.blockDim = dim3(TcCfg<NsOp<1, false>>::kThreads);
        cfg.dynamicSmemBytes = (size_t)k.smem;
        int clusters = 0;
        cudaError_t e = cudaFuncSetAttribute(k.fn, cudaFuncAttributeMaxDynamicSharedMemorySize, k.smem);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&clusters, k.fn, &cfg);
        if (e != cudaSuccess) return op_cuda_error("preparing the orthogonalisation", e);
        n.room[s][p] = std::max(1, std::min(clusters, d.num_sms / k.ctas));
      }
    cudaError_t e = cudaFuncSetAttribute(ps_ortho_small_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSoSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(ps_ortho_small_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSoSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(ps_ortho_small_kernel<1>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(ps_ortho_small_kernel<2>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return op_cuda_error("preparing the orthogonalisation", e);
    n.ready = true;
  }
  *room = n.room[split][pair];
  return PS_OK;
}

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }
size_t round256(size_t n) { return (n + 255) / 256 * 256; }
bool empty(const NsItem& it) { return it.rows == 0 || it.cols == 0; }

// Where a matrix's working memory lies.
struct NsLayout {
  long long m, n, pitch_x, pitch_e;
  size_t x[2][2], e[2], f[2], d, fd, parts, end;
  long long units;
};

NsLayout layout(const NsItem& it, bool split, size_t at) {
  NsLayout l;
  l.m = std::min(it.rows, it.cols);
  l.n = std::max(it.rows, it.cols);
  l.pitch_x = ceil_div(l.n, 64) * 64;
  l.pitch_e = ceil_div(l.m, 64) * 64;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += round256(bytes);
    return here;
  };
  const size_t x = (size_t)l.m * (size_t)l.pitch_x * 2, e = (size_t)l.m * (size_t)l.pitch_e * 2;
  for (int b = 0; b < 2; ++b)
    for (int p = 0; p < 2; ++p) l.x[b][p] = take(x);
  for (int p = 0; p < 2; ++p) l.e[p] = take(p == 0 || split ? e : 0);
  for (int p = 0; p < 2; ++p) l.f[p] = take(p == 0 || split ? e : 0);
  const size_t d = (size_t)ceil_div(l.m, 256) * 256 * sizeof(float);      // (read by whole tiles)
  l.d = take(d);
  l.fd = take(d);
  l.units = ceil_div(it.rows, kNsUnitRows) * ceil_div(it.cols, kNsUnitCols);
  l.parts = take(it.parts ? 0 : (size_t)l.units * sizeof(double));
  l.end = at;
  return l;
}

// A plane by boxes of `rows` x `cols`, rows of 128 bytes in 128-byte swizzle or of 64 in 64-byte swizzle.
bool make_map(EncodeTiled encode, CUtensorMap* m, const void* p, long long rows, long long cols, long long pitch, int box_rows,
              int box_cols) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)pitch * 2};
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, step[2] = {1, 1};
  return encode(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(p), dims, strides, box, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Matrices whose products of one kind go out together: as many as a workspace of 128 MB holds, which L2 keeps, or, where
// that is fewer, as have this many tiles, so that what a tile waits for has long been done.  (One group of 200 of 192 x 192 instead of
// four, to fp32: 644 and 347 us; half as many groups for 24 layers 1024 wide, 4.3 GB: 16.4 and 17.8 ms.)
constexpr long long kNsGroupTiles = 2 * 74;
constexpr int kNsGroupBytesLog = 27;

// What a tile costs besides its products, in elements of k.
constexpr long long kNsTileCost = 256;

// Pairs of CTAs (256 x 256 tiles) fetch half as much from L2 per product as single ones (128 x 128), which waste less where
// sides are not multiples of 256, and share out what there is more evenly.  Pairs are taken where they compute at most
// 1.2 times as much, every pair has a tile even of A, and there are more than 200 in all.  Single | pairs, us:
//   to fp32  20 x 1024 x 1024 1385 | 1152, 200 x 192 x 192 350 | 306, 32 x 200 x 2571 525 | 606, 16 x 640 x 2560 983 | 1066
//   to bf16  24 x 1024 x 4096 2779 | 2213, 24 x 512 x 512 209 | 253, 96 x 300 x 300 323 | 425
constexpr long long kNsPairs = 74, kNsPairsFrom = 200;
bool take_pairs(const std::vector<NsItem>& items) {
  long long rows = 0, square = 0, all[2] = {0, 0};
  for (const NsItem& it : items) {
    if (empty(it)) continue;
    const long long m = std::min(it.rows, it.cols), n = std::max(it.rows, it.cols);
    rows += ceil_div(m, 256) * ceil_div(n, 256);
    square += ceil_div(m, 256) * ceil_div(m, 256);
    for (int p = 0; p < 2; ++p) {
      const long long tm = ceil_div(m, 128 << p), tn = ceil_div(n, 128 << p);
      all[p] += 2 * tm * tm + tm * tn;
    }
  }
  return rows > kNsPairsFrom && square >= kNsPairs && 5 * 4 * all[1] <= 6 * all[0];
}

}  // namespace

// A list of small matrices only stays in shared memory: CTAs per matrix, 0 for other lists.  There one matrix may be done
// before another is read, so a result that lies where another matrix comes from takes the general form, which reads all
// sources first.
static int small_ctas(const std::vector<NsItem>& items) {
  struct Range { uintptr_t first, end; int of; };
  std::vector<Range> srcs;
  long long widest = 0;
  uintptr_t longest = 0;
  auto range = [](const void* p, long long ld, const NsItem& it, size_t es, int of) {
    const uintptr_t first = reinterpret_cast<uintptr_t>(p);
    return Range{first, first + ((size_t)(it.rows - 1) * (size_t)ld + (size_t)it.cols) * es, of};
  };
  for (size_t i = 0; i < items.size(); ++i) {
    const NsItem& it = items[i];
    if (empty(it)) continue;
    if (std::min(it.rows, it.cols) > kSoRows || std::max(it.rows, it.cols) > kSoCtas * kSoCols) return 0;
    widest = std::max(widest, std::max(it.rows, it.cols));
    srcs.push_back(range(it.src, it.ld_src, it, it.src_bf16 ? 2 : 4, (int)i));
    longest = std::max(longest, srcs.back().end - srcs.back().first);
  }
  if (srcs.empty()) return 0;
  std::sort(srcs.begin(), srcs.end(), [](const Range& a, const Range& b) { return a.first < b.first; });
  for (size_t i = 0; i < items.size(); ++i) {
    const NsItem& it = items[i];
    if (empty(it) || !it.dst) continue;
    const Range d = range(it.dst, it.ld_dst, it, it.out == kNsOutBf16 ? 2 : 4, (int)i);
    const uintptr_t reach = d.first > longest ? d.first - longest : 0;       // (only sources that start from here on can overlap)
    auto s = std::lower_bound(srcs.begin(), srcs.end(), reach, [](const Range& a, uintptr_t v) { return a.first < v; });
    for (; s != srcs.end() && s->first < d.end; ++s)
      if (s->of != d.of && s->end > d.first) return 0;
  }
  // One CTA where it can hold a matrix.  Else 128 columns each rather than 256, so four CTAs at least: what every CTA does for
  // itself gets shorter, adding up A does not get longer (four of 128 x 512: 81 us on two CTAs each, 66 on four).  Seven
  // clusters of sixteen run at a time; for more than two turns the general form is as fast or faster (12 | 16 | 32 of
  // 128 x 4096 to bf16: 155 | 232 | 389 us here, 191 | 218 | 341 there), and for 2048 columns clusters of eight (20 to fp32:
  // 193 us, on sixteen 258).
  if (widest <= kSoCols) return 1;
  if (widest > kSoCtas / 2 * kSoCols) return srcs.size() <= 14 ? kSoCtas : 0;
  int ctas = 4;
  while (ctas < kSoCtas / 2 && ctas * (kSoCols / 2) < widest) ctas *= 2;
  return ctas;
}

size_t NsPlan::workspace(const std::vector<NsItem>& items, bool split) {
  if (small_ctas(items)) return 256;
  size_t at = 0;
  long long tiles = 0, units = 0;
  for (const NsItem& it : items) {
    if (empty(it)) continue;
    const NsLayout l = layout(it, split, at);
    at = l.end;
    const long long tm = ceil_div(l.m, 128), tn = ceil_div(l.n, 128);
    if (tm > (1ll << 13) || tn > (1ll << 20)) return 0;
    tiles += kNsSteps * (2 * tm * tm + tm * tn);
    units += l.units;
    if (tiles > kNsMaxTiles || units > kNsMaxTiles) return 0;
  }
  return std::max<size_t>(at, 256);
}

NsPlan::~NsPlan() {
  if (mem_) cudaFree(mem_);              // (waits for launches that still use it)
}

void NsPlan::adopt(NsPlan& old) {
  std::swap(mem_, old.mem_);             // (what this one had goes with the old one)
  std::swap(cap_, old.cap_);
}

int NsPlan::build(const std::vector<NsItem>& items, bool split, void* workspace, int* status, cudaStream_t stream) {
  small_ = small_ctas(items);
  pair_ = take_pairs(items);
  const long long tile = pair_ ? 256 : 128;
  int room = 0;
  int rc = ns_device(split, pair_, &room);
  if (rc) return rc;
  EncodeTiled encode;
  rc = op_encoder(&encode);
  if (rc) return rc;
  char* ws = static_cast<char*>(workspace);
  std::vector<const NsItem*> live;
  for (const NsItem& it : items)
    if (!empty(it)) live.push_back(&it);
  const size_t n = live.size();
  if (n == 0) return PS_OK;
  std::vector<CUtensorMap> maps(small_ ? 0 : kNsMaps * n);
  std::vector<NsMat> mats(n);
  std::vector<NsTile> list;
  std::vector<int> begin, owner;
  std::vector<int2> units;
  std::memset(mats.data(), 0, n * sizeof(NsMat));
  std::memset(maps.data(), 0, maps.size() * sizeof(CUtensorMap));
  size_t at = 0;
  long long sym_tiles = 0, square_tiles = 0;
  for (const NsItem* it : live) {
    const long long tm = ceil_div(std::min(it->rows, it->cols), tile);
    square_tiles += tm * tm;
  }
  // Few tiles: all of them have a CTA anyway, and storing a tile twice takes an epilogue 4 us longer (3 x 777 x 300 to
  // fp32: 215 us mirrored, 187 us not)
  const bool mirror = square_tiles > room;
  for (size_t i = 0; i < n; ++i) {
    const NsItem& it = *live[i];
    NsMat& M = mats[i];
    M.m = (int)std::min(it.rows, it.cols);
    M.n = (int)std::max(it.rows, it.cols);
    M.flip = it.rows > it.cols;
    M.out = it.out;
    M.src = it.src;
    M.ld_src = it.ld_src;
    M.src_bf16 = it.src_bf16;
    M.dst = it.dst;
    M.ld_dst = it.ld_dst;
    const size_t es = it.out == kNsOutBf16 ? 2 : 4;
    M.wide = !M.flip && (reinterpret_cast<uintptr_t>(it.dst) & 31u) == 0 && it.ld_dst * (long long)es % 32 == 0;
    M.decay = it.decay;
    M.step = it.step;
    M.stat = it.stat;
    if (small_) continue;
    const NsLayout l = layout(it, split, at);
    at = l.end;
    auto half_at = [&](size_t o) { return reinterpret_cast<__half*>(ws + o); };
    M.pitch_x = l.pitch_x;
    M.pitch_e = l.pitch_e;
    bool ok = true;
    CUtensorMap* map = &maps[kNsMaps * i];
    auto plane = [&](int at_map, const void* p, long long cols, long long pitch, int box_rows, int box_cols) {
      ok = ok && make_map(encode, map + at_map, p, l.m, cols, pitch, box_rows, box_cols);
    };
    for (int b = 0; b < 2; ++b)
      for (int p = 0; p < 2; ++p) {
        M.x[b][p] = half_at(l.x[b][p]);
        plane(2 * b + p, M.x[b][p], l.n, l.pitch_x, split ? 32 : 64, 64);
        plane(kNsTall + 2 * b + p, M.x[b][p], l.n, l.pitch_x, 128, 32);
      }
    for (int p = 0; p < (split ? 2 : 1); ++p) {
      M.e[p] = half_at(l.e[p]);
      M.f[p] = half_at(l.f[p]);
      if (!split) {
        plane(4, M.e[p], l.m, l.pitch_e, 64, 64);
        plane(6, M.f[p], l.m, l.pitch_e, 64, 64);
      }
      plane(kNsTall + 4 + p, M.e[p], l.m, l.pitch_e, 128, 32);
      plane(kNsTall + 6 + p, M.f[p], l.m, l.pitch_e, 128, 32);
      plane(kNsMirror + p, M.e[p], l.m, l.pitch_e, 32, 32);
      plane(kNsMirror + 2 + p, M.f[p], l.m, l.pitch_e, 32, 32);
    }
    if (!ok) return op_cuda_error("tensor map", cudaErrorInvalidValue);
    M.d = reinterpret_cast<float*>(ws + l.d);
    M.fd = reinterpret_cast<float*>(ws + l.fd);
    M.parts = it.parts ? it.parts : reinterpret_cast<double*>(ws + l.parts);
    M.nparts = it.parts ? it.nparts : (int)l.units;
    if (!it.parts) norms_ = true;
    const int tm = (int)ceil_div(l.m, tile), tn = (int)ceil_div(l.n, tile);
    M.mirror = mirror;
    for (int a = 0; a < tm; ++a) {
      const int ctas = pair_ && l.m - a * tile > 128 ? 2 : 1;
      M.parts_s += (mirror ? a + 1 : tm) * ctas;
      M.parts_x += tn * ctas;
    }
    sym_tiles += mirror ? tm * (tm + 1) / 2 : tm * tm;
    for (long long u = 0; u < l.units; ++u) units.push_back(make_int2((int)i, (int)u));
  }
  // the tiles: matrices dealt to groups, a group's products one kind after the other
  const size_t groups = std::max<size_t>(1, std::min({n, (size_t)(sym_tiles / kNsGroupTiles), at >> kNsGroupBytesLog}));
  for (size_t g = 0; !small_ && g < groups; ++g)
    for (int step = 0; step < kNsSteps; ++step)
      for (int product = 0; product < 3; ++product)
        for (size_t i = g; i < n; i += groups) {
          const int tm = (int)ceil_div(mats[i].m, tile), tn = (int)ceil_div(mats[i].n, tile);
          for (int a = 0; a < tm; ++a)
            for (int b = 0; b < (product == 2 ? tn : mirror ? a + 1 : tm); ++b)
              list.push_back(NsTile{(int)i, (short)step, (short)product, a, b});
        }
  // each tile to the CTA (or pair) that has least to do so far, every CTA's in the order of all
  if (!small_) {
    const int workers = (int)std::min<size_t>(list.size(), (size_t)room);
    using Load = std::pair<long long, int>;
    std::vector<Load> loads;
    for (int w = 0; w < workers; ++w) loads.push_back(Load(0, w));
    begin.assign((size_t)workers + 1, 0);
    for (const NsTile& t : list) {       // (a heap of loads: least first)
      std::pop_heap(loads.begin(), loads.end(), std::greater<Load>());
      Load& l = loads.back();
      owner.push_back(l.second);
      ++begin[(size_t)l.second + 1];
      l.first += (t.product == 0 ? mats[(size_t)t.mat].n : mats[(size_t)t.mat].m) + kNsTileCost;
      std::push_heap(loads.begin(), loads.end(), std::greater<Load>());
    }
    for (int w = 0; w < workers; ++w) begin[(size_t)w + 1] += begin[(size_t)w];
    std::vector<NsTile> dealt(list.size());
    std::vector<int> at_worker(begin.begin(), begin.end() - 1);
    for (size_t t = 0; t < list.size(); ++t) dealt[(size_t)at_worker[(size_t)owner[t]]++] = list[t];
    list.swap(dealt);
    grid_ = workers * (pair_ ? 2 : 1);
  }
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t here = off;
    off += round256(bytes);
    return here;
  };
  const size_t maps_off = take(maps.size() * sizeof(CUtensorMap));
  mats_off_ = take(n * sizeof(NsMat));
  list_off_ = take(list.size() * sizeof(NsTile));
  begin_off_ = take(begin.size() * sizeof(int));
  units_off_ = take(units.size() * sizeof(int2));
  const size_t done_off = take(n * sizeof(unsigned int) * 32);         // a line each
  const size_t status_off = take(sizeof(int));
  cudaError_t e = cudaSuccess;
  if (off > cap_) {
    if (mem_) cudaFree(mem_);
    mem_ = nullptr;
    cap_ = 4096;                         // (powers of two: the next set's tables are likely to fit)
    while (cap_ < off) cap_ *= 2;
    if (cap_ > (64u << 20)) cap_ = off;
    void* mem = nullptr;
    e = cudaMalloc(&mem, cap_);
    if (e != cudaSuccess) {
      cap_ = 0;
      return op_cuda_error("tables of the orthogonalisation", e);
    }
    mem_ = static_cast<unsigned char*>(mem);
  }
  for (size_t i = 0; i < n; ++i) {
    mats[i].maps = reinterpret_cast<const CUtensorMap*>(mem_ + maps_off) + kNsMaps * i;
    mats[i].done = reinterpret_cast<unsigned int*>(mem_ + done_off) + 32 * i;
  }
  auto put = [&](size_t o, const void* p, size_t bytes) {
    if (e == cudaSuccess && bytes) e = cudaMemcpyAsync(mem_ + o, p, bytes, cudaMemcpyHostToDevice, stream);
  };
  put(maps_off, maps.data(), maps.size() * sizeof(CUtensorMap));
  put(mats_off_, mats.data(), n * sizeof(NsMat));
  put(list_off_, list.data(), list.size() * sizeof(NsTile));
  put(begin_off_, begin.data(), begin.size() * sizeof(int));
  put(units_off_, units.data(), units.size() * sizeof(int2));
  if (e == cudaSuccess) e = cudaMemsetAsync(mem_ + done_off, 0, status_off + sizeof(int) - done_off, stream);
  const cudaError_t w = cudaStreamSynchronize(stream);   // before other streams use it, and before the lists here are gone
  if (e == cudaSuccess) e = w;
  if (e != cudaSuccess) return op_cuda_error("tables of the orthogonalisation", e);
  status_ = status ? status : reinterpret_cast<int*>(mem_ + status_off);
  count_ = (int)n;
  units_ = (int)units.size();
  split_ = split;
  return PS_OK;
}

int NsPlan::run(cudaStream_t stream, PsStat* stats) const {
  if (!count_) return PS_OK;
  const NsMat* mats = reinterpret_cast<const NsMat*>(mem_ + mats_off_);
  const int2* units = reinterpret_cast<const int2*>(mem_ + units_off_);
  if (small_)
    return op_launch("orthogonalisation", split_ ? ps_ortho_small_kernel<2> : ps_ortho_small_kernel<1>, (unsigned)(count_ * small_),
                     kSoThreads, kSoSmem, small_, stream, SoArgs{mats, status_, small_, stats});
  int rc = PS_OK;
  if (norms_) rc = op_launch("orthogonalisation", ps_ortho_norm_kernel, (unsigned)units_, kNsThreads, 0, 1, stream, mats, units);
  if (!rc) rc = op_launch("orthogonalisation", ps_ortho_prepare_kernel, (unsigned)units_, kNsThreads, 0, 1, stream, mats, units, stats);
  if (rc) return rc;
  NsArgs a;
  a.status = status_;
  a.mats = mats;
  a.list = reinterpret_cast<const NsTile*>(mem_ + list_off_);
  a.begin = reinterpret_cast<const int*>(mem_ + begin_off_);
  a.stats = stats;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid_);
  cfg.blockDim = dim3(TcCfg<NsOp<1, false>>::kThreads);
  const NsKernel kernel = kernel_of(split_, pair_);
  cfg.dynamicSmemBytes = (size_t)kernel.smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;           // tiles wait for tiles of other CTAs: all have to be running
  attr[0].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel.fn, a);
  if (e != cudaSuccess) return op_cuda_error("orthogonalisation", e);
  return PS_OK;
}

int NsPlan::status(int* out) const {
  *out = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess && status_) e = cudaMemcpy(out, status_, sizeof(int), cudaMemcpyDeviceToHost);
  return e == cudaSuccess ? PS_OK : op_cuda_error("status of the orthogonalisation", e);
}

constexpr uint32_t kOrthoMagic = 0x50534f32u;    // "PSO2"

}  // namespace psb

using namespace psb;

struct ps_ortho {
  uint32_t magic = kOrthoMagic;
  int device = 0;
  void* workspace = nullptr;
  NsPlan plan;
};

namespace {
bool alive(const ps_ortho* o) { return o && o->magic == kOrthoMagic; }
bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
}  // namespace

extern "C" {

int ps_ortho_create(ps_ortho** out, int device, int n, const ps_matrix* srcs, int src_dtype, const ps_matrix* dsts, int dst_dtype) {
  if (!out) return PS_ERR_BAD_ARG;
  *out = nullptr;
  if (device < 0 || n < 0 || (n > 0 && (!srcs || !dsts))) return PS_ERR_BAD_ARG;
  if ((src_dtype != PS_F32 && src_dtype != PS_BF16) || (dst_dtype != PS_F32 && dst_dtype != PS_BF16)) return PS_ERR_BAD_ARG;
  ps_ortho* o = nullptr;
  int rc = PS_OK;
  try {
    std::vector<NsItem> items((size_t)n);
    for (int i = 0; i < n; ++i) {
      const ps_matrix &s = srcs[i], &d = dsts[i];
      if (s.rows < 0 || s.cols < 0 || s.rows > kNsMaxDim || s.cols > kNsMaxDim || d.rows != s.rows || d.cols != s.cols)
        return PS_ERR_BAD_ARG;
      if (s.rows == 0 || s.cols == 0) continue;
      if (!s.data || !d.data || s.ld < s.cols || d.ld < d.cols) return PS_ERR_BAD_ARG;
      if (misaligned(s.data, src_dtype == PS_BF16 ? 2 : 4) || misaligned(d.data, dst_dtype == PS_BF16 ? 2 : 4)) return PS_ERR_ALIGN;
      NsItem& it = items[(size_t)i];
      it.rows = s.rows;
      it.cols = s.cols;
      it.src = s.data;
      it.ld_src = s.ld;
      it.src_bf16 = src_dtype == PS_BF16;
      it.dst = d.data;
      it.ld_dst = d.ld;
      it.out = dst_dtype == PS_BF16 ? kNsOutBf16 : kNsOutF32;
    }
    const bool split = dst_dtype == PS_F32;
    const size_t bytes = NsPlan::workspace(items, split);
    if (!bytes) return PS_ERR_TOO_LARGE;
    std::vector<const void*> to;
    for (const NsItem& it : items)
      if (it.dst) to.push_back(it.dst);
    std::sort(to.begin(), to.end());
    if (std::adjacent_find(to.begin(), to.end()) != to.end()) return PS_ERR_BAD_ARG;
    DeviceScope on(device);
    cudaError_t e = on.error;
    if (e != cudaSuccess) return op_cuda_error("cudaSetDevice", e);
    o = new ps_ortho();
    o->device = device;
    e = cudaMalloc(&o->workspace, bytes);
    rc = e == cudaSuccess ? o->plan.build(items, split, o->workspace) : op_cuda_error("ps_ortho_create", e);
    if (!rc) {
      *out = o;
      return PS_OK;
    }
  } catch (const std::bad_alloc&) {
    rc = PS_ERR_NOMEM;
  }
  if (o) {
    DeviceScope on(device);
    if (o->workspace) cudaFree(o->workspace);
    delete o;
  }
  return rc;
}

int ps_ortho_run(ps_ortho* o, void* stream) {
  if (!alive(o)) return PS_ERR_BAD_HANDLE;
  DeviceScope on(o->device);
  if (on.error != cudaSuccess) return op_cuda_error("cudaSetDevice", on.error);
  return o->plan.run(static_cast<cudaStream_t>(stream));
}

int ps_ortho_status(ps_ortho* o, int* status_out) {
  if (!alive(o)) return PS_ERR_BAD_HANDLE;
  if (!status_out) return PS_ERR_BAD_ARG;
  DeviceScope on(o->device);
  if (on.error != cudaSuccess) return op_cuda_error("cudaSetDevice", on.error);
  return o->plan.status(status_out);
}

int ps_ortho_destroy(ps_ortho* o) {
  if (!alive(o)) return PS_ERR_BAD_HANDLE;
  DeviceScope on(o->device);
  cudaError_t e = on.error;
  if (e == cudaSuccess && o->workspace) e = cudaFree(o->workspace);      // waits for runs that still use it
  o->magic = 0;
  delete o;
  return e == cudaSuccess ? PS_OK : op_cuda_error("ps_ortho_destroy", e);
}

}  // extern "C"
