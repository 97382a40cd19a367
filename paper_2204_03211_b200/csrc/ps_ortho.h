// Orthogonalisation of a list of matrices, as the list's handle (ps_ortho.cu) and the service (ps_service.cu) use it.
#pragma once

#include <cuda_runtime.h>

#include <vector>

#include "ps_op.h"
#include "ps_types.cuh"

namespace psb {

enum { kNsOutF32 = 0, kNsOutBf16 = 1, kNsOutUpdate = 2 };

struct NsItem {                          // one matrix, rows x cols with strides in elements
  long long rows = 0, cols = 0;
  const void* src = nullptr;
  long long ld_src = 0;
  bool src_bf16 = false;
  void* dst = nullptr;
  long long ld_dst = 0;
  int out = kNsOutF32;
  float decay = 1.f, step = 1.f;         // kNsOutUpdate: dst = dst * decay - step * O
  double* parts = nullptr;               // partial sums of src's squares that are there already; nullptr: computed here
  int nparts = 0;
  unsigned int stat = 0;                 // its record among the `stats` of a run
};

// The device tables of one list.  The workspace is its owner's; runs that share one must not overlap on the GPU.
class NsPlan {
 public:
  ~NsPlan();
  NsPlan() = default;
  NsPlan(const NsPlan&) = delete;
  NsPlan& operator=(const NsPlan&) = delete;

  // Bytes of workspace that a list needs; split: three products of halves (binary32 results).  0: too large a list.
  static size_t workspace(const std::vector<NsItem>& items, bool split);
  // Makes the tables for the current device, copies them on `stream` and waits until they are there.  Throws
  // std::bad_alloc only.  `status`: the device word in which a bounded wait that ran out is noted; nullptr: one of its own.
  int build(const std::vector<NsItem>& items, bool split, void* workspace, int* status = nullptr,
            cudaStream_t stream = cudaStreamLegacy);
  // Takes over the memory of a plan that no launch uses any more, for the tables of the next build.
  void adopt(NsPlan& old);
  size_t bytes() const { return cap_; }
  // stats (device), unless NULL: the matrices' records, to whose device times what the run takes is added.
  int run(cudaStream_t stream, PsStat* stats = nullptr) const;
  int status(int* out) const;            // waits for the device

 private:
  unsigned char* mem_ = nullptr;
  size_t cap_ = 0;
  int* status_ = nullptr;
  size_t mats_off_ = 0, list_off_ = 0, begin_off_ = 0, units_off_ = 0;
  int count_ = 0, units_ = 0, grid_ = 0;
  int small_ = 0;                        // > 0: in shared memory, with so many CTAs per matrix
  bool split_ = false, pair_ = false, norms_ = false;
};

}  // namespace psb
