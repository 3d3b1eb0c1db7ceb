// The handle behind the C ABI and the helpers that its host sources share.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>
#include <string>

#include "peat.h"
#include "peat_internal.h"

namespace peat {
struct OpsState;
void ops_destroy(OpsState* s);
}  // namespace peat

struct peat_handle_s {
  int device = 0;
  int nsm = 0;
  int64_t max_segments = 4096;
  int max_ctas = 0;
  // compare workspace
  peat::Partial* partials = nullptr;
  peat::SegAcc* acc = nullptr;   // per-segment integer totals, zero between calls
  uint32_t* glist = nullptr;      // per-CTA lists of general-path pairs (stage 1 scratch)
  unsigned int* status_host = nullptr;  // mapped pinned error word written by the kernels
  unsigned int* status_dev = nullptr;
  unsigned int wait_limit = 1u << 24;   // polls before a pipeline wait gives up
  void* stage1_event = nullptr;         // profiling aid: recorded after each compare's stage-1 launch
  int64_t* d_offsets = nullptr;  // offsets (nseg + 1) then CTA bounds (nctas + 1)
  int64_t* h_offsets = nullptr;  // pinned staging of the same
  int64_t* d_single = nullptr;   // one-tensor calls: {0, n} then CTA bounds, written on the device
  // what d_single holds: the key of its last write (dtype, n, p0, nctas, stream)
  bool single_valid = false;
  int single_dtype = -1, single_nctas = 0;
  int64_t single_n = -1, single_p0 = 0;
  cudaStream_t single_stream = nullptr;
  cudaEvent_t staged = nullptr;  // the last staging copy has been consumed
  bool staged_pending = false;
  // mean-of-top-errors workspace, zero between calls
  peat::TopkState* topk = nullptr;
  peat::TopkListEntry* topk_list = nullptr;
  // context-statistics accumulators (one per segment), zero between calls
  peat::TsAcc* tsacc = nullptr;
  // injector staging (grown on demand)
  int64_t* d_inj = nullptr;
  int64_t* h_inj = nullptr;
  size_t inj_cap = 0;  // in int64 elements
  // 8-bit compare: pinned staging of offsets and work items, device copy plus item records
  int64_t* h_f8 = nullptr;
  void* d_f8 = nullptr;
  size_t f8_hcap = 0, f8_dcap = 0;  // bytes
  // state of the playback operators (ops_api.cpp), made by their first call
  peat::OpsState* ops = nullptr;
  std::string err;
};

namespace peat {

struct DeviceGuard {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
    if (prev != dev) ok = cudaSetDevice(dev) == cudaSuccess;
  }
  ~DeviceGuard() {
    int cur = -1;
    if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
  }
};

inline peat_status_t fail(peat_handle_t h, peat_status_t st, const std::string& msg) {
  if (h) h->err = msg;
  return st;
}

inline peat_status_t cuda_fail(peat_handle_t h, cudaError_t e, const char* what) {
  cudaGetLastError();  // clear a sticky non-fatal error state
  return fail(h, PEAT_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

}  // namespace peat
