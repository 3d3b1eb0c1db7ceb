// The host side of the playback operators (csrc/ops_api.cpp) against a runtime of
// plain host memory, in which calls fail, launches are refused and streams are
// being captured as a check asks for it.  No GPU: the kernels are stand-ins that
// look at the words they are given.
//
//   ops_host NAME     runs one check; exit code 0 if it holds
#include <cuda_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <new>
#include <string>
#include <vector>

#include "ops_internal.h"
#include "peat_handle.h"

namespace {

struct Runtime {
  bool capturing = false;
  bool fail_memset = false;
  bool fail_new = false;
  size_t largest = (size_t)-1;  // block that can be had
  int fail_pinned = 0;          // the pinned allocation from here on that fails (1: the next)
  int fail_step = -1;        // the quantiser's launch that fails
  int dirty = 0;             // words that a kernel should have found zero
  int allocations = 0;       // device, pinned and event allocations
  std::map<void*, size_t> device;
  peat::QuantParams quant;   // of the last quantiser launch
  size_t live() const {
    size_t n = 0;
    for (auto& b : device) n += b.second;
    return n;
  }
} rt;

void zero_or_count(const unsigned int* w, int64_t n) {
  for (int64_t i = 0; i < n; i++) rt.dirty += w[i] != 0;
}

int failures = 0;
void check(bool ok, const char* what, int line) {
  if (ok) return;
  std::printf("line %d: %s\n", line, what);
  failures++;
}
#define CHECK(x) check((x), #x, __LINE__)

}  // namespace

void* operator new(size_t n) {
  if (rt.fail_new) throw std::bad_alloc();
  if (void* p = std::malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, size_t) noexcept { std::free(p); }

// ---- the runtime ----
extern "C" {
cudaError_t cudaGetDevice(int* d) { return *d = 0, cudaSuccess; }
cudaError_t cudaSetDevice(int) { return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
const char* cudaGetErrorString(cudaError_t) { return "made to fail"; }
cudaError_t cudaDeviceSynchronize() { return cudaSuccess; }
cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) {
  *s = rt.capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
  return cudaSuccess;
}
cudaError_t cudaMalloc(void** p, size_t n) {
  if (n > rt.largest) return cudaErrorMemoryAllocation;
  *p = std::malloc(n ? n : 1);
  std::memset(*p, 0xab, n);
  rt.device[*p] = n;
  rt.allocations++;
  return cudaSuccess;
}
cudaError_t cudaFree(void* p) {
  rt.device.erase(p);
  std::free(p);
  return cudaSuccess;
}
cudaError_t cudaMallocHost(void** p, size_t n) {
  if (rt.fail_pinned && --rt.fail_pinned == 0) return cudaErrorMemoryAllocation;
  rt.allocations++;
  *p = std::malloc(n);
  return cudaSuccess;
}
cudaError_t cudaFreeHost(void* p) { return std::free(p), cudaSuccess; }
cudaError_t cudaMemset(void* p, int v, size_t n) { return std::memset(p, v, n), cudaSuccess; }
cudaError_t cudaMemsetAsync(void* p, int v, size_t n, cudaStream_t) {
  if (rt.fail_memset) return cudaErrorUnknown;
  return std::memset(p, v, n), cudaSuccess;
}
cudaError_t cudaMemcpyAsync(void* d, const void* s, size_t n, cudaMemcpyKind, cudaStream_t) {
  return std::memcpy(d, s, n), cudaSuccess;
}
cudaError_t cudaEventCreateWithFlags(cudaEvent_t* e, unsigned) {
  rt.allocations++;
  *e = reinterpret_cast<cudaEvent_t>(std::malloc(1));
  return cudaSuccess;
}
cudaError_t cudaEventDestroy(cudaEvent_t e) { return std::free(e), cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaEventSynchronize(cudaEvent_t) { return cudaSuccess; }
}

// ---- the kernels ----
namespace peat {
cudaError_t launch_quant8(int, int step, const QuantParams& p, int, cudaStream_t) {
  rt.quant = p;
  if (step == rt.fail_step) return cudaErrorLaunchFailure;
  if (step == QUANT_MAXIMA) {
    zero_or_count(p.colmax, p.cols);
    for (int64_t i = 0; i < p.cols; i++) p.colmax[i] = 1;
  } else {
    for (int64_t i = 0; i < p.zero_n; i++) p.zero[i] = 0;
    for (int64_t i = 0; i < p.zero2_n; i++) p.zero2[i] = 0;
  }
  return cudaSuccess;
}
bool quant8_packs(int, int, const QuantParams&) { return false; }
cudaError_t launch_mm8_direct(int, const Mm8Params&, int, cudaStream_t) { return cudaSuccess; }
double mm8_direct_time(int64_t, int64_t, int64_t, bool, int) { return 1e30; }
Mm8TcPlan mm8_tc_plan(int64_t M, int64_t N, int64_t K, int) {
  Mm8TcPlan p = {};
  p.bytes = 2 * (size_t)(M + N) * K;
  return p;
}
double mm8_tc_time(const Mm8TcPlan&, int64_t, int) { return 1.0; }
cudaError_t launch_mm8_pack(const Mm8Params&, const Mm8TcPlan&, char*, unsigned int*, int, cudaStream_t) {
  return cudaSuccess;
}
cudaError_t launch_mm8_tc(int, const Mm8Params&, const Mm8TcPlan&, char*, unsigned int*, bool, unsigned int*,
                          unsigned int, int, cudaStream_t) {
  return cudaSuccess;
}
int gn_block() { return 256; }
cudaError_t launch_gradnorm(const GnParams& p, const GnEntry*, int, cudaStream_t) {
  zero_or_count(p.tickets, p.count);
  zero_or_count(p.done, 1);
  return cudaSuccess;
}
}  // namespace peat

namespace {

struct Host {
  peat_handle_s h;
  std::vector<char> space = std::vector<char>(1 << 20);  // stands for the caller's tensors: no kernel touches them
  Host() { h.nsm = 152; }
  ~Host() { peat::ops_destroy(h.ops); }
  void* data() { return reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(space.data()) + 255) & ~(uintptr_t)255); }
  peat_status_t columns(int64_t cols) {
    return peat_quantize_i8(&h, data(), 1000, cols, cols, PEAT_F32, 1, static_cast<int8_t*>(data()), 1000, nullptr,
                            nullptr, 0, nullptr);
  }
  peat_status_t product(int64_t rows) {
    const int8_t* x = static_cast<int8_t*>(data());
    return peat_matmul_i8(&h, x, 500, nullptr, x, 500, nullptr, nullptr, rows, 1000, 500, data(), 1000, PEAT_F32, nullptr);
  }
  peat_status_t norm(int64_t count) {
    std::vector<peat_grad_t> list(count, peat_grad_t{data(), nullptr, 3, PEAT_F32, 0});
    return peat_grad_norm(&h, list.data(), count, PEAT_NORM_2, 1.0f, static_cast<peat_gradnorm_t*>(data()), nullptr,
                          nullptr);
  }
};

// Words that a failed launch left as they were are cleared before the next call
// takes them, a capture that was refused in between or not.
void words_after_a_failed_launch() {
  for (bool refused : {false, true}) {
    Host u;
    CHECK(u.columns(100) == PEAT_OK);
    rt.fail_step = peat::QUANT_COLUMNS;
    CHECK(u.columns(100) == PEAT_ERR_CUDA);
    rt.fail_step = -1;
    if (refused) {
      rt.capturing = true;
      CHECK(u.columns(100000) == PEAT_ERR_UNSUPPORTED);
      rt.capturing = false;
    }
    for (int i = 0; i < 3; i++) CHECK(u.columns(100) == PEAT_OK);
    CHECK(rt.dirty == 0);
  }
}

// New workspace whose clearing failed is cleared by the next call that takes it.
void words_after_a_failed_clear() {
  Host u;
  CHECK(u.columns(0) == PEAT_OK && u.norm(1) == PEAT_OK);
  rt.fail_memset = true;
  CHECK(u.columns(10000) == PEAT_ERR_CUDA);
  CHECK(u.norm(5000) == PEAT_ERR_CUDA);
  rt.fail_memset = false;
  CHECK(u.columns(10000) == PEAT_OK);
  CHECK(rt.dirty == 0);
  CHECK(u.norm(5000) == PEAT_OK);
  CHECK(rt.dirty == 0);
}

// Sizes that grow call by call: few allocations, and blocks that a graph may use
// do not add up to a multiple of the sizes.  Where memory is short, a call gets
// by with what it needs.
void growing_sizes() {
  for (bool captured : {false, true}) {
    rt.allocations = 0;
    Host u;
    CHECK(u.product(1000) == PEAT_OK);
    if (captured) {
      rt.capturing = true;
      CHECK(u.product(1000) == PEAT_OK);
      rt.capturing = false;
    }
    for (int64_t m = 1000; m <= 20000; m += 100) CHECK(u.product(m) == PEAT_OK);
    const size_t need = 2 * (20000 + 1000) * (size_t)500;
    CHECK(rt.live() <= (captured ? 5 : 2) * need);
    CHECK(rt.allocations <= 16);
  }
  Host u;
  CHECK(u.product(1000) == PEAT_OK);
  rt.largest = 2 * (1100 + 1000) * (size_t)500 + 1000;
  CHECK(u.product(1100) == PEAT_OK);
  CHECK(u.product(1200) == PEAT_ERR_ALLOC);
  rt.largest = (size_t)-1;
  CHECK(u.product(1200) == PEAT_OK);
  // zeroed words: all of a block that grew by more than its call needs, on boundaries of 16 bytes
  for (int64_t n = 5000; n <= 20000; n += 501) {
    CHECK(u.norm(n) == PEAT_OK && u.columns(2 * n) == PEAT_OK);
    CHECK(reinterpret_cast<uintptr_t>(rt.quant.colmax) % 16 == 0);
  }
  CHECK(rt.dirty == 0);
}

// After a first call of its size a gradient list allocates nothing, a long one
// neither, whichever staging buffer its turn brings.
void lists_allocate_once() {
  Host u;
  for (int64_t n : {5, 801, 2500, 900, 6000}) {
    CHECK(u.norm(n) == PEAT_OK);
    const int before = rt.allocations;
    for (int i = 0; i < 9; i++) CHECK(u.norm(n) == PEAT_OK);
    CHECK(rt.allocations == before);
  }
  // staging that could not be had: the call says so, and the next one tries again
  rt.fail_pinned = 2;
  CHECK(u.norm(20000) == PEAT_ERR_ALLOC);
  for (int i = 0; i < 9; i++) CHECK(u.norm(20000) == PEAT_OK);
}

// The row distance of a matrix of one row is not used: it does not keep its
// kernel from whole vectors.
void one_row_is_aligned() {
  Host u;
  int8_t* q = static_cast<int8_t*>(u.data());
  auto quantize = [&](int64_t rows, int64_t ldq, int64_t at) {
    CHECK(peat_quantize_i8(&u.h, u.data(), rows, 1001, 1008, PEAT_F16, 0, q + at, ldq, nullptr, nullptr, 0, nullptr) == PEAT_OK);
    return rt.quant.vec_q;
  };
  CHECK(quantize(1, 1001, 0) && quantize(2, 1008, 0) && quantize(2, 1008, 8));
  CHECK(!quantize(2, 1001, 0) && !quantize(1, 1001, 3));
  auto transpose = [&](int64_t cols, int64_t ldq, int64_t at) {
    CHECK(peat_quantize_i8(&u.h, u.data(), 11, cols, 1008, PEAT_F16, 1, q + at, ldq, nullptr, nullptr, 0, nullptr) == PEAT_OK);
    return rt.quant.vec_q;
  };
  CHECK(transpose(1, 11, 0) && transpose(2, 12, 4) && !transpose(2, 11, 0) && !transpose(1, 11, 2));
  auto aligned = [&](int64_t at, int64_t M, int64_t lda, int64_t N, int64_t ldb) {
    return peat::mm8_aligned(peat::Mm8Params{q + at, q, lda, ldb, nullptr, nullptr, nullptr, nullptr, 0, M, N, 1001});
  };
  CHECK(aligned(0, 1, 1001, 5, 1008) && aligned(0, 5, 1008, 1, 1001) && aligned(0, 1, 1001, 1, 1001) &&
        aligned(16, 5, 1008, 5, 1008));
  CHECK(!aligned(0, 2, 1001, 5, 1008) && !aligned(0, 5, 1008, 2, 1001) && !aligned(8, 1, 1001, 5, 1008));
}

// Host memory that runs out is a status with a text of its own, and the handle works on.
void host_memory() {
  Host u;
  CHECK(peat_quantize_i8(&u.h, nullptr, 1, 1, 1, PEAT_F32, 0, nullptr, 0, nullptr, nullptr, 0, nullptr) == PEAT_ERR_INVALID_ARG);
  const std::string before = u.h.err;
  std::vector<peat_grad_t> list(3, peat_grad_t{u.data(), nullptr, 3, PEAT_F32, 0});
  rt.fail_new = true;
  const peat_status_t st = peat_grad_norm(&u.h, list.data(), 3, PEAT_NORM_2, 1.0f, static_cast<peat_gradnorm_t*>(u.data()),
                                          nullptr, nullptr);
  rt.fail_new = false;
  CHECK(st == PEAT_ERR_ALLOC && u.h.err != before && !u.h.err.empty());
  CHECK(u.norm(3) == PEAT_OK);
}

const struct {
  const char* name;
  void (*run)();
} CHECKS[] = {
    {"words_after_a_failed_launch", words_after_a_failed_launch},
    {"words_after_a_failed_clear", words_after_a_failed_clear},
    {"growing_sizes", growing_sizes},
    {"lists_allocate_once", lists_allocate_once},
    {"one_row_is_aligned", one_row_is_aligned},
    {"host_memory", host_memory},
};

}  // namespace

int main(int argc, char** argv) {
  for (auto& c : CHECKS)
    if (argc == 2 && !std::strcmp(argv[1], c.name)) {
      c.run();
      return failures != 0;
    }
  for (auto& c : CHECKS) std::printf("%s\n", c.name);
  return argc == 1 ? 0 : 2;
}
