// The host side of the 4-bit products and of the norm (csrc/ops4_api.cpp) against a
// runtime of plain host memory: refusals, workspace, what the launches are given.
// No GPU: the kernels are stand-ins that keep their parameters.
//
//   ops4_host NAME     runs one check; exit code 0 if it holds
#include <cuda_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "ops_internal.h"
#include "peat_handle.h"

namespace {

struct Runtime {
  bool capturing = false, fail_launch = false;
  size_t largest = (size_t)-1;  // block that can be had
  int launches = 0, allocations = 0;
  std::map<void*, size_t> device;
  std::vector<peat::Quant4Params> quants;
  peat::Mm4Params product;
  peat::RmsParams norm;
  peat::RmsBackParams back;
} rt;

int failures = 0;
void check(bool ok, const char* what, int line) {
  if (ok) return;
  std::printf("line %d: %s\n", line, what);
  failures++;
}
#define CHECK(x) check((x), #x, __LINE__)

cudaError_t launched() {
  if (rt.fail_launch) return cudaErrorLaunchFailure;
  rt.launches++;
  return cudaSuccess;
}

}  // namespace

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
  *p = std::aligned_alloc(256, (n + 255) / 256 * 256 + 256);
  rt.device[*p] = n;
  rt.allocations++;
  return cudaSuccess;
}
cudaError_t cudaFree(void* p) {
  rt.device.erase(p);
  std::free(p);
  return cudaSuccess;
}
cudaError_t cudaFreeHost(void* p) { return std::free(p), cudaSuccess; }
cudaError_t cudaEventDestroy(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaMemset(void* p, int v, size_t n) { return std::memset(p, v, n), cudaSuccess; }
cudaError_t cudaMemsetAsync(void* p, int v, size_t n, cudaStream_t) { return std::memset(p, v, n), cudaSuccess; }
}

// ---- the kernels ----
namespace peat {
void ops_destroy(OpsState*);
cudaError_t launch_quant4(int, int, int, const Quant4Params& p, int, cudaStream_t) {
  rt.quants.push_back(p);
  return launched();
}
cudaError_t launch_mm4(int, int, const Mm4Params& p, unsigned int*, unsigned int, int, cudaStream_t) {
  rt.product = p;
  return launched();
}
cudaError_t launch_rmsnorm(int, const RmsParams& p, int, cudaStream_t) {
  rt.norm = p;
  return launched();
}
RmsBackPlan rms_back_plan(int, int64_t rows, int64_t cols, int) { return RmsBackPlan{(int)((rows + 7) / 8), 8, cols > 8192}; }
cudaError_t launch_rmsnorm_backward(int, const RmsBackPlan&, const RmsBackParams& p, cudaStream_t) {
  rt.back = p;
  return launched();
}
}  // namespace peat

#include "ops_state.h"

namespace peat {
void ops_destroy(OpsState* s) {
  if (!s) return;
  for (void* p : {(void*)s->done, s->rounded, s->tops, s->norm}) cudaFree(p);
  for (void* p : s->kept) cudaFree(p);
  delete s;
}
}  // namespace peat

namespace {

struct Host {
  peat_handle_s h;
  std::vector<char> space = std::vector<char>(1 << 20);  // stands for the caller's tensors: no kernel touches them
  Host() { h.nsm = 152; }
  ~Host() { peat::ops_destroy(h.ops); }
  char* data() { return reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(space.data()) + 255) & ~(uintptr_t)255); }
  uint8_t* bytes() { return reinterpret_cast<uint8_t*>(data()); }
  float* floats() { return reinterpret_cast<float*>(data()); }
};

// Every argument of a quantisation that is not valid is refused, and nothing launched.
void quantize_refusals() {
  struct Q {
    const void* x;
    int64_t rows = 4, cols = 40, ldx = 40;
    int dtype = PEAT_F32, format = PEAT_NVFP4, axis = 0;
    uint8_t* q;
    int64_t ldq = 32;
    uint8_t* bs;
    float* scale;
    void* values = nullptr;
    int64_t ldv = 40;
  };
  Host u;
  const Q good{u.data(), 4, 40, 40, PEAT_F32, PEAT_NVFP4, 0, u.bytes(), 32, u.bytes(), u.floats(), nullptr, 40};
  auto run = [&](const Q& a) {
    return peat_quantize_f4(&u.h, a.x, a.rows, a.cols, a.ldx, (peat_dtype_t)a.dtype, (peat_f4_t)a.format, a.axis, a.q, a.ldq, a.bs,
                            a.scale, a.values, a.ldv, nullptr);
  };
  CHECK(run(good) == PEAT_OK && rt.launches == 1);
  CHECK(rt.quants.back().width == 48 && rt.quants.back().tiles == 1);
  std::vector<Q> bad;
  auto with = [&](auto change) {
    Q a = good;
    change(a);
    bad.push_back(a);
  };
  with([](Q& a) { a.dtype = PEAT_F64; });
  with([](Q& a) { a.format = 2; });
  with([](Q& a) { a.axis = 2; });
  with([](Q& a) { a.rows = -1; });
  with([](Q& a) { a.cols = -1; });
  with([](Q& a) { a.ldx = 39; });
  with([](Q& a) { a.x = nullptr; });
  with([](Q& a) { a.x = (const char*)a.x + 2; });
  with([](Q& a) { a.q = nullptr; });
  with([](Q& a) { a.bs = nullptr; });
  with([](Q& a) { a.scale = nullptr; });
  with([](Q& a) { a.scale = (float*)((char*)a.scale + 2); });
  with([](Q& a) { a.format = PEAT_MXFP4; });  // (has no scale)
  with([](Q& a) { a.q += 8; });
  with([](Q& a) { a.ldq = 24; });
  with([](Q& a) { a.ldq = 16; });
  with([](Q& a) { a.bs += 8; });
  with([&](Q& a) { a.values = u.data(), a.ldv = 39; });
  with([&](Q& a) { a.values = u.data() + 2; });
  rt.launches = 0;
  for (size_t i = 0; i < bad.size(); i++) {
    u.h.err.clear();
    const peat_status_t st = run(bad[i]);
    if (st != PEAT_ERR_INVALID_ARG || u.h.err.empty()) std::printf("refusal %zu: %d\n", i, (int)st), failures++;
  }
  CHECK(rt.launches == 0);
  Q big = good;
  big.rows = ((int64_t)1 << 31) - 200;
  CHECK(run(big) == PEAT_ERR_UNSUPPORTED);
  big = good;  // (columns of blocks are counted in 32 bits with what a step reaches beyond)
  big.rows = 1, big.cols = big.ldx = ((int64_t)1 << 30) + 32, big.ldq = big.cols / 2;
  CHECK(run(big) == PEAT_ERR_UNSUPPORTED);
  big.axis = 1, big.rows = big.cols, big.cols = 1;
  CHECK(run(big) == PEAT_ERR_UNSUPPORTED);
  // one row needs no distance of its own; nothing to do is no error
  Q one = good;
  one.rows = 1, one.ldq = 24;
  CHECK(run(one) == PEAT_OK && rt.launches == 1);
  Q none = good;
  none.rows = 0, none.x = nullptr, none.q = nullptr, none.bs = nullptr;
  CHECK(run(none) == PEAT_OK && rt.launches == 1);
  // rows of nothing have scale 0
  u.floats()[3] = 5.0f;
  none.rows = 4, none.cols = 0;
  CHECK(run(none) == PEAT_OK && rt.launches == 1 && u.floats()[3] == 0.0f);
  rt.fail_launch = true;
  CHECK(run(good) == PEAT_ERR_CUDA);
  rt.fail_launch = false;
}

void product_refusals() {
  Host u;
  struct P {
    int format = PEAT_MXFP4;
    const uint8_t* a;
    int64_t lda = 64;
    const uint8_t* abs;
    const uint8_t* b;
    int64_t ldb = 64;
    int64_t M = 5, N = 7, K = 128;
    void* out;
    int64_t ldo = 7;
    int dtype = PEAT_F32;
  };
  const P good{PEAT_MXFP4, u.bytes(), 64, u.bytes(), u.bytes(), 64, 5, 7, 128, u.data(), 7, PEAT_F32};
  auto run = [&](const P& a) {
    return peat_matmul_f4(&u.h, (peat_f4_t)a.format, a.a, a.lda, a.abs, nullptr, a.b, a.ldb, u.bytes(), nullptr, nullptr, a.M, a.N,
                          a.K, a.out, a.ldo, (peat_dtype_t)a.dtype, nullptr);
  };
  CHECK(run(good) == PEAT_OK && rt.launches == 1);
  std::vector<P> bad;
  auto with = [&](auto change) {
    P a = good;
    change(a);
    bad.push_back(a);
  };
  with([](P& a) { a.format = 5; });
  with([](P& a) { a.a = nullptr; });
  with([](P& a) { a.a += 8; });
  with([](P& a) { a.lda = 72; });
  with([](P& a) { a.lda = 48; });
  with([](P& a) { a.abs = nullptr; });
  with([](P& a) { a.abs += 1; });
  with([](P& a) { a.b = nullptr; });
  with([](P& a) { a.ldb = 63; });
  with([](P& a) { a.M = -1; });
  with([](P& a) { a.K = -32; });
  with([](P& a) { a.K = 112; });
  with([](P& a) { a.out = nullptr; });
  with([](P& a) { a.out = (char*)a.out + 2; });
  with([](P& a) { a.ldo = 6; });
  with([](P& a) { a.dtype = 100; });
  for (size_t i = 0; i < bad.size(); i++) {
    u.h.err.clear();
    const peat_status_t st = run(bad[i]);
    if (st != PEAT_ERR_INVALID_ARG || u.h.err.empty()) std::printf("refusal %zu: %d\n", i, (int)st), failures++;
  }
  CHECK(rt.launches == 1);
  P big = good;
  big.M = big.N = (int64_t)1 << 30, big.ldo = (int64_t)1 << 30;
  CHECK(run(big) == PEAT_ERR_UNSUPPORTED);
  P none = good;
  none.M = 0, none.a = nullptr, none.out = nullptr;
  CHECK(run(none) == PEAT_OK && rt.launches == 1);
  P flat = good;  // no k: the operands are not looked at
  flat.K = 0, flat.a = flat.b = flat.abs = nullptr;
  CHECK(run(flat) == PEAT_OK && rt.launches == 2);
  // an expired wait is told once
  unsigned int word = 1;
  u.h.status_host = &word;
  CHECK(run(good) == PEAT_ERR_TIMEOUT && run(good) == PEAT_OK);
  u.h.status_host = nullptr;
}

// Operands that are rounded on the way: places of their own in the workspace, of the
// size that their rows need, on 256-byte boundaries.
void operands() {
  Host u;
  auto op = [&](int64_t rows, int64_t cols, int axis) {
    return peat_operand_f4_t{u.data(), nullptr, nullptr, rows, cols, cols, PEAT_BF16, axis};
  };
  for (int format : {PEAT_MXFP4, PEAT_NVFP4})
    for (int axes = 0; axes < 4; axes++) {
      const int64_t M = 300, N = 130, K = 1001;
      const peat_operand_f4_t a = axes & 1 ? op(K, M, 1) : op(M, K, 0), b = axes & 2 ? op(K, N, 1) : op(N, K, 0);
      rt.quants.clear();
      CHECK(peat_product_f4(&u.h, (peat_f4_t)format, &a, &b, nullptr, u.data(), N, PEAT_F32, nullptr) == PEAT_OK);
      CHECK(rt.quants.size() == 2 && rt.product.M == M && rt.product.N == N && rt.product.K == (format == PEAT_MXFP4 ? 1024 : 1008));
      const int64_t tiles = format == PEAT_MXFP4 ? 8 : 16;
      struct Range {
        uintptr_t lo, hi;
      };
      std::vector<Range> used;
      auto take = [&](const void* p, size_t n) {
        const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
        CHECK(lo % 256 == 0);
        for (const Range& r : used) CHECK(lo >= r.hi || lo + n <= r.lo);
        used.push_back({lo, lo + n});
      };
      const int64_t rows[2] = {M, N};
      for (int i = 0; i < 2; i++) {
        const peat::Quant4Params& q = rt.quants[i];
        take(q.q, rows[i] * q.ldq);
        take(q.block_scale, (rows[i] + 127) / 128 * tiles * 512);
        if (format == PEAT_NVFP4) take(q.scale, rows[i] * 4);
        if (format == PEAT_NVFP4 && (axes >> i & 1)) {  // the operands' maxima do not meet
          const uintptr_t lo = reinterpret_cast<uintptr_t>(q.tops);
          const size_t n = sizeof(unsigned int) * peat::QUANT4_CHUNKS * rows[i];
          for (const Range& r : used) CHECK(lo >= r.hi || lo + n <= r.lo);
          used.push_back({lo, lo + n});
        }
        CHECK(q.overlap == (i == 1));
        CHECK(q.tiles == tiles && q.ldq % 16 == 0 && q.ldq >= q.width / 2 && (format == PEAT_NVFP4 || !q.scale));
        CHECK((i ? rt.product.b : rt.product.a) == q.q && (i ? rt.product.sb : rt.product.sa) == q.scale);
      }
      for (const Range& r : used) {  // inside a block that was allocated
        bool in = false;
        for (auto& d : rt.device) in |= r.lo >= (uintptr_t)d.first && r.hi <= (uintptr_t)d.first + d.second;
        CHECK(in);
      }
    }
  // operands that do not belong together, or are not valid
  const peat_operand_f4_t a = op(3, 64, 0), b = op(5, 64, 0), longer = op(5, 96, 0);
  auto run = [&](const peat_operand_f4_t* x, const peat_operand_f4_t* y, int t = PEAT_F32, int format = PEAT_MXFP4) {
    return peat_product_f4(&u.h, (peat_f4_t)format, x, y, nullptr, u.data(), 5, (peat_dtype_t)t, nullptr);
  };
  CHECK(run(&a, &b) == PEAT_OK);
  CHECK(run(&a, &longer) == PEAT_ERR_INVALID_ARG && run(nullptr, &b) == PEAT_ERR_INVALID_ARG && run(&a, &b, 100) == PEAT_ERR_INVALID_ARG);
  for (int i = 0; i < 8; i++) {
    peat_operand_f4_t c = b;
    if (i == 0) c.rows = -1;
    if (i == 1) c.ld = 63;
    if (i == 2) c.dtype = 7;
    if (i == 3) c.axis = 2;
    if (i == 4) c.data = nullptr;
    if (i == 5) c = peat_operand_f4_t{u.data(), u.bytes(), nullptr, 5, 64, 32, PEAT_F4, 1};
    if (i == 6) c = peat_operand_f4_t{u.data(), u.bytes(), u.floats(), 5, 64, 32, PEAT_F4, 0};  // (mxfp4 with scales)
    if (i == 7) c = peat_operand_f4_t{u.data(), nullptr, nullptr, 5, 64, 32, PEAT_F4, 0};
    CHECK(run(&a, &c) == PEAT_ERR_INVALID_ARG);
  }
}

// A capture takes what is there; a call that would have to grow it is refused, and
// blocks that a graph may use are kept.
void captures() {
  Host u;
  const peat_operand_f4_t a{u.data(), nullptr, nullptr, 3, 64, 64, PEAT_F32, 1};
  auto run = [&](int64_t rows) {
    peat_operand_f4_t b{u.data(), nullptr, nullptr, 3, rows, rows, PEAT_F32, 1};
    return peat_product_f4(&u.h, PEAT_NVFP4, &a, &b, nullptr, u.data(), rows, PEAT_F32, nullptr);
  };
  rt.capturing = true;
  CHECK(run(10) == PEAT_ERR_UNSUPPORTED);
  rt.capturing = false;
  CHECK(run(10) == PEAT_OK);
  rt.capturing = true;
  CHECK(run(10) == PEAT_OK && run(100000) == PEAT_ERR_UNSUPPORTED);
  rt.capturing = false;
  const size_t blocks = rt.device.size();
  CHECK(run(100000) == PEAT_OK && rt.device.size() > blocks);
  rt.largest = 1000;
  CHECK(run(1000000) == PEAT_ERR_ALLOC);
  rt.largest = (size_t)-1;
  const int before = rt.allocations;
  CHECK(run(100000) == PEAT_OK);
  const int after = rt.allocations;
  CHECK(run(100000) == PEAT_OK && rt.allocations == after && after - before <= 2);
}

void norm_refusals() {
  Host u;
  struct N {
    const void* x;
    int64_t ldx = 10;
    const void* res = nullptr;
    const void* w;
    int wt = PEAT_F32;
    int64_t rows = 3, cols = 10;
    int dtype = PEAT_BF16;
    float eps = 1e-6f;
    void* y;
    int64_t ldy = 10;
  };
  const N good{u.data(), 10, nullptr, u.data(), PEAT_F32, 3, 10, PEAT_BF16, 1e-6f, u.data(), 10};
  auto run = [&](const N& a) {
    return peat_rmsnorm(&u.h, a.x, a.ldx, a.res, 10, a.w, (peat_dtype_t)a.wt, a.rows, a.cols, (peat_dtype_t)a.dtype, a.eps, nullptr, 0,
                        a.y, a.ldy, nullptr, 0, nullptr, nullptr, 0, nullptr, nullptr);
  };
  CHECK(run(good) == PEAT_OK && rt.launches == 1 && !rt.norm.grid);
  std::vector<N> bad;
  auto with = [&](auto change) {
    N a = good;
    change(a);
    bad.push_back(a);
  };
  with([](N& a) { a.x = nullptr; });
  with([](N& a) { a.x = (const char*)a.x + 1; });
  with([](N& a) { a.ldx = 9; });
  with([&](N& a) { a.res = u.data() + 1; });
  with([](N& a) { a.w = nullptr; });
  with([](N& a) { a.w = (const char*)a.w + 2; });
  with([](N& a) { a.wt = PEAT_F16; });
  with([](N& a) { a.rows = -1; });
  with([](N& a) { a.dtype = PEAT_F64; });
  with([](N& a) { a.eps = -1.0f; });
  with([](N& a) { a.eps = __builtin_inff(); });
  with([](N& a) { a.eps = __builtin_nanf(""); });
  with([](N& a) { a.y = nullptr; });
  with([](N& a) { a.y = (char*)a.y + 1; });
  with([](N& a) { a.ldy = 9; });
  for (size_t i = 0; i < bad.size(); i++) {
    u.h.err.clear();
    const peat_status_t st = run(bad[i]);
    if (st != PEAT_ERR_INVALID_ARG || u.h.err.empty()) std::printf("refusal %zu: %d\n", i, (int)st), failures++;
  }
  CHECK(rt.launches == 1);
  N none = good;
  none.rows = 0, none.x = nullptr;
  CHECK(run(none) == PEAT_OK && rt.launches == 1);
  N whole = good;
  whole.cols = whole.ldx = whole.ldy = 16;
  CHECK(run(whole) == PEAT_OK && rt.norm.grid);
  auto back = [&](int64_t rows, int64_t cols, const void* g, void* gx, float* gw, const float* rstd, int64_t ld) {
    return peat_rmsnorm_backward(&u.h, g, ld, nullptr, 0, u.data(), ld, u.data(), PEAT_F32, rstd, rows, cols, PEAT_BF16, gx, ld, gw,
                                 nullptr);
  };
  rt.launches = 0;
  CHECK(back(9, 16, u.data(), u.data(), u.floats(), u.floats(), 16) == PEAT_OK && rt.launches == 1 && rt.back.grid);
  bool in = false;
  for (auto& d : rt.device) in |= d.first == rt.back.parts && d.second >= 2 * 16 * 4;
  CHECK(in);
  CHECK(back(9, 9000, u.data(), u.data(), u.floats(), u.floats(), 9000) == PEAT_OK);
  CHECK((char*)rt.back.dots >= (char*)rt.back.parts + 2 * 9000 * 4);
  rt.launches = 0;
  for (int i = 0; i < 5; i++)
    CHECK(back(9, 16, i == 0 ? nullptr : u.data() + (i == 1), i < 2 || i > 2 ? u.data() : nullptr, i == 2 ? nullptr : u.floats(),
               i == 3 ? nullptr : u.floats(), i == 4 ? 15 : 16) == PEAT_ERR_INVALID_ARG);
  CHECK(rt.launches == 0);
  CHECK(back(0, 16, nullptr, nullptr, u.floats(), nullptr, 16) == PEAT_OK && rt.launches == 1);  // no rows: the sums are 0
  CHECK(back(0, 16, nullptr, nullptr, nullptr, nullptr, 16) == PEAT_OK && rt.launches == 1);
  CHECK(back(9, (int64_t)1 << 28, u.data(), u.data(), u.floats(), u.floats(), (int64_t)1 << 28) == PEAT_ERR_UNSUPPORTED);
}

}  // namespace

int main(int argc, char** argv) {
  const std::map<std::string, void (*)()> checks = {{"quantize_refusals", quantize_refusals},
                                                    {"product_refusals", product_refusals},
                                                    {"operands", operands},
                                                    {"captures", captures},
                                                    {"norm_refusals", norm_refusals}};
  if (argc != 2 || !checks.count(argv[1])) return 2;
  checks.at(argv[1])();
  return failures ? 1 : 0;
}
