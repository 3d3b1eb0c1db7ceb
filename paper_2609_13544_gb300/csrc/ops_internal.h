// Internal declarations of the playback operators (include/peat_ops.h).
#pragma once
#include <atomic>
#include <cstdint>

#include <cuda_runtime.h>

#include "peat.h"
#include "peat_ops.h"

namespace peat {

// a kernel's dynamic shared memory limit, raised once on each device (done: ordinals below 64)
template <typename K>
inline cudaError_t allow_smem(K kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// ---- 8-bit quantisation (quant8.cu) ----
struct QuantParams {
  const void* x;
  int64_t rows, cols, ldx;
  int8_t* q;  // or null
  int64_t ldq;
  float* scale;   // or null
  void* values;  // or null
  int64_t ldv;
  int vec_x;  // x's rows start on 16-byte boundaries
  int vec_q;  // q's rows start on boundaries of a vector's integers (axis 0: 8 or 4 bytes; axis 1: 4 bytes)
  int vec_v;  // values' rows start on 16-byte boundaries
  // columns: their largest patterns, zero before the call (null: the rows are few
  // and every CTA finds its own), and what to clear for a later one
  unsigned int* colmax;
  unsigned int* zero;
  int64_t zero_n;
  // the integers as a product's packed operand (mm8_tc.cu) in place of q; null: not
  void* packed;
  int kb, kc;        // its blocks of 64 k, and of 256
  int64_t prows;     // its rows, a multiple of 256
  unsigned int* norms;  // its sums of squares, zero before (null: not needed)
  unsigned int* zero2;  // those of an earlier call, cleared for a later one
  int64_t zero2_n;
  int overlap;  // the kernel before this one on the stream is nothing to it
};
// whether a packed operand can be made (rows that fit a CTA's registers)
bool quant8_packs(int dtype, int axis, const QuantParams& p);
// Rows up to which columns need no launch for their maxima: at 512 of 4096
// bfloat16 columns the one launch takes 6.4 us and the two 8.3.
constexpr int64_t QUANT_FEW_ROWS = 512;
// rows; or for columns first their maxima, then the integers
enum { QUANT_ROWS, QUANT_MAXIMA, QUANT_COLUMNS };
cudaError_t launch_quant8(int dtype, int step, const QuantParams& p, int nsm, cudaStream_t s);

// ---- 8-bit products (matmul8.cu) ----
struct Mm8Params {
  const int8_t* a;  // [M, K]
  const int8_t* b;  // [N, K]
  int64_t lda, ldb;
  const float* sa;    // or null
  const float* sb;    // or null
  const float* bias;  // or null
  void* out;
  int64_t ldo;
  int64_t M, N, K;
};
cudaError_t launch_mm8_direct(int out_dtype, const Mm8Params& p, int nsm, cudaStream_t s);
// the tensor-core path (mm8_tc.cu): tiles of 256 x 256, the operands packed in a workspace
struct Mm8TcPlan {
  int kb, kc;      // blocks of 64 k, and of 256
  int64_t mt, nt;  // tiles
  int splits;      // parts of a tile's k range: 1, 2 or 4
  size_t a_off, b_off, sum_off, bytes;  // workspace
  int64_t na_words, nb_words;            // sums of squares of a's and of b's blocks (0: not needed)
};
double mm8_direct_time(int64_t M, int64_t N, int64_t K, bool aligned, int nsm);  // expected microseconds
// whether the rows of an operand start on 16-byte boundaries (one row has no use for a distance)
inline bool mm8_rows_aligned(const int8_t* x, int64_t ld, int64_t rows) {
  return reinterpret_cast<uintptr_t>(x) % 16 == 0 && (ld % 16 == 0 || rows <= 1);
}
inline bool mm8_aligned(const Mm8Params& p) {
  return mm8_rows_aligned(p.a, p.lda, p.M) && mm8_rows_aligned(p.b, p.ldb, p.N);
}
Mm8TcPlan mm8_tc_plan(int64_t M, int64_t N, int64_t K, int nsm);
double mm8_tc_time(const Mm8TcPlan& p, int64_t K, int nsm);
// norms: na_words, then nb_words; which: bit 0 a, bit 1 b
cudaError_t launch_mm8_pack(const Mm8Params& p, const Mm8TcPlan& plan, char* ws, unsigned int* norms, int which,
                            cudaStream_t s);
// scales_late: the scales may be made by the kernel before
cudaError_t launch_mm8_tc(int out_dtype, const Mm8Params& p, const Mm8TcPlan& plan, char* ws, unsigned int* norms,
                          bool scales_late, unsigned int* status, unsigned int wait_limit, int nsm, cudaStream_t s);

// ---- gradient lists (gradnorm.cu) ----
struct GnEntry {
  const void* g;
  void* out;
  int64_t n;
  int64_t unit0;  // the list's 16-byte units before this tensor's (each tensor that has any leads with GnParams::lead empty ones)
  int32_t dtype, pad;
};
// Entries that travel as a kernel argument, which takes up to 32 764 bytes: a
// list in memory would first have to be copied there (a call with 800 tensors
// of 80 elements takes 12 us, with 801 of them 21).
constexpr int GN_INLINE_FEW = 96, GN_INLINE = 800;
template <int N>
struct GnInlineOf {
  GnEntry e[N];
};
struct alignas(16) GnPartial {
  double s;                // sum (or maximum)
  unsigned long long bad;  // NaN and infinite elements
};
struct GnParams {
  const GnEntry* list;  // device; null: the entries are a kernel argument
  int count;
  int64_t units;        // of the whole list
  int64_t lead;         // empty units before each tensor's: what a piece costs beside its bytes
  int nwarps;           // warps of the norm pass
  int type;             // peat_norm_t
  float unscale, max_norm, eps;
  int bad_mode;
  int clip;             // 0: norm only
  GnPartial* parts;     // count + nwarps slots: warp w's part of tensor t at t + w
  GnPartial* sums;      // one for each tensor
  unsigned int* tickets;  // pieces finished, one for each tensor, zero between calls
  unsigned int* done;   // CTAs finished, zero between calls
  peat_gradnorm_t* result;
  float* norms;         // or null
};
int gn_block();  // threads of a CTA of both passes
// host: the entries, where p.list is null
cudaError_t launch_gradnorm(const GnParams& p, const GnEntry* host, int nctas, cudaStream_t s);
// 16-byte units that hold the n elements of `size` bytes at g
inline int64_t gn_units(const void* g, int64_t n, int size) {
  if (n <= 0) return 0;
  const uintptr_t a = reinterpret_cast<uintptr_t>(g);
  return (int64_t)((a + (uint64_t)n * size + 15) / 16 - a / 16);
}

}  // namespace peat
