// Host side of the playback operators declared in include/peat_ops.h:
// argument checks, workspace, launch planning.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>
#include <vector>

#include "ops_internal.h"
#include "peat_handle.h"

namespace peat {

// Words that a call finds zero and the next one clears: two halves, in turn.  A
// call that is captured into a graph has a third part, which it clears itself,
// because the graph does not run in turn with the calls after it.
struct Halves {
  void* p = nullptr;
  size_t cap = 0;  // bytes of the three parts
  int64_t used[2] = {0, 0};
  int at = 0;
  bool lost = false;  // a launch or a clearing failed: what they hold is not known
};

// Made by a handle's first call of an operator, freed with it.
struct OpsState {
  bool capturing = false;  // the call at work is being captured
  bool captured = false;   // some call was: blocks that a graph may use are kept
  std::vector<void*> kept;
  // gradient lists: device block (entries, then partial sums), and a ring of
  // pinned copies of the entries, each free again once its event has passed
  static constexpr int RING = 4;
  void* d_list = nullptr;
  size_t d_list_cap = 0;
  void* h_list[RING] = {};
  size_t h_list_cap[RING] = {};
  cudaEvent_t taken[RING] = {};
  bool pending[RING] = {};
  int next = 0;
  unsigned int* done = nullptr;  // zero between calls
  void* tickets = nullptr;       // counters of finished parts, zero between calls
  size_t tickets_cap = 0;
  Halves colmax;  // column maxima
  Halves norms;   // sums of squares of operands packed on the way
  // operands that a product rounds, and their scales
  void* rounded = nullptr;
  size_t rounded_cap = 0;
  // products: packed operands and partial sums
  void* mm = nullptr;
  size_t mm_cap = 0;
};

void ops_destroy(OpsState* s) {
  if (!s) return;
  if (s->d_list) cudaFree(s->d_list);
  if (s->done) cudaFree(s->done);
  if (s->tickets) cudaFree(s->tickets);
  if (s->colmax.p) cudaFree(s->colmax.p);
  if (s->mm) cudaFree(s->mm);
  if (s->rounded) cudaFree(s->rounded);
  if (s->norms.p) cudaFree(s->norms.p);
  for (void* p : s->kept) cudaFree(p);
  for (int i = 0; i < OpsState::RING; i++) {
    if (s->h_list[i]) cudaFreeHost(s->h_list[i]);
    if (s->taken[i]) cudaEventDestroy(s->taken[i]);
  }
  delete s;
}

}  // namespace peat

namespace {

using peat::cuda_fail;
using peat::DeviceGuard;
using peat::fail;
using peat::OpsState;

constexpr int64_t MAX_DIM = ((int64_t)1 << 31) - 1;

int type_bytes(int dt) { return dt == PEAT_F32 ? 4 : (dt == PEAT_F16 || dt == PEAT_BF16 ? 2 : 0); }
bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

peat_status_t ops_state(peat_handle_t h, cudaStream_t st, OpsState** out) {
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(st, &capture) != cudaSuccess) {
    cudaGetLastError();
    capture = cudaStreamCaptureStatusNone;
  }
  const bool capturing = capture != cudaStreamCaptureStatusNone;
  if (!h->ops) {
    if (capturing) return fail(h, PEAT_ERR_UNSUPPORTED, "a handle's first operator call cannot be captured");
    OpsState* s = new OpsState();
    if (cudaMalloc(&s->done, 256) != cudaSuccess || cudaMemset(s->done, 0, 256) != cudaSuccess ||
        cudaDeviceSynchronize() != cudaSuccess) {
      cudaGetLastError();
      peat::ops_destroy(s);
      return fail(h, PEAT_ERR_ALLOC, "operator workspace allocation failed");
    }
    h->ops = s;
  }
  h->ops->capturing = capturing;
  h->ops->captured |= capturing;
  *out = h->ops;
  return PEAT_OK;
}

// Grows a device block; its contents are not kept, and an earlier call that uses
// it is waited for by cudaFree.  A block that is outgrown is followed by one half
// as large again at least, where there is room: sizes that grow call by call
// allocate seldom, and blocks that are kept for a graph add up to at most twice
// the last one.
peat_status_t grow(peat_handle_t h, void** p, size_t* cap, size_t need) {
  if (need <= *cap) return PEAT_OK;
  if (h->ops->capturing)
    return fail(h, PEAT_ERR_UNSUPPORTED, "the workspace would have to grow: make the call once before it is captured");
  size_t room = std::max(need, *cap + *cap / 2);
  if (*p && h->ops->captured) h->ops->kept.push_back(*p);
  else if (*p) cudaFree(*p);
  *p = nullptr;
  *cap = 0;
  cudaError_t e = cudaMalloc(p, room);
  if (e != cudaSuccess && room > need) {
    cudaGetLastError();
    room = need;
    e = cudaMalloc(p, room);
  }
  if (e != cudaSuccess) {
    cudaGetLastError();
    *p = nullptr;
    return fail(h, PEAT_ERR_ALLOC, "operator workspace allocation failed");
  }
  *cap = room;
  return PEAT_OK;
}

// n counters, zero
peat_status_t tickets(peat_handle_t h, OpsState* s, size_t n, cudaStream_t st) {
  const size_t need = sizeof(unsigned int) * std::max(n, (size_t)4096);
  if (need <= s->tickets_cap) return PEAT_OK;
  peat_status_t ps = grow(h, &s->tickets, &s->tickets_cap, need);
  if (ps != PEAT_OK) return ps;
  cudaError_t e = cudaMemsetAsync(s->tickets, 0, s->tickets_cap, st);
  if (e == cudaSuccess) return PEAT_OK;
  s->tickets_cap = 0;  // the next call tries again
  return cuda_fail(h, e, "cudaMemsetAsync(counters)");
}

// a staging buffer whose last copy has been taken
peat_status_t slot_free(peat_handle_t h, OpsState* s, int slot) {
  if (!s->pending[slot]) return PEAT_OK;
  cudaError_t e = cudaEventSynchronize(s->taken[slot]);
  if (e != cudaSuccess) return cuda_fail(h, e, "cudaEventSynchronize");
  s->pending[slot] = false;
  return PEAT_OK;
}
// Staging buffers of `bytes` at least: all of the ring at once, so that only a
// first call of its size allocates; outgrown ones as `grow` has it.
peat_status_t staging(peat_handle_t h, OpsState* s, size_t bytes) {
  for (int i = 0; i < OpsState::RING; i++) {
    if (!s->taken[i] && cudaEventCreateWithFlags(&s->taken[i], cudaEventDisableTiming) != cudaSuccess) {
      cudaGetLastError();
      s->taken[i] = nullptr;
      return fail(h, PEAT_ERR_ALLOC, "operator staging allocation failed");
    }
    if (bytes <= s->h_list_cap[i]) continue;
    peat_status_t ps = slot_free(h, s, i);
    if (ps != PEAT_OK) return ps;
    const size_t room = std::max(bytes, s->h_list_cap[i] + s->h_list_cap[i] / 2);
    if (s->h_list[i]) cudaFreeHost(s->h_list[i]);
    s->h_list[i] = nullptr;
    s->h_list_cap[i] = 0;
    if (cudaMallocHost(&s->h_list[i], room) != cudaSuccess) {
      cudaGetLastError();
      s->h_list[i] = nullptr;
      return fail(h, PEAT_ERR_ALLOC, "operator staging allocation failed");
    }
    s->h_list_cap[i] = room;
  }
  return PEAT_OK;
}

// the checks of a quantisation, and its launches' parameters but for the workspace
peat_status_t quant_params(peat_handle_t h, const void* x, int64_t rows, int64_t cols, int64_t ldx, int dtype, int axis,
                           int8_t* q, int64_t ldq, float* scale, void* values, int64_t ldv, peat::QuantParams* p) {
  const int B = type_bytes(dtype);
  if (!B) return fail(h, PEAT_ERR_INVALID_ARG, "dtype must be PEAT_F32, PEAT_F16 or PEAT_BF16");
  if (axis != 0 && axis != 1) return fail(h, PEAT_ERR_INVALID_ARG, "axis must be 0 (rows) or 1 (columns)");
  if (rows < 0 || cols < 0) return fail(h, PEAT_ERR_INVALID_ARG, "rows or cols < 0");
  if (rows > MAX_DIM || cols > MAX_DIM) return fail(h, PEAT_ERR_UNSUPPORTED, "rows or cols above 2^31 - 1");
  if (ldx < cols) return fail(h, PEAT_ERR_INVALID_ARG, "ldx < cols");
  if (q && ldq < (axis == 0 ? cols : rows)) return fail(h, PEAT_ERR_INVALID_ARG, "ldq is less than a row of q");
  if (values && ldv < cols) return fail(h, PEAT_ERR_INVALID_ARG, "ldv < cols");
  const bool any = rows > 0 && cols > 0;
  if (any && !x) return fail(h, PEAT_ERR_INVALID_ARG, "x is NULL");
  if (any && !q && !values) return fail(h, PEAT_ERR_INVALID_ARG, "q and values are both NULL");
  if ((any && !aligned(x, B)) || (values && !aligned(values, B)) || (scale && !aligned(scale, 4)))
    return fail(h, PEAT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  const int E = 16 / B;
  std::memset(p, 0, sizeof(*p));
  p->x = x;
  p->rows = rows;
  p->cols = cols;
  p->ldx = ldx;
  p->q = q;
  p->ldq = ldq;
  p->scale = scale;
  p->values = values;
  p->ldv = ldv;
  p->vec_x = aligned(x, 16) && (ldx % E == 0 || rows <= 1);
  const int qa = axis == 0 ? E : 4;
  p->vec_q = q && aligned(q, qa) && (ldq % qa == 0 || (axis == 0 ? rows : cols) <= 1);
  p->vec_v = values && aligned(values, 16) && (ldv % E == 0 || rows <= 1);
  return PEAT_OK;
}

// n zeroed words out of a buffer of two halves, used in turn by the calls that
// take some: a call also clears (*zero, *zero_n) what the one before it used.
peat_status_t take(peat_handle_t h, peat::Halves* b, int64_t n, int64_t least, unsigned int** words, unsigned int** zero,
                   int64_t* zero_n, cudaStream_t st) {
  const size_t need = 3 * sizeof(unsigned int) * (size_t)((std::max(n, least) + 3) / 4 * 4);
  if (need > b->cap || (b->lost && !h->ops->capturing)) {
    peat_status_t ps = grow(h, &b->p, &b->cap, need);
    if (ps != PEAT_OK) return ps;
    b->lost = true;
    b->used[0] = b->used[1] = 0;
    cudaError_t e = cudaMemsetAsync(b->p, 0, b->cap, st);
    if (e != cudaSuccess) return cuda_fail(h, e, "cudaMemsetAsync(workspace)");
    b->lost = false;  // (a growth that was refused leaves them as they are)
  }
  const size_t half = b->cap / 3 / sizeof(unsigned int) / 4 * 4;  // (sums of squares are read in pairs)
  unsigned int* base = static_cast<unsigned int*>(b->p);
  if (h->ops->capturing) {
    *words = *zero = base + 2 * half;
    *zero_n = 0;
    cudaError_t e = cudaMemsetAsync(*words, 0, sizeof(unsigned int) * (size_t)n, st);
    return e == cudaSuccess ? PEAT_OK : cuda_fail(h, e, "cudaMemsetAsync(workspace)");
  }
  *words = base + b->at * half;
  *zero = base + (b->at ^ 1) * half;
  *zero_n = b->used[b->at ^ 1];
  b->used[b->at] = n;
  b->used[b->at ^ 1] = 0;
  b->at ^= 1;
  return PEAT_OK;
}

peat_status_t quantize(peat_handle_t h, const void* x, int64_t rows, int64_t cols, int64_t ldx, int dtype, int axis,
                       int8_t* q, int64_t ldq, float* scale, void* values, int64_t ldv, cudaStream_t st) {
  peat::QuantParams p;
  peat_status_t ps = quant_params(h, x, rows, cols, ldx, dtype, axis, q, ldq, scale, values, ldv, &p);
  if (ps != PEAT_OK) return ps;
  // nothing to write: no scale either
  if ((axis == 0 ? rows : cols) == 0) return PEAT_OK;
  DeviceGuard dg(h->device);
  if (!dg.ok) return fail(h, PEAT_ERR_CUDA, "cudaSetDevice failed");
  cudaError_t e;
  if (axis == 0 || rows <= peat::QUANT_FEW_ROWS) {
    e = peat::launch_quant8(dtype, axis == 0 ? peat::QUANT_ROWS : peat::QUANT_COLUMNS, p, h->nsm, st);
  } else {
    OpsState* s = nullptr;
    ps = ops_state(h, st, &s);
    if (ps == PEAT_OK) ps = take(h, &s->colmax, cols, 8192, &p.colmax, &p.zero, &p.zero_n, st);
    if (ps != PEAT_OK) return ps;
    e = peat::launch_quant8(dtype, peat::QUANT_MAXIMA, p, h->nsm, st);
    if (e == cudaSuccess) e = peat::launch_quant8(dtype, peat::QUANT_COLUMNS, p, h->nsm, st);
    if (e != cudaSuccess) s->colmax.lost = true;
  }
  if (e != cudaSuccess) return cuda_fail(h, e, "8-bit quantisation launch");
  return PEAT_OK;
}

// checks of a product's output and inner size
peat_status_t output_ok(peat_handle_t h, const float* sa, const float* sb, const float* bias, int64_t M, int64_t N,
                        int64_t K, const void* out, int64_t ldo, int out_dtype) {
  const int B = out_dtype == PEAT_OUT_I32 ? 4 : type_bytes(out_dtype);
  if (K > 131071) return fail(h, PEAT_ERR_UNSUPPORTED, "K above 131071: the sums may not fit 32 bits");
  if (ldo < N) return fail(h, PEAT_ERR_INVALID_ARG, "ldo is less than a row");
  if (M == 0 || N == 0) return PEAT_OK;
  // tiles are counted in 32 bits
  if (M > MAX_DIM || N > MAX_DIM || ((M + 63) / 64) * ((N + 127) / 128) > ((int64_t)1 << 27))
    return fail(h, PEAT_ERR_UNSUPPORTED, "the output is too large for one call");
  if (!out) return fail(h, PEAT_ERR_INVALID_ARG, "out is NULL");
  if (!aligned(out, B) || (sa && !aligned(sa, 4)) || (sb && !aligned(sb, 4)) || (bias && !aligned(bias, 4)))
    return fail(h, PEAT_ERR_INVALID_ARG, "a pointer is not aligned to its element type");
  if (h->status_host && *(volatile unsigned int*)h->status_host) {
    *(volatile unsigned int*)h->status_host = 0;
    return fail(h, PEAT_ERR_TIMEOUT,
                "a bounded device-side wait expired in an earlier call on this handle; its outputs are invalid");
  }
  return PEAT_OK;
}
// whether the tensor-core path takes a product
bool wide_product(peat_handle_t h, const peat::Mm8TcPlan& plan, const peat::Mm8Params& p) {
  // the packed blocks' rows are 32-bit coordinates
  const bool fits = (plan.mt + plan.nt) * 2 * plan.kb < ((int64_t)1 << 24);
  return p.K > 0 && fits &&
         peat::mm8_tc_time(plan, p.K, h->nsm) < peat::mm8_direct_time(p.M, p.N, p.K, peat::mm8_aligned(p), h->nsm);
}
unsigned int wait_limit(peat_handle_t h) { return std::min(h->wait_limit, 1u << 22); }

peat_status_t matmul(peat_handle_t h, const int8_t* a, int64_t lda, const float* sa, const int8_t* b, int64_t ldb,
                     const float* sb, const float* bias, int64_t M, int64_t N, int64_t K, void* out, int64_t ldo,
                     int out_dtype, cudaStream_t st) {
  if (out_dtype != PEAT_OUT_I32 && !type_bytes(out_dtype))
    return fail(h, PEAT_ERR_INVALID_ARG, "out_dtype must be PEAT_F32, PEAT_F16, PEAT_BF16 or PEAT_OUT_I32");
  if (M < 0 || N < 0 || K < 0) return fail(h, PEAT_ERR_INVALID_ARG, "M, N or K < 0");
  if (lda < K || ldb < K) return fail(h, PEAT_ERR_INVALID_ARG, "lda or ldb is less than a row");
  if (out_dtype == PEAT_OUT_I32 && (sa || sb || bias))
    return fail(h, PEAT_ERR_INVALID_ARG, "PEAT_OUT_I32 takes no scales and no bias");
  peat_status_t ps = output_ok(h, sa, sb, bias, M, N, K, out, ldo, out_dtype);
  if (ps != PEAT_OK || M == 0 || N == 0) return ps;
  if (K > 0 && (!a || !b)) return fail(h, PEAT_ERR_INVALID_ARG, "a or b is NULL");
  DeviceGuard dg(h->device);
  if (!dg.ok) return fail(h, PEAT_ERR_CUDA, "cudaSetDevice failed");
  const peat::Mm8Params p{a, b, lda, ldb, sa, sb, bias, out, ldo, M, N, K};
  const peat::Mm8TcPlan plan = peat::mm8_tc_plan(M, N, K, h->nsm);
  cudaError_t e;
  if (wide_product(h, plan, p)) {
    OpsState* s = nullptr;
    ps = ops_state(h, st, &s);
    const size_t norms = (plan.bytes + 255) / 256 * 256;
    if (ps == PEAT_OK)
      ps = grow(h, &s->mm, &s->mm_cap, norms + sizeof(unsigned int) * (size_t)(plan.na_words + plan.nb_words));
    if (ps != PEAT_OK) return ps;
    char* ws = static_cast<char*>(s->mm);
    unsigned int* sums = reinterpret_cast<unsigned int*>(ws + norms);
    e = peat::launch_mm8_pack(p, plan, ws, sums, 3, st);
    if (e == cudaSuccess)
      e = peat::launch_mm8_tc(out_dtype, p, plan, ws, sums, false, h->status_dev, wait_limit(h), h->nsm, st);
  } else {
    e = peat::launch_mm8_direct(out_dtype, p, h->nsm, st);
  }
  if (e != cudaSuccess) return cuda_fail(h, e, "8-bit product launch");
  return PEAT_OK;
}

// Rounds a float operand into the handle's workspace at *at, which moves on.
// Before a pass with ws NULL only the place is counted.
struct Operand {
  const int8_t* q;
  const float* scale;
  int64_t rows, K, ld;
};
bool operand_ok(const peat_operand_t* o) {
  if (!o || o->rows < 0 || o->cols < 0 || o->ld < o->cols) return false;
  if (o->dtype == PEAT_INT8) return o->axis == 0;
  return type_bytes(o->dtype) != 0 && (o->axis == 0 || o->axis == 1);
}
Operand operand_of(const peat_operand_t& o, char* ws, size_t* at) {
  Operand r;
  r.rows = o.axis ? o.cols : o.rows;
  r.K = o.axis ? o.rows : o.cols;
  if (o.dtype == PEAT_INT8) {
    r.q = static_cast<const int8_t*>(o.data);
    r.scale = o.scale;
    r.ld = o.ld;
    return r;
  }
  r.ld = (r.K + 15) / 16 * 16;
  r.scale = reinterpret_cast<const float*>(ws + *at);
  *at += ((size_t)r.rows * sizeof(float) + 255) / 256 * 256;
  r.q = reinterpret_cast<const int8_t*>(ws + *at);
  *at += ((size_t)r.rows * (size_t)r.ld + 255) / 256 * 256;
  return r;
}

peat_status_t product(peat_handle_t h, const peat_operand_t* a, const peat_operand_t* b, const float* bias, void* out,
                      int64_t ldo, int out_dtype, cudaStream_t st) {
  if (!operand_ok(a) || !operand_ok(b))
    return fail(h, PEAT_ERR_INVALID_ARG, "an operand is NULL, or its sizes, dtype or axis are not valid");
  if (!type_bytes(out_dtype)) return fail(h, PEAT_ERR_INVALID_ARG, "out_dtype must be PEAT_F32, PEAT_F16 or PEAT_BF16");
  size_t need = 0;
  Operand x = operand_of(*a, nullptr, &need), y = operand_of(*b, nullptr, &need);
  if (x.K != y.K) return fail(h, PEAT_ERR_INVALID_ARG, "the operands differ in K");
  const int64_t M = x.rows, N = y.rows, K = x.K;
  peat_status_t ps = output_ok(h, x.scale, y.scale, bias, M, N, K, out, ldo, out_dtype);
  if (ps != PEAT_OK || M == 0 || N == 0) return ps;
  if (K > 0 && (!a->data || !b->data)) return fail(h, PEAT_ERR_INVALID_ARG, "an operand's data is NULL");
  DeviceGuard dg(h->device);
  if (!dg.ok) return fail(h, PEAT_ERR_CUDA, "cudaSetDevice failed");
  OpsState* s = nullptr;
  ps = ops_state(h, st, &s);
  if (ps == PEAT_OK) ps = grow(h, &s->rounded, &s->rounded_cap, need);
  if (ps != PEAT_OK) return ps;
  char* rounded = static_cast<char*>(s->rounded);
  size_t at = 0;
  x = operand_of(*a, rounded, &at);
  y = operand_of(*b, rounded, &at);
  const peat::Mm8TcPlan plan = peat::mm8_tc_plan(M, N, K, h->nsm);
  const peat::Mm8Params p{x.q, y.q, x.ld, y.ld, x.scale, y.scale, bias, out, ldo, M, N, K};
  const bool wide = wide_product(h, plan, p);

  // Which operands are rounded, and which of them straight into packed blocks
  const peat_operand_t* in[2] = {a, b};
  const Operand* op[2] = {&x, &y};
  peat::QuantParams q[2];
  int rounded_ops = 0, packed = 0;
  int64_t columns = 0;
  for (int i = 0; i < 2; i++) {
    if (in[i]->dtype == PEAT_INT8) continue;
    ps = quant_params(h, in[i]->data, in[i]->rows, in[i]->cols, in[i]->ld, in[i]->dtype, in[i]->axis,
                      const_cast<int8_t*>(op[i]->q), op[i]->ld, const_cast<float*>(op[i]->scale), nullptr, 0, &q[i]);
    if (ps != PEAT_OK) return ps;
    rounded_ops |= 1 << i;
    if (in[i]->axis && in[i]->rows > peat::QUANT_FEW_ROWS) columns += in[i]->cols;
    q[i].kb = plan.kb;
    q[i].kc = plan.kc;
    if (wide && peat::quant8_packs(in[i]->dtype, in[i]->axis, q[i])) packed |= 1 << i;
  }
  char* ws = nullptr;
  unsigned int *norms = nullptr, *stale = nullptr, *maxima = nullptr, *zero = nullptr;
  int64_t stale_n = 0, zero_n = 0;
  const int64_t words = plan.na_words + plan.nb_words;
  if (packed) {
    ps = grow(h, &s->mm, &s->mm_cap, plan.bytes);
    if (ps != PEAT_OK) return ps;
    ws = static_cast<char*>(s->mm);
    if (words) ps = take(h, &s->norms, words, 4096, &norms, &stale, &stale_n, st);
    if (ps != PEAT_OK) return ps;
  }
  if (columns) {
    ps = take(h, &s->colmax, columns, 8192, &maxima, &zero, &zero_n, st);
    if (ps != PEAT_OK) {
      s->norms.lost = true;  // (what it was to clear)
      return ps;
    }
  }
  // A launch that needs nothing of the one before it runs beside it: the
  // packing of one operand and the rounding of the other, both operands'
  // column maxima, both operands' columns.
  cudaError_t e = cudaSuccess;
  bool beside = false;
  const int as_is = packed ? 3 & ~rounded_ops : 0;
  if (as_is) {
    e = peat::launch_mm8_pack(p, plan, ws, norms, as_is, st);
    beside = true;
  }
  int64_t at_column = 0;
  for (int i = 0; i < 2; i++) {
    if (!(rounded_ops >> i & 1) || !in[i]->axis || !columns) continue;  // (both operands' columns have K rows)
    q[i].colmax = maxima + at_column;
    at_column += in[i]->cols;
    q[i].overlap = beside;
    if (e == cudaSuccess) e = peat::launch_quant8(in[i]->dtype, peat::QUANT_MAXIMA, q[i], h->nsm, st);
    beside = true;
  }
  if (columns) beside = false;  // the columns need their maxima
  for (int i = 0; i < 2; i++) {
    if (!(rounded_ops >> i & 1)) continue;
    if (packed >> i & 1) {
      q[i].packed = ws + (i ? plan.b_off : plan.a_off);
      q[i].prows = (i ? plan.nt : plan.mt) * 256;
      q[i].norms = norms ? norms + (i ? plan.na_words : 0) : nullptr;
      q[i].zero2 = stale;
      q[i].zero2_n = stale_n;
      stale_n = 0;
    }
    if (q[i].colmax) {
      q[i].zero = zero;
      q[i].zero_n = zero_n;
      zero_n = 0;
    }
    q[i].overlap = beside && (packed >> i & 1 || in[i]->axis);
    if (e == cudaSuccess)
      e = peat::launch_quant8(in[i]->dtype, in[i]->axis ? peat::QUANT_COLUMNS : peat::QUANT_ROWS, q[i], h->nsm, st);
    beside = true;
  }
  // (a rounded operand that could not be packed on the way)
  if (e == cudaSuccess && packed && (rounded_ops & ~packed)) e = peat::launch_mm8_pack(p, plan, ws, norms, rounded_ops & ~packed, st);
  if (e == cudaSuccess && packed)
    e = peat::launch_mm8_tc(out_dtype, p, plan, ws, norms, true, h->status_dev, wait_limit(h), h->nsm, st);
  if (e != cudaSuccess) {
    s->norms.lost = s->colmax.lost = true;
    return cuda_fail(h, e, "8-bit product launch");
  }
  if (!packed) return matmul(h, x.q, x.ld, x.scale, y.q, y.ld, y.scale, bias, M, N, K, out, ldo, out_dtype, st);
  return PEAT_OK;
}

peat_status_t grad_pass(peat_handle_t h, const peat_grad_t* list, int64_t count, int type, float unscale, bool clip,
                        float max_norm, float eps, int bad, peat_gradnorm_t* result, float* norms, cudaStream_t st) {
  if (count < 0 || (count > 0 && !list)) return fail(h, PEAT_ERR_INVALID_ARG, "count < 0, or list is NULL");
  if (count > ((int64_t)1 << 24)) return fail(h, PEAT_ERR_UNSUPPORTED, "more than 2^24 tensors");
  if (type != PEAT_NORM_2 && type != PEAT_NORM_1 && type != PEAT_NORM_INF)
    return fail(h, PEAT_ERR_INVALID_ARG, "type must be one of peat_norm_t");
  if (!(unscale > 0.0f) || !std::isfinite(unscale))
    return fail(h, PEAT_ERR_INVALID_ARG, "unscale must be finite and > 0");
  if (clip && !(max_norm >= 0.0f)) return fail(h, PEAT_ERR_INVALID_ARG, "max_norm must be >= 0");
  if (clip && (!(eps >= 0.0f) || !std::isfinite(eps)))
    return fail(h, PEAT_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (clip && bad != PEAT_BAD_PROPAGATE && bad != PEAT_BAD_ZERO && bad != PEAT_BAD_KEEP)
    return fail(h, PEAT_ERR_INVALID_ARG, "bad must be one of peat_bad_t");
  if (!result || !aligned(result, 8)) return fail(h, PEAT_ERR_INVALID_ARG, "result is NULL or not 8-byte aligned");
  if (norms && !aligned(norms, 4)) return fail(h, PEAT_ERR_INVALID_ARG, "norms is not aligned");
  int64_t units = 0;
  for (int64_t t = 0; t < count; t++) {
    const peat_grad_t& e = list[t];
    const int B = type_bytes(e.dtype);
    if (!B) return fail(h, PEAT_ERR_INVALID_ARG, "a tensor's dtype must be PEAT_F32, PEAT_F16 or PEAT_BF16");
    if (e.n < 0 || e.reserved != 0) return fail(h, PEAT_ERR_INVALID_ARG, "a tensor's n < 0, or reserved not 0");
    if (e.n > ((int64_t)1 << 40)) return fail(h, PEAT_ERR_UNSUPPORTED, "a tensor of more than 2^40 elements");
    if (e.n == 0) continue;
    if (!e.g || !aligned(e.g, B)) return fail(h, PEAT_ERR_INVALID_ARG, "a tensor's g is NULL or not aligned to its type");
    if (clip && (!e.out || !aligned(e.out, B)))
      return fail(h, PEAT_ERR_INVALID_ARG, "a tensor's out is NULL or not aligned to its type");
    units += peat::gn_units(e.g, e.n, B);
  }
  // units * warps stays inside 64 bits
  if (units > ((int64_t)1 << 44)) return fail(h, PEAT_ERR_UNSUPPORTED, "the list is too large");
  DeviceGuard dg(h->device);
  if (!dg.ok) return fail(h, PEAT_ERR_CUDA, "cudaSetDevice failed");
  OpsState* s = nullptr;
  peat_status_t ps = ops_state(h, st, &s);
  if (ps != PEAT_OK) return ps;

  // a piece's own time is about that of 256 units
  const int64_t lead = 256;
  for (int64_t t = 0; t < count; t++) units += list[t].n > 0 ? lead : 0;
  // one wave; a warp has at least 64 units
  const int per = peat::gn_block() / 32;
  const int64_t warps = std::max<int64_t>(1, std::min<int64_t>((units + 63) / 64, (int64_t)h->nsm * 5 * per));
  const int nctas = (int)((warps + per - 1) / per);
  const size_t listed = count > peat::GN_INLINE ? (sizeof(peat::GnEntry) * (size_t)count + 255) / 256 * 256 : 0;
  const size_t parted = sizeof(peat::GnPartial) * (size_t)(count + warps);
  ps = grow(h, &s->d_list, &s->d_list_cap, listed + parted + sizeof(peat::GnPartial) * (size_t)count);
  if (ps != PEAT_OK) return ps;
  ps = tickets(h, s, (size_t)count, st);
  if (ps != PEAT_OK) return ps;

  peat::GnEntry inline_list[peat::GN_INLINE];
  peat::GnEntry* dst = inline_list;
  int slot = -1;
  if (listed && s->capturing)
    return fail(h, PEAT_ERR_UNSUPPORTED, "a list of more than 800 tensors cannot be captured: it is staged by the host");
  if (listed) {
    ps = staging(h, s, listed);
    if (ps != PEAT_OK) return ps;
    slot = s->next;
    s->next = (s->next + 1) % OpsState::RING;
    ps = slot_free(h, s, slot);
    if (ps != PEAT_OK) return ps;
    dst = static_cast<peat::GnEntry*>(s->h_list[slot]);
  }
  units = 0;
  for (int64_t t = 0; t < count; t++) {
    const peat_grad_t& e = list[t];
    dst[t] = peat::GnEntry{e.g, e.out, e.n, units, e.dtype, 0};
    units += peat::gn_units(e.g, e.n, type_bytes(e.dtype)) + (e.n > 0 ? lead : 0);
  }
  if (listed) {
    cudaError_t e = cudaMemcpyAsync(s->d_list, dst, sizeof(peat::GnEntry) * (size_t)count, cudaMemcpyHostToDevice, st);
    if (e != cudaSuccess) return cuda_fail(h, e, "cudaMemcpyAsync(list)");
    e = cudaEventRecord(s->taken[slot], st);
    if (e != cudaSuccess) return cuda_fail(h, e, "cudaEventRecord");
    s->pending[slot] = true;
  }
  peat::GnParams p;
  p.list = listed ? static_cast<const peat::GnEntry*>(s->d_list) : nullptr;
  p.count = (int)count;
  p.units = units;
  p.nwarps = (int)warps;
  p.type = type;
  p.unscale = unscale;
  p.max_norm = max_norm;
  p.eps = eps;
  p.bad_mode = bad;
  p.clip = clip ? 1 : 0;
  p.parts = reinterpret_cast<peat::GnPartial*>(static_cast<char*>(s->d_list) + listed);
  p.sums = reinterpret_cast<peat::GnPartial*>(static_cast<char*>(s->d_list) + listed + parted);
  p.tickets = static_cast<unsigned int*>(s->tickets);
  p.done = s->done;
  p.result = result;
  p.norms = norms;
  p.lead = lead;
  cudaError_t e = peat::launch_gradnorm(p, inline_list, nctas, st);
  if (e != cudaSuccess) return cuda_fail(h, e, "gradient norm launch");
  return PEAT_OK;
}

// nothing is thrown across the C boundary
template <typename F>
peat_status_t guarded(peat_handle_t h, F f) {
  if (!h) return PEAT_ERR_INVALID_ARG;
  try {
    return f();
  } catch (const std::bad_alloc&) {  // (texts that a string holds in itself: setting them throws nothing)
    h->err = "out of memory";
    return PEAT_ERR_ALLOC;
  } catch (...) {
    h->err = "internal error";
    return PEAT_ERR_INTERNAL;
  }
}

}  // namespace

extern "C" {

peat_status_t peat_quantize_i8(peat_handle_t h, const void* x, int64_t rows, int64_t cols, int64_t ldx,
                               peat_dtype_t dtype, int axis, int8_t* q, int64_t ldq, float* scale, void* values,
                               int64_t ldv, peat_stream_t stream) {
  return guarded(h, [&] {
    return quantize(h, x, rows, cols, ldx, dtype, axis, q, ldq, scale, values, ldv,
                    reinterpret_cast<cudaStream_t>(stream));
  });
}

peat_status_t peat_matmul_i8(peat_handle_t h, const int8_t* a, int64_t lda, const float* a_scale, const int8_t* b,
                             int64_t ldb, const float* b_scale, const float* bias, int64_t M, int64_t N, int64_t K,
                             void* out, int64_t ldo, int out_dtype, peat_stream_t stream) {
  return guarded(h, [&] {
    return matmul(h, a, lda, a_scale, b, ldb, b_scale, bias, M, N, K, out, ldo, out_dtype,
                  reinterpret_cast<cudaStream_t>(stream));
  });
}

peat_status_t peat_product_i8(peat_handle_t h, const peat_operand_t* a, const peat_operand_t* b, const float* bias,
                              void* out, int64_t ldo, peat_dtype_t out_dtype, peat_stream_t stream) {
  return guarded(h, [&] {
    return product(h, a, b, bias, out, ldo, out_dtype, reinterpret_cast<cudaStream_t>(stream));
  });
}

peat_status_t peat_grad_norm(peat_handle_t h, const peat_grad_t* list, int64_t count, peat_norm_t type,
                             float unscale, peat_gradnorm_t* result, float* norms, peat_stream_t stream) {
  return guarded(h, [&] {
    return grad_pass(h, list, count, type, unscale, false, 0.0f, 0.0f, PEAT_BAD_PROPAGATE, result, norms,
                     reinterpret_cast<cudaStream_t>(stream));
  });
}

peat_status_t peat_grad_clip(peat_handle_t h, const peat_grad_t* list, int64_t count, peat_norm_t type,
                             float unscale, float max_norm, float eps, peat_bad_t bad, peat_gradnorm_t* result,
                             float* norms, peat_stream_t stream) {
  return guarded(h, [&] {
    return grad_pass(h, list, count, type, unscale, true, max_norm, eps, bad, result, norms,
                     reinterpret_cast<cudaStream_t>(stream));
  });
}

}  // extern "C"
