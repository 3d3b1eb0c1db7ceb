// What the host sources of the playback operators share: the state behind a
// handle, its workspace, checks of arguments.
#pragma once
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
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
  // 4-bit rounding by column: the columns' maxima over parts of the rows
  void* tops = nullptr;
  size_t tops_cap = 0;
  // norm gradients: the CTAs' sums over their rows, long rows' means
  void* norm = nullptr;
  size_t norm_cap = 0;
};

constexpr int64_t MAX_DIM = ((int64_t)1 << 31) - 1;

inline int type_bytes(int dt) { return dt == PEAT_F32 ? 4 : (dt == PEAT_F16 || dt == PEAT_BF16 ? 2 : 0); }
inline bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

inline peat_status_t ops_state(peat_handle_t h, cudaStream_t st, OpsState** out) {
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
      ops_destroy(s);
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
inline peat_status_t grow(peat_handle_t h, void** p, size_t* cap, size_t need) {
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

// n zeroed words out of a buffer of two halves, used in turn by the calls that
// take some: a call also clears (*zero, *zero_n) what the one before it used.
inline peat_status_t take(peat_handle_t h, Halves* b, int64_t n, int64_t least, unsigned int** words, unsigned int** zero,
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

inline unsigned int wait_limit(peat_handle_t h) { return std::min(h->wait_limit, 1u << 22); }

// an expired wait of an earlier call, told once
inline peat_status_t expired(peat_handle_t h) {
  if (h->status_host && *(volatile unsigned int*)h->status_host) {
    *(volatile unsigned int*)h->status_host = 0;
    return fail(h, PEAT_ERR_TIMEOUT,
                "a bounded device-side wait expired in an earlier call on this handle; its outputs are invalid");
  }
  return PEAT_OK;
}

// nothing is thrown across the C boundary
template <typename F>
inline peat_status_t guarded(peat_handle_t h, F f) {
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

}  // namespace peat
