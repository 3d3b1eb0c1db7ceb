// The norm over a list of gradient tensors, and their clipping.
//
// The list is taken as one run of 16-byte units (each tensor's own, from the
// boundary at or before its first element), shared out evenly to the warps of
// one wave; a warp's part of a tensor is a piece with one partial sum.  The warp
// that hands in a tensor's last piece adds them up in a fixed order, the CTA that
// finishes last the tensors.
//
// Squares: a lane adds 64 bytes' to 128 bytes' worth of them in float32 and the
// results with their rounding errors kept (Knuth's two-sum), so the sum is good
// to float32 whatever its length, and no binary64 instruction is needed per
// element (the GPU has few).  The largest magnitude is kept beside the sum:
// where it shows that squares may have left float32's range, or that an element
// is not finite, the warp reads its piece again, scaled by a power of two, and
// counts.
//
// Bound by memory: the norm reads the list once; clipping reads it again and
// writes it, each warp's share from its end, so that what the norm read last is
// still in L2 (355 million bfloat16 elements: 357 us, from its beginning 374).
// Outputs off the input's 16-byte grid are written element by element (25.6
// million float32 elements take 72 us, on it 60).  161 float32 tensors of 25.6
// million elements take 29 us (17 of reading at 6 TB/s, the rest is starting, the
// pieces and the last CTA; their 1-norm 29, their maximum 28), 268 million
// elements of one tensor 169 (6.4 TB/s); clipping 292 bfloat16 tensors of 355
// million elements 357 (three passes over 710 MB, 6.0 TB/s).
#include <algorithm>

#include "ops_internal.h"
#include "peat_internal.h"
#include "vec16.cuh"

namespace peat {
namespace {

constexpr int GB = 256;  // threads of a CTA

__device__ __forceinline__ int elem_size(int dt) { return dt == PEAT_F32 ? 4 : 2; }

// A tensor's bytes on the grid of 16-byte units: unit j is [base + 16 j, + 16);
// only the first and the last may hold bytes that are not the tensor's.
struct Span {
  const char* base;
  int64_t lo, hi;  // the tensor's bytes, from base
  __device__ Span(const GnEntry& e) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(e.g);
    base = reinterpret_cast<const char*>(a & ~(uintptr_t)15);
    lo = (int64_t)(a & 15);
    hi = lo + e.n * elem_size(e.dtype);
  }
  __device__ bool full(int64_t j) const { return 16 * j >= lo && 16 * j + 16 <= hi; }
};
// unit j with zeros in place of what is not the tensor's
template <int DT>
__device__ __forceinline__ uint4 edge_unit(const Span& s, int64_t j) {
  if (s.full(j)) return __ldcg(reinterpret_cast<const uint4*>(s.base) + j);
  uint32_t w[4] = {0, 0, 0, 0};
  constexpr int B = DT == PEAT_F32 ? 4 : 2;
#pragma unroll
  for (int i = 0; i < 16 / B; i++) {
    const int64_t at = 16 * j + i * B;
    if (at >= s.lo && at < s.hi) {
      if (B == 4) w[i % 4] = *reinterpret_cast<const uint32_t*>(s.base + at);
      else w[i / 2] |= (uint32_t) * reinterpret_cast<const uint16_t*>(s.base + at) << (16 * (i & 1));
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// a float32 sum with its rounding errors beside it
struct Sum {
  float hi = 0.0f, lo = 0.0f;
  __device__ __forceinline__ void add(float y) {
    const float t = __fadd_rn(hi, y), z = __fsub_rn(t, hi);
    lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(t, z)), __fsub_rn(y, z)));
    hi = t;
  }
};

template <int DT, int NORM>
__device__ __forceinline__ float unit_sum(uint4 u) {
  constexpr int E = DT == PEAT_F32 ? 4 : 8;
  float x[E];
  unpack<DT>(u, x);
  if (NORM == PEAT_NORM_1) {
    float a = fabsf(x[0]), b = fabsf(x[1]);
#pragma unroll
    for (int e = 2; e < E; e += 2) a += fabsf(x[e]), b += fabsf(x[e + 1]);
    return a + b;
  } else {
    float a = x[0] * x[0], b = x[1] * x[1];
#pragma unroll
    for (int e = 2; e < E; e += 2) a = fmaf(x[e], x[e], a), b = fmaf(x[e + 1], x[e + 1], b);
    return a + b;
  }
}
// the largest magnitude of a unit; a NaN stays
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
template <int DT>
__device__ __forceinline__ float unit_max(uint4 u) {
  constexpr int E = DT == PEAT_F32 ? 4 : 8;
  float x[E];
  unpack<DT>(u, x);
  float m = fabsf(x[0]);
#pragma unroll
  for (int e = 1; e < E; e++) m = max_nan(m, fabsf(x[e]));
  return m;
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// one piece: units [j0, j1) of a tensor, by a warp; the result in lane 0
template <int DT, int NORM>
__device__ GnPartial piece(const Span& s, int64_t j0, int64_t j1) {
  const int lane = threadIdx.x & 31;
  const uint4* v = reinterpret_cast<const uint4*>(s.base);
  constexpr int U = 8;
  Sum sum;
  float m = 0.0f;     // the largest magnitude (the maximum norm alone)
  uint32_t any = 0;   // the elements' bits
  auto take = [&](uint4 u) {
    any |= u.x | u.y | u.z | u.w;
    if (NORM == PEAT_NORM_INF) m = max_nan(m, unit_max<DT>(u));
    else sum.add(unit_sum<DT, NORM>(u));
  };
  int64_t j = j0;
  if (j < j1 && !s.full(j)) {  // the tensor's first unit
    if (lane == 0) take(edge_unit<DT>(s, j));
    j++;
  }
  int64_t je = j1;
  if (j < je && !s.full(je - 1)) {  // and its last
    if (lane == 1) take(edge_unit<DT>(s, je - 1));
    je--;
  }
  auto batch = [&](const uint4 (&u)[U]) {
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int i = 0; i < U; i += 2) {
      any |= u[i].x | u[i].y | u[i].z | u[i].w;
      any |= u[i + 1].x | u[i + 1].y | u[i + 1].z | u[i + 1].w;
      if (NORM == PEAT_NORM_INF) m = max_nan(m, max_nan(unit_max<DT>(u[i]), unit_max<DT>(u[i + 1])));
      else a += unit_sum<DT, NORM>(u[i]), b += unit_sum<DT, NORM>(u[i + 1]);
    }
    if (NORM != PEAT_NORM_INF) sum.add(a + b);
  };
  uint4 u[U];
  for (; j + 32 * U <= je; j += 32 * U) {
#pragma unroll
    for (int i = 0; i < U; i++) u[i] = __ldcg(v + j + 32 * i + lane);
    batch(u);
  }
  if (j < je) {  // the rest, its loads under way at once too; zeros past the end change nothing
#pragma unroll
    for (int i = 0; i < U; i++) {
      u[i] = make_uint4(0, 0, 0, 0);
      if (j + 32 * i + lane < je) u[i] = __ldcg(v + j + 32 * i + lane);
    }
    batch(u);
  }
  GnPartial r;
  r.bad = 0;
  any = __reduce_or_sync(0xffffffffu, any);
  if (NORM == PEAT_NORM_INF) {
    r.s = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m) & 0x7fffffffu));
    if (__double2float_rn(r.s) < __uint_as_float(0x7f800000u)) return r;  // (not for a NaN)
  } else {
    const double total = warp_sum((double)sum.hi + (double)sum.lo);
    r.s = total;
    // No element was infinite or NaN, and no square too large, if the total is
    // finite.  A square below 2^-126 may be off by 2^-150: with a total of
    // 2^-70 the fewer than 2^40 of them are off by less than 2^-40 of it.
    const float t = __double2float_rn(total);
    const bool zeros = (any & (DT == PEAT_F32 ? 0x7fffffffu : 0x7fff7fffu)) == 0;
    if (t < 0x1p120f && (NORM == PEAT_NORM_1 || t >= 0x1p-70f || zeros)) return r;
  }
  // again: scaled so that the largest finite magnitude is near 1, and counted
  constexpr int E = DT == PEAT_F32 ? 4 : 8;
  uint32_t bad = 0, nan = 0, most = 0;
  for (j = j0 + lane; j < j1; j += 32) {
    float x[E];
    unpack<DT>(edge_unit<DT>(s, j), x);
#pragma unroll
    for (int e = 0; e < E; e++) {
      const uint32_t b = __float_as_uint(x[e]) & 0x7fffffffu;
      bad += b >= 0x7f800000u;
      nan |= b > 0x7f800000u;
      if (b < 0x7f800000u) most = max(most, b);
    }
  }
  most = __reduce_max_sync(0xffffffffu, most);
  r.bad = __reduce_add_sync(0xffffffffu, bad);
  nan = __reduce_or_sync(0xffffffffu, nan);
  if (r.bad) {
    r.s = nan ? __longlong_as_double(0x7ff8000000000000ll) : __longlong_as_double(0x7ff0000000000000ll);
    return r;
  }
  const int k = ilogbf(__uint_as_float(most));  // (there is a number that is not zero here)
  const float f1 = ldexpf(1.0f, -(k / 2)), f2 = ldexpf(1.0f, -(k - k / 2));
  Sum again;
  for (j = j0 + lane; j < j1; j += 32) {
    float x[E], a = 0.0f;
    unpack<DT>(edge_unit<DT>(s, j), x);
#pragma unroll
    for (int e = 0; e < E; e++) {
      const float y = x[e] * f1 * f2;
      a = NORM == PEAT_NORM_1 ? a + fabsf(y) : fmaf(y, y, a);
    }
    again.add(a);
  }
  r.s = ldexp(warp_sum((double)again.hi + (double)again.lo), NORM == PEAT_NORM_1 ? k : 2 * k);
  return r;
}

template <int NORM>
__device__ GnPartial piece_of(const GnEntry& e, int64_t j0, int64_t j1) {
  const Span s(e);
  if (e.dtype == PEAT_F32) return piece<PEAT_F32, NORM>(s, j0, j1);
  if (e.dtype == PEAT_F16) return piece<PEAT_F16, NORM>(s, j0, j1);
  return piece<PEAT_BF16, NORM>(s, j0, j1);
}

// the last tensor whose units start at or before u (one with units, for u
// below the total), by a warp: 32 tensors are looked at together
__device__ __forceinline__ int find_tensor(const GnEntry* list, int count, int64_t u) {
  int lo = 0, n = count;  // it is one of [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32, at = lo + step * (threadIdx.x & 31);
    const uint32_t before = __ballot_sync(0xffffffffu, at < lo + n && list[min(at, count - 1)].unit0 <= u);
    const int k = 31 - __clz(before);  // (lane 0's is)
    n = min(step, lo + n - (lo + k * step));
    lo += k * step;
  }
  return lo;
}
// warp w of n owns units [first(w), first(w + 1)); owner(u) has unit u
__device__ __forceinline__ int64_t first_unit(int64_t w, int64_t n, int64_t units) { return units * w / n; }
__device__ __forceinline__ int64_t owner(int64_t u, int64_t n, int64_t units) { return ((u + 1) * n - 1) / units; }

// the norm of a sum, times unscale: the 2-norm's sum, its root and the result are
// each rounded to float32, of the others the result
template <int NORM>
__device__ __forceinline__ float to_norm(double s, float unscale) {
  if (NORM == PEAT_NORM_2) {
    // the root in float32 of s = f 4^k, 1 <= f < 4 (a binary64 root is slow here)
    const long long b = __double_as_longlong(s);
    const int e = (int)(b >> 52 & 0x7ff) - 1023, k = e >> 1;  // (no subnormal s: squares of float32 values)
    if (!(s > 0.0) || e == 1024) return (float)(s * (double)unscale);
    const float f = (float)__longlong_as_double((b & 0x000fffffffffffffll) | (long long)(1023 + (e & 1)) << 52);
    return (float)((double)__fsqrt_rn(f) * (double)unscale * __longlong_as_double((long long)(1023 + k) << 52));
  }
  return (float)(s * (double)unscale);
}

// totals of one tensor or of several
struct Total {
  double s = 0.0;
  unsigned long long bad = 0;
  template <int NORM>
  __device__ __forceinline__ void add(double v, unsigned long long b) {
    s = NORM == PEAT_NORM_INF ? (v > s || isnan(v) ? v : s) : s + v;  // (a NaN stays: nothing is above it)
    bad += b;
  }
  template <int NORM>
  __device__ __forceinline__ void warp() {
#pragma unroll
    for (int o = 16; o; o /= 2) {
      const double v = __shfl_xor_sync(0xffffffffu, s, o);
      const unsigned long long b = __shfl_xor_sync(0xffffffffu, bad, o);
      add<NORM>(v, b);
    }
  }
};

// the record from the tensors' sums, by a CTA
template <int NORM, typename F>
__device__ void finish(const GnParams& p, F tensor) {
  __shared__ Total part[GB / 32];
  Total all;
  for (int t = threadIdx.x; t < p.count; t += GB) {
    const GnPartial r = tensor(t);
    if (p.norms) p.norms[t] = to_norm<NORM>(r.s, p.unscale);
    all.add<NORM>(r.s, r.bad);
  }
  all.warp<NORM>();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = all;
  __syncthreads();
  if (threadIdx.x < 32) {
    all = Total();
    if (threadIdx.x < GB / 32) all = part[threadIdx.x];
    all.warp<NORM>();
    peat_gradnorm_t r;
    r.norm = to_norm<NORM>(all.s, p.unscale);
    r.n_bad = all.bad;
    float c = 1.0f;
    if (p.clip) {
      const float q = __fdiv_rn(p.max_norm, __fadd_rn(r.norm, p.eps));
      c = q >= 1.0f ? 1.0f : q;  // (a NaN stays one)
      if (r.n_bad && p.bad_mode == PEAT_BAD_ZERO) c = 0.0f;
      if (r.n_bad && p.bad_mode == PEAT_BAD_KEEP) c = 1.0f;
    }
    r.coef = c;
    if (threadIdx.x == 0) *p.result = r;
  }
}

// The pieces of a tensor whose units the warps w0..w1 have: one for each warp
// of the first and the last CTA, one for each CTA between them, whose whole
// share is the tensor's.  (A list of one tensor of 25.6 million float32 elements
// takes 31 us; with a piece for every warp, 6080 of them, it took 46.)
constexpr int GW = GB / 32;  // warps of a CTA
struct Pieces {
  int w0, w1, head, between;  // warps; those of the first CTA, and the CTAs between
  __device__ __forceinline__ Pieces(const GnParams& p, int64_t data, int64_t next) {
    w0 = (int)owner(data, p.nwarps, p.units);
    w1 = (int)owner(next - 1, p.nwarps, p.units);
    head = min((w0 / GW + 1) * GW, w1 + 1) - w0;
    between = max(w1 / GW - w0 / GW - 1, 0);
  }
  __device__ __forceinline__ int count() const { return w1 - w0 + 1 - between * (GW - 1); }
  // whose slot piece i has
  __device__ __forceinline__ int warp(int i) const { return w0 + i + (GW - 1) * min(max(i - head, 0), between); }
  // whether a CTA is one of those between
  __device__ __forceinline__ bool whole(int c) const { return c > w0 / GW && c < w1 / GW; }
};
// a tensor's pieces together, in a fixed order, by a warp; parts: warp 0's slot
template <int NORM>
__device__ __forceinline__ GnPartial gather(const GnPartial* parts, const Pieces& of) {
  Total all;
  const int n = (int)of.count();
#pragma unroll 4
  for (int i = threadIdx.x & 31; i < n; i += 32) {
    const GnPartial* r = parts + of.warp(i);
    all.add<NORM>(__ldcg(&r->s), __ldcg(&r->bad));
  }
  all.warp<NORM>();
  GnPartial r;
  r.s = all.s;
  r.bad = all.bad;
  return r;
}
// lane 0's piece into warp w's slot; the warp that comes last adds them all up
template <int NORM>
__device__ __forceinline__ void hand_in(const GnParams& p, int t, int w, const Pieces& of, const GnPartial& r) {
  const int lane = threadIdx.x & 31;
  unsigned int n = 0;
  if (lane == 0) {
    p.parts[t + w] = r;
    __threadfence();
    n = atomicAdd(p.tickets + t, 1u);
  }
  if (__shfl_sync(0xffffffffu, n, 0) != (unsigned)(of.count() - 1)) return;
  __threadfence();
  const GnPartial all = gather<NORM>(p.parts + t, of);
  if (lane == 0) {
    p.sums[t] = all;
    p.tickets[t] = 0;
  }
}

// Warp w's pieces.  A tensor that lies in one warp's share is done with that;
// one of several pieces is added up by the warp that comes last to it.
template <int NORM>
__device__ __forceinline__ void pieces_of(const GnParams& p, const GnEntry* list, int64_t w) {
  if (w >= p.nwarps || p.units == 0) return;
  const int lane = threadIdx.x & 31;
  int64_t u = first_unit(w, p.nwarps, p.units);
  const int64_t begin = u, end = first_unit(w + 1, p.nwarps, p.units);
  if (u >= end) return;
  for (int t = find_tensor(list, p.count, u); u < end; t++) {
    const GnEntry e = list[t];
    const int64_t next = t + 1 < p.count ? list[t + 1].unit0 : p.units, stop = min(end, next);
    const int64_t data = e.unit0 + p.lead, from = max(u, data);
    u = max(u, stop);
    if (stop <= from) continue;
    const GnPartial r = piece_of<NORM>(e, from - data, stop - data);
    if (data >= begin && next <= end) {
      if (lane == 0) p.sums[t] = r;
      continue;
    }
    const Pieces of(p, data, next);
    if (of.whole(blockIdx.x)) {  // the whole CTA is here, with nothing but this tensor
      __shared__ GnPartial part[GW];
      if (lane == 0) part[threadIdx.x >> 5] = r;
      __syncthreads();
      if (threadIdx.x >= 32) return;
      Total all;
      if (lane < GW) {
        all.s = part[lane].s;
        all.bad = part[lane].bad;
      }
      all.warp<NORM>();
      GnPartial whole;
      whole.s = all.s;
      whole.bad = all.bad;
      hand_in<NORM>(p, t, blockIdx.x * GW, of, whole);
      return;
    }
    hand_in<NORM>(p, t, (int)w, of, r);
  }
}
__device__ __forceinline__ GnPartial load_sum(const GnPartial* q) {
  GnPartial r;
  r.s = __ldcg(&q->s);
  r.bad = __ldcg(&q->bad);
  return r;
}

template <int NORM, typename IN>
__global__ void __launch_bounds__(GB, 5) gn_norm(GnParams p, const __grid_constant__ IN in) {
  pdl_wait();
  pdl_trigger();
  const GnEntry* list = p.list ? p.list : in.e;
  pieces_of<NORM>(p, list, (int64_t)blockIdx.x * (GB / 32) + (threadIdx.x >> 5));
  __shared__ bool last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(p.done, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  finish<NORM>(p, [&](int t) {
    const int64_t next = t + 1 < p.count ? list[t + 1].unit0 : p.units;
    return next > list[t].unit0 + p.lead ? load_sum(p.sums + t) : GnPartial{0.0, 0ull};  // (an empty tensor has no sum)
  });
  if (threadIdx.x == 0) *p.done = 0;
}

template <int DT>
__device__ __forceinline__ uint4 scaled(uint4 u, float f, bool zero) {
  if (zero) return make_uint4(0, 0, 0, 0);
  float x[DT == PEAT_F32 ? 4 : 8];
  unpack<DT>(u, x);
#pragma unroll
  for (int e = 0; e < (DT == PEAT_F32 ? 4 : 8); e++) x[e] = __fmul_rn(x[e], f);
  return pack<DT>(x);
}
// unit j element by element: the tensor's ends, and outputs off the input's grid
template <int DT>
__device__ __forceinline__ void put_elements(const Span& s, char* out, int64_t j, uint4 u) {
  constexpr int B = DT == PEAT_F32 ? 4 : 2;
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 16 / B; i++) {
    const int64_t at = 16 * j + i * B;
    if (at < s.lo || at >= s.hi) continue;
    if (B == 4) *reinterpret_cast<uint32_t*>(out + at) = w[i % 4];
    else *reinterpret_cast<uint16_t*>(out + at) = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
  }
}
template <int DT>
__device__ void scale_piece(const GnEntry& e, int64_t j0, int64_t j1, float f, bool zero) {
  const Span s(e);
  const int lane = threadIdx.x & 31;
  char* out = static_cast<char*>(e.out) - s.lo;  // unit j's place
  const uint4* v = reinterpret_cast<const uint4*>(s.base);
  const bool same = ((reinterpret_cast<uintptr_t>(e.g) ^ reinterpret_cast<uintptr_t>(e.out)) & 15) == 0;
  constexpr int U = 4;
  int64_t j = j0, je = j1;
  if (same) {
    if (j < je && !s.full(j)) {
      if (lane == 0) put_elements<DT>(s, out, j, scaled<DT>(edge_unit<DT>(s, j), f, zero));
      j++;
    }
    if (j < je && !s.full(je - 1)) {
      if (lane == 1) put_elements<DT>(s, out, je - 1, scaled<DT>(edge_unit<DT>(s, je - 1), f, zero));
      je--;
    }
    // last units first: they are what the norm pass read last, and the first to be found in L2
    uint4* o = reinterpret_cast<uint4*>(out);
    for (int64_t k = je - 1 - lane; k + lane >= j; k -= 32 * U) {
      uint4 u[U];
#pragma unroll
      for (int i = 0; i < U; i++) u[i] = k - 32 * i >= j ? __ldcs(v + k - 32 * i) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < U; i++)
        if (k - 32 * i >= j) __stcs(o + k - 32 * i, scaled<DT>(u[i], f, zero));
    }
  } else {
    for (j += lane; j < je; j += 32) put_elements<DT>(s, out, j, scaled<DT>(edge_unit<DT>(s, j), f, zero));
  }
}

// warp w's share of n of the list, scaled by f (or set to zero)
__device__ __forceinline__ void scale_share(const GnParams& p, const GnEntry* list, int64_t w, int64_t n, float f,
                                            bool zero) {
  const int64_t u = first_unit(w, n, p.units);
  int64_t end = first_unit(w + 1, n, p.units);
  if (u >= end) return;
  for (int t = find_tensor(list, p.count, end - 1); end > u; t--) {
    const GnEntry e = list[t];
    const int64_t data = e.unit0 + p.lead, start = max(u, data);
    if (start < end && !(f == 1.0f && !zero && e.out == e.g)) {
      if (e.dtype == PEAT_F32) scale_piece<PEAT_F32>(e, start - data, end - data, f, zero);
      else if (e.dtype == PEAT_F16) scale_piece<PEAT_F16>(e, start - data, end - data, f, zero);
      else scale_piece<PEAT_BF16>(e, start - data, end - data, f, zero);
    }
    end = min(end, max(u, e.unit0));
  }
}
template <typename IN>
__global__ void __launch_bounds__(GB) gn_scale(GnParams p, const __grid_constant__ IN in) {
  pdl_wait();
  pdl_trigger();
  const GnEntry* list = p.list ? p.list : in.e;
  const int64_t n = (int64_t)gridDim.x * (GB / 32);
  const float f = __fmul_rn(p.unscale, __ldcg(&p.result->coef));
  const bool zero = p.bad_mode == PEAT_BAD_ZERO && __ldcg(&p.result->n_bad) != 0;
  scale_share(p, list, (int64_t)blockIdx.x * (GB / 32) + (threadIdx.x >> 5), n, f, zero);
}

}  // namespace

int gn_block() { return GB; }

template <typename IN>
static cudaError_t norm_and_scale(const GnParams& p, const IN& in, int nctas, cudaStream_t s) {
  auto kernel = p.type == PEAT_NORM_1
                    ? gn_norm<PEAT_NORM_1, IN>
                    : (p.type == PEAT_NORM_INF ? gn_norm<PEAT_NORM_INF, IN> : gn_norm<PEAT_NORM_2, IN>);
  cudaError_t e = launch_dependent(kernel, (unsigned)nctas, GB, 0, s, p, in);
  if (e == cudaSuccess && p.clip && p.units > 0) e = launch_dependent(gn_scale<IN>, (unsigned)nctas, GB, 0, s, p, in);
  return e;
}
cudaError_t launch_gradnorm(const GnParams& p, const GnEntry* host, int nctas, cudaStream_t s) {
  if (p.list) return norm_and_scale(p, GnInlineOf<1>{}, nctas, s);
  if (p.count <= GN_INLINE_FEW) {
    GnInlineOf<GN_INLINE_FEW> in;
    std::copy(host, host + p.count, in.e);
    return norm_and_scale(p, in, nctas, s);
  }
  GnInlineOf<GN_INLINE> in;
  std::copy(host, host + p.count, in.e);
  return norm_and_scale(p, in, nctas, s);
}
}  // namespace peat
