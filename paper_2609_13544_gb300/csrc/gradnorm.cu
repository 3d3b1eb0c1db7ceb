// The norm over a list of gradient tensors, and their clipping.
//
// The list is taken as one run of 16-byte units (each tensor's own, from the
// boundary at or before its first element), shared out evenly to the warps of
// one wave; a warp's part of a tensor is a piece with one partial sum.  The CTA
// that finishes last adds the pieces up, tensor by tensor, in a fixed order.
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
// writes it, in the opposite order, so that what the norm read last is still
// in L2.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ops_internal.h"

namespace peat {
namespace {

constexpr int GB = 256;

__device__ __forceinline__ int elem_size(int dt) { return dt == PEAT_F32 ? 4 : 2; }

template <int DT>
__device__ __forceinline__ void unpack(uint4 u, float (&x)[DT == PEAT_F32 ? 4 : 8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if (DT == PEAT_F32) {
      x[i] = __uint_as_float(w[i]);
    } else if (DT == PEAT_BF16) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}
template <int DT>
__device__ __forceinline__ uint4 pack(const float (&x)[DT == PEAT_F32 ? 4 : 8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if (DT == PEAT_F32) {
      w[i] = __float_as_uint(x[i]);
    } else if (DT == PEAT_BF16) {
      __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<uint32_t*>(&b);
    } else {
      __half2 b = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<uint32_t*>(&b);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

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
template <int DT>
__device__ __forceinline__ uint32_t unit_max(uint32_t m, uint4 u) {  // patterns without sign: one word, or two half-words
  if (DT == PEAT_F32) {
    return max(max(m, u.x & 0x7fffffffu), max(max(u.y & 0x7fffffffu, u.z & 0x7fffffffu), u.w & 0x7fffffffu));
  } else {
    const uint32_t a = __vmaxu2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), b = __vmaxu2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu);
    return __vmaxu2(m, __vmaxu2(a, b));
  }
}
// the largest pattern as float32 bits (infinities and NaNs at or above 0x7f800000)
template <int DT>
__device__ __forceinline__ uint32_t max_bits(uint32_t m) {
  if (DT == PEAT_F32) return m;
  m = max(m & 0xffffu, m >> 16);
  if (DT == PEAT_BF16) return m << 16;
  return __float_as_uint(__half2float(__ushort_as_half((unsigned short)m)));
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
  uint32_t m = 0;
  int64_t j = j0;
  if (j < j1 && !s.full(j)) {  // the tensor's first unit
    if (lane == 0) {
      const uint4 u = edge_unit<DT>(s, j);
      if (NORM != PEAT_NORM_INF) sum.add(unit_sum<DT, NORM>(u));
      m = unit_max<DT>(m, u);
    }
    j++;
  }
  int64_t je = j1;
  if (j < je && !s.full(je - 1)) {  // and its last
    if (lane == 1) {
      const uint4 u = edge_unit<DT>(s, je - 1);
      if (NORM != PEAT_NORM_INF) sum.add(unit_sum<DT, NORM>(u));
      m = unit_max<DT>(m, u);
    }
    je--;
  }
  for (; j + 32 * U <= je; j += 32 * U) {
    uint4 u[U];
#pragma unroll
    for (int i = 0; i < U; i++) u[i] = __ldcg(v + j + 32 * i + lane);
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int i = 0; i < U; i += 2) {
      if (NORM != PEAT_NORM_INF) a += unit_sum<DT, NORM>(u[i]), b += unit_sum<DT, NORM>(u[i + 1]);
      m = unit_max<DT>(unit_max<DT>(m, u[i]), u[i + 1]);
    }
    if (NORM != PEAT_NORM_INF) sum.add(a + b);
  }
  for (j += lane; j < je; j += 32) {
    const uint4 u = __ldcg(v + j);
    if (NORM != PEAT_NORM_INF) sum.add(unit_sum<DT, NORM>(u));
    m = unit_max<DT>(m, u);
  }
  const uint32_t top = __reduce_max_sync(0xffffffffu, max_bits<DT>(m));
  GnPartial r;
  r.bad = r.nan = 0;
  const float big = __uint_as_float(top);
  // squares of numbers between 2^-40 and 2^50 and their sums stay well inside
  // float32's range; below, a number 2^23 times smaller than the largest may
  // lose its square, which is then below 2^-46 of the sum
  const bool fine = top < 0x7f800000u && (NORM == PEAT_NORM_INF || (NORM == PEAT_NORM_1 ? big < 0x1p100f : (big < 0x1p50f && (big >= 0x1p-40f || top == 0))));
  if (fine) {
    r.s = NORM == PEAT_NORM_INF ? (double)big : warp_sum((double)sum.hi + (double)sum.lo);
    return r;
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
      nan += b > 0x7f800000u;
      if (b < 0x7f800000u) most = max(most, b);
    }
  }
  most = __reduce_max_sync(0xffffffffu, most);
  r.bad = __reduce_add_sync(0xffffffffu, bad);
  r.nan = __reduce_add_sync(0xffffffffu, nan);
  if (r.bad) {
    r.s = r.nan ? __longlong_as_double(0x7ff8000000000000ll) : __longlong_as_double(0x7ff0000000000000ll);
    return r;
  }
  const int k = ilogbf(__uint_as_float(most));  // (not zero here)
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

// the last tensor whose units start at or before u (one with units, for u below the total)
__device__ __forceinline__ int find_tensor(const GnEntry* list, int count, int64_t u) {
  int lo = 0, hi = count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (list[mid].unit0 <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
// warp w of n owns units [first(w), first(w + 1)); owner(u) has unit u
__device__ __forceinline__ int64_t first_unit(int64_t w, int64_t n, int64_t units) { return units * w / n; }
__device__ __forceinline__ int64_t owner(int64_t u, int64_t n, int64_t units) { return ((u + 1) * n - 1) / units; }

// the norm of a sum, times unscale, once rounded
template <int NORM>
__device__ __forceinline__ float to_norm(double s, float unscale) {
  return (float)((NORM == PEAT_NORM_2 ? sqrt(s) : s) * (double)unscale);
}

// the pieces of every tensor, in order, by the CTA that finished last
template <int NORM>
__device__ void finish(const GnParams& p, const GnEntry* list) {
  __shared__ double wsum[GB / 32];
  __shared__ unsigned long long wbad[GB / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  double all = 0.0;
  unsigned long long bad = 0;
  for (int t = warp; t < p.count; t += GB / 32) {
    const int64_t u0 = list[t].unit0, u1 = t + 1 < p.count ? list[t + 1].unit0 : p.units;
    double s = 0.0;
    unsigned long long nb = 0;
    if (u1 > u0) {
      const int64_t w0 = owner(u0, p.nwarps, p.units), w1 = owner(u1 - 1, p.nwarps, p.units);
      for (int64_t w = w0 + lane; w <= w1; w += 32) {
        const double v = __ldcg(&p.parts[t + w].s);
        s = NORM == PEAT_NORM_INF ? (v > s || isnan(v) ? v : s) : s + v;  // (a NaN stays: nothing is above it)
        nb += __ldcg(&p.parts[t + w].bad);
      }
    }
    if (NORM == PEAT_NORM_INF) {
#pragma unroll
      for (int o = 16; o; o /= 2) {
        const double v = __shfl_xor_sync(0xffffffffu, s, o);
        s = v > s || isnan(v) ? v : s;
      }
    } else {
      s = warp_sum(s);
    }
#pragma unroll
    for (int o = 16; o; o /= 2) nb += __shfl_xor_sync(0xffffffffu, nb, o);
    bad += nb;
    all = NORM == PEAT_NORM_INF ? (s > all || isnan(s) ? s : all) : all + s;
    if (lane == 0 && p.norms) p.norms[t] = to_norm<NORM>(s, p.unscale);
  }
  if (lane == 0) wsum[warp] = all, wbad[warp] = bad;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < GB / 32; w++) {
      const double s = wsum[w];
      all = NORM == PEAT_NORM_INF ? (s > all || isnan(s) ? s : all) : all + s;
      bad += wbad[w];
    }
    peat_gradnorm_t r;
    r.norm = to_norm<NORM>(all, p.unscale);
    r.n_bad = bad;
    float c = 1.0f;
    if (p.clip) {
      const float q = __fdiv_rn(p.max_norm, __fadd_rn(r.norm, p.eps));
      c = q >= 1.0f ? 1.0f : q;  // (a NaN stays one)
      if (bad && p.bad_mode == PEAT_BAD_ZERO) c = 0.0f;
      if (bad && p.bad_mode == PEAT_BAD_KEEP) c = 1.0f;
    }
    r.coef = c;
    *p.result = r;
    *p.done = 0;
  }
}

template <int NORM>
__global__ void __launch_bounds__(GB) gn_norm(GnParams p, const __grid_constant__ GnInline in) {
  const GnEntry* list = p.list ? p.list : in.e;
  const int64_t w = (int64_t)blockIdx.x * (GB / 32) + (threadIdx.x >> 5);
  if (w < p.nwarps && p.units > 0) {
    int64_t u = first_unit(w, p.nwarps, p.units);
    const int64_t end = first_unit(w + 1, p.nwarps, p.units);
    for (int t = find_tensor(list, p.count, u); u < end; t++) {
      const GnEntry e = list[t];
      const int64_t stop = min(end, t + 1 < p.count ? list[t + 1].unit0 : p.units);
      if (stop > u) {
        const GnPartial r = piece_of<NORM>(e, u - e.unit0, stop - e.unit0);
        if ((threadIdx.x & 31) == 0) p.parts[t + w] = r;
        u = stop;
      }
    }
  }
  __shared__ bool last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(p.done, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  finish<NORM>(p, list);
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
    uint4* o = reinterpret_cast<uint4*>(out);
    for (; j + 32 * U <= je; j += 32 * U) {
      uint4 u[U];
#pragma unroll
      for (int i = 0; i < U; i++) u[i] = __ldcg(v + j + 32 * i + lane);
#pragma unroll
      for (int i = 0; i < U; i++) __stcs(o + j + 32 * i + lane, scaled<DT>(u[i], f, zero));
    }
    for (j += lane; j < je; j += 32) __stcs(o + j, scaled<DT>(__ldcg(v + j), f, zero));
  } else {
    for (j += lane; j < je; j += 32) put_elements<DT>(s, out, j, scaled<DT>(edge_unit<DT>(s, j), f, zero));
  }
}

__global__ void __launch_bounds__(GB) gn_scale(GnParams p, const __grid_constant__ GnInline in) {
  const GnEntry* list = p.list ? p.list : in.e;
  const int64_t n = (int64_t)gridDim.x * (GB / 32);
  const int64_t w = n - 1 - ((int64_t)blockIdx.x * (GB / 32) + (threadIdx.x >> 5));
  const float f = __fmul_rn(p.unscale, __ldcg(&p.result->coef));
  const bool zero = p.bad_mode == PEAT_BAD_ZERO && __ldcg(&p.result->n_bad) != 0;
  int64_t u = first_unit(w, n, p.units);
  const int64_t end = first_unit(w + 1, n, p.units);
  if (u >= end) return;
  for (int t = find_tensor(list, p.count, u); u < end; t++) {
    const GnEntry e = list[t];
    const int64_t stop = min(end, t + 1 < p.count ? list[t + 1].unit0 : p.units);
    if (stop <= u) continue;
    if (!(f == 1.0f && !zero && e.out == e.g)) {
      if (e.dtype == PEAT_F32) scale_piece<PEAT_F32>(e, u - e.unit0, stop - e.unit0, f, zero);
      else if (e.dtype == PEAT_F16) scale_piece<PEAT_F16>(e, u - e.unit0, stop - e.unit0, f, zero);
      else scale_piece<PEAT_BF16>(e, u - e.unit0, stop - e.unit0, f, zero);
    }
    u = stop;
  }
}

}  // namespace

int gn_block() { return GB; }

cudaError_t launch_gradnorm(const GnParams& p, const GnInline& in, int nctas, cudaStream_t s) {
  if (p.type == PEAT_NORM_1) gn_norm<PEAT_NORM_1><<<nctas, GB, 0, s>>>(p, in);
  else if (p.type == PEAT_NORM_INF) gn_norm<PEAT_NORM_INF><<<nctas, GB, 0, s>>>(p, in);
  else gn_norm<PEAT_NORM_2><<<nctas, GB, 0, s>>>(p, in);
  return cudaGetLastError();
}
cudaError_t launch_gradscale(const GnParams& p, const GnInline& in, int nctas, cudaStream_t s) {
  gn_scale<<<nctas, GB, 0, s>>>(p, in);
  return cudaGetLastError();
}

}  // namespace peat
