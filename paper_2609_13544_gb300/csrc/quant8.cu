// Rounding of a matrix to 8-bit integers with one scale for each row or column.
//
// Over a row (or column): amax = max |x|, scale = amax / 127, r = 127 / amax,
// q = rint(x r), all float32.  The maximum is one that keeps NaNs, so it finds
// both amax and whether the row is finite; it is handed on as a bit pattern
// without sign, which order as the magnitudes do, infinities and NaNs on top.
//
// Bound by memory: a row is read once and kept in registers between the
// maximum and the rounding; columns are read twice, as far as they fit from L2
// the second time.
#include <algorithm>

#include "ops_internal.h"
#include "peat_internal.h"
#include "vec16.cuh"

namespace peat {
namespace {

template <int DT>
struct Elem;
template <>
struct Elem<PEAT_F32> {
  using T = float;
  static constexpr int E = 4;  // elements of a 16-byte vector
  static constexpr uint32_t INF = 0x7f800000u;
  static __device__ __forceinline__ uint32_t bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
  static __device__ __forceinline__ float mag(uint32_t b) { return __uint_as_float(b); }
  static __device__ __forceinline__ float up(float v) { return v; }
  static __device__ __forceinline__ float down(float v) { return v; }
};
template <>
struct Elem<PEAT_F16> {
  using T = __half;
  static constexpr int E = 8;
  static constexpr uint32_t INF = 0x7c00u;
  static __device__ __forceinline__ uint32_t bits(__half v) { return __half_as_ushort(v) & 0x7fffu; }
  static __device__ __forceinline__ float mag(uint32_t b) { return __half2float(__ushort_as_half((unsigned short)b)); }
  static __device__ __forceinline__ float up(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half down(float v) { return __float2half_rn(v); }
};
template <>
struct Elem<PEAT_BF16> {
  using T = __nv_bfloat16;
  static constexpr int E = 8;
  static constexpr uint32_t INF = 0x7f80u;
  static __device__ __forceinline__ uint32_t bits(__nv_bfloat16 v) { return __bfloat16_as_ushort(v) & 0x7fffu; }
  static __device__ __forceinline__ float mag(uint32_t b) { return __uint_as_float(b << 16); }
  static __device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 down(float v) { return __float2bfloat16_rn(v); }
};

// a 16-byte vector as its elements
template <int DT>
union Vec {
  uint4 u;
  typename Elem<DT>::T e[Elem<DT>::E];
  __device__ Vec() {}
};

// elementwise maximum of the magnitudes; a NaN on either side stays (as a NaN
// pattern, above every number's).  The types' own maxima: the packed integer
// ones are several instructions each on this GPU.
__device__ __forceinline__ uint32_t max_f32(uint32_t m, uint32_t v) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(m)), "f"(fabsf(__uint_as_float(v))));
  return __float_as_uint(r) & 0x7fffffffu;
}
__device__ __forceinline__ uint32_t max_f16x2(uint32_t m, uint32_t v) {
  uint32_t r;
  asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(m), "r"(v & 0x7fff7fffu));
  return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t m, uint32_t v) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(m), "r"(v & 0x7fff7fffu));
  return r;
}
template <int DT>
__device__ __forceinline__ uint32_t max_word(uint32_t m, uint32_t v) {
  return DT == PEAT_F32 ? max_f32(m, v) : (DT == PEAT_F16 ? max_f16x2(m, v) : max_bf16x2(m, v));
}
template <int DT>
__device__ __forceinline__ uint4 mag_max(uint4 m, uint4 v) {
  return make_uint4(max_word<DT>(m.x, v.x), max_word<DT>(m.y, v.y), max_word<DT>(m.z, v.z), max_word<DT>(m.w, v.w));
}
template <int DT>
__device__ __forceinline__ uint32_t mag_fold(uint4 m) {  // the largest of the vector
  const uint32_t a = max_word<DT>(max_word<DT>(m.x, m.y), max_word<DT>(m.z, m.w));
  return DT == PEAT_F32 ? a : max(a & 0xffffu, a >> 16);
}

// r and scale of a row from its largest pattern
template <int DT>
__device__ __forceinline__ void factors(uint32_t m, float& r, float& scale) {
  if (m >= Elem<DT>::INF) {
    r = 0.0f;
    scale = __uint_as_float(0x7fc00000u);
    return;
  }
  const float amax = Elem<DT>::mag(m);
  r = __fdiv_rn(127.0f, amax);
  scale = __fdiv_rn(amax, 127.0f);
  if (!(r <= 3.402823466e38f)) r = scale = 0.0f;  // amax 0, or too small for a finite r
}
// The integer of x: the float32 product x r, added to 1.5 2^23, has it in its
// low bits, rounded to nearest even (conversion instructions run at an eighth of
// the additions' rate).  A row that is not finite has r = 0, and 0 x NaN must
// not get through.
constexpr float MAGIC = 12582912.0f;
__device__ __forceinline__ float whole(float x, float r, bool finite) {
  return finite ? __fadd_rn(__fmul_rn(x, r), MAGIC) : MAGIC;
}
__device__ __forceinline__ float number(float w) { return __fsub_rn(w, MAGIC); }
__device__ __forceinline__ int8_t byte_of(float w) { return (int8_t)__float_as_uint(w); }
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040),
                     __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
}

// the first `left` elements of a vector at p (left < E: one by one, zero beyond)
template <int DT, bool VEC>
__device__ __forceinline__ uint4 load_vec(const typename Elem<DT>::T* p, int64_t left) {
  if (VEC && left >= Elem<DT>::E) return __ldg(reinterpret_cast<const uint4*>(p));
  Vec<DT> v;
  v.u = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < Elem<DT>::E; e++)
    if (e < left) v.e[e] = p[e];
  return v.u;
}

// a vector's integers (in float32, see whole) from its row's or its columns' factors
template <int DT, bool FINITE>
__device__ __forceinline__ void wholes(uint4 v, float r, float (&w)[Elem<DT>::E]) {
  float x[Elem<DT>::E];
  unpack<DT>(v, x);
#pragma unroll
  for (int e = 0; e < Elem<DT>::E; e++) w[e] = whole(x[e], r, FINITE);
}
// a vector's values at o, of which `left` exist
template <int DT>
__device__ __forceinline__ void store_values(typename Elem<DT>::T* o, const float (&y)[Elem<DT>::E], bool vec, int64_t left) {
  Vec<DT> v;
  v.u = pack<DT>(y);
  if (vec && left >= Elem<DT>::E) {
    __stcs(reinterpret_cast<uint4*>(o), v.u);
  } else {
#pragma unroll
    for (int e = 0; e < Elem<DT>::E; e++)
      if (e < left) o[e] = v.e[e];
  }
}

// integers and values of one vector of a row
template <int DT>
__device__ __forceinline__ void store_row_vec(const QuantParams& p, uint4 v, int64_t row, int64_t col, int64_t left,
                                              float r, float scale, bool finite) {
  using L = Elem<DT>;
  float w[L::E];
  if (finite) wholes<DT, true>(v, r, w);
  else wholes<DT, false>(v, r, w);
  if (p.q) {
    int8_t* q = p.q + row * p.ldq + col;
    if (p.vec_q && left >= L::E) {
      if (L::E == 8)
        *reinterpret_cast<uint2*>(q) = make_uint2(pack4(w[0], w[1], w[2], w[3]), pack4(w[4 % L::E], w[5 % L::E], w[6 % L::E], w[7 % L::E]));
      else
        *reinterpret_cast<uint32_t*>(q) = pack4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < L::E; e++)
        if (e < left) q[e] = byte_of(w[e]);
    }
  }
  if (p.values) {
    float y[L::E];
#pragma unroll
    for (int e = 0; e < L::E; e++) y[e] = __fmul_rn(number(w[e]), scale);
    store_values<DT>(static_cast<typename L::T*>(p.values) + row * p.ldv + col, y, p.vec_v, left);
  }
}

constexpr int QT = 256;  // threads of a CTA

// A kernel that needs nothing of the one before it (QuantParams::overlap) runs
// beside it, and waits for it at its end, so that whoever waits for this one
// has waited for both.
__device__ __forceinline__ void begin(const QuantParams& p) {
  if (!p.overlap) pdl_wait();
  pdl_trigger();
}
__device__ __forceinline__ void end(const QuantParams& p) {
  if (p.overlap) pdl_wait();
}

// the largest pattern over the TPR threads of a row (32: a warp, QT: the CTA)
template <int TPR>
__device__ __forceinline__ uint32_t row_max(uint32_t m) {
  m = __reduce_max_sync(0xffffffffu, m);
  if (TPR == 32) return m;
  __shared__ uint32_t part[QT / 32];
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  __syncthreads();
  uint32_t t = part[threadIdx.x & (QT / 32 - 1)];
  return __reduce_max_sync(0xffffffffu, t);
}

// A row by TPR threads, NV vectors each, held in registers.
template <int DT, int TPR, int NV>
__global__ void __launch_bounds__(QT) quant_rows(QuantParams p) {
  using L = Elem<DT>;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * (QT / TPR) + threadIdx.x / TPR;
  if (row >= p.rows) return;  // (whole warps; with TPR = QT there is a row for every CTA)
  const typename L::T* x = static_cast<const typename L::T*>(p.x) + row * p.ldx;
  uint4 v[NV];
  uint4 m = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < NV; i++) {
    const int64_t col = (int64_t)(i * TPR + lane) * L::E;
    v[i] = make_uint4(0, 0, 0, 0);
    if (col + L::E <= p.cols) v[i] = __ldg(reinterpret_cast<const uint4*>(x + col));
  }
  if (p.cols % L::E) {  // the row's last vector
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int64_t col = (int64_t)(i * TPR + lane) * L::E;
      if (col < p.cols && col + L::E > p.cols) v[i] = load_vec<DT, false>(x + col, p.cols - col);
    }
  }
#pragma unroll
  for (int i = 0; i < NV; i++) m = mag_max<DT>(m, v[i]);
  const uint32_t top = row_max<TPR>(mag_fold<DT>(m));
  float r, scale;
  factors<DT>(top, r, scale);
  const bool finite = top < L::INF;
  if (p.scale && lane == 0) p.scale[row] = scale;
#pragma unroll
  for (int i = 0; i < NV; i++) {
    const int64_t col = (int64_t)(i * TPR + lane) * L::E;
    if (col < p.cols) store_row_vec<DT>(p, v[i], row, col, p.cols - col, r, scale, finite);
  }
}

// where the integers of operand row `row`, k on, lie in a packed operand (see
// mm8_tc.cu): 16 KB blocks of 128 rows by 64 k, 16-byte pieces of 8 k swizzled
__device__ __forceinline__ char* packed_at(const QuantParams& p, int64_t row, int64_t k) {
  const int r = (int)(row & 127);
  return static_cast<char*>(p.packed) + ((row >> 7) * p.kb + (k >> 6)) * 16384 + r * 128 +
         ((((int)k >> 3 & 7) ^ (r & 7)) * 16) + ((int)k & 7) * 2;
}
__device__ __forceinline__ uint32_t half_pair(float a, float b) {
  const __half2 h = __floats2half2_rn(number(a), number(b));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void clear_earlier(const QuantParams& p) {
  const int64_t n = (int64_t)gridDim.x * gridDim.y * QT;
  for (int64_t i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * QT + threadIdx.x; i < p.zero2_n; i += n) p.zero2[i] = 0;
}

// quant_rows with a packed operand for its output, zeros in its margins.  A
// group of threads takes `each` rows one after another, the next one's vectors
// on their way, and hands on the largest sums of squares of all of them.
template <int DT, int TPR, int NV>
__global__ void __launch_bounds__(QT) quant_rows_packed(QuantParams p, int each) {
  using L = Elem<DT>;
  begin(p);
  clear_earlier(p);
  __shared__ uint32_t part[2][QT / 32];
  const int lane = threadIdx.x % TPR;
  const int64_t row0 = ((int64_t)blockIdx.x * (QT / TPR) + threadIdx.x / TPR) * each;
  const bool ragged = p.cols % L::E != 0;
  auto load = [&](int64_t row, uint4 (&v)[NV]) {
    const bool real = row < p.rows;
    const typename L::T* x = static_cast<const typename L::T*>(p.x) + row * p.ldx;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int64_t col = (int64_t)(i * TPR + lane) * L::E;
      v[i] = make_uint4(0, 0, 0, 0);
      if (real && col + L::E <= p.cols) v[i] = __ldg(reinterpret_cast<const uint4*>(x + col));
    }
    if (real && ragged) {  // the row's last vector
#pragma unroll
      for (int i = 0; i < NV; i++) {
        const int64_t col = (int64_t)(i * TPR + lane) * L::E;
        if (col < p.cols && col + L::E > p.cols) v[i] = load_vec<DT, false>(x + col, p.cols - col);
      }
    }
  };
  unsigned most[NV];
#pragma unroll
  for (int i = 0; i < NV; i++) most[i] = 0;
  uint4 next[NV];
  load(row0, next);
  for (int it = 0; it < each; it++) {
    const int64_t row = row0 + it;
    uint4 v[NV];
    uint4 m = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NV; i++) {
      v[i] = next[i];
      m = mag_max<DT>(m, v[i]);
    }
    if (it + 1 < each) load(row + 1, next);
    uint32_t top = __reduce_max_sync(0xffffffffu, mag_fold<DT>(m));
    if (TPR > 32) {
      if ((threadIdx.x & 31) == 0) part[it & 1][threadIdx.x >> 5] = top;
      __syncthreads();
      top = __reduce_max_sync(0xffffffffu, part[it & 1][threadIdx.x & (QT / 32 - 1)]);
    }
    float r, scale;
    factors<DT>(top, r, scale);
    const bool finite = top < L::INF;
    if (lane == 0 && row < p.rows) p.scale[row] = scale;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int64_t k = (int64_t)(i * TPR + lane) * L::E;
      float w[L::E];
      if (finite) wholes<DT, true>(v[i], r, w);
      else wholes<DT, false>(v[i], r, w);
      if (k < (int64_t)p.kb * 64) {
        char* d = packed_at(p, row, k);
        if (L::E == 8)
          *reinterpret_cast<uint4*>(d) = make_uint4(half_pair(w[0], w[1]), half_pair(w[2], w[3]), half_pair(w[4 % L::E], w[5 % L::E]),
                                                    half_pair(w[6 % L::E], w[7 % L::E]));
        else
          *reinterpret_cast<uint2*>(d) = make_uint2(half_pair(w[0], w[1]), half_pair(w[2], w[3]));
      }
      if (p.norms) {  // a warp's vectors are 256 k, or half of them
        float ss = 0.0f;  // (exact: below 2^17)
#pragma unroll
        for (int e = 0; e < L::E; e++) ss = fmaf(number(w[e]), number(w[e]), ss);
        most[i] = max(most[i], __reduce_add_sync(0xffffffffu, (unsigned)ss));
      }
    }
  }
  if (p.norms && (threadIdx.x & 31) == 0) {
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int64_t first = (int64_t)(i * TPR + (lane & ~31)) * L::E;
      if (first < (int64_t)p.kb * 64)
        atomicMax(p.norms + (row0 >> 7) * p.kc * 2 + (L::E == 8 ? first / 256 * 2 : first / 128), most[i]);
    }
  }
  end(p);
}

// A row by a CTA, read twice: rows too long for the registers, and (VEC false) rows off the 16-byte grid,
// which are taken element by element.
template <int DT, bool VEC>
__global__ void __launch_bounds__(QT) quant_rows_twice(QuantParams p) {
  using L = Elem<DT>;
  pdl_wait();
  pdl_trigger();
  const int64_t row = blockIdx.x;
  const typename L::T* x = static_cast<const typename L::T*>(p.x) + row * p.ldx;
  uint32_t top = 0;
  if (VEC) {
    uint4 m = make_uint4(0, 0, 0, 0);
#pragma unroll 4
    for (int64_t col = (int64_t)threadIdx.x * L::E; col < p.cols; col += QT * L::E)
      m = mag_max<DT>(m, load_vec<DT, true>(x + col, p.cols - col));
    top = mag_fold<DT>(m);
  } else {
#pragma unroll 8
    for (int64_t col = threadIdx.x; col < p.cols; col += QT) top = max(top, L::bits(x[col]));
  }
  top = row_max<QT>(top);
  float r, scale;
  factors<DT>(top, r, scale);
  const bool finite = top < L::INF;
  if (p.scale && threadIdx.x == 0) p.scale[row] = scale;
  if (VEC) {
#pragma unroll 2
    for (int64_t col = (int64_t)threadIdx.x * L::E; col < p.cols; col += QT * L::E)
      store_row_vec<DT>(p, load_vec<DT, true>(x + col, p.cols - col), row, col, p.cols - col, r, scale, finite);
  } else {
    int8_t* q = p.q ? p.q + row * p.ldq : nullptr;
    typename L::T* o = p.values ? static_cast<typename L::T*>(p.values) + row * p.ldv : nullptr;
#pragma unroll 4
    for (int64_t col = threadIdx.x; col < p.cols; col += QT) {
      const float w = whole(L::up(x[col]), r, finite);
      if (q) q[col] = byte_of(w);
      if (o) o[col] = L::down(__fmul_rn(number(w), scale));
    }
  }
}

// Columns, in two launches (one for few rows).  The first finds each column's maximum: a thread
// has a 16-byte vector of columns (VEC false: one column) and walks down a
// share of the rows, the shares meet by atomic maxima of the patterns.  The
// second reads the matrix again, last rows first, so that it finds in L2 what
// the first read last, in tiles of 128 rows by 128 bytes, and writes the
// integers transposed through shared memory, 128 contiguous ones of a column
// at a time.  (One launch of clusters that keep a strip of columns to
// themselves, meet in distributed shared memory and read the strip again from
// L2 took 101 us for 16384 x 4096 bfloat16 values where these take 75: its
// phases wait for each other.)
template <int DT, bool VEC>
__global__ void __launch_bounds__(QT) quant_colmax(QuantParams p, int vl, int64_t rows_each) {
  using L = Elem<DT>;
  begin(p);
  __shared__ uint4 part[QT];
  const int lx = threadIdx.x % vl, ly = threadIdx.x / vl, nl = QT / vl;
  const int64_t r0 = (int64_t)blockIdx.y * rows_each, r1 = min(p.rows, r0 + rows_each);
  const int64_t col = ((int64_t)blockIdx.x * vl + lx) * (VEC ? L::E : 1), left = p.cols - col;
  const typename L::T* x = static_cast<const typename L::T*>(p.x) + col;
  uint4 m = make_uint4(0, 0, 0, 0);
  if (left > 0) {
    constexpr int U = 8;  // rows in flight; past the end the last row again, which changes no maximum
    if (VEC && left >= L::E) {
      for (int64_t r = r0 + ly; r < r1; r += U * nl) {
        uint4 u[U];
#pragma unroll
        for (int i = 0; i < U; i++) u[i] = __ldg(reinterpret_cast<const uint4*>(x + min(r + i * nl, r1 - 1) * p.ldx));
#pragma unroll
        for (int i = 0; i < U; i++) m = mag_max<DT>(m, u[i]);
      }
    } else if (VEC) {
      for (int64_t r = r0 + ly; r < r1; r += nl) m = mag_max<DT>(m, load_vec<DT, false>(x + r * p.ldx, left));
    } else {
      for (int64_t r = r0 + ly; r < r1; r += U * nl) {
        uint32_t u[U];
#pragma unroll
        for (int i = 0; i < U; i++) u[i] = L::bits(x[min(r + i * nl, r1 - 1) * p.ldx]);
#pragma unroll
        for (int i = 0; i < U; i++) m.x = max(m.x, u[i]);
      }
    }
  }
  part[threadIdx.x] = m;
  __syncthreads();
  if (ly == 0 && left > 0) {
    for (int k = 1; k < nl; k++) {
      if (VEC) m = mag_max<DT>(m, part[k * vl + lx]);
      else m.x = max(m.x, part[k * vl + lx].x);
    }
    if (VEC) {
      const uint32_t w[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
      for (int e = 0; e < L::E; e++) {
        const uint32_t b = L::E == 4 ? w[e % 4] : (e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu);
        if (e < left) atomicMax(p.colmax + col + e, b);
      }
    } else {
      atomicMax(p.colmax + col, m.x);
    }
  }
  end(p);
}

constexpr int TR = 128;  // rows of a tile
template <int DT, bool VEC, bool PACK>
__global__ void __launch_bounds__(QT, PACK ? 2 : 3) quant_cols(QuantParams p, int64_t rows_each) {
  using L = Elem<DT>;
  constexpr int CW = 8 * L::E;  // columns of a tile
  __shared__ __align__(16) float rs[CW], ss[CW];
  __shared__ uint32_t bads[2], tops[CW];
  __shared__ __align__(16) uint32_t tile[CW * (PACK ? TR / 2 : TR / 4 + 1)];  // integers: bytes, or packed binary16
  __shared__ float squares[PACK ? QT / 32 : 1][CW];
  const int tx = threadIdx.x & 7, ty = threadIdx.x >> 3;
  const int64_t c0 = (int64_t)blockIdx.x * CW, col = c0 + tx * L::E;
  const int64_t left = p.cols - col;  // may be <= 0
  // (a packed operand's k go on to a whole block: zeros)
  const int64_t r0 = (int64_t)(gridDim.y - 1 - blockIdx.y) * rows_each,
                r1 = min(PACK ? (int64_t)p.kb * 64 : p.rows, r0 + rows_each);
  const typename L::T* x = static_cast<const typename L::T*>(p.x) + col;
  begin(p);
  if (PACK) clear_earlier(p);
  // the other buffer of maxima is the next call's: zero again
  {
    const int64_t n = (int64_t)gridDim.x * gridDim.y * QT;
    for (int64_t i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * QT + threadIdx.x; i < p.zero_n; i += n) p.zero[i] = 0;
  }
  auto load = [&](int64_t t0, uint4 (&v)[4]) {
    const typename L::T* q = x + (t0 + ty * 4) * p.ldx;
    if (VEC && left >= L::E && t0 + TR <= min(r1, p.rows)) {
#pragma unroll
      for (int j = 0; j < 4; j++) v[j] = __ldg(reinterpret_cast<const uint4*>(q + j * p.ldx));
    } else {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        v[j] = make_uint4(0, 0, 0, 0);
        if (t0 + ty * 4 + j < min(r1, p.rows) && left > 0) v[j] = load_vec<DT, VEC>(q + j * p.ldx, left);
      }
    }
  };
  uint4 v[4];
  load(r0, v);
  if (!p.colmax) {  // few rows: every CTA finds its columns' maxima itself
    __shared__ uint4 part[QT / 32][8];
    uint4 m = make_uint4(0, 0, 0, 0);
    if (left > 0) {
      for (int64_t row = ty; row < p.rows; row += 4 * (QT / 8)) {
        uint4 u[4];
#pragma unroll
        for (int j = 0; j < 4; j++) u[j] = load_vec<DT, VEC>(x + min(row + j * (QT / 8), p.rows - 1) * p.ldx, left);
#pragma unroll
        for (int j = 0; j < 4; j++) m = mag_max<DT>(m, u[j]);
      }
    }
#pragma unroll
    for (int o = 8; o <= 16; o *= 2)
      m = mag_max<DT>(m, make_uint4(__shfl_xor_sync(0xffffffffu, m.x, o), __shfl_xor_sync(0xffffffffu, m.y, o),
                                    __shfl_xor_sync(0xffffffffu, m.z, o), __shfl_xor_sync(0xffffffffu, m.w, o)));
    if ((threadIdx.x & 31) < 8) part[threadIdx.x >> 5][tx] = m;
    __syncthreads();
    if (threadIdx.x < CW) {
      uint32_t top = 0;
      const int c = threadIdx.x;
      for (int w = 0; w < QT / 32; w++) {
        const uint32_t b = reinterpret_cast<const uint32_t*>(&part[w][0])[c * 4 / L::E];
        top = max(top, L::E == 4 ? b : (c & 1 ? b >> 16 : b & 0xffffu));
      }
      tops[c] = top;
    }
  }
  if (threadIdx.x < CW) {
    const int c = threadIdx.x;
    const uint32_t top = c0 + c >= p.cols ? 0 : (p.colmax ? __ldcg(p.colmax + c0 + c) : tops[c]);
    float r, scale;
    factors<DT>(top, r, scale);
    rs[c] = r;
    ss[c] = scale;
    const uint32_t vote = __ballot_sync(0xffffffffu, top >= L::INF);
    if ((c & 31) == 0) bads[c >> 5] = vote;
    if (p.scale && blockIdx.y == 0 && c0 + c < p.cols) p.scale[c0 + c] = scale;
  }
  __syncthreads();
  float r[L::E], scale[L::E];
#pragma unroll
  for (int e = 0; e < L::E; e += 4) {
    *reinterpret_cast<float4*>(r + e) = *reinterpret_cast<const float4*>(rs + tx * L::E + e);
    *reinterpret_cast<float4*>(scale + e) = *reinterpret_cast<const float4*>(ss + tx * L::E + e);
  }
  const uint32_t bad = bads[tx * L::E >> 5] >> (tx * L::E & 31) & ((1u << L::E) - 1u);

  for (int64_t t0 = r0; t0 < r1; t0 += TR) {
    float w[4][L::E];
#pragma unroll
    for (int j = 0; j < 4; j++) {
      unpack<DT>(v[j], w[j]);
      if (bad) {
#pragma unroll
        for (int e = 0; e < L::E; e++) w[j][e] = whole(w[j][e], r[e], !(bad >> e & 1));
      } else {
#pragma unroll
        for (int e = 0; e < L::E; e++) w[j][e] = whole(w[j][e], r[e], true);
      }
    }
    if (t0 + TR < r1) load(t0 + TR, v);  // the next tile is on its way
    if (!PACK && p.values) {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int64_t row = t0 + ty * 4 + j;
        if (row >= r1 || left <= 0) continue;
        float y[L::E];
#pragma unroll
        for (int e = 0; e < L::E; e++) y[e] = __fmul_rn(number(w[j][e]), scale[e]);
        store_values<DT>(static_cast<typename L::T*>(p.values) + row * p.ldv + col, y, p.vec_v, left);
      }
    }
    if constexpr (PACK) {
      // k pairs of a column side by side, its 16-byte pieces swizzled by the
      // thread column against bank conflicts; then 8 lanes write a row of a block
      __syncthreads();  // the tile's last readers are done
      char* bytes = reinterpret_cast<char*>(tile);
#pragma unroll
      for (int e = 0; e < L::E; e++)
        *reinterpret_cast<uint2*>(bytes + (tx * L::E + e) * (TR * 2) + ((ty >> 1 ^ tx) * 16) + (ty & 1) * 8) =
            make_uint2(half_pair(w[0][e], w[1][e]), half_pair(w[2][e], w[3][e]));
      if (p.norms) {
#pragma unroll
        for (int e = 0; e < L::E; e++) {
          float ss = 0.0f;
#pragma unroll
          for (int j = 0; j < 4; j++) ss = fmaf(number(w[j][e]), number(w[j][e]), ss);
          ss += __shfl_xor_sync(0xffffffffu, ss, 8);
          ss += __shfl_xor_sync(0xffffffffu, ss, 16);
          if ((threadIdx.x & 31) < 8) squares[threadIdx.x >> 5][tx * L::E + e] = ss;
        }
      }
      __syncthreads();
      const int piece = threadIdx.x & 7;
#pragma unroll
      for (int i = threadIdx.x >> 3; i < CW * 2; i += QT / 8) {
        const int c = i >> 1, block = i & 1;
        const int64_t k = t0 + block * 64 + piece * 8;
        if (k >= (int64_t)p.kb * 64) continue;
        const uint4 u = *reinterpret_cast<const uint4*>(bytes + c * (TR * 2) + (block * 8 + (piece ^ (c / L::E))) * 16);
        *reinterpret_cast<uint4*>(packed_at(p, c0 + c, k)) = u;
      }
      if (p.norms && threadIdx.x < CW) {  // (exact: below 2^22)
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < QT / 32; i++) ss += squares[i][threadIdx.x];
        const unsigned most = __reduce_max_sync(0xffffffffu, (unsigned)ss);
        if ((threadIdx.x & 31) == 0) atomicMax(p.norms + (c0 >> 7) * p.kc * 2 + t0 / 128, most);
      }
    } else if (p.q) {
      constexpr int TP = TR / 4 + 1;
      __syncthreads();  // the tile's last readers are done
#pragma unroll
      for (int e = 0; e < L::E; e++) tile[(tx * L::E + e) * TP + ty] = pack4(w[0][e], w[1][e], w[2][e], w[3][e]);
      __syncthreads();
      const int lane = threadIdx.x & 31;
      const int64_t row = t0 + lane * 4;
      for (int c = threadIdx.x >> 5; c < CW; c += QT / 32) {
        if (c0 + c >= p.cols || row >= p.rows) continue;
        const uint32_t u = tile[c * TP + lane];
        int8_t* q = p.q + (c0 + c) * p.ldq + row;
        if (p.vec_q && row + 4 <= p.rows) {
          *reinterpret_cast<uint32_t*>(q) = u;
        } else {
#pragma unroll
          for (int b = 0; b < 4; b++)
            if (row + b < p.rows) q[b] = (int8_t)(u >> (8 * b));
        }
      }
    }
  }
  end(p);
}

template <int DT>
cudaError_t rows_launch(const QuantParams& p, int nsm, cudaStream_t s) {
  constexpr int E = Elem<DT>::E;
  if (!p.vec_x) return launch_dependent(quant_rows_twice<DT, false>, (unsigned)p.rows, QT, 0, s, p);
  const int64_t nv = (p.cols + E - 1) / E;
  auto go = [&](void (*kernel)(QuantParams), int tpr) {
    return launch_dependent(kernel, (unsigned)((p.rows + QT / tpr - 1) / (QT / tpr)), QT, 0, s, p);
  };
  if (p.packed) {
    const int64_t pv = (int64_t)p.kb * 64 / E;
    auto pack = [&](void (*kernel)(QuantParams, int), int tpr) {
      const int64_t groups = p.prows / (QT / tpr);
      int each = 1;  // rows of a thread group (of one block of 128): up to 8, while every SM has 4 CTAs
      while (each < 8 && groups / (2 * each) >= 4 * nsm) each *= 2;
      return launch_dependent(kernel, (unsigned)(groups / each), QT, 0, s, p, each);
    };
    if (pv <= 32) return pack(quant_rows_packed<DT, 32, 1>, 32);
    if (pv <= 64) return pack(quant_rows_packed<DT, 32, 2>, 32);
    if (pv <= 128) return pack(quant_rows_packed<DT, 32, 4>, 32);
    if (pv <= 256) return pack(quant_rows_packed<DT, QT, 1>, QT);
    if (pv <= 512) return pack(quant_rows_packed<DT, QT, 2>, QT);
    if (pv <= 1024) return pack(quant_rows_packed<DT, QT, 4>, QT);
    return pack(quant_rows_packed<DT, QT, 8>, QT);
  }
  if (nv <= 32) return go(quant_rows<DT, 32, 1>, 32);
  if (nv <= 64) return go(quant_rows<DT, 32, 2>, 32);
  if (nv <= 128) return go(quant_rows<DT, 32, 4>, 32);
  if (nv <= 256) return go(quant_rows<DT, QT, 1>, QT);
  if (nv <= 512) return go(quant_rows<DT, QT, 2>, QT);
  if (nv <= 1024) return go(quant_rows<DT, QT, 4>, QT);
  if (nv <= 2048) return go(quant_rows<DT, QT, 8>, QT);
  return go(quant_rows_twice<DT, true>, QT);
}

template <int DT, bool VEC>
cudaError_t cols_launch(const QuantParams& p, bool maxima, int nsm, cudaStream_t s) {
  constexpr int E = Elem<DT>::E, CW = 8 * E;
  const int64_t per = VEC ? E : 1, nv = (p.cols + per - 1) / per;
  int vl = 8;
  while (vl < 32 && vl < nv) vl *= 2;  // wider CTAs would mean more shares of the rows, and atomics for each
  const int64_t wide = (nv + vl - 1) / vl, lanes = QT / vl;
  // one wave of as many CTAs as an SM holds, `least` rows or more for each
  auto shares = [&](int64_t across, int64_t least, int64_t rows_unit, int64_t resident, int64_t* each) {
    int64_t n = std::min(resident * nsm / across, (p.rows + least - 1) / least);
    n = std::max<int64_t>(1, std::min<int64_t>(n, 65535));
    *each = ((p.rows + n - 1) / n + rows_unit - 1) / rows_unit * rows_unit;
    return (unsigned)std::max<int64_t>(1, (p.rows + *each - 1) / std::max<int64_t>(*each, 1));
  };
  int64_t each = 1;
  if (maxima) {
    const unsigned ny = shares(wide, 8 * lanes, 1, 5, &each);
    if (p.rows == 0) return cudaSuccess;
    return launch_dependent(quant_colmax<DT, VEC>, dim3((unsigned)wide, ny), QT, 0, s, p, vl, std::max<int64_t>(each, 1));
  }
  if (p.packed) {
    const int64_t strips = p.prows / CW, K = (int64_t)p.kb * 64;
    int64_t n = std::max<int64_t>(1, std::min(std::min<int64_t>(2 * nsm / strips, (K + TR - 1) / TR), (int64_t)65535));
    each = ((K + n - 1) / n + TR - 1) / TR * TR;
    n = (K + each - 1) / each;
    return launch_dependent(quant_cols<DT, VEC, true>, dim3((unsigned)strips, (unsigned)n), QT, 0, s, p, each);
  }
  const int64_t strips = (p.cols + CW - 1) / CW;
  const unsigned ty = shares(strips, TR, TR, 3, &each);
  return launch_dependent(quant_cols<DT, VEC, false>, dim3((unsigned)strips, ty), QT, 0, s, p, std::max<int64_t>(each, TR));
}

template <int DT>
cudaError_t quant_launch(int step, const QuantParams& p, int nsm, cudaStream_t s) {
  if (step == QUANT_ROWS) return rows_launch<DT>(p, nsm, s);
  const bool maxima = step == QUANT_MAXIMA;
  return p.vec_x ? cols_launch<DT, true>(p, maxima, nsm, s) : cols_launch<DT, false>(p, maxima, nsm, s);
}

}  // namespace

bool quant8_packs(int dtype, int axis, const QuantParams& p) {
  return p.vec_x && (axis == 1 || (int64_t)p.kb * 64 / (dtype == PEAT_F32 ? 4 : 8) <= 8 * QT);
}

cudaError_t launch_quant8(int dtype, int step, const QuantParams& p, int nsm, cudaStream_t s) {
  if (dtype == PEAT_F32) return quant_launch<PEAT_F32>(step, p, nsm, s);
  if (dtype == PEAT_F16) return quant_launch<PEAT_F16>(step, p, nsm, s);
  return quant_launch<PEAT_BF16>(step, p, nsm, s);
}

}  // namespace peat
