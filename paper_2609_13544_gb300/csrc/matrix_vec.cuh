// Matrices of float32, binary16 or bfloat16 by 16-byte vectors: element types,
// magnitudes, rounding to 8-bit integers, loads and stores at any multiple of the
// element's size.
#pragma once
#include <type_traits>

#include "vec16.cuh"

namespace peat {

template <int DT>
struct Elem;
template <>
struct Elem<PEAT_F32> {
  using T = float;
  static constexpr int E = 4;  // elements of a 16-byte vector
  static constexpr uint32_t INF = 0x7f800000u;
  static __device__ __forceinline__ float mag(uint32_t b) { return __uint_as_float(b); }
};
template <>
struct Elem<PEAT_F16> {
  using T = __half;
  static constexpr int E = 8;
  static constexpr uint32_t INF = 0x7c00u;
  static __device__ __forceinline__ float mag(uint32_t b) { return __half2float(__ushort_as_half((unsigned short)b)); }
};
template <>
struct Elem<PEAT_BF16> {
  using T = __nv_bfloat16;
  static constexpr int E = 8;
  static constexpr uint32_t INF = 0x7f80u;
  static __device__ __forceinline__ float mag(uint32_t b) { return __uint_as_float(b << 16); }
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

// the larger magnitude, under some sign; a NaN stays
template <int DT>
__device__ __forceinline__ uint32_t max_abs(uint32_t a, uint32_t b) {
  uint32_t r;
  if (DT == PEAT_F32) asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(*reinterpret_cast<float*>(&r)) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)));
  else if (DT == PEAT_F16) asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// the largest magnitude's pattern of a vector
template <int DT>
__device__ __forceinline__ uint32_t vec_top(uint4 v) {
  const uint32_t m = max_abs<DT>(max_abs<DT>(v.x, v.y), max_abs<DT>(v.z, v.w));
  return DT == PEAT_F32 ? m & 0x7fffffffu : max(m & 0x7fffu, m >> 16 & 0x7fffu);
}

// ---- 8-bit integers ----
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

// Vectors of E elements at any multiple of the element's size.  On the 16-byte
// grid one load; off it the two aligned vectors that hold it, shifted together.
// A vector that is not whole (`left` elements exist), or whose aligned vectors
// reach beyond the matrix, is left for load_edge.
template <int DT, bool GRID>
struct Source {
  using T = typename Elem<DT>::T;
  uintptr_t lo, hi;  // the matrix's bytes
  __device__ Source(const void* at, int64_t rows, int64_t cols, int64_t ld) {
    const T* x = static_cast<const T*>(at);
    lo = reinterpret_cast<uintptr_t>(x);
    hi = reinterpret_cast<uintptr_t>(x + (rows - 1) * ld + cols);
  }
  __device__ __forceinline__ bool whole(const T* p, int64_t left) const {
    if (left < Elem<DT>::E) return false;
    const uintptr_t a = reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15;
    return GRID || (a >= lo && a + 32 <= hi);
  }
  __device__ __forceinline__ uint4 load(const T* p) const {
    if (GRID) return __ldg(reinterpret_cast<const uint4*>(p));
    const uint4* a = on_grid(p);
    return shifted(__ldg(a), __ldg(a + 1), (int)(reinterpret_cast<uintptr_t>(p) & 15));
  }
  static __device__ __forceinline__ const uint4* on_grid(const T* p) {
    return reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15);
  }
};
// the first `left` elements of a vector, one by one, zeros beyond
template <int DT>
__device__ __forceinline__ uint4 load_edge(const typename Elem<DT>::T* p, int64_t left) {
  Vec<DT> v;
  v.u = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < Elem<DT>::E; e++)
    if (e < left) v.e[e] = p[e];
  return v.u;
}

// A vector's values at o, of which `left` (any number) exist, by G lanes that
// have consecutive vectors of a row.  Where the row is off the 16-byte grid a
// lane writes the aligned vector that ends inside its own, the last elements of
// the vector before in front: the lane before's, or for lane 0 `carry`, the last
// lane's of the call before, unless this is the first.  What no vector of the
// group precedes or follows goes one by one.  All lanes of a group call it.
template <int DT, int G>
__device__ __forceinline__ void store_values(typename Elem<DT>::T* o, const float (&y)[Elem<DT>::E], bool on_grid,
                                             int64_t left, uint4& carry, bool first, bool last) {
  constexpr int E = Elem<DT>::E, B = 16 / E;
  Vec<DT> v;
  v.u = pack<DT>(y);
  if (on_grid) {
    if (left >= E) {
      __stcs(reinterpret_cast<uint4*>(o), v.u);
    } else {
#pragma unroll
      for (int e = 0; e < E; e++)
        if (e < left) o[e] = v.e[e];
    }
    return;
  }
  const int lane = threadIdx.x % G;
  // (a rotation: lane 0 receives the last lane's, for the next call)
  auto turned = [&](uint32_t x, uint32_t& kept) {
    const uint32_t t = __shfl_sync(0xffffffffu, x, (lane + G - 1) % G, G);
    const uint32_t before = lane == 0 ? kept : t;
    kept = t;
    return before;
  };
  const uint4 before = make_uint4(turned(v.u.x, carry.x), turned(v.u.y, carry.y), turned(v.u.z, carry.z), turned(v.u.w, carry.w));
  const int s = (int)(reinterpret_cast<uintptr_t>(o) & 15) / B;  // elements from the grid to o
  const bool alone = first && lane == 0;
  Vec<DT> w;
  w.u = s ? shifted(before, v.u, 16 - s * B) : v.u;
  if ((!alone || s == 0) && left >= E - s) {
    __stcs(reinterpret_cast<uint4*>(o - s), w.u);
  } else {
#pragma unroll
    for (int e = 0; e < E; e++)
      if ((!alone || e >= s) && e - s < left) o[e - s] = w.e[e];
  }
  if (last && lane == G - 1) {  // its own last elements
#pragma unroll
    for (int e = 0; e < E; e++)
      if (e >= E - s && e < left) o[e] = v.e[e];
  }
}

// E elements of a row, APART columns from one to the next, as a vector; and back.  A
// warp's are side by side, whatever the row's alignment.
template <int DT, int APART, typename Col>
__device__ __forceinline__ uint4 load_apart(const typename Elem<DT>::T* row, Col col, Col cols) {
  using U = std::conditional_t<DT == PEAT_F32, uint32_t, uint16_t>;
  constexpr int E = Elem<DT>::E, PER = DT == PEAT_F32 ? 1 : 2;
  uint32_t w[4] = {0, 0, 0, 0};
  const U* p = reinterpret_cast<const U*>(row + col);
  U x[E];
  if (col + (E - 1) * APART < cols) {  // (without a condition on each load, or they wait for one another)
#pragma unroll
    for (int e = 0; e < E; e++) x[e] = p[e * APART];
  } else {
#pragma unroll
    for (int e = 0; e < E; e++) x[e] = col + e * APART < cols ? p[e * APART] : (U)0;
  }
#pragma unroll
  for (int e = 0; e < E; e++) w[e / PER] |= (uint32_t)x[e] << (e % PER * 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int DT, int APART, typename Col>
__device__ __forceinline__ void put_apart(typename Elem<DT>::T* row, uint4 u, Col col, Col cols) {
  Vec<DT> v;
  v.u = u;
  typename Elem<DT>::T* o = row + col;
#pragma unroll
  for (int e = 0; e < Elem<DT>::E; e++)
    if (col + e * APART < cols) o[e * APART] = v.e[e];
}
// Between such vectors and those of consecutive elements, G lanes' at a time, by way
// of `place` (16 bytes a lane of the warp); all lanes of the warp together.
template <int DT, int G>
__device__ __forceinline__ uint4 gathered(uint4 u, uint4* place) {
  using T = typename Elem<DT>::T;
  const int lane = threadIdx.x & (G - 1);
  uint4* mine = place + (threadIdx.x & 31 & ~(G - 1));
  Vec<DT> v;
  v.u = u;
  __syncwarp();
#pragma unroll
  for (int e = 0; e < Elem<DT>::E; e++) reinterpret_cast<T*>(mine)[e * G + lane] = v.e[e];
  __syncwarp();
  return mine[lane];
}
template <int DT, int G>
__device__ __forceinline__ uint4 spread(uint4 u, uint4* place) {
  using T = typename Elem<DT>::T;
  const int lane = threadIdx.x & (G - 1);
  uint4* mine = place + (threadIdx.x & 31 & ~(G - 1));
  __syncwarp();
  mine[lane] = u;
  __syncwarp();
  Vec<DT> v;
#pragma unroll
  for (int e = 0; e < Elem<DT>::E; e++) v.e[e] = reinterpret_cast<const T*>(mine)[e * G + lane];
  return v.u;
}

}  // namespace peat
