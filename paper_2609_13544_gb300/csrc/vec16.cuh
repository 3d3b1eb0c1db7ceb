// A 16-byte vector of float32, binary16 or bfloat16 as float32 numbers, and back;
// vectors off the 16-byte grid.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "peat.h"

namespace peat {

// bytes [by, by + 16) of the 32 of a and b
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b, int by) {
  uint32_t t[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  const bool one = by & 4, two = by & 8;
#pragma unroll
  for (int i = 0; i < 7; i++) t[i] = one ? t[i + 1] : t[i];
#pragma unroll
  for (int i = 0; i < 5; i++) t[i] = two ? t[i + 2] : t[i];
  const int bits = (by & 3) * 8;
  return make_uint4(__funnelshift_r(t[0], t[1], bits), __funnelshift_r(t[1], t[2], bits),
                    __funnelshift_r(t[2], t[3], bits), __funnelshift_r(t[3], t[4], bits));
}
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

// Two float32 operations in one instruction, each rounded to nearest as the single
// ones; but the compiler makes one fma of a mul2 whose result only an add2 takes.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 x, y, w;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mul.rn.f32x2 w, x, y;\n mov.b64 {%0, %1}, w;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 x, y, w;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n add.rn.f32x2 w, x, y;\n mov.b64 {%0, %1}, w;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n .reg .b64 x, y, z, w;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %5};\n mov.b64 z, {%6, %7};\n"
      " fma.rn.f32x2 w, x, y, z;\n mov.b64 {%0, %1}, w;\n}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 minus(float2 a) { return make_float2(-a.x, -a.y); }
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
// elements 2 i and 2 i + 1
template <int N>
__device__ __forceinline__ float2 pair(const float (&x)[N], int i) { return make_float2(x[2 * i], x[2 * i + 1]); }
template <int N>
__device__ __forceinline__ void put_pair(float (&x)[N], int i, float2 v) { x[2 * i] = v.x, x[2 * i + 1] = v.y; }

}  // namespace peat
