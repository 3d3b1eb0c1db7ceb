// 4-bit floating-point values (1 sign, 2 exponent and 1 mantissa bit: 0, 0.5, 1,
// 1.5, 2, 3, 4, 6) and the scales of their blocks.
//
// The scales of 128 rows by 4 blocks lie together in 512 bytes, row r and block k
// at (r mod 32) 16 + (r div 32) 4 + k: 32 lanes of 16 bytes, the image in which
// the matrix instruction wants them in tensor memory.
#pragma once
#include <cuda_fp16.h>

#include "ops_internal.h"

namespace peat {

template <int FMT>
struct F4 {  // PEAT_MXFP4: a power of two for 32 values
  static constexpr int BLOCK = 32;
};
template <>
struct F4<PEAT_NVFP4> {  // an 8-bit float for 16, below a float32 scale of the row
  static constexpr int BLOCK = 16;
};
constexpr int SCALE_TILE = 512;
constexpr float F4_TOP = 2688.0f;  // the largest code times the largest block scale, 6 x 448

__device__ __forceinline__ int64_t scale_at(int64_t row, int64_t block, int64_t tiles) {
  const int r = (int)(row & 127);
  return ((row >> 7) * tiles + (block >> 2)) * SCALE_TILE + (r & 31) * 16 + (r >> 5) * 4 + (int)(block & 3);
}

// the codes of eight values, the first in the lowest bits: to the nearest, ties
// to the even code, at most 6 in magnitude
__device__ __forceinline__ uint32_t codes8(const float (&x)[8]) {
  uint32_t r;
  asm("{\n .reg .b8 a, b, c, d;\n"
      " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
      " mov.b32 %0, {a, b, c, d};\n}"
      : "=r"(r)
      : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return r;
}
__device__ __forceinline__ uint32_t codes4(float x0, float x1, float x2, float x3) {
  uint16_t r;
  asm("{\n .reg .b8 a, b;\n"
      " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      " mov.b16 %0, {a, b};\n}"
      : "=h"(r)
      : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
  return r;
}
// the values of four codes in the low 16 bits
__device__ __forceinline__ void values4(uint32_t c, float (&v)[4]) {
  uint32_t lo, hi;
  asm("{\n .reg .b8 a, b;\n mov.b16 {a, b}, %2;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n}"
      : "=r"(lo), "=r"(hi)
      : "h"((uint16_t)c));
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&lo)), y = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  v[0] = x.x, v[1] = x.y, v[2] = y.x, v[3] = y.y;
}
// the nearest 8-bit float (4 exponent, 3 mantissa bits) of 0 <= u, at most 448
__device__ __forceinline__ uint32_t e4m3(float u) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(u));
  return r & 0xff;
}
// the value of such a byte (not NaN): its bits are a float32's but for the bias
__device__ __forceinline__ float e4m3_value(uint32_t b) { return __uint_as_float(b << 20) * 0x1p120f; }

// What a block's rounding needs: a value's code is that of (x * t) * r, a code's
// value (code * f) * s.
struct Block4 {
  float r, f;
  uint32_t byte;
};
// of a row: the factor t before the block's and the scale s
struct Row4 {
  float t, s;
  bool finite;
};
template <int FMT>
__device__ __forceinline__ Row4 row4(float amax, bool finite) {
  if (FMT == PEAT_MXFP4) return Row4{1.0f, 1.0f, true};
  if (!finite) return Row4{0.0f, __uint_as_float(0x7fc00000u), false};
  const float t = __fdiv_rn(F4_TOP, amax);
  if (!(t <= 3.402823466e38f)) return Row4{0.0f, 0.0f, true};  // amax 0, or too small for a finite t
  return Row4{t, __fdiv_rn(amax, F4_TOP), true};
}
// the reciprocals of the 8-bit floats by their bytes, of 0 and NaN 0: a look-up a
// block in place of a division; all threads of the CTA
constexpr int RECIPROCALS = 128;
__device__ __forceinline__ void make_reciprocals(float* table) {
  for (int i = threadIdx.x; i < RECIPROCALS; i += blockDim.x)
    table[i] = i == 0 || i == RECIPROCALS - 1 ? 0.0f : __fdiv_rn(1.0f, e4m3_value((uint32_t)i));
}
// x / 6, rounded once, for x >= 2^-100: by the divisor's reciprocal in two parts
// (Brisebarre, Muller and Raina 2004; checked for every such x up to 2^12)
__device__ __forceinline__ float sixth(float x) {
  constexpr float HI = 0x1.555556p-3f, LO = -0x1.555556p-28f;
  return __fmaf_rn(x, HI, __fmul_rn(x, LO));
}
// amax: of the block (mxfp4: NaN or infinite where finite is not set)
template <int FMT>
__device__ __forceinline__ Block4 block4(float amax, bool finite, const Row4& row, const float* reciprocals) {
  if (FMT == PEAT_MXFP4) {
    const int e = max((int)(__float_as_uint(amax) >> 23), 2);  // + 129
    return finite ? Block4{__uint_as_float((uint32_t)(256 - e) << 23),
                           e > 2 ? __uint_as_float((uint32_t)(e - 2) << 23) : 0x1p-127f, (uint32_t)(e - 2)}
                  : Block4{0.0f, __uint_as_float(0x7fc00000u), 255};
  }
  const uint32_t b = row.finite ? e4m3(sixth(__fmul_rn(amax, row.t))) : 0;
  return Block4{reciprocals[b], 0.0f, b};
}
template <int FMT>
__device__ __forceinline__ float scaled4(float x, const Row4& row, const Block4& b) {
  return FMT == PEAT_MXFP4 ? __fmul_rn(x, b.r) : __fmul_rn(__fmul_rn(x, row.t), b.r);
}
// whether a block's codes are those of its numbers, not zeros
template <int FMT>
__device__ __forceinline__ bool coded(bool finite, const Block4& b) { return FMT == PEAT_MXFP4 ? finite : b.byte != 0; }
// the values of four codes; nvfp4: a code times its block's scale fits binary16 exactly
template <int FMT>
__device__ __forceinline__ void decoded4(uint32_t c, const Row4& row, const Block4& b, float (&v)[4]) {
  if (FMT == PEAT_MXFP4) {
    values4(c, v);
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = __fmul_rn(v[i], b.f);
    return;
  }
  uint32_t lo, hi, f;
  asm("{\n .reg .b8 a, b;\n mov.b16 {a, b}, %3;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
      " cvt.rn.f16x2.e4m3x2 %2, %4;\n}"
      : "=r"(lo), "=r"(hi), "=r"(f)
      : "h"((uint16_t)c), "h"((uint16_t)(b.byte * 0x101u)));
  const __half2 h = *reinterpret_cast<const __half2*>(&f);
  const float2 x = __half22float2(__hmul2(*reinterpret_cast<const __half2*>(&lo), h));
  const float2 y = __half22float2(__hmul2(*reinterpret_cast<const __half2*>(&hi), h));
  v[0] = __fmul_rn(x.x, row.s), v[1] = __fmul_rn(x.y, row.s), v[2] = __fmul_rn(y.x, row.s), v[3] = __fmul_rn(y.y, row.s);
}

}  // namespace peat
