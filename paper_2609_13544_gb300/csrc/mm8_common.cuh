// Pieces shared by the kernels of the 8-bit products: loads of any alignment,
// 8-bit integers as binary16 values, the scaled output.
//
// An 8-bit integer is exact in binary16, the product of two is below 2^14, and
// float32 holds every integer up to 2^24: a sum over at most 512 products
// (2^23) is exact in a float32 accumulator whatever the order, so the binary16
// matrix instructions give the integer product.  Longer sums are carried in
// int32 between runs of that length.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ops_internal.h"
#include "vec16.cuh"

namespace peat {

constexpr int MM8_EXACT_K = 512;  // products whose float32 sum is exact

// 16 integers of a row from p on, of which `left` (may be <= 0) exist; zeros
// beyond.  MODE 16: p is 16-byte aligned; else any alignment, by the two aligned
// vectors that hold them where those lie inside [lo, hi), the tensor's span.
template <int MODE>
__device__ __forceinline__ uint4 load16(const int8_t* p, int64_t left, const int8_t* lo, const int8_t* hi) {
  if (left <= 0) return make_uint4(0, 0, 0, 0);
  uint4 v;
  if (MODE == 16 && left >= 16) return __ldg(reinterpret_cast<const uint4*>(p));
  const uintptr_t a = reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15;
  if (MODE == 16 && p + 16 <= hi) {
    v = __ldg(reinterpret_cast<const uint4*>(p));
  } else if (MODE != 16 && a >= reinterpret_cast<uintptr_t>(lo) && a + 32 <= reinterpret_cast<uintptr_t>(hi)) {
    const uint4* w = reinterpret_cast<const uint4*>(a);
    v = shifted(__ldg(w), __ldg(w + 1), (int)(reinterpret_cast<uintptr_t>(p) & 15));
  } else {  // the tensor's first and last bytes
    uint32_t t[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; i++)
      if (i < left) t[i >> 2] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
    v = make_uint4(t[0], t[1], t[2], t[3]);
  }
  if (left < 16) {  // clear what belongs to the row's padding or to the next row
    const int n = (int)left;
    auto keep = [n](uint32_t x, int at) {
      const int b = n - at;
      return b >= 4 ? x : (b <= 0 ? 0u : x & ((1u << (8 * b)) - 1u));
    };
    v.x = keep(v.x, 0);
    v.y = keep(v.y, 4);
    v.z = keep(v.z, 8);
    v.w = keep(v.w, 12);
  }
  return v;
}

// four integers as two pairs of binary16: the byte v + 128 under the exponent
// of 1024 is 1024 + 128 + v, exactly
__device__ __forceinline__ void to_half(uint32_t w, uint32_t& lo, uint32_t& hi) {
  w ^= 0x80808080u;
  const __half2 bias = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));  // 1152
  uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
  __half2 x = __hsub2(*reinterpret_cast<__half2*>(&a), bias), y = __hsub2(*reinterpret_cast<__half2*>(&b), bias);
  lo = *reinterpret_cast<uint32_t*>(&x);
  hi = *reinterpret_cast<uint32_t*>(&y);
}

// out types: the value of an integer sum
template <int OUT>
struct Mm8Out;
template <>
struct Mm8Out<PEAT_F32> {
  using T = float;
  static __device__ __forceinline__ T make(int acc, float s, float b) { return __fadd_rn(__fmul_rn((float)acc, s), b); }
};
template <>
struct Mm8Out<PEAT_F16> {
  using T = __half;
  static __device__ __forceinline__ T make(int acc, float s, float b) {
    return __float2half_rn(__fadd_rn(__fmul_rn((float)acc, s), b));
  }
};
template <>
struct Mm8Out<PEAT_BF16> {
  using T = __nv_bfloat16;
  static __device__ __forceinline__ T make(int acc, float s, float b) {
    return __float2bfloat16_rn(__fadd_rn(__fmul_rn((float)acc, s), b));
  }
};
template <>
struct Mm8Out<PEAT_OUT_I32> {
  using T = int;
  static __device__ __forceinline__ T make(int acc, float, float) { return acc; }
};

}  // namespace peat
