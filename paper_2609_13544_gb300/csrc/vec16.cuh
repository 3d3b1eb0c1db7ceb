// A 16-byte vector of float32, binary16 or bfloat16 as float32 numbers, and back.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "peat.h"

namespace peat {

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

}  // namespace peat
