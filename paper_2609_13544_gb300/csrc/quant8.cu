// Rounding of a matrix to 8-bit integers with one scale for each row or column.
//
// Over a row (or column): amax = max |x|, scale = amax / 127, r = 127 / amax,
// q = rint(x r), all float32.  The maximum is taken on the bit patterns
// without their sign, which order as the magnitudes do and put infinities and
// NaNs above every number, so one integer maximum finds both amax and whether
// the row is finite.
//
// Bound by memory: a row is read once and kept in registers between the
// maximum and the rounding; a strip of columns is read twice, the second time
// from L2.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ops_internal.h"

namespace cg = cooperative_groups;

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

// elementwise maximum of the magnitudes' bit patterns: four words, or eight half-words
template <int DT>
__device__ __forceinline__ uint4 mag_max(uint4 m, uint4 v) {
  if (DT == PEAT_F32) {
    return make_uint4(max(m.x, v.x & 0x7fffffffu), max(m.y, v.y & 0x7fffffffu), max(m.z, v.z & 0x7fffffffu),
                      max(m.w, v.w & 0x7fffffffu));
  } else {
    return make_uint4(__vmaxu2(m.x, v.x & 0x7fff7fffu), __vmaxu2(m.y, v.y & 0x7fff7fffu),
                      __vmaxu2(m.z, v.z & 0x7fff7fffu), __vmaxu2(m.w, v.w & 0x7fff7fffu));
  }
}
template <int DT>
__device__ __forceinline__ uint32_t mag_fold(uint4 m) {  // the largest of the vector
  if (DT == PEAT_F32) return max(max(m.x, m.y), max(m.z, m.w));
  const uint32_t a = __vmaxu2(__vmaxu2(m.x, m.y), __vmaxu2(m.z, m.w));
  return max(a & 0xffffu, a >> 16);
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
// the integer of x; a non-finite row has r = 0, and 0 x NaN must not get through
template <int DT>
__device__ __forceinline__ int whole(float x, float r, bool finite) {
  return finite ? __float2int_rn(__fmul_rn(x, r)) : 0;
}
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
  return __byte_perm(__byte_perm((uint32_t)a, (uint32_t)b, 0x0040), __byte_perm((uint32_t)c, (uint32_t)d, 0x0040), 0x5410);
}

// the first `left` elements of a vector at p (left < E: one by one, zero beyond)
template <int DT, bool VEC>
__device__ __forceinline__ Vec<DT> load_vec(const typename Elem<DT>::T* p, int64_t left) {
  Vec<DT> v;
  if (VEC && left >= Elem<DT>::E) {
    v.u = __ldg(reinterpret_cast<const uint4*>(p));
    return v;
  }
  v.u = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < Elem<DT>::E; e++)
    if (e < left) v.e[e] = p[e];
  return v;
}

// integers and values of one vector of a row
template <int DT>
__device__ __forceinline__ void store_row_vec(const QuantParams& p, const Vec<DT>& v, int64_t row, int64_t col,
                                              int64_t left, float r, float scale, bool finite) {
  using L = Elem<DT>;
  int w[L::E];
#pragma unroll
  for (int e = 0; e < L::E; e++) w[e] = whole<DT>(L::up(v.e[e]), r, finite);
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
        if (e < left) q[e] = (int8_t)w[e];
    }
  }
  if (p.values) {
    typename L::T* o = static_cast<typename L::T*>(p.values) + row * p.ldv + col;
    Vec<DT> y;
#pragma unroll
    for (int e = 0; e < L::E; e++) y.e[e] = L::down(__fmul_rn((float)w[e], scale));
    if (p.vec_v && left >= L::E) {
      *reinterpret_cast<uint4*>(o) = y.u;
    } else {
#pragma unroll
      for (int e = 0; e < L::E; e++)
        if (e < left) o[e] = y.e[e];
    }
  }
}

constexpr int QT = 256;  // threads of a CTA

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
  const int lane = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * (QT / TPR) + threadIdx.x / TPR;
  if (row >= p.rows) return;  // (whole warps; with TPR = QT there is a row for every CTA)
  const typename L::T* x = static_cast<const typename L::T*>(p.x) + row * p.ldx;
  Vec<DT> v[NV];
  uint4 m = make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < NV; i++) {
    const int64_t col = (int64_t)(i * TPR + lane) * L::E;
    v[i].u = make_uint4(0, 0, 0, 0);
    if (col < p.cols) v[i] = load_vec<DT, true>(x + col, p.cols - col);
  }
#pragma unroll
  for (int i = 0; i < NV; i++) m = mag_max<DT>(m, v[i].u);
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

// A row by a CTA, read twice: rows too long for the registers, and (VEC false) rows off the 16-byte grid,
// which are taken element by element.
template <int DT, bool VEC>
__global__ void __launch_bounds__(QT) quant_rows_twice(QuantParams p) {
  using L = Elem<DT>;
  const int64_t row = blockIdx.x;
  const typename L::T* x = static_cast<const typename L::T*>(p.x) + row * p.ldx;
  uint32_t top = 0;
  if (VEC) {
    uint4 m = make_uint4(0, 0, 0, 0);
#pragma unroll 4
    for (int64_t col = (int64_t)threadIdx.x * L::E; col < p.cols; col += QT * L::E)
      m = mag_max<DT>(m, load_vec<DT, true>(x + col, p.cols - col).u);
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
      const int w = whole<DT>(L::up(x[col]), r, finite);
      if (q) q[col] = (int8_t)w;
      if (o) o[col] = L::down(__fmul_rn((float)w, scale));
    }
  }
}

// Columns: a cluster takes a strip of 128 bytes of columns (64 or 32), its
// CTAs a share of the rows each.  The maxima meet in distributed shared memory;
// then each CTA reads its share again (from L2: it has just been read) in
// tiles of 128 rows and writes the integers transposed through shared memory,
// 128 contiguous ones a column.
constexpr int TR = 128;  // rows of a tile
template <int DT, bool VEC>
__global__ void __launch_bounds__(QT) quant_cols(QuantParams p) {
  using L = Elem<DT>;
  constexpr int CW = 8 * L::E;  // columns of a strip
  __shared__ uint4 part[QT / 32][8];
  __shared__ uint4 mine[8];
  __shared__ uint32_t tile[CW][TR / 4 + 1];
  cg::cluster_group cl = cg::this_cluster();
  const int S = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int tx = threadIdx.x & 7, ty = threadIdx.x >> 3;
  const int64_t col = ((int64_t)blockIdx.x / S) * CW + tx * L::E;
  const int64_t left = p.cols - col;  // may be <= 0
  const int64_t tiles = (p.rows + TR - 1) / TR;
  const int64_t r0 = tiles * rank / S * TR, r1 = min(p.rows, tiles * (rank + 1) / S * TR);
  const typename L::T* x = static_cast<const typename L::T*>(p.x) + col;

  uint4 m = make_uint4(0, 0, 0, 0);
  if (left > 0) {
#pragma unroll 8
    for (int64_t r = r0 + ty; r < r1; r += 32) m = mag_max<DT>(m, load_vec<DT, VEC>(x + r * p.ldx, left).u);
  }
#pragma unroll
  for (int o = 8; o <= 16; o *= 2) {
    uint4 t;
    t.x = __shfl_xor_sync(0xffffffffu, m.x, o);
    t.y = __shfl_xor_sync(0xffffffffu, m.y, o);
    t.z = __shfl_xor_sync(0xffffffffu, m.z, o);
    t.w = __shfl_xor_sync(0xffffffffu, m.w, o);
    m = mag_max<DT>(m, t);
  }
  if ((threadIdx.x & 31) < 8) part[threadIdx.x >> 5][tx] = m;
  __syncthreads();
  if (threadIdx.x < 8) {
#pragma unroll
    for (int w = 0; w < QT / 32; w++) m = mag_max<DT>(m, part[w][tx]);
    mine[tx] = m;
  }
  cl.sync();
  m = mine[tx];
  for (int k = 1; k < S; k++) {
    int o = rank + k;
    o = o < S ? o : o - S;
    m = mag_max<DT>(m, *cl.map_shared_rank(&mine[tx], o));
  }
  float r[L::E], scale[L::E];
  uint32_t bad = 0;
#pragma unroll
  for (int e = 0; e < L::E; e++) {
    const uint32_t w = e < 2 * (L::E / 4) ? (e < L::E / 4 ? m.x : m.y) : (e < 3 * (L::E / 4) ? m.z : m.w);
    const uint32_t b = L::E == 4 ? w : (e & 1 ? w >> 16 : w & 0xffffu);
    factors<DT>(b, r[e], scale[e]);
    if (b >= L::INF) bad |= 1u << e;
    if (p.scale && rank == 0 && ty == 0 && e < left) p.scale[col + e] = scale[e];
  }

  for (int64_t t0 = r0; t0 < r1; t0 += TR) {
    Vec<DT> v[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const int64_t row = t0 + ty * 4 + j;
      v[j].u = make_uint4(0, 0, 0, 0);
      if (row < r1 && left > 0) v[j] = load_vec<DT, VEC>(x + row * p.ldx, left);
    }
    int w[4][L::E];
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
      for (int e = 0; e < L::E; e++) w[j][e] = whole<DT>(L::up(v[j].e[e]), r[e], !(bad >> e & 1));
    if (p.values) {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int64_t row = t0 + ty * 4 + j;
        if (row >= r1 || left <= 0) continue;
        typename L::T* o = static_cast<typename L::T*>(p.values) + row * p.ldv + col;
        Vec<DT> y;
#pragma unroll
        for (int e = 0; e < L::E; e++) y.e[e] = L::down(__fmul_rn((float)w[j][e], scale[e]));
        if (p.vec_v && left >= L::E) {
          *reinterpret_cast<uint4*>(o) = y.u;
        } else {
#pragma unroll
          for (int e = 0; e < L::E; e++)
            if (e < left) o[e] = y.e[e];
        }
      }
    }
    if (p.q) {
      __syncthreads();  // the tile's last readers are done
#pragma unroll
      for (int e = 0; e < L::E; e++) tile[tx * L::E + e][ty] = pack4(w[0][e], w[1][e], w[2][e], w[3][e]);
      __syncthreads();
      const int lane = threadIdx.x & 31;
      const int64_t row = t0 + lane * 4;
      const int64_t c0 = ((int64_t)blockIdx.x / S) * CW;
      for (int c = threadIdx.x >> 5; c < CW; c += QT / 32) {
        if (c0 + c >= p.cols || row >= p.rows) continue;
        const uint32_t u = tile[c][lane];
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
  cl.sync();  // the others may still read this CTA's maxima
}

template <int DT>
cudaError_t rows_launch(const QuantParams& p, cudaStream_t s) {
  constexpr int E = Elem<DT>::E;
  if (!p.vec_x) {
    quant_rows_twice<DT, false><<<(unsigned)p.rows, QT, 0, s>>>(p);
    return cudaGetLastError();
  }
  const int64_t nv = (p.cols + E - 1) / E;
  auto grid = [&](int tpr) { return (unsigned)((p.rows + QT / tpr - 1) / (QT / tpr)); };
  if (nv <= 32) quant_rows<DT, 32, 1><<<grid(32), QT, 0, s>>>(p);
  else if (nv <= 64) quant_rows<DT, 32, 2><<<grid(32), QT, 0, s>>>(p);
  else if (nv <= 128) quant_rows<DT, 32, 4><<<grid(32), QT, 0, s>>>(p);
  else if (nv <= 256) quant_rows<DT, QT, 1><<<grid(QT), QT, 0, s>>>(p);
  else if (nv <= 512) quant_rows<DT, QT, 2><<<grid(QT), QT, 0, s>>>(p);
  else if (nv <= 1024) quant_rows<DT, QT, 4><<<grid(QT), QT, 0, s>>>(p);
  else if (nv <= 2048) quant_rows<DT, QT, 8><<<grid(QT), QT, 0, s>>>(p);
  else quant_rows_twice<DT, true><<<(unsigned)p.rows, QT, 0, s>>>(p);
  return cudaGetLastError();
}

template <int DT, bool VEC>
cudaError_t cols_launch(const QuantParams& p, int nsm, cudaStream_t s) {
  constexpr int CW = 8 * Elem<DT>::E;
  const int64_t strips = (p.cols + CW - 1) / CW, tiles = (p.rows + TR - 1) / TR;
  // split the rows until there are a few CTAs for each SM, two tiles or more each
  int S = 1;
  while (S < 8 && strips * S < 4 * (int64_t)nsm && tiles >= 4 * S) S *= 2;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)S;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(strips * S));
  cfg.blockDim = dim3(QT);
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, quant_cols<DT, VEC>, p);
}

template <int DT>
cudaError_t quant_launch(int axis, const QuantParams& p, int nsm, cudaStream_t s) {
  if (axis == 0) return rows_launch<DT>(p, s);
  return p.vec_x ? cols_launch<DT, true>(p, nsm, s) : cols_launch<DT, false>(p, nsm, s);
}

}  // namespace

cudaError_t launch_quant8(int dtype, int axis, const QuantParams& p, int nsm, cudaStream_t s) {
  if (dtype == PEAT_F32) return quant_launch<PEAT_F32>(axis, p, nsm, s);
  if (dtype == PEAT_F16) return quant_launch<PEAT_F16>(axis, p, nsm, s);
  return quant_launch<PEAT_BF16>(axis, p, nsm, s);
}

}  // namespace peat
