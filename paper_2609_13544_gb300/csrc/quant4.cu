// Rounding of a matrix to 4-bit floating point with a scale for each block of 32
// (a power of two) or 16 (an 8-bit float, below a float32 scale of the row).
//
// The blocks lie along the product's axis: along the rows (axis 0), or down the
// columns, whose codes come out transposed (axis 1).
//
// Bound by memory.  A lane holds one 16-byte vector of a row, so a block's
// maximum is a few shuffles; down the columns a thread holds the whole block.
#include <algorithm>

#include "f4.cuh"
#include "matrix_vec.cuh"
#include "peat_internal.h"

namespace peat {
namespace {

constexpr int QT = 256;  // threads of a CTA

// the largest of two magnitudes' patterns of a vector
template <int DT>
__device__ __forceinline__ uint32_t vec_top(uint4 v) {
  return mag_fold<DT>(mag_max<DT>(make_uint4(0, 0, 0, 0), v));
}

// one vector of a row: codes, block scale, values; all lanes of a warp together
template <int DT, int FMT, int G>
__device__ __forceinline__ void put_vec(const Quant4Params& p, uint4 v, int64_t row, int64_t col, const Row4& r) {
  using L = Elem<DT>;
  constexpr int LANES = F4<FMT>::BLOCK / L::E;  // that have a block
  uint32_t top = vec_top<DT>(v);
#pragma unroll
  for (int o = 1; o < LANES; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  const bool finite = top < L::INF;
  const Block4 b = block4<FMT>(L::mag(top), finite, r);
  const bool good = FMT == PEAT_MXFP4 ? finite : b.r > 0.0f;
  float x[L::E];
  unpack<DT>(v, x);
#pragma unroll
  for (int e = 0; e < L::E; e++) x[e] = good ? scaled4<FMT>(x[e], r, b) : 0.0f;
  uint32_t c;
  if constexpr (L::E == 8) c = codes8(x);
  else c = codes4(x[0], x[1], x[2], x[3]);
  if (p.q && row < p.rows && col < p.width) {
    uint8_t* q = p.q + row * p.ldq + col / 2;
    if (L::E == 8) *reinterpret_cast<uint32_t*>(q) = c;
    else *reinterpret_cast<uint16_t*>(q) = (uint16_t)c;
  }
  const int64_t block = col / F4<FMT>::BLOCK;
  if (p.block_scale && (threadIdx.x & (LANES - 1)) == 0 && block < p.tiles * 4)
    p.block_scale[scale_at(row, block, p.tiles)] = (uint8_t)b.byte;
  if (p.values) {
    float y[L::E], four[4];
#pragma unroll
    for (int e = 0; e < L::E; e += 4) {
      values4(c >> (4 * e), four);
#pragma unroll
      for (int i = 0; i < 4; i++) y[e + i] = value4<FMT>(four[i], r, b);
    }
    uint4 none = make_uint4(0, 0, 0, 0);
    store_values<DT, G>(static_cast<typename L::T*>(p.values) + row * p.ldv + col, y, p.vec_v,
                        row < p.rows ? p.cols - col : -16, none, true, true);
  }
}

// Rows: TPR threads have a row, NV vectors each at a time.  nvfp4 needs the row's
// largest magnitude before the first code: a row that TPR NV vectors do not hold
// is read twice (from L2 the second time).  mxfp4 takes longer rows in pieces,
// one a CTA.
template <int DT, int FMT, int TPR, int NV, bool GRID>
__global__ void __launch_bounds__(QT) quant4_rows(Quant4Params p, int64_t groups) {
  using L = Elem<DT>;
  pdl_wait();
  pdl_trigger();
  constexpr int G = TPR < 32 ? TPR : 32;
  __shared__ uint32_t part[QT / 32];
  const int lane = threadIdx.x % TPR;
  const int64_t group = blockIdx.x % groups;  // of rows
  const int64_t piece0 = blockIdx.x / groups, pieces = gridDim.x / groups;
  const int64_t row = group * (QT / TPR) + threadIdx.x / TPR;
  const Source<DT, GRID> source(p.x, p.rows, p.cols, p.ldx);
  const typename L::T* x = static_cast<const typename L::T*>(p.x) + row * p.ldx;
  const int64_t cols = row < p.rows ? p.cols : 0;
  const int64_t wide = p.tiles * 4 * F4<FMT>::BLOCK;  // with the margin of the scales' tiles
  auto load = [&](int64_t at, uint4 (&v)[NV]) {
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int64_t col = at + (int64_t)(i * TPR + lane) * L::E;
      v[i] = make_uint4(0, 0, 0, 0);
      if (source.whole(x + col, cols - col)) v[i] = source.load(x + col);
      else if (col < cols) v[i] = load_edge<DT>(x + col, cols - col);
    }
  };
  constexpr int64_t PIECE = (int64_t)TPR * NV * L::E;
  uint4 v[NV];
  Row4 r = row4<FMT>(0.0f, true);
  if (FMT == PEAT_NVFP4) {
    uint4 m = make_uint4(0, 0, 0, 0);
    int64_t at = 0;
    do {
      load(at, v);
#pragma unroll
      for (int i = 0; i < NV; i++) m = mag_max<DT>(m, v[i]);
      at += PIECE;
    } while (at < p.cols);
    uint32_t top = mag_fold<DT>(m);
#pragma unroll
    for (int o = G / 2; o; o /= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (TPR > 32) {
      if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
      __syncthreads();
      const int w0 = threadIdx.x / TPR * (TPR / 32);
#pragma unroll
      for (int w = 0; w < TPR / 32; w++) top = max(top, part[w0 + w]);
    }
    r = row4<FMT>(L::mag(top), top < L::INF);
    if (p.scale && lane == 0 && row < p.rows) p.scale[row] = r.s;
  }
  for (int64_t at = piece0 * PIECE; at < wide; at += pieces * PIECE) {
    if (FMT == PEAT_MXFP4 || p.cols > PIECE) load(at, v);
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int64_t col = at + (int64_t)(i * TPR + lane) * L::E;
      if (at + (int64_t)i * TPR * L::E < wide) put_vec<DT, FMT, G>(p, v[i], row, col, r);
    }
  }
}

// Columns: a warp has 32 rows of 32 columns (16-bit types by pairs: 64), a thread
// the blocks of its own, 16 bytes of codes each.
template <int DT, int FMT, bool PAIRS>
__global__ void __launch_bounds__(QT) quant4_columns(Quant4Params p, int64_t wide) {
  using L = Elem<DT>;
  using T = typename L::T;
  pdl_wait();
  pdl_trigger();
  for (int64_t i = (int64_t)blockIdx.x * QT + threadIdx.x; i < p.zero_n; i += (int64_t)gridDim.x * QT) p.zero[i] = 0;
  constexpr int C = PAIRS ? 2 : 1, BLOCK = F4<FMT>::BLOCK, NB = 32 / BLOCK;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c0 = ((int64_t)blockIdx.x % wide) * (32 * C) + lane * C;
  const int64_t r0 = ((int64_t)blockIdx.x / wide) * (QT / 32 * 32) + warp * 32;
  const T* x = static_cast<const T*>(p.x) + r0 * p.ldx + c0;
  uint32_t w[32];  // (16-bit: of C columns)
  const int64_t rows = min((int64_t)32, p.rows - r0), cols = p.cols - c0;
#pragma unroll
  for (int i = 0; i < 32; i++) {
    w[i] = 0;
    if (i >= rows || cols <= 0) continue;
    if (DT == PEAT_F32) w[i] = __ldg(reinterpret_cast<const uint32_t*>(x + i * p.ldx));
    else if (PAIRS && cols > 1) w[i] = __ldg(reinterpret_cast<const uint32_t*>(x + i * p.ldx));
    else w[i] = __ldg(reinterpret_cast<const uint16_t*>(x + i * p.ldx));
  }
#pragma unroll
  for (int c = 0; c < C; c++) {
    const int64_t col = c0 + c;
    Row4 r = row4<FMT>(0.0f, true);
    if (FMT == PEAT_NVFP4) {
      const uint32_t top = col < p.cols ? __ldcg(p.colmax + col) : 0;
      r = row4<FMT>(L::mag(top), top < L::INF);
      if (p.scale && r0 == 0 && col < p.cols) p.scale[col] = r.s;
    }
    auto bits = [&](int i) { return DT == PEAT_F32 ? w[i] : (c ? w[i] >> 16 : w[i] & 0xffffu); };
    auto number = [&](int i) {
      const uint32_t b = bits(i);
      if (DT == PEAT_F32) return __uint_as_float(b);
      if (DT == PEAT_BF16) return __uint_as_float(b << 16);
      return __half2float(__ushort_as_half((unsigned short)b));
    };
    uint32_t code[4];
#pragma unroll
    for (int n = 0; n < NB; n++) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < BLOCK; i++) top = max(top, bits(n * BLOCK + i) & (DT == PEAT_F32 ? 0x7fffffffu : 0x7fffu));
      const bool finite = top < L::INF;
      const Block4 b = block4<FMT>(L::mag(top), finite, r);
      const bool good = FMT == PEAT_MXFP4 ? finite : b.r > 0.0f;
#pragma unroll
      for (int j = 0; j < BLOCK / 8; j++) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] = good ? scaled4<FMT>(number(n * BLOCK + j * 8 + e), r, b) : 0.0f;
        code[n * (BLOCK / 8) + j] = codes8(y);
      }
      const int64_t block = r0 / BLOCK + n;
      if (p.block_scale && block < p.tiles * 4) p.block_scale[scale_at(col, block, p.tiles)] = (uint8_t)b.byte;
      if (p.values && col < p.cols) {
        T* o = static_cast<T*>(p.values) + (r0 + n * BLOCK) * p.ldv + col;
#pragma unroll
        for (int j = 0; j < BLOCK; j += 4) {
          float v[4];
          values4(code[(n * BLOCK + j) / 8] >> (4 * (j & 4)), v);
#pragma unroll
          for (int e = 0; e < 4; e++)
            if (n * BLOCK + j + e < rows) {
              const float y = value4<FMT>(v[e], r, b);
              if constexpr (DT == PEAT_F32) o[(j + e) * p.ldv] = y;
              else if constexpr (DT == PEAT_F16) o[(j + e) * p.ldv] = __float2half_rn(y);
              else o[(j + e) * p.ldv] = __float2bfloat16_rn(y);
            }
        }
      }
    }
    // whole blocks: 16 or 8 bytes of a 16-byte unit
    const int64_t left = (p.width - r0) / 2;
    if (p.q && col < p.cols && left > 0) {
      uint8_t* q = p.q + col * p.ldq + r0 / 2;
      if (left >= 16) *reinterpret_cast<uint4*>(q) = make_uint4(code[0], code[1], code[2], code[3]);
      else *reinterpret_cast<uint2*>(q) = make_uint2(code[0], code[1]);
    }
  }
}

template <int DT, int FMT, int TPR, int NV>
cudaError_t rows_of(const Quant4Params& p, int nsm, cudaStream_t s) {
  constexpr int E = Elem<DT>::E;
  const int64_t rows = p.block_scale ? (p.rows + 127) / 128 * 128 : p.rows;
  const int64_t groups = (rows + QT / TPR - 1) / (QT / TPR);
  // pieces of a row where it is taken apart: until the SMs have eight CTAs each
  const int64_t wide = p.tiles * 4 * F4<FMT>::BLOCK, piece = (int64_t)TPR * NV * E;
  int64_t pieces = 1;
  if (FMT == PEAT_MXFP4) pieces = std::max<int64_t>(1, std::min<int64_t>((wide + piece - 1) / piece, (8 * (int64_t)nsm + groups - 1) / groups));
  const dim3 grid((unsigned)(groups * pieces));
  if (p.vec_x) return launch_dependent(quant4_rows<DT, FMT, TPR, NV, true>, grid, QT, 0, s, p, groups);
  return launch_dependent(quant4_rows<DT, FMT, TPR, NV, false>, grid, QT, 0, s, p, groups);
}
template <int DT, int FMT>
cudaError_t rows(const Quant4Params& p, int nsm, cudaStream_t s) {
  const int64_t vecs = p.tiles * 4 * F4<FMT>::BLOCK / Elem<DT>::E;
  if (vecs <= 16) return rows_of<DT, FMT, 16, 1>(p, nsm, s);
  if (vecs <= 32) return rows_of<DT, FMT, 32, 1>(p, nsm, s);
  if (vecs <= 64) return rows_of<DT, FMT, 32, 2>(p, nsm, s);
  if (FMT == PEAT_MXFP4 || vecs <= 128) return rows_of<DT, FMT, 32, 4>(p, nsm, s);
  if (vecs <= 512) return rows_of<DT, FMT, 128, 4>(p, nsm, s);
  if (vecs <= 1024) return rows_of<DT, FMT, 256, 4>(p, nsm, s);
  return rows_of<DT, FMT, 256, 8>(p, nsm, s);
}
template <int DT, int FMT>
cudaError_t columns(const Quant4Params& p, cudaStream_t s) {
  constexpr bool SMALL = DT != PEAT_F32;
  const bool pairs = SMALL && p.pairs;
  const int64_t cols = p.block_scale ? (p.cols + 127) / 128 * 128 : p.cols;
  const int64_t height = p.tiles * 4 * F4<FMT>::BLOCK, wide = (cols + (pairs ? 63 : 31)) / (pairs ? 64 : 32);
  const dim3 grid((unsigned)(wide * ((height + QT - 1) / QT)));
  if (pairs) return launch_dependent(quant4_columns<DT, FMT, SMALL>, grid, QT, 0, s, p, wide);
  return launch_dependent(quant4_columns<DT, FMT, false>, grid, QT, 0, s, p, wide);
}
template <int DT>
cudaError_t of_type(int format, int axis, const Quant4Params& p, int nsm, cudaStream_t s) {
  if (format == PEAT_MXFP4) return axis ? columns<DT, PEAT_MXFP4>(p, s) : rows<DT, PEAT_MXFP4>(p, nsm, s);
  return axis ? columns<DT, PEAT_NVFP4>(p, s) : rows<DT, PEAT_NVFP4>(p, nsm, s);
}

}  // namespace

cudaError_t launch_quant4(int dtype, int format, int axis, const Quant4Params& p, int nsm, cudaStream_t s) {
  switch (dtype) {
    case PEAT_F32: return of_type<PEAT_F32>(format, axis, p, nsm, s);
    case PEAT_F16: return of_type<PEAT_F16>(format, axis, p, nsm, s);
    default: return of_type<PEAT_BF16>(format, axis, p, nsm, s);
  }
}

}  // namespace peat
