// Rounding of a matrix to 4-bit floating point with a scale for each block of 32
// (a power of two) or 16 (an 8-bit float, below a float32 scale of the row).
//
// The blocks lie along the product's axis: along the rows (axis 0), or down the
// columns, whose codes come out transposed (axis 1).
//
// Bound by memory.  A lane holds one 16-byte vector of a row, so a block's
// maximum is a few shuffles; down the columns a thread holds the whole block.
#include <algorithm>
#include <type_traits>

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

// where a row's outputs lie
template <int DT>
struct Out4 {
  uint8_t* q;            // or null
  uint8_t* block_scale;  // or null
  typename Elem<DT>::T* values;  // or null
};
template <int DT>
__device__ __forceinline__ Out4<DT> out_of(const Quant4Params& p, int64_t row, bool margin) {
  Out4<DT> o;
  o.q = p.q && row < p.rows ? p.q + row * p.ldq : nullptr;
  o.block_scale = p.block_scale && !margin ? p.block_scale + scale_at(row, 0, p.tiles) : nullptr;
  o.values = p.values ? static_cast<typename Elem<DT>::T*>(p.values) + row * p.ldv : nullptr;
  return o;
}

// one vector of a row: codes, block scale, values; all lanes of a warp together
template <int DT, int FMT, int G, bool GRID, typename Col>
__device__ __forceinline__ void put_vec(const Quant4Params& p, uint4 v, const Out4<DT>& o, Col col, Col left, const Row4& r,
                                        const float* reciprocals) {
  using L = Elem<DT>;
  constexpr int LANES = F4<FMT>::BLOCK / L::E;  // that have a block
  uint32_t top = vec_top<DT>(v);
#pragma unroll
  for (int n = 1; n < LANES; n *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, n));
  const bool finite = top < L::INF;
  const Block4 b = block4<FMT>(L::mag(top), finite, r, reciprocals);
  float x[L::E];
  unpack<DT>(v, x);
#pragma unroll
  for (int e = 0; e < L::E; e++) x[e] = scaled4<FMT>(x[e], r, b);
  uint32_t c;
  if constexpr (L::E == 8) c = codes8(x);
  else c = codes4(x[0], x[1], x[2], x[3]);
  c = coded<FMT>(finite, b) ? c : 0;
  if (o.q && col < (Col)p.width) {
    if (L::E == 8) *reinterpret_cast<uint32_t*>(o.q + col / 2) = c;
    else *reinterpret_cast<uint16_t*>(o.q + col / 2) = (uint16_t)c;
  }
  if (o.block_scale && (threadIdx.x & (LANES - 1)) == 0 && col < (Col)(p.tiles * 4 * F4<FMT>::BLOCK)) {
    const Col block = col / F4<FMT>::BLOCK;
    o.block_scale[(int64_t)(block >> 2) * SCALE_TILE + (block & 3)] = (uint8_t)b.byte;
  }
  if (o.values) {
    float y[L::E], four[4];
#pragma unroll
    for (int e = 0; e < L::E; e += 4) {
      decoded4<FMT>(c >> (4 * e), r, b, four);
#pragma unroll
      for (int i = 0; i < 4; i++) y[e + i] = four[i];
    }
    if constexpr (GRID) {
      if (left > 0) __stcs(reinterpret_cast<uint4*>(o.values + col), pack<DT>(y));
    } else {
      uint4 none = make_uint4(0, 0, 0, 0);
      store_values<DT, G>(o.values + col, y, p.vec_v, left, none, true, true);
    }
  }
}

// (16384 x 4096 bfloat16 to codes: mxfp4 36 us, nvfp4 44, bound by the bytes under way:
// two vectors a thread and twice the threads took 43 and 51.)
// Rows: TPR threads have a unit, NV vectors each, one unit after another with the
// next one's loads under way.  A unit is a row, or with mxfp4, which needs nothing
// of the row beyond its blocks, one of `pieces` of it.  LONG (nvfp4): rows that
// these threads do not hold, read twice, from L2 the second time.  GRID: x's and
// values' rows start on 16-byte boundaries and are whole vectors.
template <int DT, int FMT, int TPR, int NV, bool GRID, bool LONG>
__global__ void __launch_bounds__(QT, NV > 2 ? 2 : 4) quant4_rows(Quant4Params p, int64_t rows, int pieces, int64_t step_row, int step_piece) {
  using L = Elem<DT>;
  using T = typename L::T;
  using Col = std::conditional_t<LONG, int64_t, int>;
  pdl_wait();
  pdl_trigger();
  constexpr int G = TPR < 32 ? TPR : 32, GROUPS = QT / TPR;
  constexpr Col PIECE = TPR * NV * L::E;
  __shared__ uint32_t part[2][QT / 32];
  __shared__ float reciprocals[FMT == PEAT_NVFP4 ? RECIPROCALS : 1];
  if (FMT == PEAT_NVFP4) {
    make_reciprocals(reciprocals);
    __syncthreads();
  }
  const int lane = threadIdx.x % TPR;
  const Source<DT, GRID> source(p.x, p.rows, p.cols, p.ldx);
  const Col wide = (Col)(p.tiles * 4 * F4<FMT>::BLOCK);  // with the margin of the scales' tiles
  uint4 v[NV];
  auto load = [&](int64_t row, Col at) {
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const Col cols = row < p.rows ? (Col)p.cols : 0;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const Col col = at + (i * TPR + lane) * L::E;
      v[i] = make_uint4(0, 0, 0, 0);
      if constexpr (GRID) {
        if (col < cols) v[i] = source.load(x + col);
      } else {
        if (source.whole(x + col, cols - col)) v[i] = source.load(x + col);
        else if (col < cols) v[i] = load_edge<DT>(x + col, cols - col);
      }
    }
  };
  // the units of this CTA's first group, and how many steps it takes over them
  const int64_t first = (int64_t)blockIdx.x * GROUPS, units = rows * pieces, step = (int64_t)gridDim.x * GROUPS;
  int64_t unit = first + threadIdx.x / TPR;
  int64_t row = pieces == 1 ? unit : unit / pieces;
  int piece = pieces == 1 ? 0 : (int)(unit - row * pieces);
  auto after = [&](int64_t& r, int& q) {
    r += step_row;
    q += step_piece;
    if (q >= pieces) q -= pieces, r++;
  };
  if (!LONG) load(row, piece * PIECE);
  int turn = 0;
  for (int64_t at_unit = first; at_unit < units; at_unit += step, turn ^= 1) {
    const bool margin = row >= rows;  // (a group beyond the last unit)
    const int64_t here = row;
    const Col at0 = LONG ? 0 : piece * PIECE;
    after(row, piece);
    uint4 w[NV];
    if (!LONG) {
#pragma unroll
      for (int i = 0; i < NV; i++) w[i] = v[i];
      if (at_unit + step < units) load(row, piece * PIECE);
    }
    Row4 r = row4<FMT>(0.0f, true);
    if (FMT == PEAT_NVFP4) {
      uint4 m = make_uint4(0, 0, 0, 0);
      if (LONG) {
        for (Col at = 0; at < (Col)p.cols; at += PIECE) {
          load(here, at);
#pragma unroll
          for (int i = 0; i < NV; i++) m = mag_max<DT>(m, v[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NV; i++) m = mag_max<DT>(m, w[i]);
      }
      uint32_t top = mag_fold<DT>(m);
      if (TPR >= 32) {
        top = __reduce_max_sync(0xffffffffu, top);
      } else {
#pragma unroll
        for (int o = G / 2; o; o /= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      }
      if (TPR > 32) {
        if ((threadIdx.x & 31) == 0) part[turn][threadIdx.x >> 5] = top;
        __syncthreads();
        const int w0 = threadIdx.x / TPR * (TPR / 32);
#pragma unroll
        for (int k = 0; k < TPR / 32; k++) top = max(top, part[turn][w0 + k]);
      }
      r = row4<FMT>(L::mag(top), top < L::INF);
      if (p.scale && lane == 0 && here < p.rows) p.scale[here] = r.s;
    }
    const Out4<DT> o = out_of<DT>(p, here, margin);
    const Col cols = here < p.rows ? (Col)p.cols : -16;
    for (Col at = at0; at < (LONG ? wide : at0 + 1); at += PIECE) {
      if (LONG) {
        load(here, at);
#pragma unroll
        for (int i = 0; i < NV; i++) w[i] = v[i];
      }
#pragma unroll
      for (int i = 0; i < NV; i++) {
        const Col begin = at + i * TPR * L::E, col = begin + lane * L::E;
        if (begin < wide) put_vec<DT, FMT, G, GRID, Col>(p, w[i], o, col, here < p.rows ? cols - col : -16, r, reciprocals);
      }
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
  __shared__ float reciprocals[FMT == PEAT_NVFP4 ? RECIPROCALS : 1];
  if (FMT == PEAT_NVFP4) {
    make_reciprocals(reciprocals);
    __syncthreads();
  }
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
      const Block4 b = block4<FMT>(L::mag(top), finite, r, reciprocals);
#pragma unroll
      for (int j = 0; j < BLOCK / 8; j++) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] = scaled4<FMT>(number(n * BLOCK + j * 8 + e), r, b);
        code[n * (BLOCK / 8) + j] = coded<FMT>(finite, b) ? codes8(y) : 0;
      }
      const int64_t block = r0 / BLOCK + n;
      if (p.block_scale && block < p.tiles * 4) p.block_scale[scale_at(col, block, p.tiles)] = (uint8_t)b.byte;
      if (p.values && col < p.cols) {
        T* o = static_cast<T*>(p.values) + (r0 + n * BLOCK) * p.ldv + col;
#pragma unroll
        for (int j = 0; j < BLOCK; j += 4) {
          float v[4];
          decoded4<FMT>(code[(n * BLOCK + j) / 8] >> (4 * (j & 4)), r, b, v);
#pragma unroll
          for (int e = 0; e < 4; e++)
            if (n * BLOCK + j + e < rows) {
              const float y = v[e];
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

template <int DT, int FMT, int TPR, int NV, bool LONG = false>
cudaError_t rows_of(const Quant4Params& p, int nsm, cudaStream_t s) {
  constexpr int E = Elem<DT>::E, GROUPS = QT / TPR;
  const int64_t rows = p.block_scale ? (p.rows + 127) / 128 * 128 : p.rows;
  const int64_t wide = p.tiles * 4 * F4<FMT>::BLOCK, piece = (int64_t)TPR * NV * E;
  const int pieces = FMT == PEAT_MXFP4 ? (int)((wide + piece - 1) / piece) : 1;
  // as many CTAs as are at work at once
  const int64_t grid = std::min<int64_t>((rows * pieces + GROUPS - 1) / GROUPS, (NV > 2 ? 2 : 4) * (int64_t)nsm), step = grid * GROUPS;
  const bool all = p.vec_x && (!p.values || p.vec_v) && p.cols % E == 0;
  return launch_dependent(all ? quant4_rows<DT, FMT, TPR, NV, true, LONG> : quant4_rows<DT, FMT, TPR, NV, false, LONG>,
                          dim3((unsigned)grid), QT, 0, s, p, rows, pieces, step / pieces, (int)(step % pieces));
}
template <int DT, int FMT>
cudaError_t rows(const Quant4Params& p, int nsm, cudaStream_t s) {
  const int64_t vecs = p.tiles * 4 * F4<FMT>::BLOCK / Elem<DT>::E;
  if (vecs <= 16) return rows_of<DT, FMT, 16, 1>(p, nsm, s);
  if (vecs <= 32) return rows_of<DT, FMT, 32, 1>(p, nsm, s);
  if (vecs <= 64) return rows_of<DT, FMT, 32, 2>(p, nsm, s);
  if (FMT == PEAT_MXFP4 || vecs <= 128) return rows_of<DT, FMT, 32, 4>(p, nsm, s);
  if constexpr (FMT == PEAT_NVFP4) {
    if (vecs <= 256) return rows_of<DT, FMT, 64, 4>(p, nsm, s);
    if (vecs <= 512) return rows_of<DT, FMT, 128, 4>(p, nsm, s);
    if (vecs <= 1024) return rows_of<DT, FMT, 256, 4>(p, nsm, s);
    return rows_of<DT, FMT, 256, 4, true>(p, nsm, s);
  }
  return cudaErrorNotSupported;
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
