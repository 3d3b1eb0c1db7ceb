// Rounding of a matrix to 8-bit integers with one scale for each row or column.
//
// Over a row (or column): amax = max |x|, scale = amax / 127, r = 127 / amax,
// q = rint(x r), all float32.  The maximum is one that keeps NaNs, so it finds
// both amax and whether the row is finite; it is handed on as a bit pattern
// without sign, which order as the magnitudes do, infinities and NaNs on top.
//
// Bound by memory: a row is read once and kept in registers between the
// maximum and the rounding; columns are read twice.
#include <algorithm>

#include "matrix_vec.cuh"
#include "ops_internal.h"
#include "peat_internal.h"

namespace peat {
namespace {

// a vector's integers (in float32, see whole) from its row's factor
template <int DT, bool FINITE>
__device__ __forceinline__ void wholes(uint4 v, float r, float (&w)[Elem<DT>::E]) {
  float x[Elem<DT>::E];
  unpack<DT>(v, x);
#pragma unroll
  for (int e = 0; e < Elem<DT>::E; e++) w[e] = whole(x[e], r, FINITE);
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
__device__ __forceinline__ void clear_earlier(const QuantParams& p) {
  const int64_t n = (int64_t)gridDim.x * gridDim.y * QT;
  for (int64_t i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * QT + threadIdx.x; i < p.zero2_n; i += n) p.zero2[i] = 0;
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

// integers (q, or the packed operand), values and the sum of squares of one
// vector of a row; all lanes of a warp together
template <int DT, bool PACK, int G>
__device__ __forceinline__ void put_row_vec(const QuantParams& p, uint4 v, int64_t row, int64_t col, float r,
                                            float scale, bool finite, unsigned& most, uint4& carry, bool first, bool last) {
  using L = Elem<DT>;
  float w[L::E];
  if (finite) wholes<DT, true>(v, r, w);
  else wholes<DT, false>(v, r, w);
  if (PACK) {
    if (col < (int64_t)p.kb * 64) {
      char* d = packed_at(p, row, col);
      if (L::E == 8)
        *reinterpret_cast<uint4*>(d) = make_uint4(half_pair(w[0], w[1]), half_pair(w[2], w[3]),
                                                  half_pair(w[4 % L::E], w[5 % L::E]), half_pair(w[6 % L::E], w[7 % L::E]));
      else
        *reinterpret_cast<uint2*>(d) = make_uint2(half_pair(w[0], w[1]), half_pair(w[2], w[3]));
    }
    if (p.norms) {  // a warp's vectors are 256 k, or half of them
      float ss = 0.0f;  // (exact: below 2^17)
#pragma unroll
      for (int e = 0; e < L::E; e++) ss = fmaf(number(w[e]), number(w[e]), ss);
      most = max(most, __reduce_add_sync(0xffffffffu, (unsigned)ss));
    }
    return;
  }
  const int64_t left = row < p.rows ? p.cols - col : -16;
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
    store_values<DT, G>(static_cast<typename L::T*>(p.values) + row * p.ldv + col, y, p.vec_v, left, carry,
                        first, last);
  }
}

// Rows, `each` one after another by TPR threads with NV vectors each, held in
// registers between the maximum and the rounding.  PACK: into a packed operand,
// with zeros in its margins, and the largest sums of squares handed on once for
// all rows.  16384 x 4096 bfloat16 with values take 49 us, 5.5 TB/s; 11590 x 1749
// binary16 with values, rows off the grid, 40 (on it, x 1752: 17).
template <int DT, int TPR, int NV, bool PACK, bool GRID>
__global__ void __launch_bounds__(QT) quant_rows(QuantParams p, int each) {
  using L = Elem<DT>;
  begin(p);
  if (PACK) clear_earlier(p);
  __shared__ uint32_t part[2][QT / 32];
  const int lane = threadIdx.x % TPR;
  const int64_t row0 = ((int64_t)blockIdx.x * (QT / TPR) + threadIdx.x / TPR) * each;
  const Source<DT, GRID> source(p.x, p.rows, p.cols, p.ldx);
  const bool ragged = p.cols % L::E != 0 || !GRID;
  auto load = [&](int64_t row, uint4 (&v)[NV]) {
    const typename L::T* x = static_cast<const typename L::T*>(p.x) + row * p.ldx;
    const int64_t cols = row < p.rows ? p.cols : 0;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int64_t col = (int64_t)(i * TPR + lane) * L::E;
      v[i] = make_uint4(0, 0, 0, 0);
      if (source.whole(x + col, cols - col)) v[i] = source.load(x + col);
    }
    if (ragged) {
#pragma unroll
      for (int i = 0; i < NV; i++) {
        const int64_t col = (int64_t)(i * TPR + lane) * L::E;
        if (col < cols && !source.whole(x + col, cols - col)) v[i] = load_edge<DT>(x + col, cols - col);
      }
    }
  };
  unsigned most[NV];
#pragma unroll
  for (int i = 0; i < NV; i++) most[i] = 0;
  for (int it = 0; it < each; it++) {
    const int64_t row = row0 + it;
    uint4 v[NV];
    uint4 m = make_uint4(0, 0, 0, 0);
    load(row, v);
#pragma unroll
    for (int i = 0; i < NV; i++) m = mag_max<DT>(m, v[i]);
    const uint32_t group = TPR >= 32 ? 0xffffffffu : ((1u << (TPR & 31)) - 1u) << (threadIdx.x & 31 & ~(TPR - 1));
    uint32_t top = __reduce_max_sync(group, mag_fold<DT>(m));
    if (TPR > 32) {
      if ((threadIdx.x & 31) == 0) part[it & 1][threadIdx.x >> 5] = top;
      __syncthreads();
      top = __reduce_max_sync(0xffffffffu, part[it & 1][threadIdx.x & (QT / 32 - 1)]);
    }
    float r, scale;
    factors<DT>(top, r, scale);
    const bool finite = top < L::INF;
    if (lane == 0 && row < p.rows && p.scale) p.scale[row] = scale;
    uint4 carry = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NV; i++)
      put_row_vec<DT, PACK, (TPR < 32 ? TPR : 32)>(p, v[i], row, (int64_t)(i * TPR + lane) * L::E, r, scale, finite, most[i],
                                                   carry, TPR > 32 || i == 0, TPR > 32 || i == NV - 1);
  }
  if (PACK && p.norms && (threadIdx.x & 31) == 0) {
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int64_t first = (int64_t)(i * TPR + (lane & ~31)) * L::E;
      if (first < (int64_t)p.kb * 64)
        atomicMax(p.norms + (row0 >> 7) * p.kc * 2 + (L::E == 8 ? first / 256 * 2 : first / 128), most[i]);
    }
  }
  end(p);
}

// A row too long for the registers, by a CTA that reads it twice.
template <int DT, bool GRID>
__global__ void __launch_bounds__(QT) quant_long_rows(QuantParams p) {
  using L = Elem<DT>;
  begin(p);
  __shared__ uint32_t part[QT / 32];
  const int64_t row = blockIdx.x;
  const typename L::T* x = static_cast<const typename L::T*>(p.x) + row * p.ldx;
  const Source<DT, GRID> source(p.x, p.rows, p.cols, p.ldx);
  auto load = [&](int64_t col) {
    const int64_t left = p.cols - col;
    if (left <= 0) return make_uint4(0, 0, 0, 0);
    return source.whole(x + col, left) ? source.load(x + col) : load_edge<DT>(x + col, left);
  };
  uint4 m = make_uint4(0, 0, 0, 0);
#pragma unroll 4
  for (int64_t col = (int64_t)threadIdx.x * L::E; col < p.cols; col += QT * L::E) m = mag_max<DT>(m, load(col));
  uint32_t top = __reduce_max_sync(0xffffffffu, mag_fold<DT>(m));
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
  __syncthreads();
  top = __reduce_max_sync(0xffffffffu, part[threadIdx.x & (QT / 32 - 1)]);
  float r, scale;
  factors<DT>(top, r, scale);
  if (p.scale && threadIdx.x == 0) p.scale[row] = scale;
  unsigned most = 0;
  uint4 carry = make_uint4(0, 0, 0, 0);
  for (int64_t first = 0; first < p.cols; first += QT * L::E) {
    const int64_t col = first + (int64_t)threadIdx.x * L::E;
    put_row_vec<DT, false, 32>(p, load(col), row, col, r, scale, top < L::INF, most, carry, true, true);
  }
  end(p);
}

// Columns, in two launches (one for few rows, QUANT_FEW_ROWS).  The first finds
// each column's maximum: a thread has a 16-byte vector of columns and walks down
// a share of the rows, the shares meet by atomic maxima of the patterns (order
// makes no difference to a maximum).  The second reads the matrix again (last
// rows first, which L2 may still hold, it takes no less time), in tiles of 128
// rows by 128 bytes, and writes the integers transposed through shared memory,
// 128 contiguous ones of a column at a time.  16384 x 4096 bfloat16 with values
// take 73 us, 5.5 TB/s of what the two launches read and write; with q alone 71.
// (One launch of clusters that keep a strip of columns to themselves, meet in
// distributed shared memory and read the strip again from L2 took 101 us: its
// phases wait for each other.)  Rows off the 16-byte grid take two aligned loads
// for a vector in the second launch, and their values go through shared memory,
// an element a lane: 16384 x 4095 take 173 us, with q alone 125, bound by
// instructions (two elements a lane: 202; values from the registers: 232).
template <int DT>
__global__ void __launch_bounds__(QT, 4) quant_colmax(QuantParams p, int vl, int64_t rows_each) {
  using L = Elem<DT>;
  begin(p);
  __shared__ uint4 part[QT];
  const int lx = threadIdx.x % vl, ly = threadIdx.x / vl, nl = QT / vl;
  const int64_t r0 = (int64_t)blockIdx.y * rows_each, r1 = min(p.rows, r0 + rows_each);
  const int64_t col = ((int64_t)blockIdx.x * vl + lx) * L::E, left = p.cols - col;
  const Source<DT, true> source(p.x, p.rows, p.cols, p.ldx);
  const typename L::T* x = static_cast<const typename L::T*>(p.x) + col;
  uint4 m = make_uint4(0, 0, 0, 0);
  constexpr int U = 8;  // rows in flight; past the end the last row again, which changes no maximum
  if (left >= L::E) {
    for (int64_t r = r0 + ly; r < r1; r += U * nl) {
      uint4 u[U];
#pragma unroll
      for (int i = 0; i < U; i++) u[i] = source.load(x + min(r + i * nl, r1 - 1) * p.ldx);
#pragma unroll
      for (int i = 0; i < U; i++) m = mag_max<DT>(m, u[i]);
    }
  } else {
    for (int64_t r = r0 + ly; r < r1 && left > 0; r += nl) m = mag_max<DT>(m, load_edge<DT>(x + r * p.ldx, left));
  }
  part[threadIdx.x] = m;
  __syncthreads();
  if (ly == 0 && left > 0) {
    for (int k = 1; k < nl; k++) m = mag_max<DT>(m, part[k * vl + lx]);
    const uint32_t w[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
    for (int e = 0; e < L::E; e++) {
      const uint32_t b = L::E == 4 ? w[e % 4] : (e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu);
      if (e < left) atomicMax(p.colmax + col + e, b);
    }
  }
  end(p);
}
// The same where rows are off the 16-byte grid: a thread has a column, an
// element a load (shifting vectors together takes more instructions: 48 us for
// 16384 x 4095 bfloat16, this 33).
template <int DT>
__global__ void __launch_bounds__(QT, 8) quant_colmax_off(QuantParams p, int64_t rows_each) {
  using T = typename Elem<DT>::T;
  begin(p);
  const int64_t r0 = (int64_t)blockIdx.y * rows_each, r1 = min(p.rows, r0 + rows_each);
  const int64_t col = (int64_t)blockIdx.x * QT + threadIdx.x;
  if (col < p.cols && r0 < r1) {
    const T* x = static_cast<const T*>(p.x) + col;
    constexpr int U = 16;
    uint32_t m = 0;
    auto bits = [](T v) {
      if constexpr (DT == PEAT_F32) return __float_as_uint(v);
      else return (uint32_t)*reinterpret_cast<const unsigned short*>(&v);
    };
    int64_t r = r0;
    for (; r + U <= r1; r += U) {
      uint32_t v[U];
#pragma unroll
      for (int i = 0; i < U; i++) v[i] = bits(__ldg(x + (r + i) * p.ldx));
#pragma unroll
      for (int i = 0; i < U; i++) m = max_word<DT>(m, v[i]);
    }
    for (; r < r1; r++) m = max_word<DT>(m, bits(__ldg(x + r * p.ldx)));
    atomicMax(p.colmax + col, m);
  }
  end(p);
}

constexpr int TR = 128;  // rows of a tile
template <int DT, bool PACK, bool GRID>
__global__ void __launch_bounds__(QT, 3) quant_cols(QuantParams p, int64_t rows_each) {
  using L = Elem<DT>;
  constexpr int CW = 8 * L::E;  // columns of a tile
  __shared__ __align__(16) float rs[CW], ss[CW];
  __shared__ uint32_t bads[2], tops[CW];
  // integers as bytes, or packed binary16; values
  __shared__ __align__(16) uint32_t tile[PACK ? CW * TR / 2 : TR * 32];
  __shared__ float squares[PACK ? QT / 32 : 1][CW];
  const int tx = threadIdx.x & 7, ty = threadIdx.x >> 3;
  const int64_t c0 = (int64_t)blockIdx.x * CW, col = c0 + tx * L::E;
  const int64_t left = p.cols - col;  // may be <= 0
  // (a packed operand's k go on to a whole block: zeros)
  const int64_t r0 = (int64_t)blockIdx.y * rows_each,
                r1 = min(PACK ? (int64_t)p.kb * 64 : p.rows, r0 + rows_each);
  const typename L::T* x = static_cast<const typename L::T*>(p.x) + col;
  begin(p);
  if (PACK) clear_earlier(p);
  // the other buffer of maxima is the next call's: zero again
  {
    const int64_t n = (int64_t)gridDim.x * gridDim.y * QT;
    for (int64_t i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * QT + threadIdx.x; i < p.zero_n; i += n) p.zero[i] = 0;
  }
  const Source<DT, GRID> source(p.x, p.rows, p.cols, p.ldx);
  auto load = [&](int64_t t0, uint4 (&v)[4]) {
    const typename L::T* q = x + (t0 + ty * 4) * p.ldx;
    const int64_t rows = min(r1, p.rows) - t0 - ty * 4;  // of the thread's four
    if (GRID && left >= L::E && rows >= 4) {
#pragma unroll
      for (int j = 0; j < 4; j++) v[j] = source.load(q + j * p.ldx);
      return;
    }
    int edges = 0;  // vectors to be read one by one
#pragma unroll
    for (int j = 0; j < 4; j++) {
      v[j] = make_uint4(0, 0, 0, 0);
      const bool whole = j < rows && source.whole(q + j * p.ldx, left);
      if (whole) v[j] = source.load(q + j * p.ldx);
      else if (j < rows && left > 0) edges |= 1 << j;
    }
    if (edges) {
#pragma unroll
      for (int j = 0; j < 4; j++)
        if (edges >> j & 1) v[j] = load_edge<DT>(q + j * p.ldx, left);
    }
  };
  if (!p.colmax) {  // few rows: every CTA finds its columns' maxima itself
    __shared__ uint4 part[QT / 32][8];
    uint4 m = make_uint4(0, 0, 0, 0);
    if (left > 0) {
      for (int64_t row = ty; row < p.rows; row += 4 * (QT / 8)) {
        uint4 u[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const typename L::T* q = x + min(row + j * (QT / 8), p.rows - 1) * p.ldx;
          u[j] = source.whole(q, left) ? source.load(q) : load_edge<DT>(q, left);
        }
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
    uint4 v[4];
    load(t0, v);
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
    if (!PACK && p.values) {
      typename L::T* o = static_cast<typename L::T*>(p.values) + t0 * p.ldv + c0;
      const int rows = (int)min((int64_t)TR, r1 - t0);
      if (!p.vec_v) __syncthreads();  // the tile's last readers are done
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int row = ty * 4 + j;
        float y[L::E];
#pragma unroll
        for (int e = 0; e < L::E; e++) y[e] = __fmul_rn(number(w[j][e]), scale[e]);
        if (p.vec_v) {
          uint4 none = make_uint4(0, 0, 0, 0);
          if (row < rows) store_values<DT, 32>(o + row * p.ldv + tx * L::E, y, true, left, none, true, true);
        } else {
          reinterpret_cast<uint4*>(tile)[row * 8 + tx] = pack<DT>(y);
        }
      }
      if (!p.vec_v) {  // rows off the grid: along them, an element a lane
        __syncthreads();
        const typename L::T* from = reinterpret_cast<const typename L::T*>(tile);
        const int lane = threadIdx.x & 31;
#pragma unroll 4
        for (int row = threadIdx.x >> 5; row < rows; row += QT / 32)
#pragma unroll
          for (int c = lane; c < CW; c += 32)
            if (c0 + c < p.cols) o[row * p.ldv + c] = from[row * CW + c];
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

template <int DT, bool PACK, bool GRID>
cudaError_t rows_launch(const QuantParams& p, int nsm, cudaStream_t s) {
  constexpr int E = Elem<DT>::E;
  const int64_t rows = PACK ? p.prows : p.rows, nv = ((PACK ? (int64_t)p.kb * 64 : p.cols) + E - 1) / E;
  auto go = [&](void (*kernel)(QuantParams, int), int tpr) {
    const int64_t groups = (rows + QT / tpr - 1) / (QT / tpr);
    int each = 1;  // rows of a thread group (of one block of 128): up to 8, while every SM has 4 CTAs
    while (each < 8 && groups / (2 * each) >= 4 * nsm) each *= 2;
    return launch_dependent(kernel, (unsigned)((groups + each - 1) / each), QT, 0, s, p, each);
  };
  // (short rows share a warp)
  if (nv <= 8) return go(quant_rows<DT, 8, 1, PACK, GRID>, 8);
  if (nv <= 16) return go(quant_rows<DT, 8, 2, PACK, GRID>, 8);
  if (nv <= 32) return go(quant_rows<DT, 8, 4, PACK, GRID>, 8);
  if (nv <= 64) return go(quant_rows<DT, 32, 2, PACK, GRID>, 32);
  if (nv <= 128) return go(quant_rows<DT, 32, 4, PACK, GRID>, 32);
  // a warp a row needs no meeting of warps, but takes longer for one row
  if (nv <= 256 && rows >= 8 * nsm) return go(quant_rows<DT, 32, 8, PACK, GRID>, 32);
  // (16384 x 4096 bfloat16 to q: 36 us, a CTA a row 42; into packed operands, with
  // 8 warps an SM then, 2 us slower for 2048 x 4096)
  if constexpr (!PACK && GRID)
    if (nv > 256 && nv <= 512 && rows >= 8 * nsm) return go(quant_rows<DT, 32, 16, false, true>, 32);
  if (nv <= 256) return go(quant_rows<DT, QT, 1, PACK, GRID>, QT);
  if (nv <= 512) return go(quant_rows<DT, QT, 2, PACK, GRID>, QT);
  if (nv <= 1024) return go(quant_rows<DT, QT, 4, PACK, GRID>, QT);
  if (nv <= 2048) return go(quant_rows<DT, QT, 8, PACK, GRID>, QT);
  return launch_dependent(quant_long_rows<DT, GRID>, (unsigned)p.rows, QT, 0, s, p);
}

template <int DT, bool GRID>
cudaError_t cols_launch(const QuantParams& p, bool maxima, int nsm, cudaStream_t s) {
  constexpr int E = Elem<DT>::E, CW = 8 * E;
  // one wave of as many CTAs as an SM holds, `least` rows or more for each
  auto shares = [&](int64_t rows, int64_t across, int64_t least, int64_t unit, int64_t resident, int64_t* each) {
    int64_t n = std::min(resident * nsm / across, (rows + least - 1) / least);
    if (maxima) n = std::min<int64_t>(n, 160);  // (690 shares' atomics on the same 256 columns took 50 us)
    n = std::max<int64_t>(1, std::min<int64_t>(n, 65535));
    *each = std::max<int64_t>(1, ((rows + n - 1) / n + unit - 1) / unit) * unit;
    return (unsigned)std::max<int64_t>(1, (rows + *each - 1) / *each);
  };
  int64_t each = 1;
  if (maxima) {
    if (p.rows == 0) return cudaSuccess;
    if constexpr (!GRID) {
      const int64_t wide = (p.cols + QT - 1) / QT;
      const unsigned ny = shares(p.rows, wide, 32, 16, 8, &each);
      return launch_dependent(quant_colmax_off<DT>, dim3((unsigned)wide, ny), QT, 0, s, p, each);
    }
    const int64_t nv = (p.cols + E - 1) / E;
    int vl = 8;
    while (vl < 32 && vl < nv) vl *= 2;  // wider CTAs would mean more shares of the rows, and atomics for each
    const int64_t wide = (nv + vl - 1) / vl;
    const unsigned ny = shares(p.rows, wide, 8 * (QT / vl), 1, 4, &each);
    return launch_dependent(quant_colmax<DT>, dim3((unsigned)wide, ny), QT, 0, s, p, vl, each);
  }
  if (p.packed) {
    const unsigned strips = (unsigned)(p.prows / CW), ny = shares((int64_t)p.kb * 64, strips, TR, TR, 3, &each);
    return launch_dependent(quant_cols<DT, true, GRID>, dim3(strips, ny), QT, 0, s, p, each);
  }
  const unsigned strips = (unsigned)((p.cols + CW - 1) / CW), ny = shares(p.rows, strips, TR, TR, 3, &each);
  return launch_dependent(quant_cols<DT, false, GRID>, dim3(strips, ny), QT, 0, s, p, each);
}

template <int DT, bool GRID>
cudaError_t quant_launch(int step, const QuantParams& p, int nsm, cudaStream_t s) {
  if (step != QUANT_ROWS) return cols_launch<DT, GRID>(p, step == QUANT_MAXIMA, nsm, s);
  return p.packed ? rows_launch<DT, true, GRID>(p, nsm, s) : rows_launch<DT, false, GRID>(p, nsm, s);
}
template <int DT>
cudaError_t quant_launch(int step, const QuantParams& p, int nsm, cudaStream_t s) {
  return p.vec_x ? quant_launch<DT, true>(step, p, nsm, s) : quant_launch<DT, false>(step, p, nsm, s);
}

}  // namespace

bool quant8_packs(int dtype, int axis, const QuantParams& p) {
  return axis == 1 || (int64_t)p.kb * 64 / (dtype == PEAT_F32 ? 4 : 8) <= 8 * QT;
}

cudaError_t launch_quant8(int dtype, int step, const QuantParams& p, int nsm, cudaStream_t s) {
  if (dtype == PEAT_F32) return quant_launch<PEAT_F32>(step, p, nsm, s);
  if (dtype == PEAT_F16) return quant_launch<PEAT_F16>(step, p, nsm, s);
  return quant_launch<PEAT_BF16>(step, p, nsm, s);
}

}  // namespace peat
