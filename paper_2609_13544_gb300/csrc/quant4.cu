// Rounding of a matrix to 4-bit floating point with a scale for each block of 32
// (a power of two) or 16 (an 8-bit float, below a float32 scale of the row).
//
// The blocks lie along the product's axis: along the rows (axis 0), or down the
// columns, whose codes come out transposed (axis 1).
//
// Bound by memory (16384 x 4096 bfloat16 to nvfp4 values by row: 46 us, 5.8 TB/s),
// next to it by the instructions of a value's rounding.  A lane holds one 16-byte
// vector of a row, so a block's maximum is a few shuffles; down the columns a thread
// holds the whole block.
#include <algorithm>
#include <type_traits>

#include "f4.cuh"
#include "matrix_vec.cuh"
#include "peat_internal.h"

namespace peat {
namespace {

constexpr int QT = 256;  // threads of a CTA

// A kernel that needs nothing of the one before it (Quant4Params::overlap) runs
// beside it, and waits for it at its end, so that whoever waits for this one has
// waited for both.
__device__ __forceinline__ void begin(const Quant4Params& p) {
  if (!p.overlap) pdl_wait();
  pdl_trigger();
}
__device__ __forceinline__ void end(const Quant4Params& p) {
  if (p.overlap) pdl_wait();
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

// one vector of a row: codes, block scale (at), values; all lanes of a warp together.
// FULL: the whole group's vectors lie inside the matrix.
template <int DT, int FMT, int G, bool GRID, bool FULL, typename Col>
__device__ __forceinline__ void put_vec(const Quant4Params& p, uint4 v, const Out4<DT>& o, Col col, Col left, uint8_t* at,
                                        const Row4& r, const float* reciprocals, uint4* place) {
  using L = Elem<DT>;
  constexpr int LANES = F4<FMT>::BLOCK / L::E;  // that have a block
  if (!GRID) v = gathered<DT, G>(v, place);
  uint32_t top = vec_top<DT>(v);
#pragma unroll
  for (int n = 1; n < LANES; n *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, n));
  const bool finite = top < L::INF;
  const Block4 b = block4<FMT>(L::mag(top), finite, r, reciprocals);
  float x[L::E];
  unpack<DT>(v, x);
  if (FMT == PEAT_NVFP4) {
#pragma unroll
    for (int e = 0; e < L::E / 2; e++) put_pair(x, e, mul2(pair(x, e), both(r.t)));
  }
#pragma unroll
  for (int e = 0; e < L::E / 2; e++) put_pair(x, e, mul2(pair(x, e), both(b.r)));
  uint32_t c;
  if constexpr (L::E == 8) c = codes8(x);
  else c = codes4(x[0], x[1], x[2], x[3]);
  c = coded<FMT>(finite, b) ? c : 0;
  if (o.q && (FULL || col < (Col)p.width)) {
    if (L::E == 8) *reinterpret_cast<uint32_t*>(o.q + col / 2) = c;
    else *reinterpret_cast<uint16_t*>(o.q + col / 2) = (uint16_t)c;
  }
  if (o.block_scale && (threadIdx.x & (LANES - 1)) == 0 && (FULL || col < (Col)(p.tiles * 4 * F4<FMT>::BLOCK))) *at = (uint8_t)b.byte;
  if (o.values) {
    float y[L::E], four[4];
#pragma unroll
    for (int e = 0; e < L::E; e += 4) {
      decoded4<FMT>(c >> (4 * e), r, b, four);
#pragma unroll
      for (int i = 0; i < 4; i++) y[e + i] = four[i];
    }
    if constexpr (GRID) {
      if (FULL || left > 0) __stcs(reinterpret_cast<uint4*>(o.values + col), pack<DT>(y));
    } else {
      // (the group's first column, its lanes' elements side by side)
      const Col lane = threadIdx.x & (G - 1);
      put_apart<DT, G>(o.values + (col - lane * L::E), spread<DT, G>(pack<DT>(y), place), lane, left + lane * L::E);
    }
  }
}

// Rows: TPR threads have a unit, NV vectors each, one unit after another with the
// next one's loads under way.  A unit is a row, or with mxfp4, which needs nothing
// of the row beyond its blocks, one of `pieces` of it.  LONG (nvfp4): rows that
// these threads do not hold, read twice, from L2 the second time.  GRID: x's and
// values' rows start on 16-byte boundaries and are whole vectors; off it a warp's
// elements are read side by side and change places in shared memory (10273 x 3863
// bfloat16 to values: mxfp4 67 us, nvfp4 78, with the codes 69 and 81; by aligned
// vectors shifted together about a third more).
// (16384 x 4096 bfloat16 to codes: mxfp4 31 us, nvfp4 37, where the bytes take 25;
// two vectors a thread and twice the threads were a fifth slower.)
template <int DT, int FMT, int TPR, int NV, bool GRID, bool LONG>
__global__ void __launch_bounds__(QT, NV > 2 ? 2 : 4) quant4_rows(Quant4Params p, int64_t rows, int pieces, int64_t step_row, int step_piece) {
  using L = Elem<DT>;
  using T = typename L::T;
  using Col = std::conditional_t<LONG, int64_t, int>;
  begin(p);
  constexpr int G = TPR < 32 ? TPR : 32, GROUPS = QT / TPR;
  constexpr Col PIECE = TPR * NV * L::E;
  __shared__ uint32_t part[2][QT / 32];
  __shared__ uint4 places[GRID ? 1 : QT];
  uint4* place = places + (GRID ? 0 : threadIdx.x & ~31);
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
    if (GRID && at + PIECE <= cols) {  // (without a condition on each load, or they wait for one another)
#pragma unroll
      for (int i = 0; i < NV; i++) v[i] = source.load(x + at + (i * TPR + lane) * L::E);
      return;
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
      if constexpr (GRID) {
        const Col col = at + (i * TPR + lane) * L::E;
        v[i] = col < cols ? source.load(x + col) : make_uint4(0, 0, 0, 0);
      } else {  // a group's elements side by side; gathered before their use
        const Col begin = at + (i * TPR + lane / G * G) * L::E;
        v[i] = load_apart<DT, G, Col>(x, begin + (lane & (G - 1)), cols);
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
    const Col cols = (Col)p.cols;
    constexpr Col NONE = -(1 << 28);  // elements left of a row that is not the matrix's, seen from any lane's column
    for (Col at = at0; at < (LONG ? wide : at0 + 1); at += PIECE) {
      if (LONG) {
        load(here, at);
#pragma unroll
        for (int i = 0; i < NV; i++) w[i] = v[i];
      }
      // where the lane's block scales go: a vector further on, whole tiles further (or there is one vector)
      constexpr int TILE = 4 * F4<FMT>::BLOCK, NEXT = TPR * L::E / TILE;
      static_assert(NV == 1 || TPR * L::E % TILE == 0, "tiles of scales");
      const Col block = (at + lane * L::E) / F4<FMT>::BLOCK;
      uint8_t* scales = o.block_scale + (int64_t)(block >> 2) * SCALE_TILE + (block & 3);
      // (one way for a warp of two rows, of which the second may be beyond the last: its shuffles are all lanes')
      bool whole = GRID && at + PIECE <= (Col)p.cols && here < p.rows;
      if (GRID && TPR < 32) whole = __all_sync(0xffffffffu, whole);
      if (whole) {
#pragma unroll
        for (int i = 0; i < NV; i++)
          put_vec<DT, FMT, G, GRID, true, Col>(p, w[i], o, at + (i * TPR + lane) * L::E, 1, scales + i * (NEXT * SCALE_TILE), r, reciprocals, place);
      } else {
#pragma unroll
        for (int i = 0; i < NV; i++) {
          const Col begin = at + i * TPR * L::E, col = begin + lane * L::E;
          if (begin < wide)
            put_vec<DT, FMT, G, GRID, false, Col>(p, w[i], o, col, here < p.rows ? cols - col : NONE, scales + i * (NEXT * SCALE_TILE), r,
                                                  reciprocals, place);
        }
      }
    }
  }
  end(p);
}

// ---- columns ------------------------------------------------------------------
// A warp has C columns a lane (16-bit types by pairs, where rows allow it).
template <int DT, bool PAIRS>
__device__ __forceinline__ uint32_t column_word(const typename Elem<DT>::T* x, int64_t cols) {
  if (cols <= 0) return 0;
  if (DT == PEAT_F32 || (PAIRS && cols > 1)) return __ldg(reinterpret_cast<const uint32_t*>(x));
  return __ldg(reinterpret_cast<const uint16_t*>(x));
}

// nvfp4: the largest patterns of each column over one of the parts of the rows,
// [parts, cols].  A lane has a vector of a row, off the 16-byte grid a word.  (16384 x
// 4096 bfloat16: half of nvfp4's 63 us.)
template <int DT, bool GRID, bool PAIRS>
__global__ void __launch_bounds__(QT) quant4_maxima(Quant4Params p, int64_t wide, int64_t each) {
  using L = Elem<DT>;
  using T = typename L::T;
  begin(p);
  constexpr int C = GRID ? L::E : (PAIRS ? 2 : 1), W = GRID ? 4 : 1, U = GRID ? 4 : 8, ROWS = QT / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c0 = ((int64_t)blockIdx.x % wide) * (32 * C) + lane * C, chunk = (int64_t)blockIdx.x / wide;
  const int64_t r0 = chunk * each, r1 = min(p.rows, r0 + each), cols = p.cols - c0;
  const T* x = static_cast<const T*>(p.x) + c0;
  uint32_t m[W];
#pragma unroll
  for (int k = 0; k < W; k++) m[k] = 0;
  auto load = [&](int64_t row, uint32_t (&w)[W]) {
    if constexpr (GRID) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(x + row * p.ldx));
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {
      w[0] = column_word<DT, PAIRS>(x + row * p.ldx, cols);
    }
  };
  int64_t r = r0 + warp;
  if (cols > 0) {
    for (; r + (U - 1) * ROWS < r1; r += U * ROWS) {  // (without a condition on each load, or they wait for one another)
      uint32_t w[U][W];
#pragma unroll
      for (int u = 0; u < U; u++) load(r + u * ROWS, w[u]);
#pragma unroll
      for (int u = 0; u < U; u++)
#pragma unroll
        for (int k = 0; k < W; k++) m[k] = max_word<DT>(m[k], w[u][k]);
    }
    for (; r < r1; r += ROWS) {
      uint32_t w[W];
      load(r, w);
#pragma unroll
      for (int k = 0; k < W; k++) m[k] = max_word<DT>(m[k], w[k]);
    }
  }
  __shared__ uint32_t part[ROWS][W][32];
#pragma unroll
  for (int k = 0; k < W; k++) part[warp][k][lane] = m[k];
  __syncthreads();
  if (warp) return;
  unsigned int* top = p.tops + chunk * p.cols + c0;
#pragma unroll
  for (int k = 0; k < W; k++) {
#pragma unroll
    for (int j = 1; j < ROWS; j++) m[k] = max_word<DT>(m[k], part[j][k][lane]);
    constexpr int PER = C / W;  // columns of a word
#pragma unroll
    for (int c = 0; c < PER; c++)
      if (k * PER + c < cols) top[k * PER + c] = DT == PEAT_F32 ? m[k] & 0x7fffffffu : (c ? m[k] >> 16 : m[k]) & 0x7fffu;
  }
  end(p);
}

// A warp has 32 rows, a thread the blocks of its columns, 16 bytes of codes each: the
// codes come out transposed without a way through shared memory, in units of half a
// sector that L2 puts together.  (To codes: 4096 x 4096 bfloat16 mxfp4 9.0 us, 16384 x
// 4096 31, the latter bound by memory.)
template <int DT, int FMT, bool PAIRS, bool VALUES>
__global__ void __launch_bounds__(QT) quant4_columns(Quant4Params p, int64_t wide, int chunks) {
  using L = Elem<DT>;
  using T = typename L::T;
  begin(p);
  constexpr int C = PAIRS ? 2 : 1, BLOCK = F4<FMT>::BLOCK, NB = 32 / BLOCK;
  __shared__ float reciprocals[FMT == PEAT_NVFP4 ? RECIPROCALS : 1];
  __shared__ uint32_t most[FMT == PEAT_NVFP4 ? QT : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c0 = ((int64_t)blockIdx.x % wide) * (32 * C) + lane * C;
  const int64_t r0 = ((int64_t)blockIdx.x / wide) * QT + warp * 32;
  const T* x = static_cast<const T*>(p.x) + r0 * p.ldx + c0;
  uint32_t w[32];  // (16-bit: of C columns)
  const int64_t rows = min((int64_t)32, p.rows - r0), cols = p.cols - c0;
  if (rows == 32 && cols >= C) {  // (without a condition on each load, or they wait for one another)
#pragma unroll
    for (int i = 0; i < 32; i++) {
      if constexpr (DT == PEAT_F32 || PAIRS) w[i] = __ldg(reinterpret_cast<const uint32_t*>(x + i * p.ldx));
      else w[i] = __ldg(reinterpret_cast<const uint16_t*>(x + i * p.ldx));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; i++) w[i] = i < rows ? column_word<DT, PAIRS>(x + i * p.ldx, cols) : 0;
  }
  if (FMT == PEAT_NVFP4) {
    // the columns' maxima over the parts, by all threads: a column's by every (32 C)-th
    make_reciprocals(reciprocals);
    constexpr int WIDE = 32 * C;
    const int64_t col = ((int64_t)blockIdx.x % wide) * WIDE + threadIdx.x % WIDE;
    uint32_t top = 0;
    if (col < p.cols)
      for (int k = threadIdx.x / WIDE; k < chunks; k += QT / WIDE) top = max(top, __ldcg(p.tops + k * p.cols + col));
    most[threadIdx.x] = top;
    __syncthreads();
  }
  Row4 r[C];
  Block4 b[C][NB];
  uint32_t code[C][4];
#pragma unroll
  for (int c = 0; c < C; c++) {
    const int64_t col = c0 + c;
    r[c] = row4<FMT>(0.0f, true);
    if (FMT == PEAT_NVFP4) {
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < QT / (32 * C); k++) top = max(top, most[k * (32 * C) + lane * C + c]);
      r[c] = row4<FMT>(L::mag(top), top < L::INF);
      if (p.scale && r0 == 0 && col < p.cols) p.scale[col] = r[c].s;
    }
    auto bits = [&](int i) { return DT == PEAT_F32 ? w[i] : (c ? w[i] >> 16 : w[i] & 0xffffu); };
    auto number = [&](int i) {
      if (DT == PEAT_F32) return __uint_as_float(w[i]);
      if (DT == PEAT_BF16) return __uint_as_float(c ? w[i] & 0xffff0000u : w[i] << 16);
      return __half2float(__ushort_as_half((unsigned short)bits(i)));
    };
#pragma unroll
    for (int n = 0; n < NB; n++) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < BLOCK; i++) top = max(top, bits(n * BLOCK + i) & (DT == PEAT_F32 ? 0x7fffffffu : 0x7fffu));
      const bool finite = top < L::INF;
      b[c][n] = block4<FMT>(L::mag(top), finite, r[c], reciprocals);
#pragma unroll
      for (int j = 0; j < BLOCK / 8; j++) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] = scaled4<FMT>(number(n * BLOCK + j * 8 + e), r[c], b[c][n]);
        code[c][n * (BLOCK / 8) + j] = coded<FMT>(finite, b[c][n]) ? codes8(y) : 0;
      }
      const int64_t block = r0 / BLOCK + n;
      if (p.block_scale && block < p.tiles * 4) p.block_scale[scale_at(col, block, p.tiles)] = (uint8_t)b[c][n].byte;
    }
    // whole blocks: 16 or 8 bytes of a 16-byte unit
    const int64_t left = (p.width - r0) / 2;
    if (p.q && col < p.cols && left > 0) {
      uint8_t* q = p.q + col * p.ldq + r0 / 2;
      if (left >= 16) *reinterpret_cast<uint4*>(q) = make_uint4(code[c][0], code[c][1], code[c][2], code[c][3]);
      else *reinterpret_cast<uint2*>(q) = make_uint2(code[c][0], code[c][1]);
    }
  }
  end(p);  // (mxfp4; nvfp4 needs its maxima first)
  if (!VALUES || cols <= 0) return;
  T* o = static_cast<T*>(p.values) + r0 * p.ldv + c0;
  const bool both = PAIRS && cols > 1 && p.pairs_v;
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    float v[C][4];
#pragma unroll
    for (int c = 0; c < C; c++) decoded4<FMT>(code[c][i / 8] >> (4 * (i & 4)), r[c], b[c][i / BLOCK], v[c]);
#pragma unroll
    for (int e = 0; e < 4; e++) {
      if (i + e >= rows) break;
      T* at = o + (i + e) * p.ldv;
      if constexpr (DT == PEAT_F32) {
        *at = v[0][e];
      } else {
        uint32_t two;
        if constexpr (DT == PEAT_F16) {
          const __half2 h = __floats2half2_rn(v[0][e], v[C - 1][e]);
          two = *reinterpret_cast<const uint32_t*>(&h);
        } else {
          const __nv_bfloat162 h = __floats2bfloat162_rn(v[0][e], v[C - 1][e]);
          two = *reinterpret_cast<const uint32_t*>(&h);
        }
        if (both) {
          *reinterpret_cast<uint32_t*>(at) = two;
        } else {
          *reinterpret_cast<uint16_t*>(at) = (uint16_t)two;
          if (C == 2 && cols > 1) *reinterpret_cast<uint16_t*>(at + 1) = (uint16_t)(two >> 16);
        }
      }
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
template <int DT, int FMT, bool PAIRS>
cudaError_t columns_by(Quant4Params p, int nsm, cudaStream_t s) {
  constexpr int WIDE = PAIRS ? 64 : 32;
  int chunks = 0;
  if (FMT == PEAT_NVFP4) {
    // parts of the rows for the maxima: until the SMs have four CTAs each, 64 rows or more
    const bool grid = p.vec_x && p.cols % Elem<DT>::E == 0;
    const int64_t broad = grid ? 32 * Elem<DT>::E : WIDE, groups = (p.cols + broad - 1) / broad;
    chunks = (int)std::max<int64_t>(1, std::min<int64_t>({QUANT4_CHUNKS, p.rows / 64, 4 * (int64_t)nsm / groups}));
    const int64_t each = (p.rows + chunks - 1) / chunks;
    cudaError_t e = launch_dependent(grid ? quant4_maxima<DT, true, PAIRS> : quant4_maxima<DT, false, PAIRS>,
                                     (unsigned)(groups * chunks), QT, 0, s, p, groups, each);
    if (e != cudaSuccess) return e;
    p.overlap = 0;
  }
  const int64_t cols = p.block_scale ? (p.cols + 127) / 128 * 128 : p.cols;
  const int64_t height = p.tiles * 4 * F4<FMT>::BLOCK, wide = (cols + WIDE - 1) / WIDE;
  return launch_dependent(p.values ? quant4_columns<DT, FMT, PAIRS, true> : quant4_columns<DT, FMT, PAIRS, false>,
                          (unsigned)(wide * ((height + QT - 1) / QT)), QT, 0, s, p, wide, chunks);
}
template <int DT, int FMT>
cudaError_t columns(const Quant4Params& p, int nsm, cudaStream_t s) {
  if constexpr (DT != PEAT_F32)
    if (p.pairs) return columns_by<DT, FMT, true>(p, nsm, s);
  return columns_by<DT, FMT, false>(p, nsm, s);
}
template <int DT>
cudaError_t of_type(int format, int axis, const Quant4Params& p, int nsm, cudaStream_t s) {
  if (format == PEAT_MXFP4) return axis ? columns<DT, PEAT_MXFP4>(p, nsm, s) : rows<DT, PEAT_MXFP4>(p, nsm, s);
  return axis ? columns<DT, PEAT_NVFP4>(p, nsm, s) : rows<DT, PEAT_NVFP4>(p, nsm, s);
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
