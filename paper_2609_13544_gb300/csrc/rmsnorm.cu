// The root-mean-square norm of a residual stream, with the stream's addition
// before it and the rounding to 8-bit integers behind it, and its gradients.
//
//   s = x + residual in the tensors' type, v = sum s^2 / n, rstd = 1 / sqrt(v + eps),
//   y = (s rstd) weight; 8 bits: amax = max |y|, q = rint(y (127 / amax))
//
// The sum of squares is carried with its rounding errors (two float32 numbers,
// good to 2^-40 or so), so that v is the 64-bit sum's float32 value: the integers
// near a rounding border then do not depend on the order of the sum.  Rows whose
// squares leave float32's range are summed in binary64.
//
// Bound by memory (16384 x 4096 bfloat16 with residual and 8-bit values: 87 us, 6.1
// TB/s; gradients with the stream's 90 us, 5.9 TB/s), next to it by the instructions
// of the sum's kept errors and of the rounding: a row is read once and kept in
// registers between the two reductions; the gradients of the weights are summed in
// registers over a CTA's rows, then over the CTAs in a fixed order.
#include <algorithm>
#include <type_traits>

#include "matrix_vec.cuh"
#include "ops_internal.h"
#include "peat_internal.h"

namespace peat {
namespace {

template <int TPR>
constexpr int threads_of() { return TPR > 256 ? TPR : 256; }

// (hi, lo) + x, the rounding error of the sum kept in lo
__device__ __forceinline__ void add_kept(float& hi, float& lo, float x) {
  const float t = __fadd_rn(hi, x), z = __fsub_rn(t, hi);
  lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(t, z)), __fsub_rn(x, z)));
  hi = t;
}
// (hi, lo) over the lanes of a group of N, the same bits in all of them
template <int N>
__device__ __forceinline__ void lanes_kept(float& hi, float& lo) {
#pragma unroll
  for (int o = N / 2; o; o /= 2) {
    const float h = __shfl_xor_sync(0xffffffffu, hi, o), l = __shfl_xor_sync(0xffffffffu, lo, o);
    lo = __fadd_rn(lo, l);
    add_kept(hi, lo, h);
  }
}
template <int TPR>
__device__ __forceinline__ double sum_wide(double x, double* part) {
#pragma unroll
  for (int o = 16; o; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (TPR > 32) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    const double* p = part + threadIdx.x / TPR * (TPR / 32);
    x = p[0];
#pragma unroll
    for (int w = 1; w < TPR / 32; w++) x += p[w];
  }
  return x;
}
template <int TPR>
__device__ __forceinline__ float sum_plain(float x, float* part) {
#pragma unroll
  for (int o = 16; o; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (TPR > 32) {
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    const float* p = part + threadIdx.x / TPR * (TPR / 32);
    x = p[0];
#pragma unroll
    for (int w = 1; w < TPR / 32; w++) x += p[w];
  }
  return x;
}
// A thread's E elements of a row of `cols`.  GRID (every matrix's rows start on
// 16-byte boundaries and are whole vectors): a vector from column `col` on.  Off the
// grid: elements `APART` columns apart, so that a warp's are side by side, whatever
// the alignment (10273 x 3863 bfloat16, 8-bit values with the residual: 101 us; by
// vectors shifted together from aligned ones 142).
template <int DT, bool GRID, int APART, typename Col>
__device__ __forceinline__ uint4 load_vec(const typename Elem<DT>::T* row, Col col, Col cols) {
  if constexpr (GRID) {
    return col < cols ? __ldg(reinterpret_cast<const uint4*>(row + col)) : make_uint4(0, 0, 0, 0);
  } else {
    return load_apart<DT, APART>(row, col, cols);
  }
}
template <int DT, bool GRID, int APART, typename Col>
__device__ __forceinline__ void put_vec(typename Elem<DT>::T* row, const float (&y)[Elem<DT>::E], Col col, Col cols) {
  if constexpr (GRID) {
    if (col < cols) __stcs(reinterpret_cast<uint4*>(row + col), pack<DT>(y));
  } else {
    put_apart<DT, APART>(row, pack<DT>(y), col, cols);
  }
}
// the weights of these columns
template <int DT, bool GRID, int APART, typename Col>
__device__ __forceinline__ void weights(const void* w, int f32, Col col, Col cols, float (&x)[Elem<DT>::E]) {
  constexpr int E = Elem<DT>::E;
  if (DT != PEAT_F32 && !f32) {
    unpack<DT>(load_vec<DT, GRID, APART>(static_cast<const typename Elem<DT>::T*>(w), col, cols), x);
    return;
  }
  const float* p = static_cast<const float*>(w);
  if constexpr (GRID) {
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const float4 f = col < cols ? __ldg(reinterpret_cast<const float4*>(p + col + e)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      x[e] = f.x, x[e + 1] = f.y, x[e + 2] = f.z, x[e + 3] = f.w;
    }
  } else {
    if (col + (E - 1) * APART < cols) {
#pragma unroll
      for (int e = 0; e < E; e++) x[e] = __ldg(p + col + e * APART);
    } else {
#pragma unroll
      for (int e = 0; e < E; e++) x[e] = col + e * APART < cols ? __ldg(p + col + e * APART) : 0.0f;
    }
  }
}

// a vector of a matrix that this kernel has written (the thread's own elements)
template <int DT, bool GRID, int APART, typename Col>
__device__ __forceinline__ uint4 load_own(const typename Elem<DT>::T* row, Col col, Col cols) {
  if constexpr (GRID) return col < cols ? *reinterpret_cast<const uint4*>(row + col) : make_uint4(0, 0, 0, 0);
  else return load_vec<DT, GRID, APART>(row, col, cols);
}

// ---- forward ------------------------------------------------------------------
// TPR threads have a row, NV vectors each, one row after another; the next row's
// loads are under way while this one's factors are found (101 us for 111 when that
// came, 16384 x 4096 bfloat16; two float32 operations an instruction: 97; a row's
// maxima by magnitude instructions and a fourth CTA: 88).  LONG: rows that these
// threads do not hold, read again for each of the three passes.
template <int DT, int TPR, int NV, bool GRID, bool LONG>
__global__ void __launch_bounds__(threads_of<TPR>(), LONG || TPR > 256 ? 1 : TPR <= 64 ? 3 : 4) rms_forward(RmsParams p) {
  using L = Elem<DT>;
  using T = typename L::T;
  using Col = std::conditional_t<LONG, int64_t, int>;
  constexpr int E = L::E, QT = threads_of<TPR>(), GROUPS = QT / TPR;
  constexpr int64_t PIECE = (int64_t)TPR * NV * E;
  constexpr int WARPS = TPR / 32;
  __shared__ float2 sums[TPR > 32 ? QT : 1], found[GROUPS], factor[GROUPS];
  __shared__ double wide[QT / 32];
  __shared__ uint32_t tops[QT / 32];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const Col end = LONG ? (Col)p.cols : 1;
  const bool round = p.q || p.values || p.scale;
  uint4 s[NV], u[NV];
  auto column = [&](Col at, int i) { return at + (GRID ? (i * TPR + lane) * E : i * TPR * E + lane); };
  auto fetch = [&](int64_t row, Col at) {
    const Col cols = row < p.rows ? (Col)p.cols : 0;
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const T* r = static_cast<const T*>(p.residual) + row * p.ldr;
    if (GRID && at + (Col)PIECE <= cols) {  // (without a condition on each load, or they wait for one another)
#pragma unroll
      for (int i = 0; i < NV; i++) s[i] = __ldg(reinterpret_cast<const uint4*>(x + column(at, i)));
      if (!p.residual) return;
#pragma unroll
      for (int i = 0; i < NV; i++) u[i] = __ldg(reinterpret_cast<const uint4*>(r + column(at, i)));
      return;
    }
#pragma unroll
    for (int i = 0; i < NV; i++) s[i] = load_vec<DT, GRID, TPR>(x, column(at, i), cols);
    if (!p.residual) return;
#pragma unroll
    for (int i = 0; i < NV; i++) u[i] = load_vec<DT, GRID, TPR>(r, column(at, i), cols);
  };
  auto added = [&](uint4 (&v)[NV]) {  // s = x + residual, rounded to the type
#pragma unroll
    for (int i = 0; i < NV; i++) {
      v[i] = s[i];
      if (!p.residual) continue;
      float a[E], b[E];
      unpack<DT>(s[i], a);
      unpack<DT>(u[i], b);
#pragma unroll
      for (int e = 0; e < E / 2; e++) put_pair(a, e, add2(pair(a, e), pair(b, e)));
      v[i] = pack<DT>(a);
    }
  };
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  if (!LONG) fetch((int64_t)blockIdx.x * GROUPS + group, 0);
  for (int64_t row0 = (int64_t)blockIdx.x * GROUPS; row0 < p.rows; row0 += step) {
    const int64_t row = row0 + group;
    const bool live = row < p.rows;
    const Col cols = live ? (Col)p.cols : 0;
    T* sum = p.sum ? static_cast<T*>(p.sum) + row * p.lds : nullptr;
    uint4 v[NV];
    auto again = [&](Col at) {  // a piece of a long row, from where the first pass left it
      if (!LONG) return;
      if (!sum) {
        fetch(row, at);
        added(v);
        return;
      }
#pragma unroll
      for (int i = 0; i < NV; i++) v[i] = load_own<DT, GRID, TPR>(sum, column(at, i), cols);
    };
    float hi = 0.0f, lo = 0.0f;
    for (Col at = 0; at < end; at += (Col)PIECE) {
      if (LONG) fetch(row, at);
      added(v);
      if (!LONG && row0 + step < p.rows) fetch(row + step, 0);
      // Squares on top of one that none exceeds: what a sum's rounding leaves of a
      // square is then the difference of two sums away (Dekker's short form)
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < NV; i++) top = max(top, vec_top<DT>(v[i]));
      const float most = L::mag(top), base = __fmul_ru(most, most);
      float2 t = both(base), rest = both(0.0f);
#pragma unroll
      for (int i = 0; i < NV; i++) {
        float a[E];
        unpack<DT>(v[i], a);
        if (sum) put_vec<DT, GRID, TPR>(sum, a, column(at, i), cols);
#pragma unroll
        for (int e = 0; e < E / 2; e++) {
          const float2 x = pair(a, e), w = fma2(x, x, t);
          rest = add2(rest, fma2(x, x, add2(t, minus(w))));
          t = w;
        }
      }
      lo = __fadd_rn(lo, __fadd_rn(rest.x, rest.y));
      if (LONG) add_kept(hi, lo, t.x);
      else hi = t.x;
      add_kept(hi, lo, -base);
      add_kept(hi, lo, t.y);
      add_kept(hi, lo, -base);
    }
    // One warp adds up the warps' sums and finds the row's factor for all: the
    // divisions would be a quarter of every thread's instructions.
    if (TPR > 32) {
      sums[threadIdx.x] = make_float2(hi, lo);
      __syncthreads();
    }
    bool fine = true;
    float rstd = 0.0f;
    if (lane < 32) {
#pragma unroll
      for (int k = 1; k < WARPS; k++) {
        const float2 f = sums[group * TPR + k * 32 + lane];
        lo = __fadd_rn(lo, f.y);
        add_kept(hi, lo, f.x);
      }
      lanes_kept<32>(hi, lo);
      // (hi + lo) / n, rounded once: the quotient and what it leaves
      const float n = (float)(int)p.cols, quotient = __fdiv_rn(hi, n);
      const float mean = __fadd_rn(quotient, __fdiv_rn(__fadd_rn(__fmaf_rn(-quotient, n, hi), lo), n));
      fine = (hi < 0x1p126f && hi > 0x1p-70f && p.cols < (1 << 24)) || !live;
      rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(mean, p.eps)));
      if (TPR > 32 && lane == 0) found[group] = make_float2(rstd, fine ? 1.0f : 0.0f);
    }
    bool widely = !fine;  // by the whole CTA where it meets at barriers
    if (TPR > 32) {
      __syncthreads();
      rstd = found[group].x;
      fine = found[group].y != 0.0f;
      widely = false;
#pragma unroll
      for (int g = 0; g < GROUPS; g++) widely |= found[g].y == 0.0f;
    }
    if (widely) {
      double t = 0.0;
      for (Col at = 0; at < end; at += (Col)PIECE) {
        again(at);
#pragma unroll
        for (int i = 0; i < NV; i++) {
          float a[E];
          unpack<DT>(v[i], a);
#pragma unroll
          for (int e = 0; e < E; e++)
            if (a[e] != 0.0f) t += (double)a[e] * (double)a[e];
        }
      }
      t = sum_wide<TPR>(t, wide);
      if (!fine) rstd = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn((float)(t / (double)p.cols), p.eps)));
    }
    if (p.rstd && lane == 0 && live) p.rstd[row] = rstd;
    if (!p.y && !round) continue;

    float y[NV][E];
    auto normed = [&](Col at) {
#pragma unroll
      for (int i = 0; i < NV; i++) {
        float w[E];
        weights<DT, GRID, TPR>(p.weight, p.weight_f32, column(at, i), (Col)p.cols, w);
        unpack<DT>(v[i], y[i]);
#pragma unroll
        for (int e = 0; e < E / 2; e++) put_pair(y[i], e, mul2(mul2(pair(y[i], e), both(rstd)), pair(w, e)));
      }
    };
    float r = 0.0f, scale = 0.0f;
    if (round) {
      // (beyond the row's end y is 0, or NaN where all of the row is)
      uint32_t top = 0;
      for (Col at = 0; at < end; at += (Col)PIECE) {
        again(at);
        normed(at);
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
          for (int e = 0; e < E; e++) top = max_f32(top, __float_as_uint(y[i][e]));
      }
      top = __reduce_max_sync(0xffffffffu, top & 0x7fffffffu);
      if (TPR > 32) {
        if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
        __syncthreads();
      }
      if (lane < 32) {
        if (TPR > 32) top = __reduce_max_sync(0xffffffffu, tops[group * WARPS + (lane & (WARPS - 1))]);
        factors<PEAT_F32>(top, r, scale);
        if (p.scale && lane == 0 && live) p.scale[row] = scale;
        if (TPR > 32 && lane == 0) factor[group] = make_float2(r, scale);
      }
      if (TPR > 32) {
        __syncthreads();
        r = factor[group].x;
        scale = factor[group].y;
      }
    }
    const bool finite = scale == scale;
    for (Col at = 0; at < end; at += (Col)PIECE) {
      if (LONG || !round) {
        again(at);
        normed(at);
      }
#pragma unroll
      for (int i = 0; i < NV; i++) {
        const Col col = column(at, i);
        if (p.y) put_vec<DT, GRID, TPR>(static_cast<T*>(p.y) + row * p.ldy, y[i], col, cols);
        if (!p.q && !p.values) continue;
        float w[E];
        if (finite) {
#pragma unroll
          for (int e = 0; e < E; e++) w[e] = __fmul_rn(y[i][e], r);  // (a pair's product and sum become one rounding)
#pragma unroll
          for (int e = 0; e < E / 2; e++) put_pair(w, e, add2(pair(w, e), both(MAGIC)));
        } else {
#pragma unroll
          for (int e = 0; e < E; e++) w[e] = MAGIC;
        }
        if (p.q) {
          int8_t* q = p.q + row * p.ldq + col;
          if constexpr (GRID) {
            if (col < cols) {
              if (E == 8)
                *reinterpret_cast<uint2*>(q) = make_uint2(pack4(w[0], w[1], w[2], w[3]), pack4(w[4 % E], w[5 % E], w[6 % E], w[7 % E]));
              else
                *reinterpret_cast<uint32_t*>(q) = pack4(w[0], w[1], w[2], w[3]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < E; e++)
              if (col + e * TPR < cols) q[e * TPR] = byte_of(w[e]);
          }
        }
        if (p.values) {
          float z[E];
#pragma unroll
          for (int e = 0; e < E / 2; e++) put_pair(z, e, mul2(add2(pair(w, e), both(-MAGIC)), both(scale)));
          put_vec<DT, GRID, TPR>(static_cast<T*>(p.values) + row * p.ldv, z, col, cols);
        }
      }
    }
  }
}

// ---- backward -----------------------------------------------------------------
//   n = s rstd, g = grad weight, c = sum (g n) / cols,
//   grad_x = rstd (g - n c) + stream, grad_weight = sum over rows of grad n
// A CTA has `each` rows for each of its groups of TPR threads, one after another,
// the next one's loads under way; a thread keeps its columns' weights and sums.
// LONG: CTA blockIdx.x has a piece of the columns (65536 pieces at most) of the rows of
// blockIdx.y, and c is there already (rms_dots), which costs a second reading (4000 x
// 12800 bfloat16: 99 us, the bytes read once 45).  Beyond a row's end grad, x and weight
// are 0.
template <int DT, int TPR, int NV, bool GRID, bool LONG>
__global__ void __launch_bounds__(threads_of<TPR>(), TPR > 256 ? 1 : 2) rms_backward(RmsBackParams p) {
  using L = Elem<DT>;
  using T = typename L::T;
  using Col = std::conditional_t<LONG, int64_t, int>;
  constexpr int E = L::E, QT = threads_of<TPR>(), GROUPS = QT / TPR;
  __shared__ float dots[2][QT / 32];
  __shared__ float met[GROUPS > 1 ? TPR * NV * E : 1];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const float n_cols = (float)(int)p.cols;
  const Col at = LONG ? (Col)blockIdx.x * (TPR * NV * E) : 0;
  const int64_t cta = LONG ? blockIdx.y : blockIdx.x, row0 = (cta * GROUPS + group) * p.each;
  constexpr int STEP = GRID ? 1 : TPR;  // columns from one element of a vector to the next
  auto column = [&](int i) { return at + (GRID ? (i * TPR + lane) * E : i * TPR * E + lane); };
  float dw[NV][E], w[NV][E];
#pragma unroll
  for (int i = 0; i < NV; i++) {
    weights<DT, GRID, TPR>(p.weight, p.weight_f32, column(i), (Col)p.cols, w[i]);
#pragma unroll
    for (int e = 0; e < E; e++) dw[i][e] = 0.0f;
  }
  uint4 d[NV], s[NV], u[NV];
  float rstd_next;
  auto fetch = [&](int64_t row) {
    const Col cols = row < p.rows ? (Col)p.cols : 0;
    const T* dp = static_cast<const T*>(p.grad) + row * p.ldg;
    const T* xp = static_cast<const T*>(p.x) + row * p.ldx;
    rstd_next = row < p.rows ? __ldg(p.rstd + row) : 0.0f;
    const bool streams = p.stream && p.grad_x;
    const T* tp = static_cast<const T*>(p.stream) + row * p.ldr;
    if (GRID && at + TPR * NV * E <= cols) {  // (without a condition on each load, or they wait for one another)
#pragma unroll
      for (int i = 0; i < NV; i++) {
        d[i] = __ldg(reinterpret_cast<const uint4*>(dp + column(i)));
        s[i] = __ldg(reinterpret_cast<const uint4*>(xp + column(i)));
      }
      if (!streams) return;
#pragma unroll
      for (int i = 0; i < NV; i++) u[i] = __ldg(reinterpret_cast<const uint4*>(tp + column(i)));
      return;
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
      d[i] = load_vec<DT, GRID, TPR>(dp, column(i), cols);
      s[i] = load_vec<DT, GRID, TPR>(xp, column(i), cols);
    }
    if (!streams) return;
#pragma unroll
    for (int i = 0; i < NV; i++) u[i] = load_vec<DT, GRID, TPR>(tp, column(i), cols);
  };
  fetch(row0);
  for (int64_t it = 0; it < p.each; it++) {
    const int64_t row = row0 + it;
    const bool live = row < p.rows;
    const float rstd = rstd_next;
    uint4 dv[NV], sv[NV], uv[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) dv[i] = d[i], sv[i] = s[i], uv[i] = u[i];
    if (it + 1 < p.each) fetch(row + 1);
    float2 c2 = both(0.0f);
#pragma unroll
    for (int i = 0; i < NV; i++) {
      float a[E], b[E];
      unpack<DT>(dv[i], a);
      unpack<DT>(sv[i], b);
#pragma unroll
      for (int e = 0; e < E / 2; e++) {
        const float2 x = pair(a, e), n = mul2(pair(b, e), both(rstd));
        put_pair(dw[i], e, fma2(x, n, pair(dw[i], e)));
        if (!LONG) c2 = fma2(mul2(x, pair(w[i], e)), n, c2);
      }
    }
    if (!p.grad_x) continue;
    float c = c2.x + c2.y;
    if (LONG) c = live ? __ldg(p.dots + row) : 0.0f;
    else c = sum_plain<TPR>(c, dots[it & 1]) / n_cols;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      float a[E], b[E], t[E];
      unpack<DT>(dv[i], a);
      unpack<DT>(sv[i], b);
#pragma unroll
      for (int e = 0; e < E / 2; e++)
        put_pair(b, e, mul2(both(rstd), fma2(minus(mul2(pair(b, e), both(rstd))), both(c), mul2(pair(a, e), pair(w[i], e)))));
      if (p.stream) {
        unpack<DT>(uv[i], t);
#pragma unroll
        for (int e = 0; e < E / 2; e++) put_pair(b, e, add2(pair(b, e), pair(t, e)));
      }
      put_vec<DT, GRID, TPR>(static_cast<T*>(p.grad_x) + row * p.ldo, b, column(i), live ? (Col)p.cols : (Col)0);
    }
  }
  if (!p.grad_weight) return;
  if (GROUPS > 1) {  // the groups' sums, one after the other
    for (int g = 0; g < GROUPS; g++) {
      if (group == g) {
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
          for (int e = 0; e < E; e++) {
            float* m = met + (i * E + e) * TPR + lane;
            dw[i][e] = g ? *m + dw[i][e] : dw[i][e];
            *m = dw[i][e];
          }
      }
      __syncthreads();
    }
    if (group != GROUPS - 1) return;
  }
  float* o = p.parts + cta * p.cols;
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int e = 0; e < E; e++)
      if (column(i) + e * STEP < p.cols) o[column(i) + e * STEP] = dw[i][e];
}

// sum (g n) / cols of each row, by a CTA: a thread's vectors one after the other, up to
// 2^17 of them, so with the rounding errors kept: EACH those of every addition, for
// float32 on the grid those of sums of up to 64 vectors (152 x 32768: 31.5 us, without
// any 30.9, with each one's 34.7)
template <int DT, bool GRID>
__global__ void __launch_bounds__(256) rms_dots(RmsBackParams p) {
  using T = typename Elem<DT>::T;
  constexpr int E = Elem<DT>::E;
  __shared__ float parts[8];
  pdl_wait();
  pdl_trigger();
  const int64_t row = blockIdx.x;
  const T* dp = static_cast<const T*>(p.grad) + row * p.ldg;
  const T* xp = static_cast<const T*>(p.x) + row * p.ldx;
  const float rstd = __ldg(p.rstd + row);
  constexpr bool EACH = !GRID || E == 8;
  float c = 0.0f, hi = 0.0f, lo = 0.0f;
  auto place = [&](int64_t at) { return at + (GRID ? threadIdx.x * E : threadIdx.x); };
  auto add = [&](uint4 d, uint4 x, int64_t at) {
    float a[E], b[E], w[E];
    unpack<DT>(d, a);
    unpack<DT>(x, b);
    weights<DT, GRID, 256>(p.weight, p.weight_f32, place(at), p.cols, w);
    float part = 0.0f;
#pragma unroll
    for (int e = 0; e < E; e++) part = __fmaf_rn(__fmul_rn(a[e], w[e]), __fmul_rn(b[e], rstd), part);
    if (EACH) add_kept(hi, lo, part);
    else c += part;
  };
  constexpr int U = GRID ? 4 : 1, PIECE = 256 * E;
  const int64_t run = EACH ? p.cols : 64 * PIECE;
  int64_t at = 0;
  for (int64_t to = min(p.cols, run);; to = min(p.cols, to + run)) {
    for (; at + U * PIECE <= to; at += U * PIECE) {  // (whole pieces: loads in a batch)
      uint4 d[U], x[U];
#pragma unroll
      for (int k = 0; k < U; k++) {
        d[k] = load_vec<DT, GRID, 256>(dp, place(at + k * PIECE), p.cols);
        x[k] = load_vec<DT, GRID, 256>(xp, place(at + k * PIECE), p.cols);
      }
#pragma unroll
      for (int k = 0; k < U; k++) add(d[k], x[k], at + k * PIECE);
    }
    for (; at < to; at += PIECE)
      add(load_vec<DT, GRID, 256>(dp, place(at), p.cols), load_vec<DT, GRID, 256>(xp, place(at), p.cols), at);
    if (!EACH) add_kept(hi, lo, c);
    if (EACH || to == p.cols) break;
    c = 0.0f;
  }
  c = sum_plain<256>(__fadd_rn(hi, lo), parts);
  if (threadIdx.x == 0) p.dots[row] = c / (float)(int)p.cols;
}

// the CTAs' sums of each column, in their order: some by each warp, then over the warps
__global__ void __launch_bounds__(1024) rms_weight_sums(const float* parts, int ctas, int64_t cols, float* out) {
  pdl_wait();
  pdl_trigger();
  __shared__ float met[32][32];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int64_t col = (int64_t)blockIdx.x * 32 + lane;
  float hi = 0.0f, lo = 0.0f;
  if (col < cols) {
    constexpr int U = 5;
    int i = part;
    for (; i + (U - 1) * warps < ctas; i += U * warps) {
      float x[U];
#pragma unroll
      for (int u = 0; u < U; u++) x[u] = __ldcg(parts + (int64_t)(i + u * warps) * cols + col);
#pragma unroll
      for (int u = 0; u < U; u++) add_kept(hi, lo, x[u]);
    }
    for (; i < ctas; i += warps) add_kept(hi, lo, __ldcg(parts + (int64_t)i * cols + col));
  }
  met[part][lane] = __fadd_rn(hi, lo);
  __syncthreads();
  if (part || col >= cols) return;
  float t = met[0][lane];
  for (int k = 1; k < warps; k++) t += met[k][lane];
  out[col] = t;
}

template <int DT, int TPR, int NV, bool LONG = false>
cudaError_t forward(const RmsParams& p, int nsm, cudaStream_t s) {
  constexpr int QT = threads_of<TPR>();
  // As many CTAs as are at work at once; without the rounding, which is bound by its
  // instructions, one less (16384 x 4096 bfloat16 with the residual: 8 bits 88 us, with
  // three CTAs an SM 96; y 82 to 85, with four 90).
  const unsigned grid = (unsigned)std::min<int64_t>((p.rows + QT / TPR - 1) / (QT / TPR),
                                                    (int64_t)nsm * (TPR > 256 ? 2 : p.q || p.values ? 4 : 3));
  if (p.grid) return launch_dependent(rms_forward<DT, TPR, NV, true, LONG>, grid, QT, 0, s, p);
  return launch_dependent(rms_forward<DT, TPR, NV, false, LONG>, grid, QT, 0, s, p);
}
template <int DT>
cudaError_t forward_of(const RmsParams& p, int nsm, cudaStream_t s) {
  const int64_t vecs = (p.cols + Elem<DT>::E - 1) / Elem<DT>::E;
  if (vecs <= 32) return forward<DT, 32, 1>(p, nsm, s);
  if (vecs <= 64) return forward<DT, 32, 2>(p, nsm, s);
  if (vecs <= 128) return forward<DT, 64, 2>(p, nsm, s);
  if (vecs <= 256) return forward<DT, 128, 2>(p, nsm, s);
  if (vecs <= 512) return forward<DT, 256, 2>(p, nsm, s);
  if (vecs <= 1024) return forward<DT, 512, 2>(p, nsm, s);
  if (vecs <= 2048) return forward<DT, 512, 4>(p, nsm, s);
  return forward<DT, 512, 4, true>(p, nsm, s);
}

struct Shape {  // of the backward kernel
  int tpr, nv;
  bool longer;
};
Shape shape_of(int64_t vecs) {
  if (vecs <= 32) return {32, 1, false};
  if (vecs <= 64) return {32, 2, false};
  if (vecs <= 128) return {64, 2, false};
  if (vecs <= 256) return {128, 2, false};
  if (vecs <= 512) return {256, 2, false};
  if (vecs <= 1024) return {512, 2, false};
  return {256, 2, true};
}
template <int DT, int TPR, int NV, bool LONG = false>
cudaError_t backward(const RmsBackParams& p, cudaStream_t s) {
  constexpr int QT = threads_of<TPR>();
  cudaError_t e = cudaSuccess;
  if (LONG && p.rows && p.grad_x) {
    e = p.grid ? launch_dependent(rms_dots<DT, true>, (unsigned)p.rows, 256, 0, s, p)
               : launch_dependent(rms_dots<DT, false>, (unsigned)p.rows, 256, 0, s, p);
    if (e != cudaSuccess) return e;
  }
  if (p.ctas) {
    constexpr int64_t PIECE = (int64_t)TPR * NV * Elem<DT>::E;
    // (a grid's y ends at 65535, the rows' CTAs at two an SM)
    const dim3 grid = LONG ? dim3((unsigned)((p.cols + PIECE - 1) / PIECE), (unsigned)p.ctas) : dim3((unsigned)p.ctas);
    e = p.grid ? launch_dependent(rms_backward<DT, TPR, NV, true, LONG>, grid, QT, 0, s, p)
               : launch_dependent(rms_backward<DT, TPR, NV, false, LONG>, grid, QT, 0, s, p);
    if (e != cudaSuccess) return e;
  }
  if (!p.grad_weight) return e;
  return launch_dependent(rms_weight_sums, (unsigned)((p.cols + 31) / 32), p.ctas > 80 ? 1024 : 256, 0, s, (const float*)p.parts, p.ctas, p.cols, p.grad_weight);
}
template <int DT>
cudaError_t backward_of(const RmsBackParams& p, cudaStream_t s) {
  const Shape k = shape_of((p.cols + Elem<DT>::E - 1) / Elem<DT>::E);
  if (k.longer) return backward<DT, 256, 2, true>(p, s);
  switch (k.tpr) {
    case 32: return k.nv == 1 ? backward<DT, 32, 1>(p, s) : backward<DT, 32, 2>(p, s);
    case 64: return backward<DT, 64, 2>(p, s);
    case 128: return backward<DT, 128, 2>(p, s);
    case 256: return backward<DT, 256, 2>(p, s);
    default: return backward<DT, 512, 2>(p, s);
  }
}

}  // namespace

cudaError_t launch_rmsnorm(int dtype, const RmsParams& p, int nsm, cudaStream_t s) {
  switch (dtype) {
    case PEAT_F32: return forward_of<PEAT_F32>(p, nsm, s);
    case PEAT_F16: return forward_of<PEAT_F16>(p, nsm, s);
    default: return forward_of<PEAT_BF16>(p, nsm, s);
  }
}

RmsBackPlan rms_back_plan(int dtype, int64_t rows, int64_t cols, int nsm) {
  const int e = dtype == PEAT_F32 ? 4 : 8;
  const Shape k = shape_of((cols + e - 1) / e);
  const int64_t groups = std::max(256, k.tpr) / k.tpr;  // of a CTA
  // two CTAs an SM; a long row's pieces fill the SMs already where there are several
  const int64_t pieces = k.longer ? (cols + (int64_t)k.tpr * k.nv * e - 1) / ((int64_t)k.tpr * k.nv * e) : 1;
  const int64_t most = std::max<int64_t>(1, 2 * (int64_t)nsm / pieces);
  RmsBackPlan r;
  r.longer = k.longer;
  r.each = std::max<int64_t>(1, (rows + most * groups - 1) / (most * groups));
  r.ctas = (int)((rows + r.each * groups - 1) / (r.each * groups));
  return r;
}

cudaError_t launch_rmsnorm_backward(int dtype, const RmsBackPlan& plan, const RmsBackParams& in, cudaStream_t s) {
  RmsBackParams p = in;
  p.ctas = plan.ctas;
  p.each = plan.each;
  switch (dtype) {
    case PEAT_F32: return backward_of<PEAT_F32>(p, s);
    case PEAT_F16: return backward_of<PEAT_F16>(p, s);
    default: return backward_of<PEAT_BF16>(p, s);
  }
}

}  // namespace peat
