// 8-bit integer products by the warp-level matrix instructions: few rows, and
// small products of any shape.
//
// Of the two operands "w" is b (its N rows are the 16-row side of the
// instruction) and "t" is a (its M rows the 8-column side).  A lane holds 16
// consecutive integers of a row; word j of the 16 makes the lane's four k
// positions of the j-th of four 16 x 8 x 16 instructions.  Which k a position
// stands for does not matter as long as both operands agree, so no shuffle and
// no transposed load is needed.
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "mm8_common.cuh"
#include "peat_internal.h"

namespace cg = cooperative_groups;

namespace peat {
namespace {

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t word(const uint4& v, int j) { return j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w; }

// sums in float32 become integers, added to `sum`
template <int NT>
__device__ __forceinline__ void drain(float (&c)[NT][4], int (&sum)[NT][4]) {
#pragma unroll
  for (int n = 0; n < NT; n++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      sum[n][i] += __float2int_rn(c[n][i]);
      c[n][i] = 0.0f;
    }
}

constexpr int64_t MM8_STREAM_N = 8192;  // rows of b from which every SM has a warp tile or more of its own

// ---- up to 16 rows of a: bound by the bytes of b -----------------------------
// A CTA of four warps takes 16 rows of b, each warp every fourth run of 64 k
// (and each CTA of a cluster a share of those runs), straight from global
// memory: every byte of b is used once, so nothing is gained by staging it.
// 1 x 4096 x 1024 takes 8 us a call, as long as the host takes to make it.
constexpr int RT = 128;  // threads
template <int OUT, int NT, int MODE>
__global__ void __launch_bounds__(RT) mm8_rows(Mm8Params p) {
  pdl_wait();
  pdl_trigger();
  __shared__ int part[4][NT * 8][17];
  cg::cluster_group cl = cg::this_cluster();
  const int S = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t n0 = ((int64_t)blockIdx.x / S) * 16;
  const int64_t runs = (p.K + 63) / 64;
  const int8_t *alo = p.a, *ahi = p.a + (p.M - 1) * p.lda + p.K, *blo = p.b, *bhi = p.b + (p.N - 1) * p.ldb + p.K;
  float c[NT][4];
  int sum[NT][4];
#pragma unroll
  for (int n = 0; n < NT; n++)
#pragma unroll
    for (int i = 0; i < 4; i++) c[n][i] = 0.0f, sum[n][i] = 0;
  const int8_t* w0 = p.b + (n0 + g) * p.ldb + 16 * t;
  const int8_t* w1 = w0 + 8 * p.ldb;
  const bool has0 = n0 + g < p.N, has1 = n0 + g + 8 < p.N;
  const int step = 4 * S;
  constexpr int U = 4;  // runs in flight
  int since = 0;
  for (int64_t r = rank * 4 + warp; r < runs; r += U * step) {
    uint4 u0[U], u1[U], x[U][NT];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int64_t k = (r + (int64_t)u * step) * 64, left = p.K - k - 16 * t;
      u0[u] = load16<MODE>(w0 + k, has0 ? left : 0, blo, bhi);
      u1[u] = load16<MODE>(w1 + k, has1 ? left : 0, blo, bhi);
#pragma unroll
      for (int n = 0; n < NT; n++)
        x[u][n] = load16<MODE>(p.a + (n * 8 + g) * p.lda + 16 * t + k, n * 8 + g < p.M ? left : 0, alo, ahi);
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
#pragma unroll
      for (int j = 0; j < 4; j++) {
        uint32_t a[4];
        to_half(word(u0[u], j), a[0], a[2]);
        to_half(word(u1[u], j), a[1], a[3]);
#pragma unroll
        for (int n = 0; n < NT; n++) {
          uint32_t b0, b1;
          to_half(word(x[u][n], j), b0, b1);
          mma16816(c[n], a, b0, b1);
        }
      }
    }
    since += U;
    if (since >= MM8_EXACT_K / 64) {
      drain(c, sum);
      since = 0;
    }
  }
  drain(c, sum);
#pragma unroll
  for (int n = 0; n < NT; n++)
#pragma unroll
    for (int i = 0; i < 4; i++) part[warp][n * 8 + 2 * t + (i & 1)][g + 8 * (i >> 1)] = sum[n][i];
  cl.sync();
  // the cluster's CTAs share the tile's elements: 16 b rows of each a row
  typename Mm8Out<OUT>::T* out = static_cast<typename Mm8Out<OUT>::T*>(p.out);
  for (int i = rank * RT + threadIdx.x; i < NT * 8 * 16; i += S * RT) {
    const int m = i >> 4, n = i & 15;
    if (m >= p.M || n0 + n >= p.N) continue;
    int v = 0;
    for (int k = 0; k < S; k++) {
      const int* q = cl.map_shared_rank(&part[0][m][n], k);
#pragma unroll
      for (int w = 0; w < 4; w++) v += q[w * NT * 8 * 17];
    }
    const float s = (p.sa ? __ldg(p.sa + m) : 1.0f) * (p.sb ? __ldg(p.sb + n0 + n) : 1.0f);
    out[m * p.ldo + n0 + n] = Mm8Out<OUT>::make(v, s, p.bias ? __ldg(p.bias + n0 + n) : 0.0f);
  }
  cl.sync();  // the others may still read this CTA's part
}

// ---- up to 64 rows of a and many of b: a stream over b ------------------------
// The rows of a are turned into binary16 once per CTA, in the very registers'
// order, and stay in shared memory (up to 4096 k of 8 rows, 2048 of 16 and 32, 1024
// of 64; longer rows are turned piece by piece for every round of tiles); every
// warp then streams 16 rows of b past them, so a byte
// of b costs its load, its conversion and its share of the instructions.  Where
// a CTA has few such tiles, 2 to 16 warps (`1 << shift`) share the runs of one
// and meet in shared memory; not where that takes more rounds (two warps a tile
// and three rounds for one and two: 29.8 us for 32 x 50257 x 1024, not 27.5).
// 16 x 50257 x 1024 to binary16 takes 17 us, 3.1 TB/s, two thirds of it the
// chain of a warp's 8 loads and of starting; 8 x 16384 x 4096 19 us, 3.6 TB/s
// (a warp a tile: 36); rows off the 16-byte grid, 13 x 30001 x 2050, 33 us (49).
constexpr int ST = 512;
template <int OUT, int NT, int MODE>
__global__ void __launch_bounds__(ST, NT <= 2 ? 2 : 1) mm8_stream(Mm8Params p, int runs_held, int shift) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) uint2 held[];  // [run][n][j][lane]
  int* met = reinterpret_cast<int*>(held + (size_t)runs_held * NT * 4 * 32) + threadIdx.x;  // [n][i][thread]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t runs = (p.K + 63) / 64, tiles = (p.N + 15) / 16;
  const int8_t *alo = p.a, *ahi = p.a + (p.M - 1) * p.lda + p.K, *blo = p.b, *bhi = p.b + (p.N - 1) * p.ldb + p.K;
  const int64_t t0 = tiles * blockIdx.x / gridDim.x, t1 = tiles * (blockIdx.x + 1) / gridDim.x;
  typename Mm8Out<OUT>::T* out = static_cast<typename Mm8Out<OUT>::T*>(p.out);
  constexpr int U = NT <= 2 ? 2 : 4;  // runs of b in flight
  const int parts = 1 << shift, part = warp & (parts - 1);
  for (int64_t round = t0; round < t1; round += ST / 32 >> shift) {
    const int64_t tile = round + (warp >> shift), n0 = tile * 16;
    const bool mine = tile < t1;
    float c[NT][4];
    int sum[NT][4];
#pragma unroll
    for (int n = 0; n < NT; n++)
#pragma unroll
      for (int i = 0; i < 4; i++) c[n][i] = 0.0f, sum[n][i] = 0;
    const int8_t* w0 = p.b + (n0 + g) * p.ldb + 16 * t;
    const int8_t* w1 = w0 + 8 * p.ldb;
    const bool has0 = mine && n0 + g < p.N, has1 = mine && n0 + g + 8 < p.N;
    for (int64_t k0 = 0; k0 < runs; k0 += runs_held) {
      const int here = (int)min((int64_t)runs_held, runs - k0);
      const int first = here * part >> shift, end = here * (part + 1) >> shift;  // of the warp
      uint4 u0[U], u1[U];
      auto load = [&](int r) {
#pragma unroll
        for (int u = 0; u < U; u++) {
          const int64_t k = (k0 + r + u) * 64, left = r + u < end ? p.K - k - 16 * t : 0;
          u0[u] = load16<MODE>(w0 + k, has0 ? left : 0, blo, bhi);
          u1[u] = load16<MODE>(w1 + k, has1 ? left : 0, blo, bhi);
        }
      };
      if (NT <= 2) load(first);  // under way while the rows of a are turned (more rows take the registers)
      if (round == t0 || runs > runs_held) {
        __syncthreads();  // the last readers are done
        for (int i = warp; i < here * NT; i += ST / 32) {
          const int n = i % NT, m = n * 8 + g;
          const int64_t k = (k0 + i / NT) * 64 + 16 * t;
          const uint4 x = load16<MODE>(p.a + m * p.lda + k, m < p.M ? p.K - k : 0, alo, ahi);
#pragma unroll
          for (int j = 0; j < 4; j++) {
            uint2 h;
            to_half(word(x, j), h.x, h.y);
            held[(i * 4 + j) * 32 + lane] = h;
          }
        }
        __syncthreads();
      }
      if (mine) {
        int since = 0;
        for (int r = first; r < end; r += U) {
          if (NT > 2 || r > first) load(r);
#pragma unroll
          for (int u = 0; u < U; u++) {
            if (r + u >= end) break;
            const uint2* x = held + (size_t)(r + u) * NT * 4 * 32 + lane;
#pragma unroll
            for (int j = 0; j < 4; j++) {
              uint32_t a[4];
              to_half(word(u0[u], j), a[0], a[2]);
              to_half(word(u1[u], j), a[1], a[3]);
#pragma unroll
              for (int n = 0; n < NT; n++) {
                const uint2 b = x[(n * 4 + j) * 32];
                mma16816(c[n], a, b.x, b.y);
              }
            }
          }
          since += U;
          if (since >= MM8_EXACT_K / 64) {
            drain(c, sum);
            since = 0;
          }
        }
        drain(c, sum);
      }
    }
    if (parts > 1) {
      if (part)
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
          for (int i = 0; i < 4; i++) met[(n * 4 + i) * ST] = sum[n][i];
      __syncthreads();
      for (int k = 1; k < parts && part == 0; k++)
#pragma unroll
        for (int n = 0; n < NT; n++)
#pragma unroll
          for (int i = 0; i < 4; i++) sum[n][i] += met[(n * 4 + i) * ST + k * 32];
      __syncthreads();
    }
    if (!mine || part) continue;
#pragma unroll
    for (int n = 0; n < NT; n++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const int64_t m = n * 8 + 2 * t + (i & 1), col = n0 + g + 8 * (i >> 1);
        if (m >= p.M || col >= p.N) continue;
        const float s = (p.sa ? __ldg(p.sa + m) : 1.0f) * (p.sb ? __ldg(p.sb + col) : 1.0f);
        out[m * p.ldo + col] = Mm8Out<OUT>::make(sum[n][i], s, p.bias ? __ldg(p.bias + col) : 0.0f);
      }
  }
}

// ---- tiles --------------------------------------------------------------------
// A CTA takes 128 rows of b by 64 rows of a, 64 k a stage, staged as bytes;
// each of its 8 warps 32 x 32, so that an integer that is turned into binary16
// serves four instructions.  128 x 1024 x 1024 takes 9 us, 64 x 4096 x 4096 17:
// a stage's conversions and instructions, 0.8 us, in a chain of K / 64 (few tiles
// have it split over a cluster).
constexpr int TT = 256, TW = 128, TA = 64, TK = 64, TSTAGES = 4;
constexpr int TSTAGE_BYTES = (TW + TA) * TK;
constexpr int T_SMEM = TSTAGES * TSTAGE_BYTES;  // 48 KB; the sums' tile (64 x 132 words) fits in it
static_assert(T_SMEM >= TA * (TW + 4) * 4, "the sums take the stages' place");

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

template <int OUT, int MODE>
__global__ void __launch_bounds__(TT, 2) mm8_tiles(Mm8Params p, int ntw) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(128) int8_t smem[];
  cg::cluster_group cl = cg::this_cluster();
  const int S = (int)cl.num_blocks(), rank = (int)cl.block_rank();
  const int tile = blockIdx.x / S;
  const int64_t n0 = (int64_t)(tile % ntw) * TW, m0 = (int64_t)(tile / ntw) * TA;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int wn = (warp & 3) * 32, wm = (warp >> 2) * 32;
  const int64_t runs = (p.K + TK - 1) / TK, r0 = runs * rank / S, r1 = runs * (rank + 1) / S;
  const int8_t *alo = p.a, *ahi = p.a + (p.M - 1) * p.lda + p.K, *blo = p.b, *bhi = p.b + (p.N - 1) * p.ldb + p.K;
  const uint32_t sbase = (uint32_t)__cvta_generic_to_shared(smem);

  // a thread's three pieces of 16 bytes of a stage: rows of b first, then of a
  const int8_t* src[3];
  bool has[3];
#pragma unroll
  for (int i = 0; i < 3; i++) {
    const int row = (threadIdx.x >> 2) + 64 * i;
    const bool isb = row < TW;
    const int64_t gr = isb ? n0 + row : m0 + row - TW;
    has[i] = gr < (isb ? p.N : p.M);
    src[i] = (isb ? p.b + (has[i] ? gr : 0) * p.ldb : p.a + (has[i] ? gr : 0) * p.lda) + 16 * (threadIdx.x & 3);
  }
  auto load = [&](int64_t r, int st) {
    const int64_t k = r * TK, left = p.K - k - 16 * (threadIdx.x & 3);
#pragma unroll
    for (int i = 0; i < 3; i++) {
      const int at = st * TSTAGE_BYTES + 64 * 64 * i + threadIdx.x * 16;
      if (MODE == 16) {
        const int bytes = has[i] && left > 0 ? (int)(left < 16 ? left : 16) : 0;
        cp_async16(sbase + at, bytes ? src[i] + k : p.a, bytes);
      } else {
        const bool isb = i < 2;
        *reinterpret_cast<uint4*>(smem + at) = load16<MODE>(src[i] + k, has[i] ? left : 0, isb ? blo : alo, isb ? bhi : ahi);
      }
    }
  };
  __shared__ float sas[TA];  // the rows' scales
  if (threadIdx.x < TA) sas[threadIdx.x] = p.sa && m0 + threadIdx.x < p.M ? __ldg(p.sa + m0 + threadIdx.x) : 1.0f;
  float c[8][4];
  int sum[8][4];
#pragma unroll
  for (int n = 0; n < 8; n++)
#pragma unroll
    for (int i = 0; i < 4; i++) c[n][i] = 0.0f, sum[n][i] = 0;

#pragma unroll
  for (int s = 0; s < TSTAGES - 1; s++) {
    if (r0 + s < r1) load(r0 + s, s);
    if (MODE == 16) asm volatile("cp.async.commit_group;" ::: "memory");
  }
  int since = 0;
  for (int64_t r = r0; r < r1; r++) {
    const int st = (int)((r - r0) % TSTAGES);
    if (MODE == 16) asm volatile("cp.async.wait_group %0;" ::"n"(TSTAGES - 2) : "memory");
    __syncthreads();  // the stage is there, and the one before it is free
    if (r + TSTAGES - 1 < r1) load(r + TSTAGES - 1, (int)((r - r0 + TSTAGES - 1) % TSTAGES));
    if (MODE == 16) asm volatile("cp.async.commit_group;" ::: "memory");
    const int8_t* sb = smem + st * TSTAGE_BYTES;
    const int8_t* sa = sb + TW * TK;
    uint4 w[4], x[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      w[i] = *reinterpret_cast<const uint4*>(sb + (wn + i * 8 + g) * TK + 16 * t);
      x[i] = *reinterpret_cast<const uint4*>(sa + (wm + i * 8 + g) * TK + 16 * t);
    }
#pragma unroll
    for (int j = 0; j < 4; j++) {
      uint32_t a[2][4], b[4][2];
#pragma unroll
      for (int i = 0; i < 2; i++) {
        to_half(word(w[2 * i], j), a[i][0], a[i][2]);
        to_half(word(w[2 * i + 1], j), a[i][1], a[i][3]);
      }
#pragma unroll
      for (int i = 0; i < 4; i++) to_half(word(x[i], j), b[i][0], b[i][1]);
#pragma unroll
      for (int i = 0; i < 2; i++)
#pragma unroll
        for (int n = 0; n < 4; n++) mma16816(c[i * 4 + n], a[i], b[n][0], b[n][1]);
    }
    if (++since == MM8_EXACT_K / TK) {
      drain(c, sum);
      since = 0;
    }
  }
  drain(c, sum);
  if (MODE == 16) asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  int* tot = reinterpret_cast<int*>(smem);  // [TA][TW + 4]
  constexpr int P = TW + 4;
#pragma unroll
  for (int i = 0; i < 2; i++)
#pragma unroll
    for (int n = 0; n < 4; n++)
#pragma unroll
      for (int e = 0; e < 4; e++)
        tot[(wm + n * 8 + 2 * t + (e & 1)) * P + wn + i * 16 + g + 8 * (e >> 1)] = sum[i * 4 + n][e];
  cl.sync();
  typename Mm8Out<OUT>::T* out = static_cast<typename Mm8Out<OUT>::T*>(p.out);
  const int col = threadIdx.x & 127;
  const int64_t n = n0 + col;
  if (n < p.N) {
    const float sb = p.sb ? __ldg(p.sb + n) : 1.0f, bias = p.bias ? __ldg(p.bias + n) : 0.0f;
    const int rows = (int)min((int64_t)TA, p.M - m0), row0 = rank * 2 + (threadIdx.x >> 7);
    if (S == 1) {
#pragma unroll 8
      for (int row = row0; row < rows; row += 2)
        out[(m0 + row) * p.ldo + n] = Mm8Out<OUT>::make(tot[row * P + col], sas[row] * sb, bias);
    } else {
      for (int row = row0; row < rows; row += 2 * S) {
        int v = 0;
        for (int k = 0; k < S; k++) v += *cl.map_shared_rank(&tot[row * P + col], k);
        out[(m0 + row) * p.ldo + n] = Mm8Out<OUT>::make(v, sas[row] * sb, bias);
      }
    }
  }
  cl.sync();  // the others may still read this CTA's sums
}

template <typename F, typename... A>
cudaError_t cluster_launch(F kernel, int64_t tiles, int S, int threads, int smem, cudaStream_t s, A... args) {
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)S;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * S));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// parts of the k range of a tile: until the SMs have two each, 8 runs of 64 k or more to start from
int tile_parts(int64_t tiles, int64_t runs, int nsm) {
  int S = 1;
  while (S < 8 && tiles * S < 2 * (int64_t)nsm && runs >= 8 * S) S *= 2;
  return S;
}

template <int OUT, int NT, int MODE>
cudaError_t stream(const Mm8Params& p, int nsm, cudaStream_t s) {
  const int64_t runs = (p.K + 63) / 64, tiles = (p.N + 15) / 16;
  constexpr int RUN = NT * 1024, CTAS = NT <= 2 ? 2 : 1, MOST = 16 * 8 * 1024;  // bytes of a held run; of all of them
  const int held = (int)std::min<int64_t>(runs, (CTAS == 2 ? MOST / 2 : MOST) / RUN);
  constexpr int MET = NT * 4 * ST * 4;  // what the parts of tiles meet in
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_smem(mm8_stream<OUT, NT, MODE>, MOST + MET, allowed);
  if (e != cudaSuccess) return e;
  const unsigned ctas = (unsigned)std::min<int64_t>(CTAS * (int64_t)nsm, tiles);
  const int64_t most = (tiles + ctas - 1) / ctas;  // tiles of a CTA
  int shift = 0;  // 2^shift parts of two runs or more
  while ((2 * most << shift) <= ST / 32 && runs >= 4 << shift) shift++;
  return launch_dependent(mm8_stream<OUT, NT, MODE>, ctas, ST, (size_t)held * RUN + (shift ? MET : 0), s, p, held, shift);
}

template <int OUT, int MODE>
cudaError_t direct(const Mm8Params& p, int nsm, cudaStream_t s) {
  const int64_t runs = (p.K + 63) / 64;
  if (p.M <= 64 && p.K > 0 && p.N >= MM8_STREAM_N) {
    if (p.M <= 8) return stream<OUT, 1, MODE>(p, nsm, s);
    if (p.M <= 16) return stream<OUT, 2, MODE>(p, nsm, s);
    if (p.M <= 32) return stream<OUT, 4, MODE>(p, nsm, s);
    return stream<OUT, 8, MODE>(p, nsm, s);
  }
  if (p.M <= 16) {
    const int64_t tiles = (p.N + 15) / 16;
    int S = 1;  // share the k runs while the SMs are not filled and every warp keeps a few
    while (S < 8 && tiles * S < 2 * (int64_t)nsm && runs >= 32 * S) S *= 2;
    if (p.M <= 8) return cluster_launch(mm8_rows<OUT, 1, MODE>, tiles, S, RT, 0, s, p);
    return cluster_launch(mm8_rows<OUT, 2, MODE>, tiles, S, RT, 0, s, p);
  }
  const int64_t ntw = (p.N + TW - 1) / TW, tiles = ntw * ((p.M + TA - 1) / TA);
  const int S = tile_parts(tiles, runs, nsm);
  // (with the static part a little above the 48 KB that need no leave)
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_smem(mm8_tiles<OUT, MODE>, T_SMEM, allowed);
  if (e != cudaSuccess) return e;
  return cluster_launch(mm8_tiles<OUT, MODE>, tiles, S, TT, T_SMEM, s, p, (int)ntw);
}

template <int OUT>
cudaError_t direct_out(const Mm8Params& p, int nsm, cudaStream_t s) {
  return mm8_aligned(p) ? direct<OUT, 16>(p, nsm, s) : direct<OUT, 1>(p, nsm, s);
}

}  // namespace

// Microseconds of a call, fitted to those measured for M from 32 to 1024, N to
// 16 384 and K to 16 384: one run of 64 k of a tile takes 0.8 (off the 16-byte
// grid, where it is loaded through registers, 1.4), an SM's CTAs share it.
double mm8_direct_time(int64_t M, int64_t N, int64_t K, bool aligned, int nsm) {
  if (M <= 16 || (M <= 64 && N >= MM8_STREAM_N)) return 0.0;  // bound by b's bytes: nothing is faster
  const int64_t tiles = ((N + TW - 1) / TW) * ((M + TA - 1) / TA), runs = (K + TK - 1) / TK;
  const int S = tile_parts(tiles, runs, nsm);
  const double share = std::max(1.0, 1.1 * (double)(tiles * S) / nsm);
  return 6.5 + (aligned ? 0.8 : 1.4) * std::ceil((double)runs / S) * share;
}

cudaError_t launch_mm8_direct(int out_dtype, const Mm8Params& p, int nsm, cudaStream_t s) {
  switch (out_dtype) {
    case PEAT_F32: return direct_out<PEAT_F32>(p, nsm, s);
    case PEAT_F16: return direct_out<PEAT_F16>(p, nsm, s);
    case PEAT_BF16: return direct_out<PEAT_BF16>(p, nsm, s);
    default: return direct_out<PEAT_OUT_I32>(p, nsm, s);
  }
}

}  // namespace peat
