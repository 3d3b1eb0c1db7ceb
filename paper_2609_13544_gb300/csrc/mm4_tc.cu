// Products of 4-bit matrices on the fifth-generation tensor cores, which scale
// each block of values by the bytes that go with it and add up in float32.
//
// A CTA makes tiles of 128 rows of one operand by `bn` rows of the other, or a pair of
// CTAs tiles of 256 by `bn` (each holds 128 rows and half of the others), which needs
// fewer bytes for an instruction; persistent over the tiles.  An instruction of 64 k
// takes about 128 cycles for any bn up to 256, so large products are bound by it at 256
// (8192 x 8192 x 8192 to bfloat16: mxfp4 168 us, 6.5 PFLOP/s, nvfp4 180; the chip's
// form of 96 k, of 1.5 times that rate, is not used: a stage's 256 k are no multiple of
// it), short k by the results' way out (16384 x 4096 x 1024: 36.5 us, with a bias 39.3,
// 21 of them bytes), small ones by the chain of copy, instruction and result (1 x 4096 x
// 1024: 4.5 us).  Two pairs in a cluster, each reading half of what both need of the
// other operand, were no faster (178 us where one pair took 171: 72 of 76 pairs find
// place, and reading is not what bounds it).
//
// A stage is 256 k: a 128-byte piece of every row, swizzled by the copy, and the
// scales' tiles, which lie in memory as the instruction wants them in tensor memory.
// Warp roles: one thread issues the copies, one the moves of scales and the matrix
// instructions, sixteen warps (eight for 128 x 128) turn accumulators into results
// while the other one fills.
//
// Few rows of a: the tile's 128 rows are b's (SWAP), so that the instruction
// spends nothing on rows that a does not have.
#include <cooperative_groups.h>

#include <algorithm>

#include "f4.cuh"
#include "peat_internal.h"
#include "tc_common.cuh"
#include "vec16.cuh"

namespace cg = cooperative_groups;

namespace peat {
namespace {

constexpr int SK = 256;                 // k of a stage
constexpr int P_BYTES = 128 * SK / 2;   // its rows on the 128-row side
constexpr int PS_BYTES = 2048, QS_BYTES = 4096;  // its scales: tiles of 64 k or more, of up to two blocks of 128 rows
constexpr int FEW_ROWS = 192, MOST_STAGES = 8;  // rows of a up to which the tile's 128 rows may be b's
// Warps for results: they take a tile's chunks of columns in turn, 32 rows each.
template <int CG, bool SWAP>
struct Warps {
  static constexpr int PARTS = SWAP || CG == 2 ? 4 : 2, EPI = 4 * PARTS, COPY = EPI, MMA = COPY + 1, THREADS = (MMA + 1) * 32;
  static constexpr int STEP = SWAP ? 16 : 64;           // columns of a chunk
  static constexpr int EDGE = SWAP ? FEW_ROWS / PARTS : STEP;  // columns of a warp
  // a place where a warp's results wait for their copy out, and its columns' scales and bias
  static constexpr int BOX = SWAP ? 0 : 4096, BYTES = EPI * (BOX + EDGE * 2 * 4);
};
constexpr int BARS = 256;
constexpr int SUM_ROW = 132;  // words from one row of sums to the next
constexpr int SMEM = 227 * 1024;
// Tensor memory: two accumulators, then a stage's scales.  A pair's accumulators have
// 256 columns and share 32 (mxfp4) or 48 of them: the next tile's instructions wait
// until the warps that have these have read them, not for the whole tile.
template <int CG, int FMT>
struct Tmem {
  static constexpr int APART = CG == 2 ? (FMT == PEAT_MXFP4 ? 224 : 208) : FEW_ROWS, SCALES = CG == 2 ? APART + 256 : 2 * FEW_ROWS;
};

constexpr int stage_bytes(int rows) { return P_BYTES + rows * (SK / 2) + PS_BYTES + QS_BYTES; }

struct Tc4Params {
  const uint8_t* ps;  // scales of the 128-row side and of the other
  const uint8_t* qs;
  const float* sp;    // of their rows, or null
  const float* sq;
  const float* bias;
  OutPlace out;
  int64_t P, Q;       // rows
  int64_t tiles;      // of scales along k
  int steps;          // instructions of 64 k
  int bn, pt, qt, stages;  // (tiles start on blocks of 128 rows of Q: bn is 128, 256, or all of them)
  int units;          // the output's rows are whole 16-byte units
  int splits;         // CTAs of a cluster that share a tile's k range: 1, 2, 4 or 8 (then a cluster has one tile)
  unsigned int* status;
  uint32_t wait_limit;
};

__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, int x, int row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(x), "r"(row), "r"(bar)
      : "memory");
}
// the same, its bytes counted on a barrier of the pair's even CTA
__device__ __forceinline__ void tma_pair(uint32_t dst, const CUtensorMap* map, int x, int row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, "
      "%3}], [%4];" ::"r"(dst),
      "l"(map), "r"(x), "r"(row), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
// arrives on the barrier (of both CTAs of a pair) once the instructions issued so far are done
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
  if (CG == 2) return commit_both(bar, 3);
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// a tile of scales into four columns of tensor memory: 32 lanes of 16 bytes, the same for each quarter of the lanes
// (of a pair: each CTA's own)
template <int CG>
__device__ __forceinline__ void scales_in(uint32_t col, uint64_t d) {
  if (CG == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(col), "l"(d) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(col), "l"(d) : "memory");
}
// 128 rows (of a pair: 256) by bn, 64 k: 4-bit values, a scale for 32 (mxfp4: two of the four bytes of a tile, from the
// byte on that the instruction's descriptor names) or for 16
template <int FMT, int CG>
__device__ __forceinline__ void mma4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool accumulate) {
#define PEAT_MMA4(GROUP, SCALES)                                                                                      \
  asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n tcgen05.mma.cta_group::" GROUP                            \
               ".kind::mxf4nvf4.block_scale.scale_vec::" SCALES " [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d),      \
               "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"((uint32_t)accumulate)                                \
               : "memory")
  if constexpr (FMT == PEAT_MXFP4 && CG == 1) PEAT_MMA4("1", "2X");
  if constexpr (FMT == PEAT_MXFP4 && CG == 2) PEAT_MMA4("2", "2X");
  if constexpr (FMT == PEAT_NVFP4 && CG == 1) PEAT_MMA4("1", "4X");
  if constexpr (FMT == PEAT_NVFP4 && CG == 2) PEAT_MMA4("2", "4X");
#undef PEAT_MMA4
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(addr));
}

// a ring's slot and the parity of its round
struct Turn {
  int s = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int n) {
    if (++s == n) s = 0, phase ^= 1;
  }
};
constexpr int GROUP = 8;
struct Place4 {
  int64_t p0, q0;
};
template <int CG>
__device__ __forceinline__ Place4 place_of(const Tc4Params& p, int u) {
  // groups of GROUP tiles of P, column by column: the CTAs at work at any time share few rows of either
  // (there are at most 2^27 tiles)
  const unsigned per = GROUP * (unsigned)p.qt, g = (unsigned)u / per, in = (unsigned)u - g * per;
  const unsigned wide = min(GROUP, p.pt - (int)g * GROUP), q = in / wide;
  return Place4{(int64_t)(g * GROUP + in - q * wide) * (CG * 128), (int64_t)q * p.bn};
}

__device__ __forceinline__ float4 load_cluster_float4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}
template <int OUT>
__device__ __forceinline__ void put_one(void* out, int64_t at, float y) {
  typename Mm8Out<OUT>::T* o = static_cast<typename Mm8Out<OUT>::T*>(out) + at;
  if constexpr (OUT == PEAT_F32) *o = y;
  else if constexpr (OUT == PEAT_F16) *o = __float2half_rn(y);
  else *o = __float2bfloat16_rn(y);
}

// 16 bytes of results from v[c] on
template <int OUT>
__device__ __forceinline__ uint4 packed(const float* v) {
  if constexpr (OUT == PEAT_F32) return *reinterpret_cast<const uint4*>(v);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if constexpr (OUT == PEAT_BF16) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    } else {
      const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Half h of 64 columns of a warp's 32 rows, a row a lane, the first or the second one in
// turn, scaled and biased, through shared memory (128-byte rows, swizzled) and out by
// copies of 32 rows, which write whole lines and leave out what lies beyond the matrix.
// (Sectors straight from the lanes, 32 rows a store, took 1.3 us a tile of 128 x 128,
// twice its instructions' time.)
template <int OUT>
__device__ __forceinline__ void put_box(char* box, const CUtensorMap* map, float (&v)[32], int h, int turn, bool scaled, float sp,
                                        const float* sq, bool biased, const float* bias, int64_t row0, int64_t col0, int64_t N) {
  constexpr int B = (int)sizeof(typename Mm8Out<OUT>::T), HALVES = B == 2 ? 2 : 1;  // that a box holds
  const int lane = threadIdx.x & 31;
  if (scaled) {
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
      const float4 f = *reinterpret_cast<const float4*>(sq + 32 * h + j);
      const float2 lo = mul2(both(sp), make_float2(f.x, f.y)), hi = mul2(both(sp), make_float2(f.z, f.w));
      // (one by one: a pair's product and the bias' sum would become one rounding)
      v[j] = __fmul_rn(v[j], lo.x);
      v[j + 1] = __fmul_rn(v[j + 1], lo.y);
      v[j + 2] = __fmul_rn(v[j + 2], hi.x);
      v[j + 3] = __fmul_rn(v[j + 3], hi.y);
    }
  }
  if (biased) {
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
      const float4 f = *reinterpret_cast<const float4*>(bias + 32 * h + j);
      put_pair(v, j / 2, add2(pair(v, j / 2), make_float2(f.x, f.y)));
      put_pair(v, j / 2 + 1, add2(pair(v, j / 2 + 1), make_float2(f.z, f.w)));
    }
  }
  if (HALVES == 1 || turn == 0) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // the place is free
    __syncwarp();
  }
  const int c0 = HALVES == 2 ? 4 * h : 0;
#pragma unroll
  for (int c = 0; c < 8 / HALVES; c++)
    *reinterpret_cast<uint4*>(box + lane * 128 + (((c0 + c) ^ (lane & 7)) * 16)) = packed<OUT>(v + c * (16 / B));
  if (HALVES == 2 && turn == 0) return;
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  const int64_t col = HALVES == 2 ? col0 : col0 + 32 * h;
  if (lane == 0 && col < N) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"((int)col),
                 "r"((int)row0), "r"(sptr(box))
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
}

// mp, mq: the codes; msp, msq: the tiles of scales, where a pair copies them; mo: out, where it can be copied to
template <int OUT, int FMT, bool SWAP, int CG>
__global__ void __launch_bounds__(Warps<CG, SWAP>::THREADS, 1)
    mm4_tc(Tc4Params p, const __grid_constant__ CUtensorMap mp, const __grid_constant__ CUtensorMap mq,
           const __grid_constant__ CUtensorMap msp, const __grid_constant__ CUtensorMap msq, const __grid_constant__ CUtensorMap mo) {
  using W = Warps<CG, SWAP>;
  constexpr int PARTS = W::PARTS, EPI_WARPS = W::EPI, COPY_WARP = W::COPY, MMA_WARP = W::MMA, EDGE = W::EDGE, STEP = W::STEP;
  extern __shared__ char raw[];
  char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const int bn = p.bn, half = bn / CG, stage = stage_bytes(half);  // rows of the other operand: the tile's, this CTA's
  // a pair's CTAs differ in their rank; the even one issues the instructions
  uint32_t rank = 0;
  if (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  // parts of a tile's k range, in stages
  uint32_t part_k = 0;
  if (CG == 1 && p.splits > 1) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(part_k));
  const bool split = CG == 1 && p.splits > 1;
  const int together = CG == 1 ? p.splits : 2, first = blockIdx.x / together, apart = gridDim.x / together;
  const int all_k = (p.steps + 3) / 4, k0 = (int)((int64_t)all_k * part_k / p.splits), k1 = (int)((int64_t)all_k * (part_k + 1) / p.splits);
  char* edges = smem + p.stages * stage;
  const uint32_t full = sptr(edges + W::BYTES), empty = full + 8 * MOST_STAGES, acc_full = empty + 8 * MOST_STAGES,
                 acc_empty = acc_full + 16, shared_empty = acc_empty + 16, last = shared_empty + 8;
  volatile uint32_t* tmem_at = reinterpret_cast<volatile uint32_t*>(edges + W::BYTES + 8 * (2 * MOST_STAGES + 6));
  static_assert(8 * (2 * MOST_STAGES + 6) + 4 <= BARS, "the barriers fit");
  constexpr int TILE_K = F4<FMT>::BLOCK * 4, PER = SK / TILE_K;  // k of a tile of scales; tiles of a stage
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int units = p.pt * p.qt, nk = k1 - k0;
  const uint32_t base = sptr(smem);

  if (threadIdx.x == 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mp) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mq) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < MOST_STAGES; i++) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; i++) {
      mbar_init(acc_full + 8 * i, 1);
      mbar_init(acc_empty + 8 * i, CG * EPI_WARPS);
    }
    mbar_init(shared_empty, CG * 4);  // the warps of one chunk of columns
    mbar_init(last, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == MMA_WARP) {
    if (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(sptr((const void*)tmem_at))
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(sptr((const void*)tmem_at))
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  if (CG == 2) cg::this_cluster().sync();
  else __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_at;
  pdl_trigger();

  bool ok = true;
  if (warp == COPY_WARP) {
    if (elect_one()) {
      pdl_wait();
      Turn at;
      int64_t seq = 0;
      for (int u = first; u < units && ok; u += apart) {
        const Place4 t = place_of<CG>(p, u);
        const int64_t pb = t.p0 >> 7, qb = t.q0 >> 7, q_end = min(t.q0 + bn, p.Q);
        const int qbs = (int)(((q_end - 1) >> 7) - qb) + 1;  // blocks of 128 rows that the tile's lie in
        const uint8_t* ps = p.ps + (pb * p.tiles + (int64_t)k0 * PER) * SCALE_TILE;
        const uint8_t* qs = p.qs + (qb * p.tiles + (int64_t)k0 * PER) * SCALE_TILE;
        int left = (int)p.tiles - k0 * PER;
        for (int k = k0; k < k1; k++, seq++, left -= PER, ps += PER * SCALE_TILE, qs += PER * SCALE_TILE) {
          if (!(ok = mbar_wait(empty + 8 * at.s, at.phase ^ 1, p.wait_limit))) break;
          const uint32_t dst = base + at.s * stage, bar = full + 8 * at.s, qd = dst + P_BYTES, sd = qd + half * (SK / 2);
          if constexpr (CG == 2) {  // all bytes of both CTAs count on the even one's barrier
            const uint32_t even = mapa(bar, 0);
            if (rank == 0) mbar_expect(bar, 2 * (P_BYTES + half * (SK / 2) + 3 * PER * SCALE_TILE));
            tma_pair(dst, &mp, k * (SK / 2), (int)(t.p0 + rank * 128), even);
            tma_pair(qd, &mq, k * (SK / 2), (int)(t.q0 + rank * half), even);
            // (past a row's last tile lie the next row's, which no instruction takes; past all of them zeros)
            const int64_t kt = (int64_t)k * PER;
            tma_pair(sd, &msp, 0, (int)((pb + rank) * p.tiles + kt), even);
            tma_pair(sd + PS_BYTES, &msq, 0, (int)(qb * p.tiles + kt), even);
            tma_pair(sd + PS_BYTES + PER * SCALE_TILE, &msq, 0, (int)((qb + 1) * p.tiles + kt), even);
            at.next(p.stages);
            continue;
          }
          const uint32_t n = (uint32_t)min(PER, left) * SCALE_TILE;
          mbar_expect(bar, P_BYTES + bn * (SK / 2) + n * (1 + qbs));
          tma_rows(dst, &mp, k * (SK / 2), (int)t.p0, bar);
          tma_rows(qd, &mq, k * (SK / 2), (int)t.q0, bar);
          bulk(sd, ps, n, bar);
          bulk(sd + PS_BYTES, qs, n, bar);
          if (qbs > 1) bulk(sd + PS_BYTES + PER * SCALE_TILE, qs + p.tiles * SCALE_TILE, n, bar);
          at.next(p.stages);
        }
      }
      // a stage's copies have landed when its instructions are done with it
      for (int j = 0; j < p.stages && j < seq; j++) {
        const int64_t q = seq - 1 - j;
        mbar_wait(empty + 8 * (int)(q % p.stages), (uint32_t)(q / p.stages & 1), END_LIMIT);
      }
    }
  } else if (warp == MMA_WARP) {
    if (rank == 0 && elect_one()) {
      // (The loop is one thread's: what it does for an instruction has to fit into the
      // one before.)
      const uint64_t desc = block_desc(0), scale_desc = (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
      const uint32_t at_q = P_BYTES >> 4, at_s = (P_BYTES + half * (SK / 2)) >> 4, tall = CG == 2 || bn > 128;
      const uint32_t idesc = (1u << 7) | (1u << 10) | ((bn / 8) << 17) | ((FMT == PEAT_MXFP4 ? 1u : 0u) << 23) | ((CG * 128u / 16) << 24);
      const uint32_t tp = tmem + Tmem<CG, FMT>::SCALES, tq = tp + 4 * PER;  // 4 and 8 columns for a tile
      static_assert(Tmem<CG, FMT>::SCALES + 12 * PER <= 512, "tensor memory has 512 columns");
      Turn at;
      uint32_t acc = 0, acc_phase = 1, shared_phase = 1;
      for (int u = first; u < units && ok && nk; u += apart) {
        if (!(ok = mbar_wait(acc_empty + 8 * acc, acc_phase, p.wait_limit))) break;
        if (CG == 2 && !(ok = mbar_wait(shared_empty, shared_phase, p.wait_limit))) break;
        shared_phase ^= 1;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + acc * Tmem<CG, FMT>::APART;
        for (int k = k0; k < k1; k++) {
          if (!(ok = mbar_wait(full + 8 * at.s, at.phase, p.wait_limit))) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t from = (base + at.s * stage) >> 4;
          const uint64_t a = desc + from, b = a + at_q, sd = scale_desc + from + at_s;
#pragma unroll
          for (int j = 0; j < PER; j++) {
            scales_in<CG>(tp + 4 * j, sd + j * (SCALE_TILE >> 4));
            scales_in<CG>(tq + 8 * j, sd + ((PS_BYTES + j * SCALE_TILE) >> 4));
            if (tall) scales_in<CG>(tq + 8 * j + 4, sd + ((PS_BYTES + (PER + j) * SCALE_TILE) >> 4));
          }
          const int here = p.steps - 4 * k;
#pragma unroll
          for (int j = 0; j < 4; j++) {
            if (j >= here) break;
            constexpr int TILE_STEPS = 4 / PER;
            mma4<FMT, CG>(d, a + 2 * j, b + 2 * j, idesc | (FMT == PEAT_MXFP4 ? (2u * (j & 1)) * 0x20000010u : 0u),
                          tp + 4 * (j / TILE_STEPS), tq + 8 * (j / TILE_STEPS), k + j > k0);
          }
          commit<CG>(empty + 8 * at.s);
          at.next(p.stages);
        }
        if (ok) commit<CG>(acc_full + 8 * acc);
        acc ^= 1;
        acc_phase ^= acc == 0;
      }
      // whatever was issued is done before the accumulators are given back
      commit<CG>(last);
      mbar_wait(last, 0, END_LIMIT);
    }
  } else {  // results: a warp has 32 of the 128 rows, and every PARTS-th chunk of columns
    pdl_wait();
    int i = 0;
    const int part = warp >> 2, quarter = warp & 3, chunks = bn / STEP;
    char* box = edges + warp * W::BOX;
    float* sq = reinterpret_cast<float*>(edges + EPI_WARPS * W::BOX) + warp * (EDGE * 2);
    float* bias = sq + EDGE;
    const bool scaled = p.sp || p.sq;
    // scales and bias of a tile, fetched while the one before is at work
    constexpr int MINE = EDGE / STEP, KEPT = (EDGE + 31) / 32;
    float sq_next[KEPT], bias_next[KEPT], sp_next = 1.0f, row_bias_next = 0.0f;
    auto column = [&](int c) { return (part + PARTS * (c / STEP)) * STEP + c % STEP; };  // the warp's c-th, of the tile
    auto fetch = [&](int u) {
      if (u >= units) return;
      const Place4 t = place_of<CG>(p, u);
      const int64_t row = t.p0 + rank * 128 + quarter * 32 + lane;
      if (p.sp && row < p.P) sp_next = __ldcg(p.sp + row);
      if (SWAP && p.bias && row < p.P) row_bias_next = __ldcg(p.bias + row);
#pragma unroll
      for (int k = 0; k < KEPT; k++) {
        const int c = k * 32 + lane;
        const bool in = c < EDGE && column(c) < bn && t.q0 + column(c) < p.Q;
        sq_next[k] = p.sq && in ? __ldcg(p.sq + t.q0 + column(c)) : 1.0f;
        bias_next[k] = !SWAP && p.bias && in ? __ldcg(p.bias + t.q0 + column(c)) : 0.0f;
      }
    };
    const uint32_t release = CG == 2 ? mapa(acc_empty, 0) : acc_empty, release_shared = CG == 2 ? mapa(shared_empty, 0) : 0;
    auto released = [&](uint32_t bar) {
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane) return;
      if (CG == 2) mbar_arrive_cluster(bar);
      else mbar_arrive(bar);
    };
    fetch(first);
    for (int u = first; u < units && ok; u += apart, i++) {
      const Place4 t = place_of<CG>(p, u);
      const int64_t row0 = t.p0 + rank * 128 + quarter * 32, row = row0 + lane;
      const float sp = sp_next, row_bias = row_bias_next;
      const int acc = i & 1;
      __syncwarp();
#pragma unroll
      for (int k = 0; k < KEPT; k++)
        if (k * 32 + lane < EDGE) {
          sq[k * 32 + lane] = sq_next[k];
          if (!SWAP) bias[k * 32 + lane] = bias_next[k];
        }
      __syncwarp();
      fetch(u + apart);
      if (nk) {
        if (!(ok = warp_wait(acc_full + 8 * acc, i / 2 & 1, p.wait_limit))) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      }
      const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + acc * Tmem<CG, FMT>::APART;
      if (split) {
        // The sums go to the stages' place (the last instruction is done with it), where
        // the cluster's other parts find them: contiguous along the output's rows.
        float* sums = reinterpret_cast<float*>(smem);
        const int r = quarter * 32 + lane;
        for (int c = part * 16; c < bn; c += PARTS * 16) {
          float v[16];
          tmem_load16(taddr + c, reinterpret_cast<uint32_t(&)[16]>(v));
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          if (SWAP) {
#pragma unroll
            for (int j = 0; j < 16; j++) sums[(c + j) * SUM_ROW + r] = v[j];
          } else {
#pragma unroll
            for (int j = 0; j < 16; j += 4)
              *reinterpret_cast<float4*>(sums + r * SUM_ROW + c + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
          }
        }
        break;
      }
      const int rows = (int)max((int64_t)0, min((int64_t)32, p.P - row0));
#pragma unroll
      for (int k = 0; k < MINE; k++) {
        const int c = part + PARTS * k;
        if (c >= chunks) break;
        const int at = k * STEP;
        const int64_t col0 = t.q0 + c * STEP;
        if constexpr (SWAP) {
          float v[16];
          if (nk) {
            tmem_load16(taddr + c * STEP, reinterpret_cast<uint32_t(&)[16]>(v));
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          } else {
#pragma unroll
            for (int j = 0; j < 16; j++) v[j] = 0.0f;
          }
          if (c + PARTS >= chunks) released(release + 8 * acc);
#pragma unroll
          for (int j = 0; j < 16; j++) {
            float y = v[j];
            if (scaled) y = __fmul_rn(y, __fmul_rn(sq[at + j], sp));
            if (p.bias) y = __fadd_rn(y, row_bias);
            if (col0 + j < p.Q && row < p.P) put_one<OUT>(p.out.out, (col0 + j) * p.out.ldo + row, y);
          }
        } else {
          // (a copy out writes whole 16-byte units: the row's last columns go by themselves if they are not)
          const bool boxed = p.out.vec && (p.units || col0 + STEP <= p.out.N);
          // Of a pair's accumulators the first ends with the shared columns, the second starts with them: the first
          // one's last half goes first (16384 x 4096 x 1024: mxfp4 37.5 us for 38.4).
          const int half0 = CG == 2 && boxed && !acc, sharing = CG == 2 && part == (acc ? 0 : 3);
          auto take = [&](float (&v)[32], int h, int turn) {  // 32 columns at a time
            if (nk) {
              tmem_load32(taddr + c * STEP + 32 * h, reinterpret_cast<uint32_t(&)[32]>(v));
              asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            } else {
#pragma unroll
              for (int j = 0; j < 32; j++) v[j] = 0.0f;
            }
            if (sharing && (FMT == PEAT_MXFP4 ? h != acc : turn == 1)) released(release_shared);
            if (turn == 1 && c + PARTS >= chunks) released(release + 8 * acc);
          };
          if (boxed) {
#pragma unroll 1
            for (int turn = 0; turn < 2; turn++) {
              const int h = turn ^ half0;
              float v[32];
              take(v, h, turn);
              if (row0 < p.P) put_box<OUT>(box, &mo, v, h, turn, scaled, sp, sq, p.out.biased, bias, row0, col0, p.out.N);
            }
          } else {
            const OutPlace off_grid{p.out.out, p.out.ldo, p.out.N, p.out.biased, false};
            uint32_t carry[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 1
            for (int h = 0; h < 2; h++) {
              float v[32];
              take(v, h, h);
              put_columns<OUT>(off_grid, v, sp, sq + 32 * h, bias + 32 * h, row0, rows, col0 + 32 * h, h == 0, h == 1, carry);
            }
          }
        }
      }
      if (part >= chunks) released(release + 8 * acc);
    }
    // (the boxes are read before the CTA ends, and written before the next kernel reads them)
    if (!SWAP && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  __syncwarp();
  if (split) {
    // The parts meet: each CTA adds up its share of the columns, in the parts' order.
    cg::this_cluster().sync();
    if (warp < EPI_WARPS && ok && first < units) {
      const Place4 t = place_of<CG>(p, first);
      // four of a row of the output at a time: of a column of sums (SWAP), or of a row's share
      const int c0 = bn * (int)part_k / p.splits, nc = bn * ((int)part_k + 1) / p.splits - c0;
      const int per = SWAP ? 5 : 5 - (__ffs(p.splits) - 1);  // (not SWAP: 128 columns)
      const uint32_t sums = sptr(smem);
      // (a thread's place along the rows is the same in all its turns)
      const int along = (threadIdx.x & ((1 << per) - 1)) * 4;
      const int64_t from = SWAP ? t.p0 + along : t.q0 + c0 + along, limit = SWAP ? p.P : p.Q;
      const float *mine = SWAP ? p.sp : p.sq, *others = SWAP ? p.sq : p.sp;
      float scale[4], bias[4];
#pragma unroll
      for (int j = 0; j < 4; j++) {
        scale[j] = mine && from + j < limit ? __ldcg(mine + from + j) : 1.0f;
        bias[j] = p.bias && from + j < limit ? __ldcg(p.bias + from + j) : 0.0f;
      }
#pragma unroll 2
      for (int i = threadIdx.x; i < 32 * nc; i += EPI_WARPS * 32) {
        const int over = i >> per;
        const int64_t m = SWAP ? t.q0 + c0 + over : t.p0 + over;  // the output's row
        if (m >= (SWAP ? p.Q : p.P)) continue;
        const uint32_t at = sums + ((SWAP ? c0 + over : over) * SUM_ROW + (SWAP ? along : c0 + along)) * 4;
        const float other = others ? __ldcg(others + m) : 1.0f;
        float4 x[8];
#pragma unroll
        for (int k = 0; k < 8; k++)
          if (k < p.splits) x[k] = load_cluster_float4(mapa(at, k));
        float y[4] = {x[0].x, x[0].y, x[0].z, x[0].w};
#pragma unroll
        for (int k = 1; k < 8; k++)
          if (k < p.splits) y[0] += x[k].x, y[1] += x[k].y, y[2] += x[k].z, y[3] += x[k].w;
#pragma unroll
        for (int j = 0; j < 4; j++) {
          if (from + j >= limit) break;
          if (p.sp || p.sq) y[j] = __fmul_rn(y[j], __fmul_rn(other, scale[j]));
          if (p.bias) y[j] = __fadd_rn(y[j], bias[j]);
          put_one<OUT>(p.out.out, m * p.out.ldo + from + j, y[j]);
        }
      }
    }
    cg::this_cluster().sync();  // the others may still read this CTA's sums
  }
  if (!ok) atomicOr_system(p.status, 1u);
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  if (CG == 2) cg::this_cluster().sync();
  else __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (CG == 2) {
    // (the last arrival in the odd CTA's shared memory, before it goes)
    if (warp == MMA_WARP && rank) warp_wait(last, 0, END_LIMIT);
    __syncwarp();
    if (warp == MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  } else if (warp == MMA_WARP) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// rows of codes; a box is 128 bytes of `box` rows, swizzled
bool rows_map(CUtensorMap* m, const uint8_t* base, int64_t rows, int64_t bytes, int64_t ld, int box) {
  EncodeFn f = encode_fn();
  if (!f) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)bytes, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? ld : (bytes + 15) / 16 * 16)};
  const cuuint32_t size[2] = {128, (cuuint32_t)box}, elem[2] = {1, 1};
  return f(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(base), dims, strides, size, elem,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// tiles of scales, `per` of them a box
bool scales_map(CUtensorMap* m, const uint8_t* base, int64_t tiles, int per) {
  EncodeFn f = encode_fn();
  if (!f) return false;
  const cuuint64_t dims[2] = {SCALE_TILE / 4, (cuuint64_t)tiles}, strides[1] = {SCALE_TILE};
  const cuuint32_t size[2] = {SCALE_TILE / 4, (cuuint32_t)per}, elem[2] = {1, 1};
  return f(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<uint8_t*>(base), dims, strides, size, elem,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// results: boxes of 32 rows of 128 bytes, swizzled
bool out_map(CUtensorMap* m, void* out, int64_t rows, int64_t cols, int64_t ld, int dtype) {
  EncodeFn f = encode_fn();
  if (!f) return false;
  const int size = dtype == PEAT_F32 ? 4 : 2;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? ld * size : (cols * size + 15) / 16 * 16)};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / size), 32}, elem[2] = {1, 1};
  const CUtensorMapDataType type = dtype == PEAT_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == PEAT_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  return f(m, type, 2, out, dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
           CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Maps {
  CUtensorMap p, q, sp, sq, out;
};
template <int OUT, int FMT, bool SWAP, int CG>
cudaError_t launch(const Tc4Params& p, const Maps& m, int nsm, cudaStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_smem(mm4_tc<OUT, FMT, SWAP, CG>, SMEM, allowed);
  if (e != cudaSuccess) return e;
  const int64_t tiles = (int64_t)p.pt * p.qt;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)(CG == 2 ? 2 : p.splits);
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  // (one CTA an SM, which has all of tensor memory)
  cfg.gridDim = dim3((unsigned)(p.splits > 1 ? p.splits * tiles : CG * std::min<int64_t>(tiles, nsm / CG)));
  cfg.blockDim = dim3(Warps<CG, SWAP>::THREADS);
  cfg.dynamicSmemBytes = SMEM;
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = CG == 2 || p.splits > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, mm4_tc<OUT, FMT, SWAP, CG>, p, m.p, m.q, m.sp, m.sq, m.out);
}
enum Kind { FEW, ONE, PAIR };  // few rows of a; tiles of a CTA; of a pair
template <int OUT, int FMT>
cudaError_t launch_kind(Kind kind, const Tc4Params& p, const Maps& m, int nsm, cudaStream_t s) {
  if (kind == FEW) return launch<OUT, FMT, true, 1>(p, m, nsm, s);
  return kind == ONE ? launch<OUT, FMT, false, 1>(p, m, nsm, s) : launch<OUT, FMT, false, 2>(p, m, nsm, s);
}
template <int OUT>
cudaError_t launch_out(int format, Kind kind, const Tc4Params& p, const Maps& m, int nsm, cudaStream_t s) {
  return format == PEAT_MXFP4 ? launch_kind<OUT, PEAT_MXFP4>(kind, p, m, nsm, s) : launch_kind<OUT, PEAT_NVFP4>(kind, p, m, nsm, s);
}

// How a product is cut into tiles: by its expected time, fitted to those measured
// for M from 1 to 16384, N to 50257 and K to 16384 (see the figures in each row).  An
// instruction takes as long for 16 columns as for 256 (its 128 rows' loads): what
// tells the ways apart are the waves, and the results' way out, which takes the
// longer of it and the instructions.  Few tiles of long rows have a cluster each,
// whose CTAs share the k range.
struct Cut {
  Kind kind;
  int bn, splits;
};
Cut cut_of(int64_t M, int64_t N, int64_t steps, bool grid, int nsm) {
  const int few = (int)((std::min<int64_t>(M, FEW_ROWS) + 15) / 16 * 16);
  const struct {
    Cut cut;
    // nanoseconds: of a call; of a wave, on the 16-byte grid and off it, at least; with instructions: and of each
    int fixed, least, least_off, tile, step;
  } ways[] = {{{FEW, few, 1}, 3400, 0, 0, 350 + 19 * few, 60},   // 16 x 50257 x 1024: 8.5 us, 192 x: 18.9
              {{ONE, 128, 1}, 3300, 1350, 3900, 450, 65},        // 2048 x 1024 x 4096: 7.7 us (a pair's 9.8)
              {{PAIR, 256, 1}, 4200, 1800, 5800, 1100, 81}};     // 16384 x 4096 x 1024: 36.5 us (a CTA's 43.2)
  Cut best = ways[1].cut;
  double shortest = 0.0;
  for (const auto& w : ways) {
    if (w.cut.kind == FEW && M > FEW_ROWS) continue;
    if (w.cut.kind != FEW && M <= 48) continue;  // (16 x 8192 x 8192: 12.0 us, with a's rows on the 128-row side 17.9)
    const int64_t rows = w.cut.kind == PAIR ? 256 : 128, at_once = w.cut.kind == PAIR ? nsm / 2 : nsm;
    const int64_t tiles = w.cut.kind == FEW ? (N + 127) / 128 : ((M + rows - 1) / rows) * ((N + w.cut.bn - 1) / w.cut.bn);
    for (int s = 1; s <= (w.cut.kind == PAIR ? 1 : 8); s *= 2) {
      // (a cluster of 8 finds place on some of the GPU's parts only; a part has two stages or more)
      if (s > 1 && (tiles > (s == 2 ? nsm / 2 : s == 4 ? nsm / 4 - 2 : nsm / 10) || steps < 8 * s)) break;
      const double waves = s > 1 ? 1.0 : (double)((tiles + at_once - 1) / at_once);
      double t = w.fixed + waves * std::max<double>(grid || s > 1 ? w.least : w.least_off, w.tile + (double)w.step * ((steps + s - 1) / s));
      if (s > 1) t += w.cut.kind == FEW ? 1600 + 3 * few : 4300;  // the parts' meeting
      if (shortest == 0.0 || t < shortest) best = Cut{w.cut.kind, w.cut.bn, s}, shortest = t;
    }
  }
  return best;
}

}  // namespace

cudaError_t launch_mm4(int format, int out_dtype, const Mm4Params& m, unsigned int* status, unsigned int wait_limit, int nsm,
                       cudaStream_t s) {
  const int block = format == PEAT_MXFP4 ? 32 : 16;
  Tc4Params p;
  p.steps = (int)((m.K + 63) / 64);
  const int size = out_dtype == PEAT_F32 ? 4 : 2;
  const bool grid = reinterpret_cast<uintptr_t>(m.out) % 16 == 0 && (m.ldo * size % 16 == 0 || m.M <= 1) && m.ldo * size < ((int64_t)1 << 40);
  Cut cut = cut_of(m.M, m.N, p.steps, grid, nsm);
  p.tiles = (m.K / block + 3) / 4;
  // (a pair's copies count tiles of scales in 32 bits)
  const int64_t tall = (std::max(m.M, m.N) + 127) / 128 * p.tiles;
  if (cut.kind == PAIR && tall >= ((int64_t)1 << 31) - 1024 - 2 * p.tiles) cut = {ONE, 128, 1};
  const bool swap = cut.kind == FEW;
  p.ps = swap ? m.b_block_scale : m.a_block_scale;
  p.qs = swap ? m.a_block_scale : m.b_block_scale;
  p.sp = swap ? m.sb : m.sa;
  p.sq = swap ? m.sa : m.sb;
  p.bias = m.bias;
  p.P = swap ? m.N : m.M;
  p.Q = swap ? m.M : m.N;
  p.bn = cut.bn;
  p.splits = cut.splits;
  const int cg = cut.kind == PAIR ? 2 : 1;
  p.pt = (int)((p.P + 128 * cg - 1) / (128 * cg));
  p.qt = (int)((p.Q + p.bn - 1) / p.bn);
  const int results = swap ? Warps<1, true>::BYTES : (cg == 2 ? Warps<2, false>::BYTES : Warps<1, false>::BYTES);
  p.stages = std::min(MOST_STAGES, (SMEM - 1024 - results - BARS) / stage_bytes(p.bn / cg));
  p.out = OutPlace{m.out, m.ldo, m.N, m.bias != nullptr, grid};
  p.units = m.N * size % 16 == 0;
  p.status = status;
  p.wait_limit = wait_limit;
  Maps maps = {};
  const int per = SK / (4 * block);
  if (m.K > 0 && (!rows_map(&maps.p, swap ? m.b : m.a, p.P, m.K / 2, swap ? m.ldb : m.lda, 128) ||
                  !rows_map(&maps.q, swap ? m.a : m.b, p.Q, m.K / 2, swap ? m.lda : m.ldb, p.bn / cg)))
    return cudaErrorNotSupported;
  if (m.K > 0 && cut.kind == PAIR && (!scales_map(&maps.sp, p.ps, (p.P + 127) / 128 * p.tiles, per) ||
                                      !scales_map(&maps.sq, p.qs, (p.Q + 127) / 128 * p.tiles, per)))
    return cudaErrorNotSupported;
  if (!swap && grid && !out_map(&maps.out, m.out, m.M, m.N, m.ldo, out_dtype)) return cudaErrorNotSupported;
  switch (out_dtype) {
    case PEAT_F32: return launch_out<PEAT_F32>(format, cut.kind, p, maps, nsm, s);
    case PEAT_F16: return launch_out<PEAT_F16>(format, cut.kind, p, maps, nsm, s);
    default: return launch_out<PEAT_BF16>(format, cut.kind, p, maps, nsm, s);
  }
}

}  // namespace peat
