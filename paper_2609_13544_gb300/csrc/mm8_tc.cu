// 8-bit integer products on the fifth-generation tensor cores: many rows.
//
// The integers are laid out as binary16 once per call (pack), in the very
// image that the matrix instruction reads from shared memory: blocks of 128
// rows by 64 k, 128-byte rows with their 16-byte pieces swizzled, so that a
// block is one contiguous 16 KB that a TMA copy moves as it lies, and ragged
// edges are zeros that pack wrote.  Converting inside the product instead would
// move every block through shared memory twice more than the instruction reads
// it, and shared memory bandwidth is what the instruction runs against.
//
// A cluster of two CTAs makes a tile of 256 x 256 (cta_group::2: each holds
// 128 rows of a and 128 of b, and the accumulators of its rows), persistent
// over the tiles.  Warp roles: one thread issues the copies, one (of the even
// CTA) the matrix instructions, eight warps turn accumulators into results
// while the other half of the 512 accumulator columns fills, and one warp
// plans: a few tiles ahead it works out each tile's place and drains and
// fetches its scales, so that neither instructions nor results wait for global
// memory.
//
// Exactness: float32 holds a sum of products exactly while it stays below
// 2^24.  pack (or the quantiser that writes the blocks itself) leaves for every
// block of 128 rows and 256 k the largest sum of squares of a row, in one word
// or as one for each half; by Cauchy and Schwarz the product of two roots
// bounds every partial sum over those 256 k, and the accumulator is drained to int32
// before the bounds add up to more than 2^24.  Full-range integers drain every
// 768 k, normally distributed ones about every 16 000; up to 1024 k nothing can
// add up to more, and no norms are made.
//
// 8192 x 8192 x 8192 to bfloat16 takes 590 us in bursts (1860 TFLOP/s) and 620 to
// 635 without a pause, at the power limit (1690 to 1755 MHz; the library's
// bfloat16 product of normal numbers 573 and 643), with extreme integers 716 to
// 727 at 2070 MHz; 16384 x 4096 x 1024 88 to 92, of which pack has 10; 2048 x
// 1024 x 4096, 32 tiles with k in two parts, 26.
// pack is bound by memory: 52 million integers take 22 us, 7 TB/s.
#include <cooperative_groups.h>

#include <algorithm>

#include "peat_internal.h"
#include "tc_common.cuh"

namespace cg = cooperative_groups;

namespace peat {
namespace {

constexpr int BLK = 128 * 64 * 2;  // bytes of a packed block
constexpr int KN = 256;            // k of one norm
constexpr int64_t FREE_K = 1024;   // products of any integers whose sum is at most 2^24

// ---------------------------------------------------------------------------
// pack
// ---------------------------------------------------------------------------
struct PackParams {
  const int8_t* x[2];
  int64_t ld[2], rows[2];
  __half* out[2];
  unsigned int* norm[2];
  int64_t K;
  int kb, kc;        // blocks of 64 and 256 k
  int64_t first_b;   // CTAs of the first matrix
};

template <int MODE>
__global__ void __launch_bounds__(256) mm8_pack(PackParams p) {
  pdl_wait();
  pdl_trigger();
  const int which = blockIdx.x >= p.first_b;
  const int64_t at = blockIdx.x - (which ? p.first_b : 0);
  const int64_t rb = at / p.kc;
  const int kc = (int)(at - rb * p.kc);
  const int8_t* x = which ? p.x[1] : p.x[0];
  const int64_t ld = which ? p.ld[1] : p.ld[0], rows = which ? p.rows[1] : p.rows[0];
  const int8_t *lo = x, *hi = x + (rows - 1) * ld + p.K;
  const int l = threadIdx.x & 15, kb = kc * 4 + (l >> 2);
  const int64_t k = (int64_t)kc * KN + l * 16, left = p.K - k;
  char* out = reinterpret_cast<char*>(which ? p.out[1] : p.out[0]) + (rb * p.kb + kb) * (int64_t)BLK;
  uint4 v[8];
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const int64_t row = rb * 128 + (threadIdx.x >> 4) + 16 * i;
    v[i] = load16<MODE>(x + row * ld + k, row < rows ? left : 0, lo, hi);
  }
  const bool odd = threadIdx.x >> 4 & 1;  // of the thread's rows: there the two 16-byte pieces change places
  if (kb < p.kb) {
    char* d = out + (threadIdx.x >> 4) * 128 + (((l & 3) * 2) ^ ((threadIdx.x >> 4) & 6)) * 16;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      uint32_t w[8];
      to_half(odd ? v[i].z : v[i].x, w[0], w[1]);
      to_half(odd ? v[i].w : v[i].y, w[2], w[3]);
      to_half(odd ? v[i].x : v[i].z, w[4], w[5]);
      to_half(odd ? v[i].y : v[i].w, w[6], w[7]);
      store_sector(d + i * (16 * 128), w);
    }
  }
  if (p.K <= FREE_K) return;  // no norms are needed
  // sums of squares of the thread's part of 8 rows; 16 lanes have a row: two
  // values change hands a step while there are several (8 shuffles, not 32)
  int ss[8];
#pragma unroll
  for (int i = 0; i < 8; i++) {
    ss[i] = __dp4a((int)v[i].x, (int)v[i].x, 0);
    ss[i] = __dp4a((int)v[i].y, (int)v[i].y, ss[i]);
    ss[i] = __dp4a((int)v[i].z, (int)v[i].z, ss[i]);
    ss[i] = __dp4a((int)v[i].w, (int)v[i].w, ss[i]);
  }
#pragma unroll
  for (int n = 4; n; n /= 2) {
    const bool high = l & n;
#pragma unroll
    for (int i = 0; i < n; i++) {
      const int give = high ? ss[i] : ss[i + n], keep = high ? ss[i + n] : ss[i];
      ss[i] = keep + __shfl_xor_sync(0xffffffffu, give, n);
    }
  }
  int most = ss[0] + __shfl_xor_sync(0xffffffffu, ss[0], 8);
  most = __reduce_max_sync(0xffffffffu, most);
  __shared__ int part[8];
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 8; w++) most = max(most, part[w]);
    reinterpret_cast<uint2*>(which ? p.norm[1] : p.norm[0])[rb * p.kc + kc] = make_uint2((unsigned)most, 0u);
  }
}

// ---------------------------------------------------------------------------
// product
// ---------------------------------------------------------------------------
constexpr int STAGES = 6, STAGE = 2 * BLK;  // a CTA's block of a and block of b
constexpr int EPI_WARPS = 8, COPY_WARP = EPI_WARPS, MMA_WARP = COPY_WARP + 1, PLAN_WARP = MMA_WARP + 1;
constexpr int THREADS = (PLAN_WARP + 1) * 32;
constexpr int MAX_GROUPS = 16;     // of 32 norm blocks: K up to 131072
struct Slot {                      // a planned tile
  int tile, mt, nt, k0, k1;        // its place; its part of the k range in blocks of 64
  int pieces;                      // times its accumulator is read
  int exact;                       // float32 holds the whole sum, over all parts of the k range
  uint32_t drain[MAX_GROUPS];      // bit i of word g: drained before norm block k0 / 4 + 32 g + i
  alignas(16) float sb[256];
  float bias[256];
};
constexpr int SLOTS = 4;
constexpr int AT_SLOTS = STAGES * STAGE, AT_BARS = AT_SLOTS + SLOTS * (int)sizeof(Slot), BARS = 256;
static_assert(AT_BARS % 16 == 0, "barriers are aligned");
constexpr int SMEM = AT_BARS + BARS + 1024;
constexpr float LIMIT = 16777216.0f;  // 2^24

struct TcParams {
  Mm8Params m;
  const uint2* na;  // sums of squares [row blocks][kc]
  const uint2* nb;
  int scales_late;  // the scales may come from the kernel before this one
  int kb, kc;
  int mt, nt;       // tiles
  int splits;       // parts of the k range of a tile: 1, 2 or 4; split tiles have a cluster each
  int4* sums;       // 128 x 256 int32 for each CTA
  int vec_out;      // out's rows start on 32-byte boundaries
  unsigned int* status;
  uint32_t wait_limit;
};

// float32 accumulators, binary16 operands, both K-major, 256 x 256
constexpr uint32_t IDESC = (1u << 4) | ((256u / 8) << 17) | ((256u / 16) << 24);
__device__ __forceinline__ void mma_256(uint32_t d, uint64_t a, uint64_t b, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(IDESC), "r"(accumulate)
      : "memory");
}
// integer sums (exact: in float32) as put_columns takes them
template <int OUT>
__device__ __forceinline__ void as_results(const int4 (&x)[8], bool exact, float (&f)[32]) {
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const int v[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if (OUT == PEAT_OUT_I32) f[4 * j + i] = __int_as_float(exact ? __float2int_rn(__int_as_float(v[i])) : v[i]);
      else f[4 * j + i] = exact ? __int_as_float(v[i]) : __int2float_rn(v[i]);
    }
  }
}
__device__ __forceinline__ int add_sum(int a, int b, bool exact) {
  return exact ? __float_as_int(__fadd_rn(__int_as_float(a), __int_as_float(b))) : a + b;
}

constexpr int GROUP = 8;
// a tile, and its part of the k range in blocks of 64
struct Place {
  int tile, mt, nt, k0, k1;
};
__device__ __forceinline__ Place place_of(const TcParams& p, int u, int part) {
  Place r;
  r.tile = u;
  // groups of GROUP rows of tiles, column by column: the clusters at work at
  // any time share few blocks of a and few of b
  const int per = GROUP * p.nt, g = r.tile / per, in = r.tile - g * per, wide = min(GROUP, p.mt - g * GROUP);
  r.nt = in / wide;
  r.mt = g * GROUP + in - r.nt * wide;
  // (kb <= 2048, splits <= 4)
  r.k0 = p.kb * part / p.splits;
  r.k1 = p.kb * (part + 1) / p.splits;
  return r;
}
// a tile's scales into its slot, by a warp
__device__ __forceinline__ void plan_scales(const TcParams& p, const Place& t, Slot* slot) {
  const int lane = threadIdx.x & 31;
  float sb[8], bias[8];
#pragma unroll
  for (int i = 0; i < 8; i++) {
    const int64_t col = (int64_t)t.nt * 256 + i * 32 + lane;
    sb[i] = p.m.sb && col < p.m.N ? __ldcg(p.m.sb + col) : 1.0f;
    bias[i] = p.m.bias && col < p.m.N ? __ldcg(p.m.bias + col) : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < 8; i++) {
    slot->sb[i * 32 + lane] = sb[i];
    slot->bias[i * 32 + lane] = bias[i];
  }
}
// a tile's place and drains into its slot, by a warp
__device__ void plan_drains(const TcParams& p, const Place& t, Slot* slot) {
  const int lane = threadIdx.x & 31;
  const uint2* na = p.na + (int64_t)t.mt * 2 * p.kc;
  const uint2* nb = p.nb + (int64_t)t.nt * 2 * p.kc;
  int pieces = 1;
  float run = 0.0f;  // the bound of what the accumulator holds
  bool exact = true;
  auto bound = [&](int c, int end) {  // of the products of norm block c
    if (c >= end) return 0.0f;
    const uint2 a0 = __ldcg(na + c), a1 = __ldcg(na + p.kc + c), b0 = __ldcg(nb + c), b1 = __ldcg(nb + p.kc + c);
    const unsigned a = max(a0.x + a0.y, a1.x + a1.y), b = max(b0.x + b0.y, b1.x + b1.y);
    return sqrtf((float)a) * sqrtf((float)b) * 1.00001f;  // (rounded up)
  };
  auto over_warp = [](float x) {
#pragma unroll
    for (int o = 16; o; o /= 2) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
  };
  if (p.m.K > FREE_K && p.splits > 1) {
    float all = 0.0f;
    for (int c = lane; c < p.kc; c += 32) all += bound(c, p.kc);
    exact = over_warp(all) <= LIMIT;
  } else if (p.m.K > FREE_K) {
    exact = false;
  }
  if (exact && lane < MAX_GROUPS) slot->drain[lane] = 0;
  for (int c0 = t.k0 / 4, w = 0; !exact && c0 * 4 < t.k1; c0 += 32, w++) {
    const float mine = bound(c0 + lane, (t.k1 + 3) / 4), all = over_warp(mine);
    uint32_t mask = 0;
    if (run + all <= LIMIT) {
      run += all;
    } else {
      for (int i = 0; i < 32; i++) {
        const float b = __shfl_sync(0xffffffffu, mine, i);
        if (run + b > LIMIT) {
          if (run > 0.0f) mask |= 1u << i;
          run = b;
        } else {
          run += b;
        }
      }
    }
    pieces += __popc(mask);
    if (lane == 0) slot->drain[w] = mask;
  }
  if (lane == 0) {
    slot->tile = t.tile;
    slot->mt = t.mt;
    slot->nt = t.nt;
    slot->k0 = t.k0;
    slot->k1 = t.k1;
    slot->pieces = pieces;
    slot->exact = exact;
  }
}

template <int OUT>
__global__ void __launch_bounds__(THREADS, 1)
    mm8_tc(TcParams p, const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb) {
  extern __shared__ char raw[];
  char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  Slot* slots = reinterpret_cast<Slot*>(smem + AT_SLOTS);
  const uint32_t full = sptr(smem + AT_BARS), empty = full + 8 * STAGES, acc_full = empty + 8 * STAGES,
                 acc_empty = acc_full + 16, last = acc_empty + 16, planned = last + 8, unplanned = planned + 8 * SLOTS;
  volatile uint32_t* tmem_at = reinterpret_cast<volatile uint32_t*>(smem + AT_BARS + 8 * (2 * STAGES + 5 + 2 * SLOTS));
  static_assert(8 * (2 * STAGES + 5 + 2 * SLOTS) + 4 <= BARS, "the barriers fit");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // a pair's CTAs differ in the last bit of their rank; the parts of a split
  // tile's k range are the pairs of one cluster
  uint32_t in_cluster;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(in_cluster));
  const uint32_t rank = in_cluster & 1, part = in_cluster >> 1, even = in_cluster & ~1u;
  const uint16_t pair = (uint16_t)(3u << even);
  const int units = p.mt * p.nt, first = blockIdx.x / (2 * p.splits), step = gridDim.x / (2 * p.splits);
  const bool split = p.splits > 1;

  if (threadIdx.x == 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&ma) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&mb) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; i++) {
      mbar_init(full + 8 * i, 1);   // the even CTA's copier; plus the bytes of both
      mbar_init(empty + 8 * i, 1);  // a commit
    }
    for (int i = 0; i < 2; i++) {
      mbar_init(acc_full + 8 * i, 1);
      mbar_init(acc_empty + 8 * i, 2 * EPI_WARPS);
    }
    mbar_init(last, 1);
    for (int i = 0; i < SLOTS; i++) {
      mbar_init(planned + 8 * i, 1);
      mbar_init(unplanned + 8 * i, EPI_WARPS + (rank == 0));  // results, and the instructions' warp
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == MMA_WARP) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(sptr((const void*)tmem_at))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  cg::this_cluster().sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_at;
  pdl_trigger();

  const OutPlace place{p.m.out, p.m.ldo, p.m.N, p.m.bias != nullptr, p.vec_out != 0};
  bool ok = true;
  float sa = 1.0f;  // of the lane's row of results
  if (warp == PLAN_WARP) {
    int i = 0;
    for (int u = first; u < units && ok; u += step, i++) {
      ok = warp_wait(unplanned + 8 * (i % SLOTS), (i / SLOTS & 1) ^ 1, p.wait_limit);
      if (!ok) break;
      const Place t = place_of(p, u, part);
      // (where the kernel before is pack, the scales are older: complete before
      // pack let this kernel start)
      if (i == 0 && p.scales_late) pdl_wait();
      plan_scales(p, t, slots + i % SLOTS);
      if (i == 0) pdl_wait();
      plan_drains(p, t, slots + i % SLOTS);
      __syncwarp();
      if (lane == 0) mbar_arrive(planned + 8 * (i % SLOTS));
    }
  } else if (warp == COPY_WARP) {
    if (elect_one()) {
      pdl_wait();
      int seq = 0;
      for (int u = first; u < units && ok; u += step) {
        const Place t = place_of(p, u, part);
        const int ra = (t.mt * 2 + (int)rank) * p.kb, rb = (t.nt * 2 + (int)rank) * p.kb;
        for (int k = t.k0; k < t.k1; k++, seq++) {
          const int s = seq % STAGES;
          if (!(ok = mbar_wait(empty + 8 * s, (seq / STAGES & 1) ^ 1, p.wait_limit))) break;
          const uint32_t dst = sptr(smem + s * STAGE), bar = mapa(full + 8 * s, even);
          if (rank == 0) mbar_expect(full + 8 * s, 2 * STAGE);
          tma_block(dst, &ma, (ra + k) * 16, bar);
          tma_block(dst + BLK, &mb, (rb + k) * 16, bar);
        }
      }
      // a stage's copies have landed when its instructions are done with it
      for (int j = 0; j < STAGES && j < seq; j++) {
        const int q = seq - 1 - j;
        mbar_wait(empty + 8 * (q % STAGES), q / STAGES & 1, END_LIMIT);
      }
    }
  } else if (warp == MMA_WARP) {
    // (one thread for the whole loop: with all lanes waiting and voting on the
    // outcome 16384 x 4096 x 1024 took 92.0 us, not 89.5)
    if (rank == 0 && elect_one()) {
      int seq = 0, chunk = 0, i = 0;
      for (int u = first; u < units && ok; u += step, i++) {
        const Slot* t = slots + i % SLOTS;
        const Place at = place_of(p, u, part);
        const int k0 = at.k0, k1 = at.k1;
        uint32_t mask = 0;
        bool fresh = true, known = false;  // the accumulator starts anew; the plan is there
        for (int k = k0; k < k1; k++, seq++) {
          const int c = k / 4 - k0 / 4;
          // (no drain comes before the fourth norm block: three hold less than 2^24)
          if (c >= 3 && (k & 3) == 0) {
            if (!known && !(ok = mbar_wait(planned + 8 * (i % SLOTS), i / SLOTS & 1, p.wait_limit))) break;
            if (!known || (c & 31) == 0) mask = t->drain[c >> 5];
            known = true;
            if (mask >> (c & 31) & 1) {
              commit_both(acc_full + 8 * (chunk & 1), pair);
              chunk++;
              fresh = true;
            }
          }
          if (fresh) {
            ok = mbar_wait(acc_empty + 8 * (chunk & 1), (chunk / 2 & 1) ^ 1, p.wait_limit);
            if (!ok) break;
          }
          const int s = seq % STAGES;
          if (!(ok = mbar_wait(full + 8 * s, seq / STAGES & 1, p.wait_limit))) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t d = tmem + (chunk & 1) * 256, base = sptr(smem + s * STAGE);
          const uint64_t a = block_desc(base), b = block_desc(base + BLK);
#pragma unroll
          for (int j = 0; j < 4; j++) mma_256(d, a + 2 * j, b + 2 * j, !(fresh && j == 0));
          commit_both(empty + 8 * s, pair);
          if (k == k1 - 1) commit_both(acc_full + 8 * (chunk & 1), pair);
          fresh = false;
        }
        chunk++;
        if (ok && !known) ok = mbar_wait(planned + 8 * (i % SLOTS), i / SLOTS & 1, p.wait_limit);
        mbar_arrive(unplanned + 8 * (i % SLOTS));
      }
      // whatever was issued is done before the accumulators are given back
      commit_both(last, pair);
      mbar_wait(last, 0, END_LIMIT);
    }
  } else {  // results: a warp has 32 rows and half of the columns
    int chunk = 0, i = 0;
    const int half = warp >> 2, quarter = warp & 3;
    const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + half * 128;
    const uint32_t release0 = mapa(acc_empty, even);
    for (int u = first; u < units && ok; u += step, i++) {
      const Slot* t = slots + i % SLOTS;
      if (!(ok = warp_wait(planned + 8 * (i % SLOTS), i / SLOTS & 1, p.wait_limit))) break;
      const int pieces = t->pieces;
      const int64_t row0 = (int64_t)t->mt * 256 + rank * 128 + quarter * 32;
      const int64_t col0 = (int64_t)t->nt * 256 + half * 128;
      const float *sb = t->sb + half * 128, *bias = t->bias + half * 128;
      const int rows = (int)max((int64_t)0, min((int64_t)32, p.m.M - row0));
      sa = p.m.sa && lane < rows ? __ldcg(p.m.sa + row0 + lane) : 1.0f;
      // One piece that is the whole sum goes straight from the accumulator to
      // the output.  Several are added up as integers in memory, in a place of
      // this CTA's.  The sum of a split tile's part (its CTA's only one) goes to
      // the stages' place in shared memory, where the other parts find it; the
      // last piece is there when the instructions are done with the stages.
      const bool whole = pieces == 1 && !split, exact = t->exact;
      const int mine = warp * (8 * 128) + lane;
      int4* sums = p.sums + (int64_t)blockIdx.x * (EPI_WARPS * 8 * 128) + mine;
      int4* shared_sums = reinterpret_cast<int4*>(smem) + mine;
      uint32_t carry[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      for (int q = 0; q < pieces && ok; q++, chunk++) {
        if (!(ok = warp_wait(acc_full + 8 * (chunk & 1), chunk / 2 & 1, p.wait_limit))) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
        for (int g = 0; g < 4; g++) {
          uint32_t v[32];
          float f[32];
          tmem_load32(taddr + (chunk & 1) * 256 + g * 32, v);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          if (g == 3) {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(release0 + 8 * (chunk & 1));
          }
#pragma unroll
          for (int j = 0; j < 32; j++) f[j] = __uint_as_float(v[j]);
          if (!whole) {
            if (exact) {  // (a split tile's)
#pragma unroll
              for (int j = 0; j < 8; j++) shared_sums[(g * 8 + j) * 32] = make_int4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
              continue;
            }
            int4 x[8];
#pragma unroll
            for (int j = 0; j < 8; j++) x[j] = q ? sums[(g * 8 + j) * 32] : make_int4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 8; j++) {
              x[j].x += __float2int_rn(f[4 * j]);
              x[j].y += __float2int_rn(f[4 * j + 1]);
              x[j].z += __float2int_rn(f[4 * j + 2]);
              x[j].w += __float2int_rn(f[4 * j + 3]);
            }
            if (q < pieces - 1) {
#pragma unroll
              for (int j = 0; j < 8; j++) sums[(g * 8 + j) * 32] = x[j];
              continue;
            }
            if (split) {
#pragma unroll
              for (int j = 0; j < 8; j++) shared_sums[(g * 8 + j) * 32] = x[j];
              continue;
            }
            as_results<OUT>(x, false, f);
          } else if (OUT == PEAT_OUT_I32) {
#pragma unroll
            for (int j = 0; j < 32; j++) f[j] = __int_as_float(__float2int_rn(f[j]));
          }
          put_columns<OUT>(place, f, sa, sb + g * 32, bias + g * 32, row0, rows, col0 + g * 32, g == 0, g == 3, carry);
        }
      }
      if (!ok || split) break;  // (a split tile's slot is still needed)
      __syncwarp();
      if (lane == 0) mbar_arrive(unplanned + 8 * (i % SLOTS));
    }
  }
  __syncwarp();
  if (split) {
    // The parts meet: each CTA adds up its share of the columns over the pairs,
    // the other parts' next ones under way while it writes.
    cg::this_cluster().sync();
    if (warp < EPI_WARPS && ok) {
      const Slot* t = slots;
      const bool exact = t->exact;
      const int half = warp >> 2, quarter = warp & 3;
      const int64_t row0 = (int64_t)t->mt * 256 + rank * 128 + quarter * 32, col0 = (int64_t)t->nt * 256 + half * 128;
      const int rows = (int)max((int64_t)0, min((int64_t)32, p.m.M - row0));
      const int4* own = reinterpret_cast<const int4*>(smem) + warp * (8 * 128) + lane;
      auto other = [&](int g, int k, int4 (&y)[8]) {  // the sums of part + k
        const uint32_t from = mapa(sptr(own + g * 8 * 32), rank + 2 * ((part + k) & (p.splits - 1)));
#pragma unroll
        for (int j = 0; j < 8; j++) y[j] = load_cluster(from + j * 512);
      };
      int4 x[8], y[8];
      auto add = [&]() {
#pragma unroll
        for (int j = 0; j < 8; j++)
          x[j] = make_int4(add_sum(x[j].x, y[j].x, exact), add_sum(x[j].y, y[j].y, exact), add_sum(x[j].z, y[j].z, exact),
                           add_sum(x[j].w, y[j].w, exact));
      };
      other(part, 1, y);
#pragma unroll 1
      for (int g = part; g < 4; g += p.splits) {
#pragma unroll
        for (int j = 0; j < 8; j++) x[j] = own[(g * 8 + j) * 32];
        add();
        for (int k = 2; k < p.splits; k++) {
          other(g, k, y);
          add();
        }
        if (g + p.splits < 4) other(g + p.splits, 1, y);
        float f[32];
        as_results<OUT>(x, exact, f);
        uint32_t carry[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        put_columns<OUT>(place, f, sa, t->sb + half * 128 + g * 32, t->bias + half * 128 + g * 32, row0, rows, col0 + g * 32,
                         true, true, carry);
      }
    }
  }
  if (!ok) atomicOr_system(p.status, 1u);
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  cg::this_cluster().sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  // (the last arrival in the odd CTA's shared memory, before it goes)
  if (warp == MMA_WARP && rank) warp_wait(last, 0, END_LIMIT);
  __syncwarp();
  if (warp == MMA_WARP)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// packed blocks as rows of 1 KB; a box of 16 of them is one block
bool block_map(CUtensorMap* m, void* base, int64_t blocks) {
  EncodeFn f = encode_fn();
  if (!f) return false;
  const cuuint64_t dims[2] = {256, (cuuint64_t)blocks * 16}, strides[1] = {1024};
  const cuuint32_t box[2] = {256, 16}, elem[2] = {1, 1};
  return f(m, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, base, dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
           CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) ==
         CUDA_SUCCESS;
}

template <int OUT>
cudaError_t tc_launch(const TcParams& p, const CUtensorMap& ma, const CUtensorMap& mb, int nsm, cudaStream_t s) {
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_smem(mm8_tc<OUT>, SMEM, allowed);
  if (e != cudaSuccess) return e;
  const int64_t tiles = (int64_t)p.mt * p.nt;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = 2 * (unsigned)p.splits;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  // persistent pairs, or a cluster for each split tile
  cfg.gridDim = dim3((unsigned)(p.splits > 1 ? tiles * 2 * p.splits : 2 * std::min<int64_t>(tiles, nsm / 2)));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = SMEM;
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, mm8_tc<OUT>, p, ma, mb);
}

}  // namespace

Mm8TcPlan mm8_tc_plan(int64_t M, int64_t N, int64_t K, int nsm) {
  Mm8TcPlan r;
  r.kb = (int)((K + 63) / 64);
  r.kc = (r.kb + 3) / 4;
  r.mt = (M + 255) / 256;
  r.nt = (N + 255) / 256;
  r.splits = 1;
  const int64_t tiles = r.mt * r.nt;
  // Time of a split in blocks of 64 k (about 520 cycles): those of the waves,
  // and what each tile pays once. Clusters of 8 do not fill the GPU (15 of them
  // run at once, of 152 SMs), those of 4 nearly do.
  double best = 0.0;
  for (int s = 1; s <= 4 && s <= r.kb; s *= 2) {
    const int64_t clusters = s == 1 ? nsm / 2 : (s == 2 ? nsm / 4 - 1 : nsm / 10);
    const double t = (double)((tiles + clusters - 1) / clusters) * ((double)r.kb / s + (s == 1 ? 2 : (s == 2 ? 10 : 8))) + 14;
    if (s == 1 || t < best) best = t, r.splits = s;
  }
  auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  size_t at = 0;
  r.a_off = at;
  at += up((size_t)r.mt * 2 * r.kb * BLK);
  r.b_off = at;
  at += up((size_t)r.nt * 2 * r.kb * BLK);
  r.na_words = K > FREE_K ? r.mt * 2 * r.kc * 2 : 0;
  r.nb_words = K > FREE_K ? r.nt * 2 * r.kc * 2 : 0;
  r.sum_off = at;
  if (K > FREE_K) at += (size_t)(r.splits > 1 ? tiles * 2 * r.splits : nsm) * (128 * 256 * sizeof(int));
  r.bytes = at;
  return r;
}

// Microseconds of a call, fitted as mm8_direct_time is: a fixed time, the waves'
// blocks, the meeting of parts, and packing beyond what the fixed time hides.
double mm8_tc_time(const Mm8TcPlan& p, int64_t K, int nsm) {
  const int64_t tiles = p.mt * p.nt, at_once = p.splits == 1 ? nsm / 2 : (p.splits == 2 ? nsm / 4 - 1 : nsm / 10);
  const double waves = (double)((tiles + at_once - 1) / at_once);
  return 10.5 + 0.27 * waves * ((double)p.kb / p.splits) + (p.splits > 1 ? 2.0 : 0.0) + (K > FREE_K ? 2.5 : 0.0) +
         std::max(0.0, (double)(p.mt + p.nt) * 256 * K * 3 / 5e6 - 3.0);
}

cudaError_t launch_mm8_pack(const Mm8Params& m, const Mm8TcPlan& plan, char* ws, unsigned int* norms, int which,
                            cudaStream_t s) {
  PackParams k;
  k.x[0] = m.a;
  k.x[1] = m.b;
  k.ld[0] = m.lda;
  k.ld[1] = m.ldb;
  k.rows[0] = m.M;
  k.rows[1] = m.N;
  k.out[0] = reinterpret_cast<__half*>(ws + plan.a_off);
  k.out[1] = reinterpret_cast<__half*>(ws + plan.b_off);
  k.norm[0] = norms;
  k.norm[1] = norms + plan.na_words;
  k.K = m.K;
  k.kb = plan.kb;
  k.kc = plan.kc;
  k.first_b = which & 1 ? plan.mt * 2 * plan.kc : 0;  // (a matrix that is not asked for has no CTAs)
  const int64_t ctas = k.first_b + (which & 2 ? plan.nt * 2 * plan.kc : 0);
  const bool aligned = (!(which & 1) || mm8_rows_aligned(m.a, m.lda, m.M)) && (!(which & 2) || mm8_rows_aligned(m.b, m.ldb, m.N));
  return launch_dependent(aligned ? mm8_pack<16> : mm8_pack<1>, (unsigned)ctas, 256, 0, s, k);
}

cudaError_t launch_mm8_tc(int out_dtype, const Mm8Params& m, const Mm8TcPlan& plan, char* ws, unsigned int* norms,
                          bool scales_late, unsigned int* status, unsigned int wait_limit, int nsm, cudaStream_t s) {
  CUtensorMap ma, mb;
  if (!block_map(&ma, ws + plan.a_off, plan.mt * 2 * plan.kb) || !block_map(&mb, ws + plan.b_off, plan.nt * 2 * plan.kb))
    return cudaErrorNotSupported;
  TcParams p;
  p.m = m;
  p.na = reinterpret_cast<const uint2*>(norms);
  p.nb = reinterpret_cast<const uint2*>(norms + plan.na_words);
  p.scales_late = scales_late;
  p.kb = plan.kb;
  p.kc = plan.kc;
  p.mt = (int)plan.mt;
  p.nt = (int)plan.nt;
  p.splits = plan.splits;
  p.sums = reinterpret_cast<int4*>(ws + plan.sum_off);
  p.vec_out = reinterpret_cast<uintptr_t>(m.out) % 32 == 0 &&
              m.ldo * (out_dtype == PEAT_F16 || out_dtype == PEAT_BF16 ? 2 : 4) % 32 == 0;
  p.status = status;
  p.wait_limit = wait_limit;
  switch (out_dtype) {
    case PEAT_F32: return tc_launch<PEAT_F32>(p, ma, mb, nsm, s);
    case PEAT_F16: return tc_launch<PEAT_F16>(p, ma, mb, nsm, s);
    case PEAT_BF16: return tc_launch<PEAT_BF16>(p, ma, mb, nsm, s);
    default: return tc_launch<PEAT_OUT_I32>(p, ma, mb, nsm, s);
  }
}

}  // namespace peat
