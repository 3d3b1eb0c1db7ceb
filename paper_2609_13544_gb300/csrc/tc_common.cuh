// Pieces shared by the products on the fifth-generation tensor cores: barriers,
// copies, accumulators, results out of them.
#pragma once
#include <cuda.h>

#include "mm8_common.cuh"

namespace peat {

// a whole 32-byte sector
__device__ __forceinline__ void store_sector(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
__device__ __forceinline__ uint32_t sptr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Arrive on a barrier of the cluster (an address of mapa).  What it tells the
// other CTA is that accumulators have been read, which the tcgen05 fence
// before it orders; a release at cluster scope would wait for this thread's
// stores to global memory, 2000 cycles of every tile.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t mapa(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ int4 load_cluster(uint32_t addr) {
  int4 v;
  asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
// waits for the barrier's phase of this parity; false after `limit` polls (a thread by itself)
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, uint32_t limit) {
  for (uint32_t i = 0; i < limit; i++) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        " selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    if (ok) return true;
  }
  return false;
}
// The same by all lanes of a warp, with one outcome: a wait may expire for some
// lanes just as the phase completes for the others, and the warp must not part
// before an instruction that takes all of it (tcgen05.ld, shuffles).
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, uint32_t limit) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, limit));
}
// one lane of the warp; unlike a test of the lane's number, the compiler knows
// that it is one (with the test a tile took 843 cycles per 64 k, with this 600)
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, q;\n}" : "=r"(p));
  return p != 0;
}
// a block into this CTA's shared memory, its bytes counted on the even CTA's barrier
__device__ __forceinline__ void tma_block(uint32_t dst, const CUtensorMap* map, int row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, "
      "%3}], [%4];" ::"r"(dst),
      "l"(map), "r"(0), "r"(row), "r"(bar)
      : "memory");
}
// shared-memory descriptor of a block: K-major, 128-byte swizzle, 8-row groups 1024 bytes apart
__device__ __forceinline__ uint64_t block_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)2 << 61);
}
// arrives on the barrier at this offset in both CTAs of the pair (their ranks'
// bits: pair) once the instructions issued so far are done
__device__ __forceinline__ void commit_both(uint32_t bar, uint16_t pair) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
      "h"(pair)
      : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]),
        "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]),
        "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(addr));
}

// N consecutive results of a row, packed
template <int OUT, int N>
__device__ __forceinline__ void results(const float* v, float sa, const float* sb, const float* bias, bool biased,
                                        uint32_t* w) {
  constexpr int B = (int)sizeof(typename Mm8Out<OUT>::T);
  if constexpr (OUT == PEAT_OUT_I32) {  // (v holds the integers' bits)
#pragma unroll
    for (int i = 0; i < N; i++) w[i] = __float_as_uint(v[i]);
  } else {
    float y[N];
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 s = *reinterpret_cast<const float4*>(sb + i);
      y[i] = __fmul_rn(v[i], __fmul_rn(sa, s.x));
      y[i + 1] = __fmul_rn(v[i + 1], __fmul_rn(sa, s.y));
      y[i + 2] = __fmul_rn(v[i + 2], __fmul_rn(sa, s.z));
      y[i + 3] = __fmul_rn(v[i + 3], __fmul_rn(sa, s.w));
      if (biased) {
        const float4 b = *reinterpret_cast<const float4*>(bias + i);
        y[i] = __fadd_rn(y[i], b.x);
        y[i + 1] = __fadd_rn(y[i + 1], b.y);
        y[i + 2] = __fadd_rn(y[i + 2], b.z);
        y[i + 3] = __fadd_rn(y[i + 3], b.w);
      }
    }
#pragma unroll
    for (int i = 0; i < N * B / 4; i++) {
      if (OUT == PEAT_F32) {
        w[i] = __float_as_uint(y[i]);
      } else if (OUT == PEAT_BF16) {
        __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
        w[i] = *reinterpret_cast<uint32_t*>(&h);
      } else {
        __half2 h = __floats2half2_rn(y[2 * i], y[2 * i + 1]);
        w[i] = *reinterpret_cast<uint32_t*>(&h);
      }
    }
  }
}
// The elements [lo, hi) of a 32-byte sector: aligned pieces, each as large as fits.
template <int OUT>
__device__ __forceinline__ void store_part(void* sector, const uint32_t (&w)[8], int lo, int hi) {
  constexpr int B = (int)sizeof(typename Mm8Out<OUT>::T), E = 32 / B;
  if (lo <= 0 && hi >= E) return store_sector(sector, w);
  char* d = static_cast<char*>(sector);
  auto in = [&](int from, int n) { return from >= lo && from + n <= hi; };
#pragma unroll
  for (int i = 0; i < 8; i += 4)
    if (in(i * 4 / B, 16 / B)) *reinterpret_cast<uint4*>(d + 4 * i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
#pragma unroll
  for (int i = 0; i < 8; i += 2)
    if (in(i * 4 / B, 8 / B) && !in((i & ~3) * 4 / B, 16 / B)) *reinterpret_cast<uint2*>(d + 4 * i) = make_uint2(w[i], w[i + 1]);
#pragma unroll
  for (int i = 0; i < 8; i++)
    if (in(i * 4 / B, 4 / B) && !in((i & ~1) * 4 / B, 8 / B)) *reinterpret_cast<uint32_t*>(d + 4 * i) = w[i];
  if (B == 2) {
#pragma unroll
    for (int i = 0; i < 16; i++)
      if (in(i, 1) && !in(i & ~1, 2)) *reinterpret_cast<uint16_t*>(d + 2 * i) = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
  }
}
// A sector's words where the row is `s` elements off the sectors: x holds the
// words before the sector's place in the row, then the eight from there on.
template <int OUT>
__device__ __forceinline__ void sector_at(const uint32_t (&x)[16], int s, uint32_t (&w)[8]) {
  constexpr int B = (int)sizeof(typename Mm8Out<OUT>::T);
  const int words = s * B / 4;
  uint32_t y[16];
  y[0] = x[0];
#pragma unroll
  for (int i = 1; i < 16; i++) y[i] = B == 2 ? __funnelshift_l(x[i - 1], x[i], 16 * (s & 1)) : x[i];
#pragma unroll
  for (int by = 4; by; by /= 2)
#pragma unroll
    for (int i = 15; i >= 9 - by; i--) y[i] = words & by ? y[max(i - by, 0)] : y[i];
#pragma unroll
  for (int i = 0; i < 8; i++) w[i] = y[8 + i];
}
// where results go: rows of ldo elements, N columns; vec: rows start on boundaries of the
// units that the caller stores (put_columns: 32 bytes; copies out of shared memory: 16)
struct OutPlace {
  void* out;
  int64_t ldo, N;
  bool biased, vec;
};
// 32 columns of a warp's 32 rows, a row a lane, in a run of such calls from left
// to right.  Each lane writes whole 32-byte sectors of its row: where the row is
// off them, its words are shifted by what it is off, the last ones of the call
// before (carry) in front, and the ends of the run go in smaller pieces.
// (Through shared memory and out along the rows, 64 bytes of a row at a time,
// half of the sectors are written in two parts: 1024 x 50257 x 1024 to binary16
// took 102 us.)
template <int OUT>
__device__ __forceinline__ void put_columns(const OutPlace& p, const float (&v)[32], float sa, const float* sb,
                                            const float* bias, int64_t row0, int rows, int64_t col0, bool first,
                                            bool last, uint32_t (&carry)[8]) {
  using T = typename Mm8Out<OUT>::T;
  constexpr int B = (int)sizeof(T), E = 32 / B;
  const int lane = threadIdx.x & 31;
  const int64_t left = p.N - col0;  // columns
  if (left <= 0) return;
  T* o = static_cast<T*>(p.out) + (row0 + lane) * p.ldo + col0;
  if (p.vec && left >= 32) {
#pragma unroll
    for (int c = 0; c < 32; c += E) {
      uint32_t w[8];
      results<OUT, E>(v + c, sa, sb + c, bias + c, p.biased, w);
      if (lane < rows) store_sector(o + c, w);
    }
    return;
  }
  const int s = (int)(reinterpret_cast<uintptr_t>(o) & 31) / B;
  const int n = lane < rows ? (int)min(left, (int64_t)32) : -32;  // the lane's columns
  o -= s;
  uint32_t x[16], w[8];
#pragma unroll
  for (int i = 0; i < 8; i++) x[i] = carry[i];
#pragma unroll
  for (int c = 0; c < 32; c += E) {
    results<OUT, E>(v + c, sa, sb + c, bias + c, p.biased, w);
#pragma unroll
    for (int i = 0; i < 8; i++) x[8 + i] = w[i];
    sector_at<OUT>(x, s, w);
    store_part<OUT>(o + c, w, first && c == 0 ? s : 0, s + n - c);
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = x[8 + i];
  }
#pragma unroll
  for (int i = 0; i < 8; i++) carry[i] = x[i];
  if (last || left <= 32) {
    sector_at<OUT>(x, s, w);
    store_part<OUT>(o + 32, w, 0, s + n - 32);
  }
}

// Polls for what a CTA has under way before it ends, whether or not an earlier
// wait of its expired.  A poll that finds nothing takes 4 us: a quarter of a
// second for each copy stage, for copies and instructions that
// take microseconds.  (Where all went well nothing hangs on these: the cluster
// meets only when the instructions are done.)
constexpr uint32_t END_LIMIT = 1u << 16;

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeFn encode_fn() {
  static EncodeFn fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<EncodeFn>(f);
  }();
  return fn;
}

}  // namespace peat
