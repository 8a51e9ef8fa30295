// Attention of many rows over the same keys (a prefix that a batch shares, new tokens over a cached prefix):
// the tile kernel, on the 5th-generation tensor cores.
//
// A worker walks the keys of one span and key/value head in steps of 128 for two tiles of rows.  Per step and
// tile: S = Q K^T into tensor memory (one thread issues tcgen05.mma, operands in shared memory), a
// warpgroup, one thread per row, reads S, keeps the row's running maximum and sum, and writes the
// probabilities back over S in 16 bits, by halves, and O += P V with P read from tensor memory.  The tiles
// take turns: while one tile's softmax runs, the tensor cores work on the other's products.  O is rescaled
// in tensor memory, by the threads that own its rows, only when a row's maximum has grown by more than 2^8.
// Tensor memory (512 columns): S/P of tile 0 and 1, O of tile 0 and 1.
//
// With head_dim 128 a worker is a pair of CTAs (cta_group::2): a tile is 256 rows, 128 in each CTA, and each
// CTA holds half of every key tile (64 keys) and of every value tile (64 columns), which the tensor cores of
// both read.  That halves what an SM draws from L2 and through its shared memory per row, and what it has to
// turn from fp8 to bf16; one CTA alone, drawing 64 KB per step, was bound by that.  With head_dim 64 half a
// value tile is narrower than a swizzled panel, and a worker is one CTA with tiles of 128 rows.
//
// The cache's 16-bit records lie in memory in the swizzled order that the tensor cores read, so keys and
// values arrive by plain bulk copies into a ring.  fp8 records land in a ring of their own and a fourth
// warpgroup turns them into bf16 (exactly, scales included) in the operands' ring.
//
// Keys here are seen by all rows: the plan gives the ends of causal spans to the row kernel.  Only a span's
// last step can be partial; its scores past the end are masked, and its value rows past the end zeroed.
//
// Bound by the tensor cores for full tiles: 4 * D multiply-adds a row and key, and, near that, the
// exponentials: one per row and key.  Work is cut into equal shares per worker; each walks its pieces.
// 9900 rows of 8 heads and 128 columns on 16384 keys, bf16, 665 GFLOP: 393 us = 1.69 PFLOP/s, 98% of what a
// library product keeps up at the card's power limit (1.72; 1.94 in a burst); fp8, 2048 rows on 32768, 282
// GFLOP: 236 us on 108 SMs, the same rate an SM.  A step of 128 keys takes
// 2400 cycles (2048 at the nominal rate); start and end of a worker take about 10000: the way of the queries and
// the first keys, the pipeline's filling, the result's way out.
#include "kv_internal.cuh"

namespace pskv {
namespace {

template <int D, int FMT>
struct Cfg {
  static constexpr bool kFp8 = FMT == PS_KV_FP8, kFp16 = FMT == PS_KV_FP16;
  static constexpr int kCtas = tile_ctas_of(D);
  static constexpr int kRows = 128 * kCtas;                      // rows of a tile
  static constexpr int kKeys = kTileKeys / kCtas;                // keys of a step that a CTA holds
  static constexpr int kCols = D / kCtas;                        // value columns that it holds: one panel
  static constexpr int kSlot = kTileKeys * 128;                  // a CTA's keys, or values, of a step
  static constexpr int kQ = 128 * D * 2;                         // a CTA's queries of one tile
  static constexpr int kRec = record_bytes(D, FMT), kHalf = half_bytes(D, FMT);
  static constexpr int kRawK = kKeys * D, kRawV = kTileKeys * 64;  // a step's fp8 codes
  static constexpr int kRaw = kFp8 ? kRawK + kRawV + 8 * 32 : 0;   // and exponents
  static constexpr int kRaws = kFp8 ? 4 : 0;
  static constexpr int kSlots = kFp8 ? 6 : 10;
  static constexpr int kWarps = kFp8 ? 16 : 12;
  static constexpr int kRegSoft = kFp8 ? 176 : 200, kRegRest = kFp8 ? 80 : 104;
  static constexpr int kSmem = 2 * kQ + kSlots * kSlot + kRaws * kRaw + 1024;  // 1024: alignment
  static_assert(kSlot == kKeys * D * 2 && kCols == 64, "a slot holds keys or values");
  // registers a thread at launch (multiples of 8): the split hands out no more than that
  static_assert(256 * kRegSoft + (kWarps * 32 - 256) * kRegRest <= 65536 / (kWarps * 32) / 8 * 8 * (kWarps * 32),
                "register split");
};

struct Bars {
  uint64_t full[10], empty[10];  // operand ring
  uint64_t raw_full[4], raw_empty[4];
  uint64_t q_ready[2], s_full[2], p_ready[2][2], o_done[2], tail_here, tail_done, drain;
  uint32_t tmem;
  uint32_t gave_up;  // by the warp that arrives on tail_here, before its last arrival
};

// ---- tcgen05
// (CTAS: the cta_group)
template <int CTAS>
__device__ __forceinline__ void tc_alloc(uint32_t dst, uint32_t cols) {
  if (CTAS == 2)
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n"
                 "tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::"r"(dst), "r"(cols) : "memory");
  else
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n"
                 "tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::"r"(dst), "r"(cols) : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tc_dealloc(uint32_t addr, uint32_t cols) {
  if (CTAS == 2)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
  else
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
// Arrives on the barrier, of both CTAs of a pair, when the products issued so far are done.
template <int CTAS>
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  if (CTAS == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3)
                 : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Arrives on the barrier of the worker's first CTA.  What it publishes is read by the tensor cores (tensor memory
// after tcgen05.wait, shared memory after a proxy fence), so the release stays at the default scope: one at the
// scope of the cluster took 500 to 1400 cycles here, a third of a step.
template <int CTAS>
__device__ __forceinline__ void arrive_first(uint32_t bar) {
  if (CTAS == 2)
    asm volatile(
        "{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %0, 0;\n"
        " mbarrier.arrive.shared::cluster.b64 _, [a];\n}\n" ::"r"(bar)
        : "memory");
  else
    mbar_arrive(bar);
}
// The relaxed arrival publishes the barriers' set-up (after fence.mbarrier_init) and nothing else, and does not wait for
// the copies in flight, as a releasing one does (3 us when the ring has just been asked for).
template <int CTAS>
__device__ __forceinline__ void arrive_worker() {
  if (CTAS == 2) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
template <int CTAS>
__device__ __forceinline__ void wait_worker() {
  if (CTAS == 2) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// D[tmem] (+)= A[smem] B[smem]
template <int CTAS>
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) {
  if (CTAS == 2)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
        : "memory");
}
// D[tmem] (+)= A[tmem] B[smem]
template <int CTAS>
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc) {
  if (CTAS == 2)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
        : "memory");
}

#define TC_R4(a, i) "=r"(a[i]), "=r"(a[i + 1]), "=r"(a[i + 2]), "=r"(a[i + 3])
#define TC_I4(a, i) "r"(a[i]), "r"(a[i + 1]), "r"(a[i + 2]), "r"(a[i + 3])
#define TC_R8(a, i) TC_R4(a, i), TC_R4(a, i + 4)
#define TC_I8(a, i) TC_I4(a, i), TC_I4(a, i + 4)

// 32 columns of the calling warp's 32 lanes, one lane a thread
__device__ __forceinline__ void tc_ld32(uint32_t (&r)[32], uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : TC_R8(r, 0), TC_R8(r, 8), TC_R8(r, 16), TC_R8(r, 24)
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t (&r)[16], uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : TC_R8(r, 0), TC_R8(r, 8)
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
      ::TC_I8(r, 0), TC_I8(r, 8), "r"(addr)
      : "memory");
}

// Two floats in a register pair
__device__ __forceinline__ uint64_t pair(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t x, float& lo, float& hi) {
  uint32_t a, b;
  asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(x));
  lo = __uint_as_float(a);
  hi = __uint_as_float(b);
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Shared-memory operand descriptor, 128-byte swizzle, groups of 8 rows (keys and queries, K-major; values,
// MN-major, one panel of 64 columns) 1024 bytes apart.
__device__ __forceinline__ uint64_t operand(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ bool elect_one() {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(ok));
  return ok != 0;
}
// f32 accumulator, M and N, A and B of one 16-bit type; mn_b: B is MN-major
__device__ __forceinline__ constexpr uint32_t instruction(bool fp16, int m, int n, bool mn_b) {
  return (1u << 4) | (fp16 ? 0u : (1u << 7) | (1u << 10)) | (mn_b ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// fp8: the codes of `n` chunks of a row, at `src(c)`, as bf16 with the row's scale applied, to `dst(2 c)` and
// `dst(2 c + 1)`.
// Codes to fp16 (one instruction for two), to floats, times the scale, to bf16: two of the ALU pipe's instructions for
// two elements, where taking the codes' bits apart needs four (256 queries on 32768 tokens: 8 us of 253).  The mark of a
// row with a NaN gives an infinity, whose product with such a row's codes, zeros, is a NaN.
template <int N, class Src, class Dst>
__device__ __forceinline__ void to_bf16(uint32_t e, bool live, Src src, Dst dst) {
  const float f = __uint_as_float(e << 23);
#pragma unroll 2
  for (int c = 0; c < N; ++c) {
    uint32_t w[4] = {0, 0, 0, 0}, o[8];
    if (live)
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                   : "r"(src(c))
                   : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t h[2];
      e4m3x4_to_f16x2(w[i], h[0], h[1]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h[k]));
        o[2 * i + k] = pack2<false>(x.x * f, x.y * f);
      }
    }
    sts128(dst(2 * c), o[0], o[1], o[2], o[3]);
    sts128(dst(2 * c + 1), o[4], o[5], o[6], o[7]);
  }
}
__device__ __forceinline__ uint32_t lds8(uint32_t addr) {
  uint16_t b;
  asm volatile("ld.shared.u8 %0, [%1];" : "=h"(b) : "r"(addr) : "memory");
  return b;
}

template <int D, int FMT>
__global__ void __launch_bounds__(Cfg<D, FMT>::kWarps * 32, 1) tiles_kernel(const AttnArgs a, const PlanDev p) {
  using C = Cfg<D, FMT>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) Bars bars;
  const uint32_t warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
  const uint32_t rank = C::kCtas == 2 ? blockIdx.x & 1u : 0u, worker = blockIdx.x / C::kCtas;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_smem = smem, ring = smem + 2 * C::kQ, raw_ring = ring + C::kSlots * C::kSlot;
  auto full = [&](uint32_t i) { return smem_u32(&bars.full[i]); };
  auto empty = [&](uint32_t i) { return smem_u32(&bars.empty[i]); };

  const uint32_t first = p.tile_off[worker], last = p.tile_off[worker + 1];
  if (warp == 8 && lane == 0) {
    for (int i = 0; i < C::kSlots; ++i) {
      // 16-bit: the copies, and at the first CTA of a pair the other's word; fp8: the converting warps
      mbar_init(full(i), C::kFp8 ? 4 * C::kCtas : rank == 0 ? C::kCtas : 1);
      mbar_init(empty(i), 1);
    }
    for (int i = 0; i < C::kRaws; ++i) {
      mbar_init(smem_u32(&bars.raw_full[i]), 1);
      mbar_init(smem_u32(&bars.raw_empty[i]), 4);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&bars.q_ready[t]), 4 * C::kCtas);
      mbar_init(smem_u32(&bars.s_full[t]), 1);
      mbar_init(smem_u32(&bars.p_ready[t][0]), 4 * C::kCtas);
      mbar_init(smem_u32(&bars.p_ready[t][1]), 4 * C::kCtas);
      mbar_init(smem_u32(&bars.o_done[t]), 1);
    }
    mbar_init(smem_u32(&bars.tail_here), 1);
    mbar_init(smem_u32(&bars.tail_done), 1);
    mbar_init(smem_u32(&bars.drain), 1);
    bars.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) tc_alloc<C::kCtas>(smem_u32(&bars.tmem), 512);
  // Every warp comes here once before it uses a barrier that others set up, tensor memory or the other CTA: the
  // softmax when its first queries are on their way.  The copying warp only says that it has set the barriers
  // up; it has to be met before it waits for anything but its own copies.
  auto all_here = [&]() {
    __syncwarp();
    tc_fence_before();
    asm volatile("barrier.cta.sync 1, %0;" ::"n"(C::kWarps * 32) : "memory");
    arrive_worker<C::kCtas>();
    wait_worker<C::kCtas>();
    tc_fence_after();
    return bars.tmem;
  };

  if (warp < 8) {
    // ================= softmax: warpgroup t owns tile t, thread r its row r =================
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegSoft));
    const uint32_t t = warp / 4, r = threadIdx.x % 128;
    uint32_t s_addr = 0, o_addr = 0;
    bool here = false;
    const float sc = fmaxf(fabsf(a.scale_log2), 1.2e-38f);  // a scale of 0 still sends masked scores to -inf
    const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
    uint32_t steps = 0, done = 0;  // phases of s_full; of o_done
    bool alive = true;
    for (uint32_t pi = first; alive && pi < last; ++pi) {
      const Piece pc = p.tile_pieces[pi];
      if (pi == first) wait_for_last();  // the plan is read before, queries and results' places after
      if (!pc.split && t * C::kRows >= pc.nrows) continue;
      const uint32_t in_tile = (pc.split ? 0 : t * C::kRows) + rank * 128 + r;
      const uint32_t row = pc.row0 + in_tile;
      const bool valid = in_tile < pc.nrows;
      const uint32_t query = pc.query0 + row / a.group, head = pc.head * a.group + row % a.group;
      {
        // a warp's 32 rows, each row's chunks by neighbouring lanes; where the rows are goes through their own places
        // in shared memory
        const int64_t mine = valid ? (int64_t)query * a.q_tok + (int64_t)head * a.q_head : INT64_MIN;
        constexpr int kLanes = D / 8, kAt = 32 / kLanes;
        const uint32_t c = lane % kLanes, rows_at = q_smem + t * C::kQ + (warp % 4) * (32 * 128);
        asm volatile("st.shared.b64 [%0], %1;" ::"r"(rows_at + lane * 8), "l"(mine) : "memory");
        __syncwarp();
        uint4 w[32 / kAt];
#pragma unroll
        for (int i = 0; i < 32 / kAt; ++i) {
          int64_t at;
          asm volatile("ld.shared.b64 %0, [%1];" : "=l"(at) : "r"(rows_at + (i * kAt + lane / kLanes) * 8) : "memory");
          w[i] = at != INT64_MIN ? __ldcg(reinterpret_cast<const uint4*>(a.q + at + 8 * c)) : make_uint4(0, 0, 0, 0);
        }
        __syncwarp();
        if (!here) {
          const uint32_t tmem = all_here();
          here = true;
          s_addr = tmem + t * 128 + ((warp % 4) * 32 << 16);
          o_addr = s_addr + 256;
        }
#pragma unroll
        for (int i = 0; i < 32 / kAt; ++i) {
          const uint32_t to = (r & ~31u) + i * kAt + lane / kLanes;
          sts128(q_smem + t * C::kQ + (c / 8) * (128 * 128) + to * 128 + (((c % 8) ^ (to & 7u)) << 4),
                 w[i].x ^ flip, w[i].y ^ flip, w[i].z ^ flip, w[i].w ^ flip);
        }
      }
      fence_async_shared();
      __syncwarp();
      if (lane == 0) arrive_first<C::kCtas>(smem_u32(&bars.q_ready[t]));

      float m = -INFINITY, l = 0.0f;
      const uint32_t j0 = pc.split ? t : 0, dj = pc.split ? 2 : 1;
      for (uint32_t j = j0; j < pc.nblocks; j += dj) {
        if (!mbar_wait_warp(smem_u32(&bars.s_full[t]), steps & 1)) {
          alive = false;
          break;
        }
        ++steps;
        tc_fence_after();
        uint32_t s[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tc_ld32(s[c], s_addr + 32 * c);
        tc_wait_ld();
        const uint32_t left = pc.end - (pc.key0 + j * kTileKeys);
        if (left < (uint32_t)kTileKeys) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if ((uint32_t)(32 * c + i) >= left) s[c][i] = 0xFF800000u;
        }
        float x4[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          x4[c] = max3(__uint_as_float(s[c][0]), __uint_as_float(s[c][1]), __uint_as_float(s[c][2]));
#pragma unroll
          for (int i = 3; i < 31; i += 2) x4[c] = max3(x4[c], __uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1]));
          x4[c] = fmaxf(x4[c], __uint_as_float(s[c][31]));
        }
        const float x = max3(fmaxf(x4[0], x4[1]), x4[2], x4[3]) * sc;
        const bool grow = x > m + 8.0f;
        if (__any_sync(0xFFFFFFFFu, grow)) {
          const float n = fmaxf(m, x), f = n == m ? 1.0f : ex2(m - n);
          m = n;
          l *= f;
          if (j > j0) {  // the product before this step's scores is done: it was issued, and so finished, first
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
              uint32_t o[16];
              tc_ld16(o, o_addr + 16 * c);
              tc_wait_ld();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              tc_st16(o_addr + 16 * c, o);
            }
          }
        }
        const float u = m == -INFINITY ? 0.0f : m;
        const uint64_t sc2 = pair(__float_as_uint(sc), __float_as_uint(sc));
        const uint64_t u2 = pair(__float_as_uint(-u), __float_as_uint(-u));
        uint64_t sum2 = 0;
        // by halves, so that the product of the first half runs beside the exponentials of the second
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int c = 2 * h; c < 2 * h + 2; ++c) {
            uint32_t pk[16];
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              float p0, p1;
              unpair(fma2(pair(s[c][i], s[c][i + 1]), sc2, u2), p0, p1);
              p0 = ex2(p0);
              p1 = ex2(p1);
              sum2 = add2(sum2, pair(__float_as_uint(p0), __float_as_uint(p1)));
              pk[i / 2] = pack2<C::kFp16>(p0, p1);
            }
            tc_st16(s_addr + 16 * c, pk);
          }
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_first<C::kCtas>(smem_u32(&bars.p_ready[t][h]));
        }
        float l0, l1;
        unpair(sum2, l0, l1);
        l += l0 + l1;
      }
      if (!alive || !mbar_wait_warp(smem_u32(&bars.o_done[t]), done & 1)) {
        alive = false;
        break;
      }
      ++done;
      tc_fence_after();
      const bool direct = pc.part_row == kDirect;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      const uint64_t at = (uint64_t)pc.part_row + t * (pc.split ? pc.split : C::kRows) + rank * 128 + r;
      // The queries are used up: their shared memory takes the warp's 32 rows, half of their columns at a time, from
      // which whole rows are stored by neighbouring lanes.  A warp uses the place of its own queries alone, 4 KB in
      // each panel: the tile's other warps may be at this or already at their next piece's queries.
      auto stage = [&](uint32_t row_l) {
        return q_smem + t * C::kQ + (warp % 4) * (32 * 128) +
               (D == 128 ? (row_l / 16) * (128 * 128) + (row_l % 16) * 256 : row_l * 128);
      };
      constexpr int kCols = D / 2, kChunks = kCols / 4;  // floats and 16-byte chunks of a row in one round
      const uint32_t row0 = in_tile - lane, live = min(32u, max(row0, (uint32_t)pc.nrows) - row0);  // of the warp's rows
      constexpr int kAt = 32 / kChunks;  // rows that the warp stores at once
      const uint32_t my = lane / kChunks, mc = lane % kChunks;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t o[kCols / 32][32];
#pragma unroll
        for (int c = 0; c < kCols / 32; ++c) tc_ld32(o[c], o_addr + half * kCols + 32 * c);
        tc_wait_ld();
#pragma unroll
        for (int c = 0; c < kCols / 32; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            sts128(stage(lane) + (((8 * c + i) ^ (lane & 7u)) << 4), o[c][4 * i], o[c][4 * i + 1],
                   o[c][4 * i + 2], o[c][4 * i + 3]);
        __syncwarp();
        auto staged = [&](uint32_t row_l, uint32_t (&x)[4]) {
          asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                       : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                       : "r"(stage(row_l) + ((mc ^ (row_l & 7u)) << 4))
                       : "memory");
        };
        if (!direct) {
          float* dst = a.part + (at - lane + my) * D + half * kCols + 4 * mc;
#pragma unroll
          for (int i = 0; i < 32 / kAt; ++i) {
            uint32_t x[4];
            staged(i * kAt + my, x);
            if (i * kAt + my < live) *reinterpret_cast<uint4*>(dst + i * kAt * D) = make_uint4(x[0], x[1], x[2], x[3]);
          }
        } else {
#pragma unroll 4
          for (int i = 0; i < 32 / kAt; ++i) {
            const uint32_t row_l = i * kAt + my;
            uint32_t x[4];
            staged(row_l, x);
            const float f = __shfl_sync(0xFFFFFFFFu, inv, row_l);
            const int64_t to = __shfl_sync(0xFFFFFFFFu, (int64_t)query * a.o_tok + (int64_t)head * a.o_head, row_l);
            if (row_l < live)
              *reinterpret_cast<uint2*>(a.out + to + half * kCols + 4 * mc) =
                  make_uint2(pack2<C::kFp16>(__uint_as_float(x[0]) * f, __uint_as_float(x[1]) * f),
                             pack2<C::kFp16>(__uint_as_float(x[2]) * f, __uint_as_float(x[3]) * f));
          }
        }
        __syncwarp();
      }
      if (valid) {
        if (!direct)
          a.part_ml[at] = make_float2(m, l);
        else if (a.lse)
          a.lse[(uint64_t)query * a.kv_heads * a.group + head] =
              l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
      }
      tc_fence_before();  // the reads of O before the next piece's products, which p_ready orders
    }
    if (!here) all_here();
    if (!alive && r == 0) atomicOr_system(a.err, kErrWait);
  } else if (warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegRest));
    if (warp == 8) {
      // ================= copies: a step's keys, then its values (fp8: all at once) =================
      uint32_t n = 0, ids = 0;  // slots (fp8: raw stages) filled
      constexpr uint32_t kN = C::kFp8 ? (C::kRaws ? C::kRaws : 1) : C::kSlots;
      // The copies of this lane: 16-bit keys (2 KB panels of this CTA's blocks) and values (its panel of
      // every block), or fp8 keys, values and exponents.  blk: the block of the step; from: in its record.
      constexpr uint32_t kOwn = C::kKeys / kBlock;  // blocks whose keys this CTA holds
      uint32_t blk[2] = {0, 0}, from[2] = {0, 0}, to[2] = {0, 0}, bytes[2] = {0, 0};
      if (!C::kFp8) {
        if (lane < 8) {
          constexpr uint32_t kPanels = D / 64;
          blk[0] = rank * kOwn + lane / kPanels;
          from[0] = (lane % kPanels) * (kBlock * 128);
          to[0] = (lane % kPanels) * (C::kKeys * 128) + (lane / kPanels) * (kBlock * 128);
          blk[1] = lane;
          from[1] = C::kHalf + rank * (kBlock * 128);
          to[1] = lane * (kBlock * 128);
          bytes[0] = bytes[1] = kBlock * 128;
        }
      } else if (lane < kOwn) {
        blk[0] = rank * kOwn + lane;
        to[0] = lane * C::kHalf;
        bytes[0] = C::kHalf;
      } else if (lane >= 8 && lane < 16) {
        blk[0] = lane - 8;
        from[0] = C::kHalf + rank * (kBlock * 64);
        to[0] = C::kRawK + (lane - 8) * (kBlock * 64);
        bytes[0] = kBlock * 64;
      } else if (lane >= 16 && lane < 24) {
        blk[0] = lane - 16;
        from[0] = 2 * C::kHalf;
        to[0] = C::kRawK + C::kRawV + (lane - 16) * 32;
        bytes[0] = 32;
      }
      __syncwarp();
      asm volatile("barrier.cta.arrive 1, %0;" ::"n"(C::kWarps * 32) : "memory");
      arrive_worker<C::kCtas>();
      wait_for_last();
      let_next_start();  // the row kernel, which does not wait for what came before this one
      bool alive = true, begun = false;
      for (uint32_t pi = first; alive && pi < last; ++pi) {
        const Piece* pp = p.tile_pieces + pi;
        const uint32_t steps = pp->nblocks, block = pp->block, head = pp->head, key0 = pp->key0, end = pp->end;
        const uint32_t nb = (end - key0 + kBlock - 1) / kBlock;  // blocks from here to the span's end
        for (uint32_t j = 0; alive && j < steps; ++j) {
          if ((j & 3u) == 0) ids = p.blocks[block + min(j * 8 + lane, nb - 1)];
          const uint32_t live = min(nb - j * 8, 8u);
#pragma unroll
          for (uint32_t part = 0; part < (C::kFp8 ? 1u : 2u); ++part, ++n) {
            const uint32_t at = n % kN;
            const uint32_t fb = C::kFp8 ? smem_u32(&bars.raw_full[at % 4]) : full(at);
            const uint32_t eb = C::kFp8 ? smem_u32(&bars.raw_empty[at % 4]) : empty(at);
            if (n >= kN) {
              if (!begun) wait_worker<C::kCtas>();
              begun = true;
              if (!mbar_wait_warp(eb, (n / kN - 1) & 1)) {
                alive = false;
                break;
              }
            }
            const uint32_t id = __shfl_sync(0xFFFFFFFFu, ids, (j & 3u) * 8 + blk[part]);
            const uint32_t mine = blk[part] < live ? bytes[part] : 0u;
            const uint32_t sum = __reduce_add_sync(0xFFFFFFFFu, mine);
            if (lane == 0) mbar_expect(fb, sum);
            __syncwarp();
            if (mine)
              bulk_load((C::kFp8 ? raw_ring + at * C::kRaw : ring + at * C::kSlot) + to[part],
                        a.pool + ((uint64_t)id * a.kv_heads + head) * C::kRec + from[part], mine, fb);
          }
        }
      }
      if (!begun) wait_worker<C::kCtas>();
      for (uint32_t i = n > kN ? n - kN : 0; i < n; ++i)  // no copy is left in flight
        alive &= mbar_wait_warp(C::kFp8 ? smem_u32(&bars.raw_full[i % kN % 4]) : full(i % kN), (i / kN) & 1);
      if (!alive && lane == 0) atomicOr_system(a.err, kErrWait);
    } else {
    const uint32_t tmem = all_here();
    if (warp == 9 && rank == 0 && elect_one()) {
      // ================= products: one thread waits and issues =================
      constexpr uint32_t id_s = instruction(C::kFp16, C::kRows, kTileKeys, false);
      constexpr uint32_t id_o = instruction(C::kFp16, C::kRows, D, true);
      uint32_t n = 0;  // slots taken
      uint32_t p_seen[2] = {0, 0}, q_seen[2] = {0, 0}, tails = 0;
      bool alive = true;
      auto wait = [&](uint32_t bar, uint32_t parity) { return alive = alive && mbar_wait(bar, parity); };
      const uint64_t q_desc[2] = {operand(q_smem), operand(q_smem + C::kQ)};
      const uint64_t ring_desc = operand(ring);
      auto scores = [&](uint32_t t, uint32_t slot) {
        const uint64_t qd = q_desc[t], kd = ring_desc + slot * (C::kSlot >> 4);
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          tc_mma_ss<C::kCtas>(tmem + t * 128, qd + (((k / 4) * (128 * 128) + (k % 4) * 32) >> 4),
                              kd + (((k / 4) * (C::kKeys * 128) + (k % 4) * 32) >> 4), id_s, k > 0);
      };
      auto values = [&](uint32_t t, uint32_t slot, int half, bool acc) {
        const uint64_t vd = ring_desc + slot * (C::kSlot >> 4);
#pragma unroll
        for (int k = 4 * half; k < 4 * half + 4; ++k)
          tc_mma_ts<C::kCtas>(tmem + 256 + t * 128, tmem + t * 128 + k * 8, vd + ((k * 16 * 128) >> 4), id_o,
                              acc || k > 0);
      };
      for (uint32_t pi = first; alive && pi < last; ++pi) {
        const Piece* pp = p.tile_pieces + pi;
        const uint32_t steps = pp->nblocks, keys = pp->end - pp->key0;
        const uint32_t tiles = pp->nrows > C::kRows ? 2 : 1;
        // ring order: keys 0, values 0, keys 1, values 1, ...: step j's keys are slot n0 + 2j, values n0 + 2j + 1
        const uint32_t n0 = n;
        auto slot = [&](uint32_t i) { return (n0 + i) % C::kSlots; };
        auto here = [&](uint32_t i) { return wait(full(slot(i)), ((n0 + i) / C::kSlots) & 1u); };
        // A step's values and its rows' next scores, by tile t; `ahead` steps lie between them.
        auto turn = [&](uint32_t t, uint32_t j, uint32_t ahead) {
          if (!wait(smem_u32(&bars.p_ready[t][0]), p_seen[t] & 1)) return false;
          tc_fence_after();
          values(t, slot(2 * j + 1), 0, j >= ahead);
          if (!wait(smem_u32(&bars.p_ready[t][1]), p_seen[t] & 1)) return false;
          ++p_seen[t];
          tc_fence_after();
          values(t, slot(2 * j + 1), 1, true);
          if (j + ahead < steps) {
            if (!here(2 * (j + ahead))) return false;
            scores(t, slot(2 * (j + ahead)));
            tc_commit<C::kCtas>(smem_u32(&bars.s_full[t]));
          } else {
            tc_commit<C::kCtas>(smem_u32(&bars.o_done[t]));
          }
          return true;
        };
        // One tile of rows alone would leave the tensor cores idle during its softmax: its even and odd steps run as
        // two tiles, each with a result of its own.
        const uint32_t ahead = pp->split ? 2 : 1;
        for (uint32_t t = 0; t < (pp->split ? 2 : tiles); ++t) {
          if (!here(pp->split ? 2 * t : 0) || !wait(smem_u32(&bars.q_ready[t]), q_seen[t] & 1)) break;
          ++q_seen[t];
          tc_fence_after();
          scores(t, slot(pp->split ? 2 * t : 0));
          tc_commit<C::kCtas>(smem_u32(&bars.s_full[t]));
          if (pp->split || t == tiles - 1) tc_commit<C::kCtas>(empty(slot(pp->split ? 2 * t : 0)));
        }
        for (uint32_t j = 0; alive && j < steps; ++j) {
          if (!here(2 * j + 1)) break;
          if (!C::kFp8 && keys - j * kTileKeys < (uint32_t)kTileKeys) {
            mbar_arrive(smem_u32(&bars.tail_here));
            if (!wait(smem_u32(&bars.tail_done), tails++ & 1)) break;
          }
          if (pp->split) {
            if (!turn(j & 1, j, 2)) break;
          } else {
            for (uint32_t t = 0; t < tiles; ++t)
              if (!turn(t, j, 1)) break;
          }
          if (alive) {
            tc_commit<C::kCtas>(empty(slot(2 * j + 1)));
            if (j + ahead < steps) tc_commit<C::kCtas>(empty(slot(2 * (j + ahead))));
          }
        }
        n = n0 + 2 * steps;
      }
      tc_commit<C::kCtas>(smem_u32(&bars.drain));
      alive = mbar_wait(smem_u32(&bars.drain), 0) && alive;  // nothing is in flight when tensor memory is freed
      if (!alive) {
        atomicOr_system(a.err, kErrWait);
        *static_cast<volatile uint32_t*>(&bars.gave_up) = 1;
        mbar_arrive(smem_u32(&bars.tail_here));  // releases the warp that waits for it
      }
    } else if (warp == 9 && rank == 1 && !C::kFp8 && elect_one()) {
      // ================= the pair's second CTA: tells the first what has arrived here =================
      uint32_t n = 0, tails = 0;
      bool alive = true;
      for (uint32_t pi = first; alive && pi < last; ++pi) {
        const Piece* pp = p.tile_pieces + pi;
        const uint32_t slots = 2 * pp->nblocks;
        const bool partial = pp->end - pp->key0 < pp->nblocks * kTileKeys;
        for (uint32_t i = 0; alive && i < slots; ++i, ++n) {
          const uint32_t at = n % C::kSlots;
          alive = mbar_wait(full(at), (n / C::kSlots) & 1);
          if (alive && partial && i == slots - 1) {
            mbar_arrive(smem_u32(&bars.tail_here));
            alive = mbar_wait(smem_u32(&bars.tail_done), tails++ & 1);
          }
          if (alive) arrive_first<C::kCtas>(full(at));
        }
      }
      if (!alive) {
        atomicOr_system(a.err, kErrWait);
        *static_cast<volatile uint32_t*>(&bars.gave_up) = 1;
        mbar_arrive(smem_u32(&bars.tail_here));
      }
    } else if (warp == 10 && !C::kFp8) {
      // ================= partial steps: value rows past the end hold other tokens or earlier steps =================
      uint32_t n = 0, tails = 0;
      bool alive = true;
      for (uint32_t pi = first; alive && pi < last; ++pi) {
        const Piece* pp = p.tile_pieces + pi;
        n += 2 * pp->nblocks;
        const uint32_t left = pp->end - (pp->key0 + (pp->nblocks - 1) * kTileKeys);
        if (left >= (uint32_t)kTileKeys) continue;
        // The whole share may run before this step comes; the issuing thread's own waits are short, and it
        // also arrives when it gives up.
        if (!__all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&bars.tail_here), tails++ & 1, 60000000000ull))) {
          alive = false;
          break;
        }
        if (*static_cast<volatile uint32_t*>(&bars.gave_up)) break;  // no step comes any more
        const uint32_t v = ring + (n - 1) % C::kSlots * C::kSlot;  // the last step's values
        for (uint32_t i = left * 8 + lane; i < kTileKeys * 8; i += 32)
          sts128(v + (i / 8) * 128 + (i % 8) * 16, 0, 0, 0, 0);
        fence_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.tail_done));
      }
      if (!alive && lane == 0) atomicOr_system(a.err, kErrWait);
    }
    }
  } else {
    // ================= fp8: records to operands, a thread a token =================
    if constexpr (C::kFp8) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegRest));
      all_here();
      const uint32_t tok = threadIdx.x % 128;
      const uint32_t kt = tok % C::kKeys, kb = kt / kBlock, vb = tok / kBlock;  // this thread's key; blocks
      constexpr int kChunks = D / 16 / C::kCtas;                               // and chunks of it: 4
      const uint32_t kc = tok / C::kKeys * kChunks;
      constexpr uint32_t kOwn = C::kKeys / kBlock;
      uint32_t n = 0, raws = 0;
      bool alive = true;
      for (uint32_t pi = first; alive && pi < last; ++pi) {
        const Piece* pp = p.tile_pieces + pi;
        const uint32_t steps = pp->nblocks, keys = pp->end - pp->key0;
        for (uint32_t j = 0; alive && j < steps; ++j, ++raws) {
          const uint32_t rs = raws % C::kRaws;
          if (!mbar_wait_warp(smem_u32(&bars.raw_full[rs]), (raws / C::kRaws) & 1)) {
            alive = false;
            break;
          }
          const uint32_t raw = raw_ring + rs * C::kRaw, exps = raw + C::kRawK + C::kRawV;
          const uint32_t left = keys - j * kTileKeys;
          for (uint32_t part = 0; part < 2; ++part, ++n) {
            const uint32_t at = n % C::kSlots;
            if (n >= (uint32_t)C::kSlots && !mbar_wait_warp(empty(at), (n / C::kSlots - 1) & 1)) {
              alive = false;
              break;
            }
            const uint32_t dst = ring + at * C::kSlot;
            if (part == 0) {
              const bool live = rank * C::kKeys + kt < left;
              const uint32_t at_e = exps + (rank * kOwn + kb) * 32 + exp_place(kt % kBlock);
              const uint32_t e = live ? lds8(at_e) : (uint32_t)kExpBias;
              to_bf16<kChunks>(
                  e, live, [&](int c) { return raw + kb * C::kHalf + offset8k<D>(kt % kBlock, kc + c); },
                  [&](int c) {
                    const uint32_t cc = 2 * kc + c;
                    return dst + (cc / 8) * (C::kKeys * 128) + kt * 128 + (((cc % 8) ^ (kt & 7u)) << 4);
                  });
            } else {
              const bool live = tok < left;
              const uint32_t at_e = exps + vb * 32 + kBlock + exp_place(tok % kBlock);
              const uint32_t e = live ? lds8(at_e) : (uint32_t)kExpBias;
              to_bf16<4>(
                  e, live, [&](int c) { return raw + C::kRawK + vb * (kBlock * 64) + offset8v(tok % kBlock, c); },
                  [&](int c) { return dst + tok * 128 + ((c ^ (tok & 7u)) << 4); });
            }
            fence_async_shared();
            __syncwarp();
            if (lane == 0) arrive_first<C::kCtas>(full(at));
          }
          if (alive && lane == 0) mbar_arrive(smem_u32(&bars.raw_empty[rs]));
        }
      }
      if (!alive && tok == 0) atomicOr_system(a.err, kErrWait);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  arrive_worker<C::kCtas>();
  wait_worker<C::kCtas>();  // no CTA leaves while the other may arrive on its barriers or read its memory
  tc_fence_after();
  if (warp == 9) tc_dealloc<C::kCtas>(bars.tmem, 512);
}

template <int D, int FMT>
cudaError_t prepare_one() {
  // setmaxnreg hands out what the launch was given: fewer registers than the split adds up to would wait for ever
  cudaFuncAttributes at{};
  cudaError_t e = cudaFuncGetAttributes(&at, tiles_kernel<D, FMT>);
  if (e != cudaSuccess) return e;
  const int threads = Cfg<D, FMT>::kWarps * 32;
  if (at.numRegs * threads < 256 * Cfg<D, FMT>::kRegSoft + (threads - 256) * Cfg<D, FMT>::kRegRest)
    return cudaErrorInvalidKernelImage;
  return cudaFuncSetAttribute(tiles_kernel<D, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D, FMT>::kSmem);
}
template <int D, int FMT>
cudaError_t launch_one(const AttnArgs& a, const PlanDev& p, bool overlap, cudaStream_t s) {
  using C = Cfg<D, FMT>;
  return launch(tiles_kernel<D, FMT>, p.tile_workers * C::kCtas, C::kWarps * 32, C::kSmem, C::kCtas, overlap, s, a, p);
}

}  // namespace

cudaError_t prepare_tiles(int D, int fmt) {
  if (D == 128)
    return fmt == PS_KV_BF16   ? prepare_one<128, PS_KV_BF16>()
           : fmt == PS_KV_FP16 ? prepare_one<128, PS_KV_FP16>()
                               : prepare_one<128, PS_KV_FP8>();
  return fmt == PS_KV_BF16   ? prepare_one<64, PS_KV_BF16>()
         : fmt == PS_KV_FP16 ? prepare_one<64, PS_KV_FP16>()
                             : prepare_one<64, PS_KV_FP8>();
}

cudaError_t launch_tiles(int D, int fmt, const AttnArgs& a, const PlanDev& p, bool overlap, cudaStream_t s) {
  if (D == 128)
    return fmt == PS_KV_BF16   ? launch_one<128, PS_KV_BF16>(a, p, overlap, s)
           : fmt == PS_KV_FP16 ? launch_one<128, PS_KV_FP16>(a, p, overlap, s)
                               : launch_one<128, PS_KV_FP8>(a, p, overlap, s);
  return fmt == PS_KV_BF16   ? launch_one<64, PS_KV_BF16>(a, p, overlap, s)
         : fmt == PS_KV_FP16 ? launch_one<64, PS_KV_FP16>(a, p, overlap, s)
                             : launch_one<64, PS_KV_FP8>(a, p, overlap, s);
}

}  // namespace pskv
