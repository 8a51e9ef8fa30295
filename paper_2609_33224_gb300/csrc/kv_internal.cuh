// Shared by the serving operators (kv*.cu): the layout of a cache block, the descriptors that a plan hands
// to the attention kernels, and the PTX wrappers they use.
//
// A cache is an array of records, one per (block, key/value head), the heads of a block next to each other.
// A record holds 16 tokens:
//   16-bit formats: K then V, each D / 64 panels of 64 columns; a panel is 16 rows x 128 bytes, 16-byte chunk
//     c of row r at chunk c ^ (r % 8).  That is the 128-byte-swizzled order that the tensor cores read from
//     shared memory (keys K-major, values MN-major, groups of 8 rows 1024 bytes apart), so plain bulk copies
//     of panels land ready for use, and ldmatrix reads them without bank conflicts.
//   fp8: K codes (16 rows of D bytes, chunk c of row r at c ^ swz(r)), V codes (D / 64 panels of 16 rows x
//     64 bytes, chunks swizzled too), then the 16 scale exponents of K and the 16 of V (biased by 127; 255:
//     the row holds a NaN, and its codes are 0), which fill one 32-byte sector: one copy brings a record with
//     its scales.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kv_plan.h"
#include "packserve_kv.h"

namespace pskv {

constexpr int kExpBias = 127;
constexpr int kExpMin = -110, kExpMax = 119, kExpNan = 255;

enum : uint32_t { kErrSlot = 1u, kErrWait = 2u };

__host__ __device__ constexpr int record_bytes(int D, int fmt) {
  return fmt == PS_KV_FP8 ? 2 * kBlock * D + 2 * kBlock : 2 * kBlock * D * 2;
}
__host__ __device__ constexpr int half_bytes(int D, int fmt) { return kBlock * D * (fmt == PS_KV_FP8 ? 1 : 2); }

// byte offset of 16-byte chunk c of token t inside the K or V part of a 16-bit record
__device__ __forceinline__ uint32_t offset16(uint32_t t, uint32_t c) {
  return (c >> 3) * (kBlock * 128) + (t >> 3) * 1024 + (t & 7u) * 128 + (((c & 7u) ^ (t & 7u)) << 4);
}
// the same inside the K part of an fp8 record, and inside its V part
template <int D>
__device__ __forceinline__ uint32_t offset8k(uint32_t t, uint32_t c) {
  return D == 128 ? t * 128 + ((c ^ (t & 7u)) << 4) : t * 64 + ((c ^ ((t >> 1) & 3u)) << 4);
}
__device__ __forceinline__ uint32_t offset8v(uint32_t t, uint32_t c) {
  return (c >> 2) * (kBlock * 64) + t * 64 + (((c & 3u) ^ ((t >> 1) & 3u)) << 4);
}
// where token t's exponent lies among the 16: the four that a lane of an m16n8 result needs next to each other
__device__ __forceinline__ uint32_t exp_place(uint32_t t) { return ((t & 7u) >> 1) * 4 + (t >> 3) * 2 + (t & 1u); }

struct PlanDev {
  const Piece* row_pieces;
  const uint32_t* row_off;  // pieces of worker w: row_off[w] .. row_off[w + 1]
  uint32_t row_workers, row_ctas;
  const Piece* tile_pieces;
  const uint32_t* tile_off;
  uint32_t tile_workers;  // CTAs, or pairs of them
  const JoinEntry* join;
  const JoinSeg* segs;
  const Fold* folds;
  uint32_t njoin, join_stride;  // entries, and rows that each gets
  uint32_t max_parts;
  const uint32_t* blocks;
};

struct AttnArgs {
  const uint8_t* pool;
  const uint16_t* q;
  int64_t q_tok, q_head;  // in elements
  uint16_t* out;
  int64_t o_tok, o_head;
  float* lse;       // [query][q head] or null
  float* part;      // [part row][D], not yet divided by the sum
  float2* part_ml;  // [part row] maximum (of the scores times log2 e) and sum
  uint32_t kv_heads, group;
  float scale_log2;
  uint32_t rows_first;  // the row kernel is the call's first: it waits for what came before
  uint32_t* err;  // mapped host word
};

struct StoreArgs {
  uint8_t* pool;
  const int64_t* slots;
  uint64_t n;
  uint64_t num_slots;
  uint32_t kv_heads;
  void* k;
  void* v;
  int64_t k_tok, k_head, v_tok, v_head;
  uint32_t* err;
};

cudaError_t launch_write(int D, int fmt, int type, const StoreArgs& a, int sms, cudaStream_t s);
cudaError_t launch_read(int D, int fmt, int type, const StoreArgs& a, int sms, cudaStream_t s);
cudaError_t launch_rows(int D, int fmt, const AttnArgs& a, const PlanDev& p, bool overlap, cudaStream_t s);
cudaError_t launch_join(int D, bool fp16, const AttnArgs& a, const PlanDev& p, bool overlap, cudaStream_t s);
cudaError_t launch_tiles(int D, int fmt, const AttnArgs& a, const PlanDev& p, bool overlap, cudaStream_t s);
cudaError_t prepare_rows(int D, int fmt);
cudaError_t prepare_tiles(int D, int fmt);
// ---- PTX ----------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_u32(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// Waits for a phase, by default one second at most (the limit of the scheduler's waits); false: it gave up.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, uint64_t limit_ns = 1000000000ull) {
  if (mbar_try(bar, parity)) return true;
  const uint64_t t0 = now_ns();
#pragma unroll 1
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try(bar, parity)) return true;
    if (now_ns() - t0 > limit_ns) return false;
  }
}
// The same for a whole warp, which goes on or gives up together.
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity) {
  return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity)) != 0;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
// A call's kernels are launched so that the next may start while the last one ends.  The call's first kernel waits for
// what came before it in the stream where it first reads or writes anything but the plan, and only then lets the next
// one start; each later one waits for the one before it (and with it all earlier ones) where it reads its results, at
// the latest before it ends.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <class... P, class... A>
cudaError_t launch(void (*kernel)(P...), unsigned grid, unsigned block, size_t smem, unsigned cluster, bool overlap,
                   cudaStream_t s, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = overlap ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <bool FP16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if (FP16) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Two bf16 as floats.
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// The scale of an fp8 row as a float; the mark of a row with a NaN gives a NaN.
__device__ __forceinline__ float exp_value(uint32_t e) {
  return __uint_as_float(e == kExpNan ? 0x7FC00000u : e << 23);
}

// Two e4m3 codes in the high bytes of the halves of x -> bf16x2, without their scale.  A code's magnitude
// bits, moved down by 4, are a bf16 whose exponent bias is 127 instead of 7 (subnormal codes become bf16
// subnormals), so a product with 2^120 gives the value, exactly.  (No code of a cache is a NaN: rows with
// one are marked by their scale.)
__device__ __forceinline__ uint32_t e4m3_to_bf16x2(uint32_t x) {
  const uint32_t y = ((x >> 4) & 0x07F007F0u) | (x & 0x80008000u);
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(y), "r"(0x7B807B80u));
  return r;
}

// The same to f16x2: the two codes in the lower or upper half of x.
__device__ __forceinline__ void e4m3x4_to_f16x2(uint32_t x, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}\n"
      : "=r"(lo), "=r"(hi)
      : "r"(x));
}

}  // namespace pskv
