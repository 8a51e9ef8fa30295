// Copies of what the cache holds: tokens moved inside it, whole blocks copied inside or from another cache.
#include "kv_internal.cuh"

namespace pskv {
namespace {

// A token's rows of a head as 16-byte chunks: the keys', the values', and with fp8 one for the two exponents.
template <int D, int FMT>
struct Held {
  static constexpr bool kFp8 = FMT == PS_KV_FP8;
  static constexpr int kRec = record_bytes(D, FMT), kHalf = half_bytes(D, FMT);
  static constexpr uint32_t kOwn = D / (kFp8 ? 16 : 8);  // chunks of a row of keys or values
  static constexpr uint32_t kChunks = 2 * kOwn + (kFp8 ? 1 : 0);
  __device__ static __forceinline__ uint32_t place(uint32_t tok, uint32_t c) {
    if (c < kOwn) return kFp8 ? offset8k<D>(tok, c) : offset16(tok, c);
    return kHalf + (kFp8 ? offset8v(tok, c - kOwn) : offset16(tok, c - kOwn));
  }
  __device__ static __forceinline__ uint4 get(const uint8_t* pool, uint64_t slot, uint32_t heads, uint32_t h, uint32_t c) {
    const uint8_t* rec = pool + (slot / kBlock * heads + h) * kRec;
    const uint32_t tok = (uint32_t)(slot % kBlock);
    if (c < 2 * kOwn) return *reinterpret_cast<const uint4*>(rec + place(tok, c));
    return make_uint4(rec[2 * kHalf + exp_place(tok)], rec[2 * kHalf + kBlock + exp_place(tok)], 0, 0);
  }
  __device__ static __forceinline__ void put(uint8_t* pool, uint64_t slot, uint32_t heads, uint32_t h, uint32_t c,
                                             uint4 x) {
    uint8_t* rec = pool + (slot / kBlock * heads + h) * kRec;
    const uint32_t tok = (uint32_t)(slot % kBlock);
    if (c < 2 * kOwn) {
      *reinterpret_cast<uint4*>(rec + place(tok, c)) = x;
    } else {
      rec[2 * kHalf + exp_place(tok)] = (uint8_t)x.x;
      rec[2 * kHalf + kBlock + exp_place(tok)] = (uint8_t)x.y;
    }
  }
};

// Whether move i happens; its slots.
__device__ __forceinline__ bool moves(const MoveArgs& a, uint64_t i, int64_t* src, int64_t* dst, bool report) {
  *src = a.src[i];
  *dst = a.dst[i];
  if (*dst < 0) return false;
  if (*dst >= (int64_t)a.num_slots || *src >= (int64_t)a.num_slots) {
    if (report) atomicOr_system(a.err, kErrSlot);
    return false;
  }
  return true;
}

// Up to kMoveTokens moves in one launch: moves of one head and column of chunks touch no other column, so a CTA takes
// a column of all tokens, reads it whole into registers and then writes it.  Columns of 64 bytes (two sectors).
// Bound by latency: the slots, the rows, their way back.  One token of 8 heads, 128 columns and 16 bits 1.5 us, 512 of
// them 3.4; by the two launches below 3.2 and 4.4.  With more tokens the CTAs (64 here) are too few: 1024 of them took
// 6.4, by two launches 5.3.
constexpr uint32_t kColumn = 4, kMoveThreads = 1024, kPer = 2;
constexpr uint32_t kMoveTokens = kMoveThreads * kPer / kColumn;

template <int D, int FMT>
__global__ void __launch_bounds__(kMoveThreads, 1) move_kernel(const MoveArgs a) {
  using H = Held<D, FMT>;
  constexpr uint32_t kColumns = (H::kChunks + kColumn - 1) / kColumn;
  const uint32_t h = blockIdx.x / kColumns, c0 = blockIdx.x % kColumns * kColumn;
  const uint32_t c = c0 + threadIdx.x % kColumn, first = threadIdx.x / kColumn, step = blockDim.x / kColumn;
  uint4 x[kPer];
#pragma unroll
  for (uint32_t k = 0; k < kPer; ++k) {
    const uint64_t i = first + k * step;
    x[k] = make_uint4(0, 0, 0, 0);
    int64_t src, dst;
    if (i < a.n && c < H::kChunks && moves(a, i, &src, &dst, blockIdx.x == 0) && src >= 0)
      x[k] = H::get(a.pool, (uint64_t)src, a.kv_heads, h, c);
  }
  __syncthreads();
#pragma unroll
  for (uint32_t k = 0; k < kPer; ++k) {
    const uint64_t i = first + k * step;
    int64_t src, dst;
    if (i < a.n && c < H::kChunks && moves(a, i, &src, &dst, false)) H::put(a.pool, (uint64_t)dst, a.kv_heads, h, c, x[k]);
  }
}

// More of them: all sources into the workspace, and from there to their places.  Bound by bytes, twice those of the
// rows: 16384 tokens, 268 MB, 65 us = 4.1 TB/s.
template <int D, int FMT, bool GATHER>
__global__ void __launch_bounds__(256) move_far_kernel(const MoveArgs a) {
  using H = Held<D, FMT>;
  const uint64_t per = (uint64_t)a.kv_heads * H::kChunks, items = a.n * per;
  for (uint64_t it = (uint64_t)blockIdx.x * 256 + threadIdx.x; it < items; it += (uint64_t)gridDim.x * 256) {
    const uint64_t i = it / per;
    const uint32_t rest = (uint32_t)(it - i * per), h = rest / H::kChunks, c = rest % H::kChunks;
    int64_t src, dst;
    if (!moves(a, i, &src, &dst, GATHER && rest == 0)) continue;
    if (GATHER)
      a.space[it] = src < 0 ? make_uint4(0, 0, 0, 0) : H::get(a.pool, (uint64_t)src, a.kv_heads, h, c);
    else
      H::put(a.pool, (uint64_t)dst, a.kv_heads, h, c, a.space[it]);
  }
}

template <int D, int FMT>
cudaError_t go(const MoveArgs& a, int sms, cudaStream_t s) {
  using H = Held<D, FMT>;
  if (a.n <= kMoveTokens) {
    const unsigned columns = (H::kChunks + kColumn - 1) / kColumn;
    const unsigned threads = (unsigned)((a.n * kColumn + 31) / 32 * 32);
    move_kernel<D, FMT><<<a.kv_heads * columns, threads < kMoveThreads ? threads : kMoveThreads, 0, s>>>(a);
    return cudaGetLastError();
  }
  const uint64_t need = (a.n * a.kv_heads * H::kChunks + 255) / 256, most = (uint64_t)sms * 64;
  const unsigned grid = (unsigned)(need < most ? need : most);
  move_far_kernel<D, FMT, true><<<grid, 256, 0, s>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  move_far_kernel<D, FMT, false><<<grid, 256, 0, s>>>(a);
  return cudaGetLastError();
}

template <int D>
cudaError_t by_format(int fmt, const MoveArgs& a, int sms, cudaStream_t s) {
  switch (fmt) {
    case PS_KV_BF16: return go<D, PS_KV_BF16>(a, sms, s);
    case PS_KV_FP16: return go<D, PS_KV_FP16>(a, sms, s);
    case PS_KV_FP8: return go<D, PS_KV_FP8>(a, sms, s);
  }
  return cudaErrorInvalidValue;
}

// A block is one run of bytes (its heads' records lie side by side).  A CTA takes a part of one, eight 16-byte loads a
// thread on their way at once.  Bound by bytes: 8192 blocks of 8 heads, 128 columns, fp8, 541 MB: 82 us = 6.6 TB/s, 97% of
// the measured copy.
constexpr uint32_t kCopyChunks = 256 * 8;

__global__ void __launch_bounds__(256) copy_kernel(const CopyArgs a) {
  const uint64_t items = a.n * a.parts;
  for (uint64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const uint64_t i = it / a.parts;
    const uint32_t part = (uint32_t)(it - i * a.parts);
    const int64_t src = a.src[i], dst = a.dst[i];
    if (dst < 0) continue;
    if ((uint64_t)dst >= a.num_blocks || (src >= 0 && (uint64_t)src >= a.from_blocks)) {
      if (threadIdx.x == 0 && part == 0) atomicOr_system(a.err, kErrSlot);
      continue;
    }
    const uint32_t lo = (uint32_t)((uint64_t)a.chunks * part / a.parts);
    const uint32_t hi = (uint32_t)((uint64_t)a.chunks * (part + 1) / a.parts);
    const uint4* from = reinterpret_cast<const uint4*>(a.from) + (uint64_t)(src < 0 ? 0 : src) * a.chunks;
    uint4* to = reinterpret_cast<uint4*>(a.pool) + (uint64_t)dst * a.chunks;
    uint4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t at = lo + k * 256 + threadIdx.x;
      x[k] = src >= 0 && at < hi ? from[at] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t at = lo + k * 256 + threadIdx.x;
      if (at < hi) to[at] = x[k];
    }
  }
}

}  // namespace

uint64_t move_space(int D, int fmt, uint32_t heads, uint64_t n) {
  if (n <= kMoveTokens) return 0;
  const uint64_t chunks = fmt == PS_KV_FP8 ? D / 8 + 1 : D / 4;
  return n * heads * chunks * 16;
}
cudaError_t launch_move(int D, int fmt, const MoveArgs& a, int sms, cudaStream_t s) {
  return D == 128 ? by_format<128>(fmt, a, sms, s) : by_format<64>(fmt, a, sms, s);
}
cudaError_t launch_copy(CopyArgs a, int sms, cudaStream_t s) {
  a.parts = (a.chunks + kCopyChunks - 1) / kCopyChunks;
  const uint64_t need = a.n * a.parts, most = (uint64_t)sms * 1024;
  copy_kernel<<<(unsigned)(need < most ? need : most), 256, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace pskv
