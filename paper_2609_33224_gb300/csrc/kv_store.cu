// Writing keys and values into the block cache and reading them back.
#include <cuda_fp8.h>

#include "kv_internal.cuh"

namespace pskv {
namespace {

template <int TYPE>
struct Elem;
template <>
struct Elem<PS_KV_BF16> {
  static constexpr int kSize = 2;
};
template <>
struct Elem<PS_KV_FP16> {
  static constexpr int kSize = 2;
};
template <>
struct Elem<PS_KV_FP32> {
  static constexpr int kSize = 4;
};

// N consecutive elements as 16-byte loads, then as floats
template <int TYPE, int N>
struct Row {
  static constexpr int kVec = N * Elem<TYPE>::kSize / 16;
  uint4 w[kVec];
  __device__ __forceinline__ void load(const void* base, int64_t elem) {
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(base) + elem * Elem<TYPE>::kSize);
#pragma unroll
    for (int i = 0; i < kVec; ++i) w[i] = __ldcs(p + i);
  }
  __device__ __forceinline__ void store(void* base, int64_t elem) const {
    uint4* p = reinterpret_cast<uint4*>(static_cast<uint8_t*>(base) + elem * Elem<TYPE>::kSize);
#pragma unroll
    for (int i = 0; i < kVec; ++i) __stcs(p + i, w[i]);
  }
  __device__ __forceinline__ void floats(float (&x)[N]) const {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(w);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (TYPE == PS_KV_FP32) {
        x[i] = __uint_as_float(u[i]);
      } else if (TYPE == PS_KV_BF16) {
        x[i] = (i & 1) ? bf16_hi(u[i / 2]) : bf16_lo(u[i / 2]);
      } else {
        const __half2 h = *reinterpret_cast<const __half2*>(&u[i / 2]);
        x[i] = (i & 1) ? __high2float(h) : __low2float(h);
      }
    }
  }
  __device__ __forceinline__ void set(const float (&x)[N]) {
    uint32_t* u = reinterpret_cast<uint32_t*>(w);
    if (TYPE == PS_KV_FP32) {
#pragma unroll
      for (int i = 0; i < N; ++i) u[i] = __float_as_uint(x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 2) u[i / 2] = pack2<TYPE == PS_KV_FP16>(x[i], x[i + 1]);
    }
  }
};

// One row's 16 elements per lane (D / 16 lanes a row): the row's scale exponent, and this lane's codes.
template <int D>
__device__ __forceinline__ uint4 quantise(const float (&x)[16], uint32_t* exp_code) {
  float amax = 0.0f;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    nan |= x[i] != x[i];
    amax = fmaxf(amax, fabsf(x[i]));  // fmaxf passes a NaN over
  }
#pragma unroll
  for (int o = 1; o < D / 16; o <<= 1) {
    amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, o));
    nan |= __shfl_xor_sync(0xFFFFFFFFu, (int)nan, o) != 0;
  }
  amax = fminf(amax, 3.402823466e38f);
  // the smallest e with amax <= 1.75 * 2^(e + 8), from the float's exponent and mantissa fields; a
  // subnormal's fields give an e below the range, as they should
  const uint32_t b = __float_as_uint(amax);
  int e = (int)(b >> 23) - kExpBias - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = min(max(e, kExpMin), kExpMax);
  const float inv = __uint_as_float((uint32_t)(kExpBias - e) << 23);
  uint4 code;
  uint32_t* c = reinterpret_cast<uint32_t*>(&code);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 a = make_float2(x[4 * i] * inv, x[4 * i + 1] * inv);
    const float2 d = make_float2(x[4 * i + 2] * inv, x[4 * i + 3] * inv);
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(a, __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(d, __NV_SATFINITE, __NV_E4M3);
    c[i] = lo | (hi << 16);
  }
  if (nan) code = make_uint4(0, 0, 0, 0);  // the scale marks the row; no code of the cache is a NaN
  *exp_code = nan ? kExpNan : (uint32_t)(e + kExpBias);
  return code;
}

// A lane's chunk of a (token, head) row of K and of V: 16 bytes of the cache each, loaded together.  Lanes
// run over the chunks of a row, then heads, then tokens, as the caller's rows lie in memory.
// Bound by bytes: reads 2 * D source elements and writes the record's rows, each once.  65536 tokens of 8 heads and
// 128 columns, bf16 to fp8, 403 MB: 63 us = 6.4 TB/s, 94% of the measured copy.
// Six blocks an SM: with the 50 registers it takes without the bound, 151 us instead of 146 for a store and a load.
template <int D, int FMT, int TYPE>
__global__ void __launch_bounds__(256, TYPE == PS_KV_FP32 ? 4 : 6) write_kernel(StoreArgs a) {
  constexpr bool kFp8 = FMT == PS_KV_FP8;
  constexpr int kN = kFp8 ? 16 : 8;  // elements of a 16-byte chunk
  constexpr int kLanes = D / kN;
  const uint32_t items = (uint32_t)a.n * a.kv_heads;  // < 2^31: longer calls are cut
  constexpr int kRec = record_bytes(D, FMT), kHalf = half_bytes(D, FMT);
  const uint32_t c = threadIdx.x % kLanes;
  const uint32_t step = gridDim.x * (256 / kLanes);
  // every lane of a warp runs the same number of rounds: the row's maximum is taken with full-warp shuffles
  const uint32_t first = blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  const uint32_t rounds = (items + step - 1) / step;
  for (uint32_t r = 0, it = first; r < rounds; ++r, it += step) {
    const bool live = it < items;
    const uint32_t t = live ? it / a.kv_heads : 0;
    const uint32_t h = live ? it - t * a.kv_heads : 0;
    const int64_t slot = live ? a.slots[t] : -1;
    bool ok = slot >= 0;
    if (ok && (uint64_t)slot >= a.num_slots) {
      ok = false;
      atomicOr_system(a.err, kErrSlot);
    }
    Row<TYPE, kN> k, v;
    if (ok) {
      k.load(a.k, (int64_t)t * a.k_tok + (int64_t)h * a.k_head + c * kN);
      v.load(a.v, (int64_t)t * a.v_tok + (int64_t)h * a.v_head + c * kN);
    } else {
#pragma unroll
      for (int i = 0; i < Row<TYPE, kN>::kVec; ++i) k.w[i] = v.w[i] = make_uint4(0, 0, 0, 0);
    }
    uint8_t* rec = a.pool + ((uint64_t)(ok ? slot : 0) / kBlock * a.kv_heads + h) * kRec;
    const uint32_t tok = (uint32_t)((uint64_t)(ok ? slot : 0) % kBlock);
    const uint32_t ko = kFp8 ? offset8k<D>(tok, c) : offset16(tok, c);
    const uint32_t vo = kHalf + (kFp8 ? offset8v(tok, c) : offset16(tok, c));
    if constexpr (kFp8) {
      float x[16];
      uint32_t ek, ev;
      k.floats(x);
      const uint4 ck = quantise<D>(x, &ek);
      v.floats(x);
      const uint4 cv = quantise<D>(x, &ev);
      if (ok) {
        *reinterpret_cast<uint4*>(rec + ko) = ck;
        *reinterpret_cast<uint4*>(rec + vo) = cv;
        if (c == 0) {
          rec[2 * kHalf + exp_place(tok)] = (uint8_t)ek;
          rec[2 * kHalf + kBlock + exp_place(tok)] = (uint8_t)ev;
        }
      }
    } else if (ok) {
      if constexpr (TYPE == FMT) {
        *reinterpret_cast<uint4*>(rec + ko) = k.w[0];
        *reinterpret_cast<uint4*>(rec + vo) = v.w[0];
      } else {
        float x[8];
        Row<FMT, 8> o;
        k.floats(x);
        o.set(x);
        *reinterpret_cast<uint4*>(rec + ko) = o.w[0];
        v.floats(x);
        o.set(x);
        *reinterpret_cast<uint4*>(rec + vo) = o.w[0];
      }
    }
  }
}

__device__ __forceinline__ void decode(const uint4& code, uint32_t e, float (&x)[16]) {
  const float s = exp_value(e);
  const uint32_t* c = reinterpret_cast<const uint32_t*>(&code);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = e4m3_to_bf16x2(__byte_perm(c[i], 0, 0x1404)), hi = e4m3_to_bf16x2(__byte_perm(c[i], 0, 0x3424));
    x[4 * i] = bf16_lo(lo) * s;
    x[4 * i + 1] = bf16_hi(lo) * s;
    x[4 * i + 2] = bf16_lo(hi) * s;
    x[4 * i + 3] = bf16_hi(hi) * s;
  }
}

// The reverse of write_kernel, with the same lanes.  131072 tokens of 8 heads and 128 columns, fp8 to bf16: 146 us
// for 807 MB, two thirds of them written; the card writes 3.9 TB/s (a fill of 2 GB), at which those take 139 us.
template <int D, int FMT, int TYPE>
__global__ void __launch_bounds__(256) read_kernel(StoreArgs a) {
  constexpr bool kFp8 = FMT == PS_KV_FP8;
  constexpr int kN = kFp8 ? 16 : 8;
  constexpr int kLanes = D / kN;
  constexpr int kRec = record_bytes(D, FMT), kHalf = half_bytes(D, FMT);
  const uint32_t items = (uint32_t)a.n * a.kv_heads;
  const uint32_t c = threadIdx.x % kLanes;
  const uint32_t step = gridDim.x * (256 / kLanes);
  for (uint32_t it = blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes; it < items; it += step) {
    const uint32_t t = it / a.kv_heads;
    const uint32_t h = it - t * a.kv_heads;
    const int64_t slot = a.slots[t];
    bool ok = slot >= 0;
    if (ok && (uint64_t)slot >= a.num_slots) {
      ok = false;
      atomicOr_system(a.err, kErrSlot);
    }
    uint4 ck = make_uint4(0, 0, 0, 0), cv = ck;
    uint32_t ek = kExpBias, ev = kExpBias;
    if (ok) {
      const uint8_t* rec = a.pool + ((uint64_t)slot / kBlock * a.kv_heads + h) * kRec;
      const uint32_t tok = (uint32_t)((uint64_t)slot % kBlock);
      ck = *reinterpret_cast<const uint4*>(rec + (kFp8 ? offset8k<D>(tok, c) : offset16(tok, c)));
      cv = *reinterpret_cast<const uint4*>(rec + kHalf + (kFp8 ? offset8v(tok, c) : offset16(tok, c)));
      if (kFp8) {
        ek = rec[2 * kHalf + exp_place(tok)];
        ev = rec[2 * kHalf + kBlock + exp_place(tok)];
      }
    }
    const int64_t ko = (int64_t)t * a.k_tok + (int64_t)h * a.k_head + c * kN;
    const int64_t vo = (int64_t)t * a.v_tok + (int64_t)h * a.v_head + c * kN;
    Row<TYPE, kN> o;
    float x[kN];
    if constexpr (kFp8) {
      decode(ck, ek, x);
      o.set(x);
      o.store(a.k, ko);
      decode(cv, ev, x);
      o.set(x);
      o.store(a.v, vo);
    } else {
      Row<FMT, 8> in;
      in.w[0] = ck;
      in.floats(x);
      o.set(x);
      o.store(a.k, ko);
      in.w[0] = cv;
      in.floats(x);
      o.set(x);
      o.store(a.v, vo);
    }
  }
}

template <bool WRITE, int D, int FMT, int TYPE>
cudaError_t go(StoreArgs a, int sms, cudaStream_t s) {
  constexpr uint64_t per = 256 / (D / (FMT == PS_KV_FP8 ? 16 : 8));
  // the last round's index stays below 2^32: a grid's rows are at most sms * 32 * per
  const uint64_t most = 0x7FFFFFFFull / a.kv_heads;  // tokens of one launch
  for (uint64_t left = a.n; left > 0;) {
    a.n = left < most ? left : most;
    const uint64_t need = (a.n * a.kv_heads + per - 1) / per;
    const unsigned grid = (unsigned)(need < (uint64_t)sms * 32 ? need : (uint64_t)sms * 32);
    if (WRITE)
      write_kernel<D, FMT, TYPE><<<grid, 256, 0, s>>>(a);
    else
      read_kernel<D, FMT, TYPE><<<grid, 256, 0, s>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    left -= a.n;
    a.slots += a.n;
    a.k = static_cast<uint8_t*>(a.k) + (int64_t)a.n * a.k_tok * Elem<TYPE>::kSize;
    a.v = static_cast<uint8_t*>(a.v) + (int64_t)a.n * a.v_tok * Elem<TYPE>::kSize;
  }
  return cudaSuccess;
}

template <bool WRITE, int D, int FMT>
cudaError_t by_type(int type, const StoreArgs& a, int sms, cudaStream_t s) {
  switch (type) {
    case PS_KV_BF16: return go<WRITE, D, FMT, PS_KV_BF16>(a, sms, s);
    case PS_KV_FP16: return go<WRITE, D, FMT, PS_KV_FP16>(a, sms, s);
    case PS_KV_FP32: return go<WRITE, D, FMT, PS_KV_FP32>(a, sms, s);
  }
  return cudaErrorInvalidValue;
}

template <bool WRITE, int D>
cudaError_t by_format(int fmt, int type, const StoreArgs& a, int sms, cudaStream_t s) {
  switch (fmt) {
    case PS_KV_BF16: return by_type<WRITE, D, PS_KV_BF16>(type, a, sms, s);
    case PS_KV_FP16: return by_type<WRITE, D, PS_KV_FP16>(type, a, sms, s);
    case PS_KV_FP8: return by_type<WRITE, D, PS_KV_FP8>(type, a, sms, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_write(int D, int fmt, int type, const StoreArgs& a, int sms, cudaStream_t s) {
  return D == 128 ? by_format<true, 128>(fmt, type, a, sms, s) : by_format<true, 64>(fmt, type, a, sms, s);
}
cudaError_t launch_read(int D, int fmt, int type, const StoreArgs& a, int sms, cudaStream_t s) {
  return D == 128 ? by_format<false, 128>(fmt, type, a, sms, s) : by_format<false, 64>(fmt, type, a, sms, s);
}

}  // namespace pskv
