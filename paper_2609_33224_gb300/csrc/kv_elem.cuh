// Rows of the caller's tensors as 16-byte loads and stores, and their rounding to a cache row's fp8 codes: shared by the
// kernels that write and read the cache.
#pragma once

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

// One row's 16 elements per lane (D / 16 lanes a row): the row's scale exponent, and this lane's codes; at_border: whether
// the row's maximum is within 2^-19 of where the exponent changes.
template <int D>
__device__ __forceinline__ uint4 quantise(const float (&x)[16], uint32_t* exp_code, bool* at_border = nullptr) {
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
  if (at_border) *at_border = (b & 0x7FFFFFu) - (0x600000u - 16) <= 32;
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

}  // namespace
}  // namespace pskv
