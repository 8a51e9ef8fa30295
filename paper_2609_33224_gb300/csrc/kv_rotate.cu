// Rotary positions: queries rotated, keys rotated and written into the block cache with their values.
#include "kv_elem.cuh"

namespace pskv {
namespace {

// A lane's 16 elements of a row, as two groups of 8.
template <int TYPE>
struct Pair {
  Row<TYPE, 8> lo, hi;
  __device__ __forceinline__ void load(const void* base, int64_t at, uint32_t e0, uint32_t e1) {
    lo.load(base, at + e0);
    hi.load(base, at + e1);
  }
  __device__ __forceinline__ void floats(float (&x)[16]) const {
    float a[8], b[8];
    lo.floats(a);
    hi.floats(b);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = a[i];
      x[8 + i] = b[i];
    }
  }
};

__device__ __forceinline__ void turn(float& a, float& b, float2 cs) {
  const float x = a, y = b;
  a = x * cs.x - y * cs.y;
  b = y * cs.x + x * cs.y;
}

// Cosine and sine (x, y) of `part` 2^-64 turns and what they lack of the exact values (z, w), to 2^-28: the angle
// less its nearest quarter turn, at most pi / 4, as a sum of two floats, its square and cube as such sums too, in the
// functions' power series (up to the 10th and 11th power: the next terms are below 2^-33 and 2^-37).
__device__ __forceinline__ float4 turn_of(uint64_t part) {
  const uint64_t quarter = (part + (1ull << 61)) >> 62;
  const uint64_t r = part - (quarter << 62);  // in 2^-64 turns, signed
  const int32_t hi = (int32_t)(r >> 32);
  const float rh = (float)hi, x = rh * 0x1p-31f;  // in half turns
  const float xl = ((float)(hi - (int32_t)rh) + (float)(uint32_t)r * 0x1p-32f) * 0x1p-31f;
  constexpr float kPi = 3.14159274f, kPiLow = -8.74227766e-8f, kSixth = 0.16666667f, kSixthLow = -4.96705e-9f;
  const float t = __fmul_rn(x, kPi), tl = __fmaf_rn(x, kPi, -t) + (x * kPiLow + xl * kPi);
  const float u = __fmul_rn(t, t), ul = __fmaf_rn(t, t, -u) + 2.0f * t * tl;
  const float cu = __fmul_rn(u, t), cl = __fmaf_rn(u, t, -cu) + (ul * t + u * tl);
  const float w = __fmul_rn(cu, kSixth), wl = __fmaf_rn(cu, kSixth, -w) + (cu * kSixthLow + cl * kSixth);
  const float c0 = __fadd_rn(1.0f, -0.5f * u), s0 = __fadd_rn(t, -w);
  const float c1 = __fadd_rn(__fadd_rn(1.0f, -c0), -0.5f * u) + ul * (u * (1.0f / 12) - 0.5f) +
                   u * u * (1.0f / 24 + u * (-1.0f / 720 + u * (1.0f / 40320 - u * (1.0f / 3628800))));
  const float s1 = __fadd_rn(__fadd_rn(t, -s0), -w) + (tl - wl) +
                   cu * u * (1.0f / 120 + u * (-1.0f / 5040 + u * (1.0f / 362880 - u * (1.0f / 39916800))));
  const float c = __fadd_rn(c0, c1), s = __fadd_rn(s0, s1);
  float4 y = make_float4(c, s, c1 - __fadd_rn(c, -c0), s1 - __fadd_rn(s, -s0));
  if (quarter & 1u) y = make_float4(-y.y, y.x, -y.w, y.z);
  if (quarter & 2u) y = make_float4(-y.x, -y.y, -y.z, -y.w);
  return y;
}

__device__ __forceinline__ uint64_t floats(float lo, float hi) { return pair(__float_as_uint(lo), __float_as_uint(hi)); }
// Rounds y + rest, y being the nearest float, to odd: a sum that is no float has its last bit set, so that what it is
// rounded to after that, to fewer bits, is its own rounding.
__device__ __forceinline__ float to_odd(float y, float rest) {
  uint32_t bits = __float_as_uint(y);
  const uint32_t some = fabsf(rest) > 0.0f && fabsf(y) > 0.0f;
  bits -= ((bits ^ __float_as_uint(rest)) >> 31) & some;  // towards zero
  return __uint_as_float(bits | some);
}
// (a c - b s, b c + a s), with the parts that c and s lack, rounded to odd.  Two floats an instruction: the products and
// their sum (a, b) c + (-b, a) s, what they lack, and the sum of it all.
__device__ __forceinline__ void turn_exactly(float& a, float& b, float2 cs, float2 rest) {
  const uint64_t x = floats(a, b), y = floats(-b, a), c = floats(cs.x, cs.x), s = floats(cs.y, cs.y), none = floats(-1.0f, -1.0f);
  const uint64_t p = mul2(x, c), q = mul2(y, s), r = add2(p, q);
  const uint64_t v = fma2(p, none, r);                                         // r - p
  const uint64_t lost = add2(fma2(fma2(v, none, r), none, p), fma2(v, none, q));  // (p - (r - v)) + (q - v)
  const uint64_t of_products = add2(fma2(x, c, mul2(p, none)), fma2(y, s, mul2(q, none)));
  const uint64_t of_turn = fma2(x, floats(rest.x, rest.x), mul2(y, floats(rest.y, rest.y)));
  const uint64_t low = add2(add2(lost, of_products), of_turn), z = add2(r, low);
  const uint64_t left = fma2(fma2(r, none, z), none, low);  // low - (z - r)
  float r0, r1, z0, z1, l0, l1;
  unpair(r, r0, r1);
  unpair(z, z0, z1);
  unpair(left, l0, l1);
  a = fabsf(r0) < INFINITY ? to_odd(z0, l0) : r0;
  b = fabsf(r1) < INFINITY ? to_odd(z1, l1) : r1;
}

template <class F>
__device__ __forceinline__ void each_pair(float (&x)[16], bool interleaved, F f) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f(x[2 * i], x[2 * i + 1], i);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f(x[i], x[8 + i], i);
  }
}

// The keys of rounds from .. to - 1 of token t once more, fp8: rows whose maximum, turned in 32 bits, is close to a border
// of the scales are turned to 2^-28 and stored again.
template <int D, int TYPE>
__device__ __noinline__ void store_exactly(const RotateArgs& a, uint64_t t, uint64_t slot, uint32_t from, uint32_t to,
                                           uint32_t e0, uint32_t e1, const float2* turns, const float2* rests) {
  constexpr int kRec = record_bytes(D, PS_KV_FP8), kHalf = half_bytes(D, PS_KV_FP8);
  constexpr uint32_t kLanes = D / 16, kRows = 32 / kLanes;
  const uint32_t lane = threadIdx.x % 32, c = lane % kLanes, tok = (uint32_t)(slot % kBlock);
  for (uint32_t r = from; r < to; ++r) {
    const uint32_t h = r * kRows + lane / kLanes;
    const bool live = h < a.s.kv_heads;
    Pair<TYPE> in;
    in.load(a.s.k, (int64_t)t * a.s.k_tok + (int64_t)(live ? h : 0) * a.s.k_head, e0, e1);
    float x[16];
    in.floats(x);
    if (16 * c < a.dims)
      each_pair(x, a.interleaved, [&](float& u, float& w, int i) { turn(u, w, turns[8 * c + i]); });
    uint32_t e;
    bool close;
    quantise<D>(x, &e, &close);
    in.floats(x);
    if (16 * c < a.dims)
      each_pair(x, a.interleaved,
                [&](float& u, float& w, int i) { turn_exactly(u, w, turns[8 * c + i], rests[8 * c + i]); });
    const uint4 code = quantise<D>(x, &e);
    if (!live || !close) continue;
    uint8_t* rec = a.s.pool + (slot / kBlock * a.s.kv_heads + h) * kRec;
    *reinterpret_cast<uint2*>(rec + offset8k<D>(tok, e0 / 16) + e0 % 16) = make_uint2(code.x, code.y);
    *reinterpret_cast<uint2*>(rec + offset8k<D>(tok, e1 / 16) + e1 % 16) = make_uint2(code.z, code.w);
    if (c == 0) rec[2 * kHalf + exp_place(tok)] = (uint8_t)e;
  }
}

// A warp takes a token and a share of its rows (queries' heads, then keys' heads), D / 16 lanes a row.  Its lanes first
// work out the token's cosines and sines, a pair of elements each, which every row then uses: the angle is
// position * (turns per position), as 64-bit fractions of a turn, so the integer product wraps at whole turns and no
// position is too far.  A lane has two groups of 8 elements that its pairs lie in: half a rotated part apart, or next to
// each other.
// All of it is in 32 bits, with one exception: in an 8-bit cache a difference of 2^-24 in the largest element may take a
// whole row to another scale, so rows whose maximum is that near to a border (one in 10^5) are turned again, to 2^-28.
// Bound by bytes: reads q, k and v and writes the rotated queries and the cache's rows, each once.  65536 tokens of 64 and
// 8 heads, 128 columns, bf16 to fp8, 2.55 GB: 421 us = 6.1 TB/s, 89% of the measured copy; all keys turned to 2^-28 took
// 456, none 410.  Four blocks an SM, whose 64 registers a thread spill 44 to 92 bytes, hide more latency than three (437)
// or two (509).  The next row loaded ahead or streaming stores gave nothing.
template <int D, int FMT, int TYPE>
__global__ void __launch_bounds__(256, TYPE == PS_KV_FP32 ? 3 : 4) rotate_kernel(const __grid_constant__ RotateArgs a) {
  constexpr bool kFp8 = FMT == PS_KV_FP8;
  constexpr int kOut = FMT == PS_KV_FP16 ? PS_KV_FP16 : PS_KV_BF16;
  constexpr uint32_t kLanes = D / 16, kRows = 32 / kLanes;
  constexpr int kRec = record_bytes(D, FMT), kHalf = half_bytes(D, FMT);
  __shared__ __align__(16) float2 turns[8][64], rests[8][64];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t c = lane % kLanes, rl = lane / kLanes;
  const bool rotated = 16 * c < a.dims, halves = rotated && !a.interleaved;
  const uint32_t e0 = halves ? 8 * c : 16 * c, e1 = halves ? a.dims / 2 + 8 * c : 16 * c + 8;
  const uint32_t q_rounds = (a.q_heads + kRows - 1) / kRows, rounds = q_rounds + (a.s.kv_heads + kRows - 1) / kRows;

  auto rotate = [&](float (&x)[16], const float2 (&cs)[8]) {
    if (rotated) each_pair(x, a.interleaved, [&](float& u, float& w, int i) { turn(u, w, cs[i]); });
  };

  const uint64_t items = a.s.n * a.shares;
  for (uint64_t it = (uint64_t)blockIdx.x * 8 + warp; it < items; it += (uint64_t)gridDim.x * 8) {
    const uint64_t t = it / a.shares;
    const uint32_t share = (uint32_t)(it - t * a.shares);
    const uint32_t from = rounds * share / a.shares, to = rounds * (share + 1) / a.shares;
    const uint64_t p = (uint64_t)a.positions[t];
    const int64_t slot = to > q_rounds ? a.s.slots[t] : -1;
    __syncwarp();
    for (uint32_t i = lane; i < a.dims / 2; i += 32) {
      const float4 y = turn_of(p * a.turns[i]);
      const float m = a.magnitude, co = __fmul_rn(y.x, m), si = __fmul_rn(y.y, m);
      turns[warp][i] = make_float2(co, si);
      rests[warp][i] = make_float2(__fmaf_rn(y.x, m, -co) + y.z * m, __fmaf_rn(y.y, m, -si) + y.w * m);
    }
    __syncwarp();
    float2 cs[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = turns[warp][rotated ? 8 * c + i : i];

    for (uint32_t r = from; r < min(to, q_rounds); ++r) {
      const uint32_t h = r * kRows + rl;
      if (h >= a.q_heads) continue;
      Pair<TYPE> in;
      in.load(a.q, (int64_t)t * a.q_tok + (int64_t)h * a.q_head, e0, e1);
      float x[16];
      in.floats(x);
      rotate(x, cs);
      Row<kOut, 8> o;
      float y[8];
      const int64_t at = (int64_t)t * a.o_tok + (int64_t)h * a.o_head;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[8 * g + i];
        o.set(y);
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.q_out) + at + (g ? e1 : e0)) = o.w[0];
      }
    }
    bool ok = slot >= 0;
    if (ok && (uint64_t)slot >= a.s.num_slots) {
      ok = false;
      if (lane == 0) atomicOr_system(a.s.err, kErrSlot);
    }
    if (!ok) continue;  // the same for the whole warp
    const uint32_t tok = (uint32_t)((uint64_t)slot % kBlock);
    bool again = false;
    for (uint32_t r = max(from, q_rounds); r < to; ++r) {
      const uint32_t h = (r - q_rounds) * kRows + rl;
      const bool live = h < a.s.kv_heads;
      Pair<TYPE> k, v;
      const int64_t row = live ? h : 0;
      k.load(a.s.k, (int64_t)t * a.s.k_tok + row * a.s.k_head, e0, e1);
      v.load(a.s.v, (int64_t)t * a.s.v_tok + row * a.s.v_head, 16 * c, 16 * c + 8);
      float x[16], y[16];
      k.floats(x);
      v.floats(y);
      rotate(x, cs);
      uint8_t* rec = a.s.pool + ((uint64_t)slot / kBlock * a.s.kv_heads + row) * kRec;
      if constexpr (kFp8) {
        uint32_t ek, ev;
        bool close;
        const uint4 ck = quantise<D>(x, &ek, &close);
        const uint4 cv = quantise<D>(y, &ev);
        again |= close;
        if (live) {
          *reinterpret_cast<uint2*>(rec + offset8k<D>(tok, e0 / 16) + e0 % 16) = make_uint2(ck.x, ck.y);
          *reinterpret_cast<uint2*>(rec + offset8k<D>(tok, e1 / 16) + e1 % 16) = make_uint2(ck.z, ck.w);
          *reinterpret_cast<uint4*>(rec + kHalf + offset8v(tok, c)) = cv;
          if (c == 0) {
            rec[2 * kHalf + exp_place(tok)] = (uint8_t)ek;
            rec[2 * kHalf + kBlock + exp_place(tok)] = (uint8_t)ev;
          }
        }
      } else if (live) {
        Row<FMT, 8> o;
        float z[8];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = x[8 * g + i];
          o.set(z);
          *reinterpret_cast<uint4*>(rec + offset16(tok, (g ? e1 : e0) / 8)) = o.w[0];
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = y[8 * g + i];
          o.set(z);
          *reinterpret_cast<uint4*>(rec + kHalf + offset16(tok, 2 * c + g)) = o.w[0];
        }
      }
    }
    if (kFp8 && __any_sync(0xFFFFFFFFu, again))
      store_exactly<D, TYPE>(a, t, (uint64_t)slot, max(from, q_rounds) - q_rounds, to - q_rounds, e0, e1, turns[warp],
                             rests[warp]);
  }
}

template <int D, int FMT, int TYPE>
cudaError_t go(RotateArgs a, int sms, cudaStream_t s) {
  constexpr uint32_t kRows = 512 / D;
  // Few tokens: their rows go to several warps each, which all work out the token's angles.
  const uint32_t rounds = (a.q_heads + kRows - 1) / kRows + (a.s.kv_heads + kRows - 1) / kRows;
  const uint64_t warps = (uint64_t)sms * 32;
  a.shares = (uint32_t)(a.s.n >= warps ? 1 : warps / a.s.n < rounds ? warps / a.s.n : rounds);
  const uint64_t need = (a.s.n * a.shares + 7) / 8, most = (uint64_t)sms * 32;
  rotate_kernel<D, FMT, TYPE><<<(unsigned)(need < most ? need : most), 256, 0, s>>>(a);
  return cudaGetLastError();
}

template <int D, int FMT>
cudaError_t by_type(int type, const RotateArgs& a, int sms, cudaStream_t s) {
  switch (type) {
    case PS_KV_BF16: return go<D, FMT, PS_KV_BF16>(a, sms, s);
    case PS_KV_FP16: return go<D, FMT, PS_KV_FP16>(a, sms, s);
    case PS_KV_FP32: return go<D, FMT, PS_KV_FP32>(a, sms, s);
  }
  return cudaErrorInvalidValue;
}

template <int D>
cudaError_t by_format(int fmt, int type, const RotateArgs& a, int sms, cudaStream_t s) {
  switch (fmt) {
    case PS_KV_BF16: return by_type<D, PS_KV_BF16>(type, a, sms, s);
    case PS_KV_FP16: return by_type<D, PS_KV_FP16>(type, a, sms, s);
    case PS_KV_FP8: return by_type<D, PS_KV_FP8>(type, a, sms, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_write_rotated(int D, int fmt, int type, const RotateArgs& a, int sms, cudaStream_t s) {
  return D == 128 ? by_format<128>(fmt, type, a, sms, s) : by_format<64>(fmt, type, a, sms, s);
}

}  // namespace pskv
