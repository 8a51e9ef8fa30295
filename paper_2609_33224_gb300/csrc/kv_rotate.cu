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

// A warp takes a token and a share of its rows (queries' heads, then keys' heads), D / 16 lanes a row.  Its lanes first
// work out the token's cosines and sines, a pair of elements each, which every row then uses: the angle is
// position * (turns per position), as 64-bit fractions of a turn, so the integer product wraps at whole turns and no
// position is too far; its upper 32 bits, less the nearest quarter turn, go to sincospif.  A lane has two groups of 8
// elements that its pairs lie in: half a rotated part apart, or next to each other.
// Bound by bytes: reads q, k and v and writes the rotated queries and the cache's rows, each once.  65536 tokens of 64 and
// 8 heads, 128 columns, bf16 to fp8, 2.55 GB: 405 us = 6.3 TB/s, 93% of the measured copy.  The next row loaded ahead,
// three or two blocks an SM (402 to 486 us) or streaming stores (409) gave no more.
template <int D, int FMT, int TYPE>
__global__ void __launch_bounds__(256, TYPE == PS_KV_FP32 ? 3 : 4) rotate_kernel(const __grid_constant__ RotateArgs a) {
  constexpr bool kFp8 = FMT == PS_KV_FP8;
  constexpr int kOut = FMT == PS_KV_FP16 ? PS_KV_FP16 : PS_KV_BF16;
  constexpr uint32_t kLanes = D / 16, kRows = 32 / kLanes;
  constexpr int kRec = record_bytes(D, FMT), kHalf = half_bytes(D, FMT);
  __shared__ __align__(16) float2 turns[8][64];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t c = lane % kLanes, rl = lane / kLanes;
  const bool rotated = 16 * c < a.dims, halves = rotated && !a.interleaved;
  const uint32_t e0 = halves ? 8 * c : 16 * c, e1 = halves ? a.dims / 2 + 8 * c : 16 * c + 8;
  const uint32_t q_rounds = (a.q_heads + kRows - 1) / kRows, rounds = q_rounds + (a.s.kv_heads + kRows - 1) / kRows;

  auto rotate = [&](float (&x)[16], const float2 (&cs)[8]) {
    if (!rotated) return;
    if (a.interleaved) {
#pragma unroll
      for (int i = 0; i < 8; ++i) turn(x[2 * i], x[2 * i + 1], cs[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) turn(x[i], x[8 + i], cs[i]);
    }
  };

  const uint64_t items = a.s.n * a.shares;
  for (uint64_t it = (uint64_t)blockIdx.x * 8 + warp; it < items; it += (uint64_t)gridDim.x * 8) {
    const uint64_t t = it / a.shares;
    const uint32_t share = (uint32_t)(it - t * a.shares);
    const uint32_t from = rounds * share / a.shares, to = rounds * (share + 1) / a.shares;
    const uint64_t p = (uint64_t)a.positions[t];
    __syncwarp();
    for (uint32_t i = lane; i < a.dims / 2; i += 32) {
      const uint32_t part = (uint32_t)((p * a.turns[i]) >> 32);  // of a turn, in 2^-32
      // to within an eighth of a turn of a quarter: what is left has as many bits as a float keeps
      const uint32_t quarter = (part + (1u << 29)) >> 30;
      float s, co;
      sincospif((float)(int32_t)(part - (quarter << 30)) * 0x1p-31f, &s, &co);
      if (quarter & 1u) {
        const float x = co;
        co = -s;
        s = x;
      }
      const float m = quarter & 2u ? -a.magnitude : a.magnitude;
      turns[warp][i] = make_float2(co * m, s * m);
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
    if (to <= q_rounds) continue;
    const int64_t slot = a.s.slots[t];
    bool ok = slot >= 0;
    if (ok && (uint64_t)slot >= a.s.num_slots) {
      ok = false;
      if (lane == 0) atomicOr_system(a.s.err, kErrSlot);
    }
    if (!ok) continue;  // the same for the whole warp
    const uint32_t tok = (uint32_t)((uint64_t)slot % kBlock);
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
        const uint4 ck = quantise<D>(x, &ek);
        const uint4 cv = quantise<D>(y, &ev);
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
