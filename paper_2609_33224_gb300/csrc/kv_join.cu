// Joining the partial results of a query's rows: those of the spans that cover it and of the pieces that a
// span's keys were cut into.
#include "kv_internal.cuh"

namespace pskv {
namespace {

// One (query, q head) row per warp, or with kWide per CTA of 8 warps, which share its parts.  Up to 32 parts at
// a time: each lane takes one part's maximum m_k and sum l_k, then all lanes add the parts' D values, D / 32 a
// lane, with the weights 2^(m_k - M): the loads of the values do not wait for one another.
// out = sum_k 2^(m_k - M) acc_k / sum_k 2^(m_k - M) l_k with the running maximum M, in 32 bits.
// Bound by the bytes of the parts (D * 4 + 8 each), which the attention kernels left in L2.
template <int D, bool FP16, bool kWide>
__global__ void __launch_bounds__(256) join_kernel(const AttnArgs a, const PlanDev p) {
  constexpr int kV = D / 32;
  constexpr uint32_t kStep = kWide ? 8 : 1;
  wait_for_last();
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t row = kWide ? blockIdx.x : blockIdx.x * 8 + warp;
  if (row >= p.njoin * a.group) return;  // kWide: the whole CTA
  const JoinEntry en = p.join[row / a.group];
  const uint32_t gi = row % a.group;
  if (gi >= en.count) return;  // the same
  const uint32_t query = en.query, head = en.head0 + gi;

  float m = -INFINITY, l = 0.0f, acc[kV];
#pragma unroll
  for (int i = 0; i < kV; ++i) acc[i] = 0.0f;
  for (uint32_t x = 0; x < en.nsegs; ++x) {
    const JoinSeg sg = p.segs[en.seg0 + x];
    const uint64_t at0 = (uint64_t)sg.row + gi, stride = (uint64_t)sg.stride * kStep;
    const uint64_t base = at0 + (kWide ? (uint64_t)warp * sg.stride : 0);
    const uint32_t n = kWide ? (sg.nparts + 7 - warp) / 8 : sg.nparts;  // this warp's parts
    for (uint32_t c = 0; c < n; c += 32) {
      const uint32_t cnt = min(32u, n - c);
      float2 ml = make_float2(-INFINITY, 0.0f);
      if (lane < cnt) ml = a.part_ml[base + (uint64_t)(c + lane) * stride];
      float mm = ml.x;
      for (uint32_t o = 16; o; o >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xFFFFFFFFu, mm, o));
      mm = fmaxf(mm, m);
      const float f = m == mm ? 1.0f : ex2(m - mm);
      m = mm;
      float w = lane < cnt ? (ml.x == mm ? 1.0f : ex2(ml.x - mm)) : 0.0f;
      float wl = w * ml.y;
      for (uint32_t o = 16; o; o >>= 1) wl += __shfl_xor_sync(0xFFFFFFFFu, wl, o);
      l = l * f + wl;
#pragma unroll
      for (int i = 0; i < kV; ++i) acc[i] *= f;
#pragma unroll 4
      for (uint32_t k = 0; k < cnt; ++k) {
        const float* src = a.part + (base + (uint64_t)(c + k) * stride) * D + lane * kV;
        float v[kV];
        if (kV == 4) {
          const float4 y = *reinterpret_cast<const float4*>(src);
          v[0] = y.x; v[1] = y.y; v[kV - 2] = y.z; v[kV - 1] = y.w;
        } else {
          const float2 y = *reinterpret_cast<const float2*>(src);
          v[0] = y.x; v[1] = y.y;
        }
        const float wk = __shfl_sync(0xFFFFFFFFu, w, k);
#pragma unroll
        for (int i = 0; i < kV; ++i) acc[i] = fmaf(v[i], wk, acc[i]);
      }
    }
  }
  if (kWide) {
    __shared__ float sm[8], sl[8], sacc[8][D];
    if (lane == 0) {
      sm[warp] = m;
      sl[warp] = l;
    }
#pragma unroll
    for (int i = 0; i < kV; ++i) sacc[warp][lane * kV + i] = acc[i];
    __syncthreads();
    if (warp != 0) return;
    float n = -INFINITY;
#pragma unroll
    for (int w = 0; w < 8; ++w) n = fmaxf(n, sm[w]);
    l = 0.0f;
#pragma unroll
    for (int i = 0; i < kV; ++i) acc[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const float f = sm[w] == n ? 1.0f : ex2(sm[w] - n);
      l += sl[w] * f;
#pragma unroll
      for (int i = 0; i < kV; ++i) acc[i] += sacc[w][lane * kV + i] * f;
    }
    m = n;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // no key: zeros (a NaN stays one)
  uint16_t* o = a.out + (int64_t)query * a.o_tok + (int64_t)head * a.o_head + lane * kV;
  uint32_t w[kV / 2];
#pragma unroll
  for (int i = 0; i < kV; i += 2) w[i / 2] = pack2<FP16>(acc[i] * inv, acc[i + 1] * inv);
  if (kV == 4)
    *reinterpret_cast<uint2*>(o) = make_uint2(w[0], w[kV / 2 - 1]);
  else
    *reinterpret_cast<uint32_t*>(o) = w[0];
  if (a.lse && lane == 0)
    a.lse[(uint64_t)query * a.kv_heads * a.group + head] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
}

template <int D, bool FP16>
cudaError_t go(const AttnArgs& a, const PlanDev& p, cudaStream_t s) {
  const uint32_t rows = p.njoin * a.group;
  // Few rows of many parts (one request on all SMs): a CTA a row.
  if (p.max_parts > 16)
    return launch(join_kernel<D, FP16, true>, rows, 256, 0, 1, true, s, a, p);
  return launch(join_kernel<D, FP16, false>, (rows + 7) / 8, 256, 0, 1, true, s, a, p);
}

}  // namespace

cudaError_t launch_join(int D, bool fp16, const AttnArgs& a, const PlanDev& p, cudaStream_t s) {
  if (D == 128) return fp16 ? go<128, true>(a, p, s) : go<128, false>(a, p, s);
  return fp16 ? go<64, true>(a, p, s) : go<64, false>(a, p, s);
}

}  // namespace pskv
