// Joining the partial results of a query's rows: those of the spans that cover it and of the pieces that a
// span's keys were cut into.
#include "kv_internal.cuh"

namespace pskv {
namespace {

// One (query, q head) row per warp, or with kWide per CTA of 8 warps, which share its parts.  A part is read
// once: its maximum and sum (all lanes the same two floats), and its D values, D / 32 per lane.
// out = sum_k 2^(m_k - M) acc_k / sum_k 2^(m_k - M) l_k with the running maximum M, in 32 bits.
// Bound by the bytes of the parts (D * 4 + 8 each), which the attention kernels left in L2.
template <int D, bool FP16, bool kWide>
__global__ void __launch_bounds__(256) join_kernel(const AttnArgs a, const PlanDev p) {
  constexpr int kV = D / 32;
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t row = kWide ? blockIdx.x : blockIdx.x * 8 + warp;
  const uint32_t rows = p.njoin * a.group;
  if (row >= rows) return;  // kWide: the whole CTA
  const uint32_t entry = p.join[row / a.group], gi = row % a.group;
  const uint32_t query = entry / a.kv_heads, kvh = entry % a.kv_heads;
  const uint32_t head = kvh * a.group + gi;

  float m = -INFINITY, l = 0.0f, acc[kV];
#pragma unroll
  for (int i = 0; i < kV; ++i) acc[i] = 0.0f;
  bool done = false;
  for (uint32_t x = p.tok_off[query]; x < p.tok_off[query + 1]; ++x) {
    const Layer ly = p.layers[p.tok_layer[x]];
    const uint32_t r = (query - ly.query0) * a.group + gi;
    const Group gr = p.groups[ly.group0 + r / ly.tile_rows * a.kv_heads + kvh];
    if (gr.part_row == kDirect) {
      done = true;  // written by the attention kernel
      break;
    }
    const uint32_t base = gr.part_row + r % ly.tile_rows;
#pragma unroll 4
    for (uint32_t k = kWide ? warp : 0; k < gr.nparts; k += kWide ? 8 : 1) {
      const uint64_t at = base + (uint64_t)k * ly.tile_rows;
      const float2 ml = a.part_ml[at];
      float v[kV];
      const float* src = a.part + at * D + lane * kV;
      if (kV == 4) {
        const float4 w = *reinterpret_cast<const float4*>(src);
        v[0] = w.x; v[1] = w.y; v[kV - 2] = w.z; v[kV - 1] = w.w;
      } else {
        const float2 w = *reinterpret_cast<const float2*>(src);
        v[0] = w.x; v[1] = w.y;
      }
      const float n = fmaxf(m, ml.x);
      const float f0 = m == n ? 1.0f : ex2(m - n), f1 = ml.x == n ? 1.0f : ex2(ml.x - n);
      m = n;
      l = l * f0 + ml.y * f1;
#pragma unroll
      for (int i = 0; i < kV; ++i) acc[i] = acc[i] * f0 + v[i] * f1;
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
    if (done || warp != 0) return;
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
  if (done) return;
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
    join_kernel<D, FP16, true><<<rows, 256, 0, s>>>(a, p);
  else
    join_kernel<D, FP16, false><<<(rows + 7) / 8, 256, 0, s>>>(a, p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_join(int D, bool fp16, const AttnArgs& a, const PlanDev& p, cudaStream_t s) {
  if (D == 128) return fp16 ? go<128, true>(a, p, s) : go<128, false>(a, p, s);
  return fp16 ? go<64, true>(a, p, s) : go<64, false>(a, p, s);
}

}  // namespace pskv
