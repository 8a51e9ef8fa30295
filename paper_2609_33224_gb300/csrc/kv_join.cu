// Joining the partial results of a query's rows: those of the spans that cover it and of the pieces that a
// span's keys were cut into.
#include <type_traits>

#include "kv_internal.cuh"

namespace pskv {
namespace {

// One (query, q head) row per warp, or with kWide per CTA of 8 warps, which share its parts.  Up to 32 parts at
// a time: each lane finds one part and takes its maximum m_k and sum l_k, then all lanes add the parts' D
// values, D / 32 a lane, with the weights 2^(m_k - M).  The loads of the first four parts' values wait for
// nothing but the parts' places: few rows are bound by the chain of dependent loads.
// out = sum_k 2^(m_k - M) acc_k / sum_k 2^(m_k - M) l_k with the running maximum M, in 32 bits.
// Bound by the bytes of the parts (D * 4 + 8 each), which the attention kernels left in L2, or, for few rows, by four
// dependent loads: 4096 rows of 8 parts (17 MB) take 8 us, 64 rows of 128 parts 5.
template <int D, bool FP16, bool kWide>
__global__ void __launch_bounds__(256, 4) join_kernel(const AttnArgs a, const PlanDev p) {
  constexpr int kV = D / 32, kAhead = 4;
  constexpr uint32_t kStep = kWide ? 8 : 1, kFull = 0xFFFFFFFFu;
  using Vec = typename std::conditional<kV == 4, float4, float2>::type;
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t row = kWide ? blockIdx.x : blockIdx.x * 8 + warp;
  // What there is to join is the plan's; the parts are the kernels' before this one.
  const bool live = row < p.njoin * p.join_stride;  // < 2^32; kWide: the same for the whole CTA
  const JoinEntry en = live ? p.join[row / p.join_stride] : JoinEntry{};
  const uint32_t gi = row % p.join_stride;
  JoinSeg ahead_seg{0, 0, 0};
  if (lane < min(32u, en.nsegs)) ahead_seg = p.segs[en.seg0 + lane];
  let_next_start();  // the next call's first kernel, which waits for this one
  wait_for_last();
  if (!live || gi >= en.count) return;
  const uint32_t query = en.query, head = en.head0 + gi;

  const float* part = a.part + lane * kV;
  float m = -INFINITY, l = 0.0f, acc[kV];
#pragma unroll
  for (int i = 0; i < kV; ++i) acc[i] = 0.0f;
  auto add = [&](const Vec& v, float w) {
    acc[0] = fmaf(v.x, w, acc[0]);
    acc[1] = fmaf(v.y, w, acc[1]);
    if constexpr (kV == 4) {
      acc[2] = fmaf(v.z, w, acc[2]);
      acc[3] = fmaf(v.w, w, acc[3]);
    }
  };
  for (uint32_t s0 = 0; s0 < en.nsegs; s0 += 32) {
    const uint32_t ns = min(32u, en.nsegs - s0);
    JoinSeg sg = ahead_seg;
    if (s0 > 0) sg = lane < ns ? p.segs[en.seg0 + s0 + lane] : JoinSeg{0, 0, 0};
    const uint32_t total = __reduce_add_sync(kFull, sg.nparts);
    for (uint32_t c = kWide ? warp : 0; c < total; c += 32 * kStep) {
      const uint32_t mine = c + lane * kStep;
      const uint32_t cnt = min(32u, (total - c + kStep - 1) / kStep);
      uint32_t at = 0;
      for (uint32_t s = 0, start = 0; s < ns; ++s) {
        const uint32_t np = __shfl_sync(kFull, sg.nparts, s), r0 = __shfl_sync(kFull, sg.row, s);
        const uint32_t st = __shfl_sync(kFull, sg.stride, s);
        if (mine >= start && mine - start < np) at = r0 + gi + (mine - start) * st;
        start += np;
      }
      float2 ml = make_float2(-INFINITY, 0.0f);
      if (lane < cnt) ml = a.part_ml[at];
      Vec ahead[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const uint32_t ak = __shfl_sync(kFull, at, k);
        if (k < (int)cnt) ahead[k] = *reinterpret_cast<const Vec*>(part + (uint64_t)ak * D);
      }
      float mm = ml.x;
      for (uint32_t o = 16; o; o >>= 1) mm = fmaxf(mm, __shfl_xor_sync(kFull, mm, o));
      mm = fmaxf(mm, m);
      const float f = m == mm ? 1.0f : ex2(m - mm);
      m = mm;
      const float w = lane < cnt ? (ml.x == mm ? 1.0f : ex2(ml.x - mm)) : 0.0f;
      float wl = w * ml.y;
      for (uint32_t o = 16; o; o >>= 1) wl += __shfl_xor_sync(kFull, wl, o);
      l = l * f + wl;
#pragma unroll
      for (int i = 0; i < kV; ++i) acc[i] *= f;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float wk = __shfl_sync(kFull, w, k);
        if (k < (int)cnt) add(ahead[k], wk);
      }
#pragma unroll 4
      for (uint32_t k = kAhead; k < cnt; ++k) {
        const uint32_t ak = __shfl_sync(kFull, at, k);
        const float wk = __shfl_sync(kFull, w, k);
        add(*reinterpret_cast<const Vec*>(part + (uint64_t)ak * D), wk);
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

// A warp takes an entry: rows of one query that have the same number of parts, at most kParts.  A lane finds the place,
// maximum and sum of a (row, part), 32 / kParts rows at once, and the rows' values are then loaded some rows together,
// with nothing to wait for between them.  The same operations in the same order as above.  Bound by the bytes of the
// parts, where the other form, a warp a row, is bound by the four loads that a row waits for, with as many rows in flight
// as there are warps.
template <int D, bool FP16, int kParts>
__global__ void __launch_bounds__(256, 4) join_entries_kernel(const AttnArgs a, const PlanDev p) {
  constexpr int kV = D / 32, kRows = 32 / kParts, kAtOnce = kRows < 4 ? kRows : 4;
  constexpr uint32_t kFull = 0xFFFFFFFFu;
  using Vec = typename std::conditional<kV == 4, float4, float2>::type;
  const uint32_t lane = threadIdx.x % 32, entry = blockIdx.x * 8 + threadIdx.x / 32;
  const bool live = entry < p.njoin;
  const JoinEntry en = live ? p.join[entry] : JoinEntry{};
  JoinSeg sg{0, 0, 0};
  if (lane < en.nsegs) sg = p.segs[en.seg0 + lane];  // at most kParts of them: each has a part
  // this lane's part of a row
  const uint32_t mine = lane % kParts;
  uint32_t at = 0, total = 0;
  for (uint32_t s = 0; s < en.nsegs; ++s) {
    const uint32_t np = __shfl_sync(kFull, sg.nparts, s), r0 = __shfl_sync(kFull, sg.row, s);
    const uint32_t st = __shfl_sync(kFull, sg.stride, s);
    if (mine >= total && mine - total < np) at = r0 + (mine - total) * st;
    total += np;
  }
  let_next_start();
  wait_for_last();
  const float* part = a.part + lane * kV;
  for (uint32_t i0 = 0; i0 < en.count; i0 += kRows) {
    const uint32_t gi = i0 + lane / kParts;
    float2 ml = make_float2(-INFINITY, 0.0f);
    if (gi < en.count && mine < total) ml = a.part_ml[at + gi];
    float m = ml.x;
#pragma unroll
    for (int o = kParts / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, o));
    const float w = mine < total ? (ml.x == m ? 1.0f : ex2(ml.x - m)) : 0.0f;
    float l = w * ml.y;
#pragma unroll
    for (int o = kParts / 2; o; o >>= 1) l += __shfl_xor_sync(kFull, l, o);
    const uint32_t rows = min((uint32_t)kRows, en.count - i0);
#pragma unroll 1
    for (uint32_t r0 = 0; r0 < rows; r0 += kAtOnce) {
      float acc[kAtOnce][kV];
#pragma unroll
      for (int r = 0; r < kAtOnce; ++r)
#pragma unroll
        for (int i = 0; i < kV; ++i) acc[r][i] = 0.0f;
#pragma unroll
      for (int k = 0; k < kParts; ++k) {
        if (k >= (int)total) break;
        const uint32_t ak = __shfl_sync(kFull, at, k);
        Vec v[kAtOnce];
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r)
          if (r0 + r < rows) v[r] = *reinterpret_cast<const Vec*>(part + (uint64_t)(ak + i0 + r0 + r) * D);
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r) {
          const float wk = __shfl_sync(kFull, w, (r0 + r) * kParts + k);
          if (r0 + r >= rows) continue;
          acc[r][0] = fmaf(v[r].x, wk, acc[r][0]);
          acc[r][1] = fmaf(v[r].y, wk, acc[r][1]);
          if constexpr (kV == 4) {
            acc[r][2] = fmaf(v[r].z, wk, acc[r][2]);
            acc[r][3] = fmaf(v[r].w, wk, acc[r][3]);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < kAtOnce; ++r) {
        const float lr = __shfl_sync(kFull, l, (r0 + r) * kParts), mr = __shfl_sync(kFull, m, (r0 + r) * kParts);
        if (r0 + r >= rows) continue;
        const float inv = lr == 0.0f ? 0.0f : 1.0f / lr;  // no key: zeros (a NaN stays one)
        const uint32_t head = en.head0 + i0 + r0 + r;
        uint16_t* o = a.out + (int64_t)en.query * a.o_tok + (int64_t)head * a.o_head + lane * kV;
        uint32_t x[kV / 2];
#pragma unroll
        for (int i = 0; i < kV; i += 2) x[i / 2] = pack2<FP16>(acc[r][i] * inv, acc[r][i + 1] * inv);
        if (kV == 4)
          *reinterpret_cast<uint2*>(o) = make_uint2(x[0], x[kV / 2 - 1]);
        else
          *reinterpret_cast<uint32_t*>(o) = x[0];
        if (a.lse && lane == 0)
          a.lse[(uint64_t)en.query * a.kv_heads * a.group + head] =
              lr == 0.0f ? -INFINITY : (mr + log2f(lr)) * 0.6931471805599453f;
      }
    }
  }
}

template <int D, bool FP16>
cudaError_t go(const AttnArgs& a, const PlanDev& p, bool overlap, cudaStream_t s) {
  const uint32_t rows = p.njoin * p.join_stride;
  // A CTA a row where there are few: 64 rows of 64 parts 7 us less than a warp a row; 2048 rows of 38 parts 3 us more.
  // With up to 8 parts a warp a row is as good from fewer rows on: 1024 rows of 8 parts 15.6 us with the attention before
  // them, 17.2 by CTAs; 512 rows of 8 14.7 and 14.0.  (Only where masked spans are: the sums of a row's parts are in
  // another order, and other batches keep theirs.)
  const uint32_t wide = p.max_parts <= 8 && (p.mask_tiles || p.mask_rows) ? 512 : 1024;
  if (p.max_parts > 4 && rows <= wide)
    return launch(join_kernel<D, FP16, true>, rows, 256, 0, 1, overlap, s, a, p);
  if (join_by_entries(p.njoin, p.join_stride, p.join_parts))
    return launch(p.join_parts <= 4 ? join_entries_kernel<D, FP16, 4> : join_entries_kernel<D, FP16, 8>, (p.njoin + 7) / 8,
                  256, 0, 1, overlap, s, a, p);
  return launch(join_kernel<D, FP16, false>, (rows + 7) / 8, 256, 0, 1, overlap, s, a, p);
}

}  // namespace

cudaError_t launch_join(int D, bool fp16, const AttnArgs& a, const PlanDev& p, bool overlap, cudaStream_t s) {
  if (D == 128) return fp16 ? go<128, true>(a, p, overlap, s) : go<128, false>(a, p, overlap, s);
  return fp16 ? go<64, true>(a, p, overlap, s) : go<64, false>(a, p, overlap, s);
}

}  // namespace pskv
