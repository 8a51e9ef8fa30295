// Attention of few rows over many keys (single-token queries, the ends of causal spans): the row kernel.
//
// A worker is one warp.  It holds 16 rows of one span and key/value head (queries x heads of the group) and
// streams the records of its run of blocks through a private ring in shared memory, one bulk copy per
// record (16 keys and values), several in flight, with no barrier between warps: per block, scores by
// mma.sync (16 rows x 16 keys), the running maximum and sum of the softmax, and the product with the
// values, all in registers.  The plan cuts the batch's (rows, head, keys) space into equal shares, one per
// worker, so that long and short spans fill the GPU alike; a share's rows leave as partial results (maximum,
// sum, unnormalised values) for join_kernel, or as the final output where nothing is to be joined.
//
// Bound by the bytes of the cache: 2 * D elements per key and head for 4 * D * 16 multiply-adds.  mma.sync
// has the smallest tile (16 rows) and takes operands and results in registers; tcgen05's 128 rows would be
// 1/8 or less filled here.  5 requests of 65536 to 131072 tokens, fp8, 8 heads, 128 columns, 1.05 GB: 166 us a pass,
// the join included, = 6.3 TB/s, 93% of the measured copy; with 44 of the 152 SMs, where memory does not bind it, it is
// bound by its instructions (ALU pipe 56%).  As a warp joins nothing with its CTA's other warps, a share's partial
// results cost 4 * D + 8 bytes a row.
#include <type_traits>

#include "kv_internal.cuh"
#include "kv_ring.h"

namespace pskv {
namespace {

// Ring of one warp: with 128 columns two records of 16 bits or three of fp8, with 64 four or seven.  More of them
// (28 KB) measured the same or 2% slower: the memory then only answers later.
constexpr int kRingBytes = 16640;

// A stage starts on a multiple of 128 bytes, so that a swizzled address is an exclusive or with a constant.
template <int D, int FMT>
constexpr int stage_bytes() {
  return (record_bytes(D, FMT) + 127) / 128 * 128;
}
template <int D, int FMT>
constexpr int ring_stages() {
  return kRingBytes / stage_bytes<D, FMT>();
}

__device__ __forceinline__ float abs_max2(uint32_t w) { return fmaxf(fabsf(bf16_lo(w)), fabsf(bf16_hi(w))); }

template <bool FP16>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (FP16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool TRANS>
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  if (TRANS)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
// Byte i of w as the exponent field of a float: a row's scale, or, for the mark of a row with a NaN, an infinity, whose
// product with such a row's codes, zeros, is the NaN that is wanted.
template <int I>
__device__ __forceinline__ float exp_byte(uint32_t w) {
  return __uint_as_float((I == 3 ? w >> 1 : w << (23 - 8 * I)) & 0x7F800000u);
}
// The same of the byte at an address.
__device__ __forceinline__ float exp_of(uint32_t addr) {
  uint16_t b;
  asm volatile("ld.shared.u8 %0, [%1];" : "=h"(b) : "r"(addr) : "memory");
  return __uint_as_float((uint32_t)b << 23);
}
__device__ __forceinline__ float min3(float a, float b, float c) {
  float r;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}
__device__ __forceinline__ void sts128_zero(uint32_t addr) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(addr), "r"(0) : "memory");
}

__device__ __forceinline__ void prefetch(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// Whether one of the two 16-bit floats in w is an infinity or a NaN.
template <bool FP16>
__device__ __forceinline__ bool not_finite2(uint32_t w) {
  constexpr uint32_t m = FP16 ? 0x7C00u : 0x7F80u;
  return (w & m) == m || ((w >> 16) & m) == m;
}
template <bool FP16>
__device__ __forceinline__ float value16(uint16_t b) {
  if (FP16) return __half2float(__ushort_as_half(b));
  return __uint_as_float((uint32_t)b << 16);
}

// Where a worker is: its next piece and the end of its pieces, its ring's next stage and that barrier's phase; whether
// it has waited for the kernel before this one.
struct Place {
  uint32_t piece, end, st, phase;
  bool waited;
};
enum Step { kDone, kTooFar, kGaveUp };

// A worker's pieces from `pl` on.  kApart (fp8): the form for queries or value scales whose magnitudes lie far apart,
// with keys, values, queries and probabilities in bf16, whose exponents reach as far as a float's; the other form leaves
// it a piece (kTooFar), with nothing of it written, and the pieces after it.  5 requests of 131072 tokens, 256 queries on
// 32768: 257 and 357 us, 166 and 248 by the other form.  The two are separate instances: as branches of a block they
// cost the common form registers (178 and 260 us).
template <int D, int FMT, bool kApart>
__device__ __forceinline__ Step run_pieces(const AttnArgs& a, const PlanDev& p, const uint32_t ring, const uint32_t bar,
                                           Place& pl) {
  constexpr bool kFp8 = FMT == PS_KV_FP8, kFp16 = FMT == PS_KV_FP16;
  constexpr int kRec = record_bytes(D, FMT), kHalf = half_bytes(D, FMT);
  constexpr int kStages = ring_stages<D, FMT>(), kStage = stage_bytes<D, FMT>();
  constexpr int kTiles = D / 8;  // n8 tiles of the output
  const uint32_t lane = threadIdx.x % 32;
  const uint32_t piece_end = pl.end;
  // what is loaded next: block `ahead_i` of piece `ahead`, into stage `ahead_st`
  uint32_t ahead = pl.piece, ahead_i = 0, ahead_st = pl.st;
  uint32_t ahead_n = 0, ahead_block = 0, ahead_head = 0, ids = 0;
  uint32_t in_flight = 0;
  auto issue = [&]() {
    if (ahead >= piece_end) return;
    if (ahead_i == 0) {
      const Piece* q = p.row_pieces + ahead;
      ahead_n = q->nblocks;
      ahead_block = q->block;
      ahead_head = q->head;
      // the piece's queries, and what it has to join in, are wanted when its turn comes
      const uint32_t row = q->row0 + lane / 2;
      if (lane / 2 < q->nrows) {
        const uint16_t* src = a.q + (int64_t)(q->query0 + row / a.group) * a.q_tok +
                              (int64_t)(ahead_head * a.group + row % a.group) * a.q_head + (lane & 1u) * (D / 2);
        prefetch(src);
      }
      if (q->nfold && lane == 0) prefetch(p.folds + q->fold0);
    }
    if ((ahead_i & 31u) == 0) ids = p.blocks[ahead_block + min(ahead_i + lane, ahead_n - 1)];
    const uint32_t id = __shfl_sync(0xFFFFFFFFu, ids, ahead_i & 31u);
    if (lane == 0) {
      mbar_expect(bar + ahead_st * 8, kRec);
      bulk_load(ring + ahead_st * kStage, a.pool + ((uint64_t)id * a.kv_heads + ahead_head) * kRec, kRec,
                bar + ahead_st * 8);
    }
    ++in_flight;
    ahead_st = ahead_st + 1 == kStages ? 0 : ahead_st + 1;
    if (++ahead_i == ahead_n) {
      ahead_i = 0;
      ++ahead;
    }
  };
#pragma unroll 1
  for (int i = 0; i < kStages; ++i) issue();

  const uint32_t quad = lane / 4, t4 = lane % 4;  // row (or key, or column) of a fragment, place in the quad
  const uint32_t mi = lane / 8, mr = lane % 8;    // ldmatrix: matrix and row whose address this lane gives
  // fp8 keys: keys 0-7 and 8-15 of a 16-byte chunk, then of the next; 16-bit: keys 0-7 of a chunk and of the next,
  // then keys 8-15.  Values: keys 0-7 and 8-15 of a chunk, then of the next.
  const uint32_t k_at = kFp8 ? offset8k<D>((mi & 1) * 8 + mr, mi >> 1) : offset16((mi >> 1) * 8 + mr, mi & 1);
  const uint32_t v_at = kHalf + (kFp8 ? offset8v((mi & 1) * 8 + mr, mi >> 1) : offset16((mi & 1) * 8 + mr, mi >> 1));
  uint32_t st = pl.st, phase = pl.phase;
  // The copies under way write this warp's memory: they are waited for, each as long as the one that is given up.
  auto leave = [&](Step how, uint32_t piece) {
    bool all = true;
    drain_ring<kStages>(st, phase, in_flight,
                        [&](uint32_t i, uint32_t parity) { all &= mbar_wait_warp(bar + i * 8, parity); });
    if (how == kGaveUp || !all) {
      if (lane == 0) atomicOr_system(a.err, kErrWait);
      return kGaveUp;
    }
    pl.piece = piece;
    pl.st = ahead_st;
    pl.phase = st + in_flight >= kStages ? phase ^ 1u : phase;
    return how;
  };

  for (uint32_t pi = pl.piece; pi < piece_end; ++pi) {
    const Piece pc = p.row_pieces[pi];
    // ---- the rows of the tile
    const uint32_t ra = pc.row0 + quad, rb = ra + 8;
    const bool va = quad < pc.nrows, vb = quad + 8 < pc.nrows;
    const uint32_t ta = ra / a.group, tb = rb / a.group;
    const uint32_t ha = pc.head * a.group + ra % a.group, hb = pc.head * a.group + rb % a.group;
    uint32_t qf[D / 16][4];
    {
      const uint16_t* qa = a.q + (int64_t)(pc.query0 + ta) * a.q_tok + (int64_t)ha * a.q_head;
      const uint16_t* qb = a.q + (int64_t)(pc.query0 + tb) * a.q_tok + (int64_t)hb * a.q_head;
#pragma unroll
      for (int kc = 0; kc < D / 16; ++kc) {
        // fp8: the key fragment of a 16-byte chunk has this lane's four neighbouring elements
        const int lo = kFp8 ? kc * 16 + t4 * 4 : kc * 16 + t4 * 2, hi = kFp8 ? lo + 2 : lo + 8;
        qf[kc][0] = va ? __ldcg(reinterpret_cast<const uint32_t*>(qa + lo)) : 0u;
        qf[kc][1] = vb ? __ldcg(reinterpret_cast<const uint32_t*>(qb + lo)) : 0u;
        qf[kc][2] = va ? __ldcg(reinterpret_cast<const uint32_t*>(qa + hi)) : 0u;
        qf[kc][3] = vb ? __ldcg(reinterpret_cast<const uint32_t*>(qb + hi)) : 0u;
      }
    }
    // fp8: codes are exact in fp16 and one instruction turns two of them into it, so the products are fp16.
    // The queries are first scaled by a power of two per row, which brings the largest element just below
    // 2^15: all but elements 2^-32 of it keep their 8 bits.  Rows with such elements, or so large that a product might
    // overflow before the key's scale brings it back, are for the other form.
    float qa_scale = a.scale_log2, qb_scale = a.scale_log2;
    if constexpr (kFp8 && !kApart) {
      float x = 0.0f, y = 0.0f;
#pragma unroll
      for (int kc = 0; kc < D / 16; ++kc) {
        x = fmaxf(x, fmaxf(abs_max2(qf[kc][0]), abs_max2(qf[kc][2])));
        y = fmaxf(y, fmaxf(abs_max2(qf[kc][1]), abs_max2(qf[kc][3])));
      }
      x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 1));
      y = fmaxf(y, __shfl_xor_sync(0xFFFFFFFFu, y, 1));
      x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 2));
      y = fmaxf(y, __shfl_xor_sync(0xFFFFFFFFu, y, 2));
      // exponents such that 2^up * max is in [2^14, 2^15); limited, so that 2^up and 2^-up are normal floats
      const int ea = min(max(14 + 127 - (int)(__float_as_uint(x) >> 23), -112), 126);
      const int eb = min(max(14 + 127 - (int)(__float_as_uint(y) >> 23), -112), 126);
      const float ua = __uint_as_float((uint32_t)(127 + ea) << 23), ub = __uint_as_float((uint32_t)(127 + eb) << 23);
      qa_scale *= __uint_as_float((uint32_t)(127 - ea) << 23);
      qb_scale *= __uint_as_float((uint32_t)(127 - eb) << 23);
      bool lost = fmaxf(fabsf(qa_scale), fabsf(qb_scale)) > 0x1p90f;
#pragma unroll
      for (int kc = 0; kc < D / 16; ++kc) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = (i & 1) ? ub : ua, lo = bf16_lo(qf[kc][i]) * u, hi = bf16_hi(qf[kc][i]) * u;
          qf[kc][i] = pack2<true>(lo, hi);
          const float2 got = __half22float2(*reinterpret_cast<const __half2*>(&qf[kc][i]));
          lost |= got.x != lo || got.y != hi;
        }
      }
      if (__any_sync(0xFFFFFFFFu, lost)) return leave(kTooFar, pi);
    }
    // fp8: the scale that the output so far is relative to, 2^5 over it, and the first such scale
    float v_ref = 0.0f, v_inv = 0.0f, v_first = 0.0f;
    // the last key each of the two rows sees, and the last that all rows of the tile see
    const int32_t last = (int32_t)pc.end - 1;
    const int32_t lim_a = min(last, pc.climit + (int32_t)ta), lim_b = min(last, pc.climit + (int32_t)tb);
    const int32_t lim_all = min(last, pc.climit + (int32_t)(pc.row0 / a.group));

    float acc[kTiles][4];
#pragma unroll
    for (int j = 0; j < kTiles; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
    float ma = -INFINITY, mb = -INFINITY, la = 0.0f, lb = 0.0f;

    for (uint32_t bi = 0; bi < pc.nblocks; ++bi) {
      const uint32_t rec = ring + st * kStage;
      if (!mbar_wait_warp(bar + st * 8, phase)) return leave(kGaveUp, pi);
      // ---- scores
      float s[2][4];
#pragma unroll
      for (int n = 0; n < 2; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
      // two codes as a bf16 operand, with their scales
      auto scaled = [](uint32_t h, float f0, float f1) {
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h));
        return pack2<false>(x.x * f0, x.y * f1);
      };
      if constexpr (kFp8) {
        // apart: the scales of this lane's keys of the fragments; the mark of a NaN gives one
        const float kf[2] = {kApart ? exp_of(rec + 2 * kHalf + exp_place(quad)) : 1.0f,
                             kApart ? exp_of(rec + 2 * kHalf + exp_place(quad + 8)) : 1.0f};
#pragma unroll
        for (int c = 0; c < D / 16; c += 2) {
          uint32_t r[4];
          ldsm4<false>(r, (rec + k_at) ^ (c << 4));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t b0, b1;
            e4m3x4_to_f16x2(r[i], b0, b1);
            if (kApart) {
              b0 = scaled(b0, kf[i & 1], kf[i & 1]);
              b1 = scaled(b1, kf[i & 1], kf[i & 1]);
            }
            mma16816<!kApart>(s[i & 1], qf[c + (i >> 1)], b0, b1);
          }
        }
      } else {
#pragma unroll
        for (int kc = 0; kc < D / 16; ++kc) {
          uint32_t r[4];
          ldsm4<false>(r, (rec + k_at + (kc / 4) * (kBlock * 128)) ^ ((2 * kc % 8) << 4));
          mma16816<kFp16>(s[0], qf[kc], r[0], r[1]);
          mma16816<kFp16>(s[1], qf[kc], r[2], r[3]);
        }
      }
      float vs[4];  // fp8: the value rows' scales of this lane's keys
      if constexpr (kFp8) {
        const uint32_t ke = lds32(rec + 2 * kHalf + t4 * 4), vx = lds32(rec + 2 * kHalf + kBlock + t4 * 4);
        const float k0 = kApart ? 1.0f : exp_byte<0>(ke), k1 = kApart ? 1.0f : exp_byte<1>(ke);
        const float k2 = kApart ? 1.0f : exp_byte<2>(ke), k3 = kApart ? 1.0f : exp_byte<3>(ke);
        s[0][0] = s[0][0] * qa_scale * k0;
        s[0][1] = s[0][1] * qa_scale * k1;
        s[0][2] = s[0][2] * qb_scale * k0;
        s[0][3] = s[0][3] * qb_scale * k1;
        s[1][0] = s[1][0] * qa_scale * k2;
        s[1][1] = s[1][1] * qa_scale * k3;
        s[1][2] = s[1][2] * qb_scale * k2;
        s[1][3] = s[1][3] * qb_scale * k3;
        // The values' scales go into the probabilities, relative to a reference near the largest and times 2^5: with
        // probabilities of at most 2^8 (below) and scales of at most twice the reference, their products stay at or
        // below 2^14.  Scales of at least 2^-10 of it leave a product its 11 bits down to probabilities of 2^-9, and
        // below that cost at most 2^-20 of the key's own value.  A key further below, beside large rows that a query
        // does not see or hardly weighs, would lose its bits: such a piece is for the other form, whose values have their
        // scales and whose output is relative to nothing.
        vs[0] = exp_byte<0>(vx);
        vs[1] = exp_byte<1>(vx);
        vs[2] = exp_byte<2>(vx);
        vs[3] = exp_byte<3>(vx);
        if constexpr (kApart) {  // the mark of a NaN stays with the probability
#pragma unroll
          for (int i = 0; i < 4; ++i) vs[i] = vs[i] < 0x1p120f ? 1.0f : vs[i];
        } else {
          float rel[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) rel[i] = vs[i] * v_inv;
          // the same for the whole warp; also where a row is marked, zero or past the end
          if (__any_sync(0xFFFFFFFFu, max3(fmaxf(rel[0], rel[1]), rel[2], rel[3]) > 0x1p6f ||
                                          min3(fminf(rel[0], rel[1]), rel[2], rel[3]) < 0x1p-5f)) {
            const int32_t here = (int32_t)pc.key0 + (int32_t)(bi * kBlock);
            // Rows of zeros have the smallest scale (or, never written, none) and weigh nothing.
            uint32_t zeros = 0;  // bit 2 * key
            if (__any_sync(0xFFFFFFFFu, min3(fminf(vs[0], vs[1]), vs[2], vs[3]) <= 0x1p-110f)) {
              bool any = false;
#pragma unroll 1
              for (uint32_t c = lane & 1; c < D / 16; c += 2) {
                const uint4 w = lds128(rec + kHalf + offset8v(lane >> 1, c));
                any |= ((w.x | w.y | w.z | w.w) & 0x7F7F7F7Fu) != 0;
              }
              const uint32_t some = __ballot_sync(0xFFFFFFFFu, any);
              zeros = ~(some | (some >> 1));
            }
            float top = 0.0f, low = INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t key = t4 * 2 + (i & 1) + (i >> 1) * 8;
              if (vs[i] < 0x1p120f && here + (int32_t)key <= last && !((zeros >> (2 * key)) & 1u)) {
                top = fmaxf(top, vs[i]);
                low = fminf(low, vs[i]);
              }
            }
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, 1));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, 2));
            const float ref = top > 2.0f * v_ref ? top : v_ref;
            // (the second: the output so far keeps its bits when it is brought to another reference)
            if (low < 0x1p-10f * ref || (v_first > 0.0f && ref * 0x1p-60f > v_first)) return leave(kTooFar, pi);
            if (ref > v_ref) {
              const uint32_t inverse = (254u << 23) - __float_as_uint(ref);  // of a power of two
              const float f = v_ref * __uint_as_float(inverse);
              v_ref = ref;
              v_inv = __uint_as_float(inverse + (5u << 23));
              if (v_first == 0.0f) v_first = ref;
#pragma unroll
              for (int j = 0; j < kTiles; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] *= f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) rel[i] = vs[i] * v_inv;
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) vs[i] = rel[i];
        }
      } else {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[n][i] *= a.scale_log2;
      }
      // ---- masks: only blocks past what every row sees
      const int32_t key0 = (int32_t)(pc.key0 + bi * kBlock);
      const bool edge = key0 + kBlock - 1 > lim_all;  // the same for the whole warp
      uint32_t bad = 0;                               // 16-bit formats: keys whose values are not all finite
      if (edge) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int32_t j = key0 + n * 8 + (int32_t)t4 * 2 + i;
            if (j > lim_a) s[n][i] = -INFINITY;
            if (j > lim_b) s[n][2 + i] = -INFINITY;
          }
        if constexpr (!kFp8) {
          // A masked key's probability is 0, but 0 times an infinity or a NaN is not: value rows past the
          // end (left there by other tokens) and rows with such a value are taken out of the product.  Of
          // the latter, those that some row sees are added below one by one.
          const uint32_t tok = lane >> 1;
          const bool past = key0 + (int32_t)tok > last;
          bool odd = false;
#pragma unroll 4
          for (int c = 0; c < D / 16; ++c) {
            const uint4 w = lds128(rec + kHalf + offset16(tok, 2 * c + (lane & 1)));
            odd |= not_finite2<kFp16>(w.x) | not_finite2<kFp16>(w.y) | not_finite2<kFp16>(w.z) | not_finite2<kFp16>(w.w);
          }
          const uint32_t odds = __ballot_sync(0xFFFFFFFFu, odd && !past);
          const bool out = past || ((odds >> (lane & ~1u)) & 3u) != 0;
          if (out) {
#pragma unroll 4
            for (int c = 0; c < D / 16; ++c) sts128_zero(rec + kHalf + offset16(tok, 2 * c + (lane & 1)));
          }
          bad = odds | (odds >> 1);  // bit 2 * key
          __syncwarp();
        }
      }
      // ---- running maximum and sum.  The maximum that the exponents refer to follows only when a new one
      // is more than 2^8 larger: up to there the probabilities and their sum are far from 32-bit overflow.
      float xa = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1]));
      float xb = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
      xa = fmaxf(xa, __shfl_xor_sync(0xFFFFFFFFu, xa, 1));
      xb = fmaxf(xb, __shfl_xor_sync(0xFFFFFFFFu, xb, 1));
      xa = fmaxf(xa, __shfl_xor_sync(0xFFFFFFFFu, xa, 2));
      xb = fmaxf(xb, __shfl_xor_sync(0xFFFFFFFFu, xb, 2));
      if (__any_sync(0xFFFFFFFFu, xa > ma + 8.0f || xb > mb + 8.0f)) {
        const float na = fmaxf(ma, xa), nb = fmaxf(mb, xb);
        const float fa = na == ma ? 1.0f : ex2(ma - na), fb = nb == mb ? 1.0f : ex2(mb - nb);
        ma = na;
        mb = nb;
        la *= fa;
        lb *= fb;
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          acc[j][0] *= fa;
          acc[j][1] *= fa;
          acc[j][2] *= fb;
          acc[j][3] *= fb;
        }
      }
      const float ua = ma == -INFINITY ? 0.0f : ma, ub = mb == -INFINITY ? 0.0f : mb;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        s[n][0] = ex2(s[n][0] - ua);
        s[n][1] = ex2(s[n][1] - ua);
        s[n][2] = ex2(s[n][2] - ub);
        s[n][3] = ex2(s[n][3] - ub);
        la += s[n][0] + s[n][1];
        lb += s[n][2] + s[n][3];
      }
      if constexpr (kFp8) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float fa = vs[2 * n + i], fb = fa;
            if (edge) {  // the scale of a masked row may be the mark of a NaN
              const int32_t j = key0 + n * 8 + (int32_t)t4 * 2 + i;
              if (j > lim_a) fa = 0.0f;
              if (j > lim_b) fb = 0.0f;
            }
            s[n][i] *= fa;
            s[n][2 + i] *= fb;
          }
      }
      // ---- product with the values
      if constexpr (kFp8) {
        const uint32_t pf[4] = {pack2<!kApart>(s[0][0], s[0][1]), pack2<!kApart>(s[0][2], s[0][3]),
                                pack2<!kApart>(s[1][0], s[1][1]), pack2<!kApart>(s[1][2], s[1][3])};
        if constexpr (kApart) {  // a marked row's codes are zeros, and stay so
          const uint32_t vx = lds32(rec + 2 * kHalf + kBlock + t4 * 4);
          vs[0] = exp_byte<0>(vx);
          vs[1] = exp_byte<1>(vx);
          vs[2] = exp_byte<2>(vx);
          vs[3] = exp_byte<3>(vx);
#pragma unroll
          for (int i = 0; i < 4; ++i) vs[i] = vs[i] < 0x1p120f ? vs[i] : 0.0f;
        }
        auto operand = [&](uint32_t h, float f0, float f1) { return kApart ? scaled(h, f0, f1) : h; };
#pragma unroll
        for (int c = 0; c < D / 16; c += 2) {
          uint32_t r[4];
          ldsm4<true>(r, (rec + v_at + (c / 4) * (kBlock * 64)) ^ ((c % 4) << 4));
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            // a chunk's 16 columns: tile 2c has the even ones, tile 2c + 1 the odd ones; the halves of a register are the
            // keys of vs[0] and vs[1], or of vs[2] and vs[3]
            uint32_t even0, odd0, even1, odd1;
            e4m3x4_to_f16x2(__byte_perm(r[i], 0, 0x3120), even0, odd0);
            e4m3x4_to_f16x2(__byte_perm(r[i + 1], 0, 0x3120), even1, odd1);
            mma16816<!kApart>(acc[2 * c + i], pf, operand(even0, vs[0], vs[1]), operand(even1, vs[2], vs[3]));
            mma16816<!kApart>(acc[2 * c + i + 1], pf, operand(odd0, vs[0], vs[1]), operand(odd1, vs[2], vs[3]));
          }
        }
      } else {
        const uint32_t pf[4] = {pack2<kFp16>(s[0][0], s[0][1]), pack2<kFp16>(s[0][2], s[0][3]),
                                pack2<kFp16>(s[1][0], s[1][1]), pack2<kFp16>(s[1][2], s[1][3])};
#pragma unroll
        for (int j = 0; j < kTiles; j += 2) {
          uint32_t r[4];
          ldsm4<true>(r, (rec + v_at + (j / 8) * (kBlock * 128)) ^ ((j % 8) << 4));
          mma16816<kFp16>(acc[j], pf, r[0], r[1]);
          mma16816<kFp16>(acc[j + 1], pf, r[2], r[3]);
        }
        if (edge) {
          if (bad & 0x55555555u) {
            const uint32_t id = p.blocks[pc.block + bi];
            const uint8_t* vals = a.pool + ((uint64_t)id * a.kv_heads + pc.head) * kRec + kHalf;
            for (uint32_t kk = 0; kk < kBlock; ++kk) {
              if (!((bad >> (2 * kk)) & 1u)) continue;
              const uint32_t from = (lane & ~3u) | ((kk % 8) / 2);
              const float c0 = kk < 8 ? ((kk & 1) ? s[0][1] : s[0][0]) : ((kk & 1) ? s[1][1] : s[1][0]);
              const float c1 = kk < 8 ? ((kk & 1) ? s[0][3] : s[0][2]) : ((kk & 1) ? s[1][3] : s[1][2]);
              const float pa = __shfl_sync(0xFFFFFFFFu, c0, from), pb = __shfl_sync(0xFFFFFFFFu, c1, from);
              const bool sa = key0 + (int32_t)kk <= lim_a, sb = key0 + (int32_t)kk <= lim_b;
#pragma unroll
              for (int j = 0; j < kTiles; ++j) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(vals + offset16(kk, j) + t4 * 4);
                const float v0 = value16<kFp16>((uint16_t)w), v1 = value16<kFp16>((uint16_t)(w >> 16));
                if (sa) {
                  acc[j][0] += pa * v0;
                  acc[j][1] += pa * v1;
                }
                if (sb) {
                  acc[j][2] += pb * v0;
                  acc[j][3] += pb * v1;
                }
              }
            }
          }
          fence_async_shared();  // the zeros above before the next copy into this stage
        }
      }
      __syncwarp();
      --in_flight;
      if (++st == kStages) {
        st = 0;
        phase ^= 1u;
      }
      issue();
    }

    // ---- the piece's result
    if constexpr (kFp8 && !kApart) {
      const float f = v_ref * 0x1p-5f;
#pragma unroll
      for (int j = 0; j < kTiles; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] *= f;
    }
    la += __shfl_xor_sync(0xFFFFFFFFu, la, 1);
    lb += __shfl_xor_sync(0xFFFFFFFFu, lb, 1);
    la += __shfl_xor_sync(0xFFFFFFFFu, la, 2);
    lb += __shfl_xor_sync(0xFFFFFFFFu, lb, 2);
    if (pc.part_row != kDirect) {
      float* oa = a.part + (uint64_t)(pc.part_row + quad) * D;
      float* ob = oa + 8 * D;
      if (va) {
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          if (kFp8) {
            if (j & 1) continue;
            *reinterpret_cast<float4*>(oa + 8 * j + 4 * t4) =
                make_float4(acc[j][0], acc[j + 1][0], acc[j][1], acc[j + 1][1]);
          } else {
            *reinterpret_cast<float2*>(oa + 8 * j + 2 * t4) = make_float2(acc[j][0], acc[j][1]);
          }
        }
        if (t4 == 0) a.part_ml[pc.part_row + quad] = make_float2(ma, la);
      }
      if (vb) {
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          if (kFp8) {
            if (j & 1) continue;
            *reinterpret_cast<float4*>(ob + 8 * j + 4 * t4) =
                make_float4(acc[j][2], acc[j + 1][2], acc[j][3], acc[j + 1][3]);
          } else {
            *reinterpret_cast<float2*>(ob + 8 * j + 2 * t4) = make_float2(acc[j][2], acc[j][3]);
          }
        }
        if (t4 == 0) a.part_ml[pc.part_row + 8 + quad] = make_float2(mb, lb);
      }
    } else {
      // The tile kernel's parts of these rows (the prefix that they share) are joined in here, which saves the
      // write and the read of this part and, mostly, the join kernel.
      if (pc.nfold && !pl.waited) {
        wait_for_last();
        pl.waited = true;
      }
      for (uint32_t fi = 0; fi < pc.nfold; ++fi) {
        const Fold fo = p.folds[pc.fold0 + fi];
        const bool ia = quad >= fo.first && quad < (uint32_t)fo.first + fo.count;
        const bool ib = quad + 8 >= fo.first && quad + 8 < (uint32_t)fo.first + fo.count;
        for (uint32_t x = 0; x < fo.nsegs; ++x) {
          const JoinSeg sg = p.segs[fo.seg0 + x];
          for (uint32_t k = 0; k < sg.nparts; ++k) {
            const uint64_t at = (uint64_t)sg.row + (uint64_t)k * sg.stride + quad - fo.first;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              if (half ? !ib : !ia) continue;
              float& m = half ? mb : ma;
              float& l = half ? lb : la;
              const float2 ml = a.part_ml[at + 8 * half];
              const float* src = a.part + (at + 8 * half) * D;
              const float n = fmaxf(m, ml.x);
              const float f0 = m == n ? 1.0f : ex2(m - n), f1 = ml.x == n ? 1.0f : ex2(ml.x - n);
              m = n;
              l = l * f0 + ml.y * f1;
#pragma unroll
              for (int j = 0; j < kTiles; ++j) {
                if (kFp8) {
                  if (j & 1) continue;
                  const float4 v = *reinterpret_cast<const float4*>(src + 8 * j + 4 * t4);
                  acc[j][2 * half] = acc[j][2 * half] * f0 + v.x * f1;
                  acc[j + 1][2 * half] = acc[j + 1][2 * half] * f0 + v.y * f1;
                  acc[j][2 * half + 1] = acc[j][2 * half + 1] * f0 + v.z * f1;
                  acc[j + 1][2 * half + 1] = acc[j + 1][2 * half + 1] * f0 + v.w * f1;
                } else {
                  const float2 v = *reinterpret_cast<const float2*>(src + 8 * j + 2 * t4);
                  acc[j][2 * half] = acc[j][2 * half] * f0 + v.x * f1;
                  acc[j][2 * half + 1] = acc[j][2 * half + 1] * f0 + v.y * f1;
                }
              }
            }
          }
        }
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (half ? !vb : !va) continue;
        const float l = half ? lb : la, m = half ? mb : ma;
        const uint32_t query = pc.query0 + (half ? tb : ta), head = half ? hb : ha;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // no key: zeros (a NaN stays one)
        uint16_t* o = a.out + (int64_t)query * a.o_tok + (int64_t)head * a.o_head;
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          const float x0 = acc[j][2 * half] * inv, x1 = acc[j][2 * half + 1] * inv;
          if (kFp8) {
            if (j & 1) continue;
            const float y0 = acc[j + 1][2 * half] * inv, y1 = acc[j + 1][2 * half + 1] * inv;
            *reinterpret_cast<uint2*>(o + 8 * j + 4 * t4) = make_uint2(pack2<kFp16>(x0, y0), pack2<kFp16>(x1, y1));
          } else {
            *reinterpret_cast<uint32_t*>(o + 8 * j + 2 * t4) = pack2<kFp16>(x0, x1);
          }
        }
        if (a.lse && t4 == 0)
          a.lse[(uint64_t)query * a.kv_heads * a.group + head] =
              l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
      }
    }
  }
  return kDone;
}

template <int D, int FMT>
__global__ void __launch_bounds__(kRowWarps * 32, 1) rows_kernel(const AttnArgs a, const PlanDev p) {
  constexpr int kStages = ring_stages<D, FMT>(), kStage = stage_bytes<D, FMT>();
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ __align__(8) uint64_t bars[kRowWarps * kStages];

  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t worker = warp * p.row_ctas + blockIdx.x;  // neighbours in the plan go to different SMs
  if (worker >= p.row_workers) {  // no barrier of the CTA is used
    wait_for_last();
    return;
  }
  const uint32_t ring = smem_u32(smem) + warp * kStages * kStage;
  const uint32_t bar = smem_u32(bars) + warp * kStages * 8;
  if (lane < kStages) mbar_init(bar + lane * 8, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncwarp();

  // The plan is read at once, the cache and the queries after what may have written them; after a tile kernel of the
  // same call, which has waited for that, at once too.
  Place pl{p.row_off[worker], p.row_off[worker + 1], 0, 0, a.rows_first != 0};
  if (pl.waited) {
    prefetch(p.row_pieces + pl.piece);
    wait_for_last();
  }
  let_next_start();
  const Step how = run_pieces<D, FMT, false>(a, p, ring, bar, pl);
  if constexpr (FMT == PS_KV_FP8)
    if (how == kTooFar) run_pieces<D, FMT, true>(a, p, ring, bar, pl);
  if (!pl.waited) wait_for_last();
}

template <int D, int FMT>
constexpr int smem_bytes() {
  return kRowWarps * ring_stages<D, FMT>() * stage_bytes<D, FMT>();
}

template <int D, int FMT>
cudaError_t prepare_one() {
  return cudaFuncSetAttribute(rows_kernel<D, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<D, FMT>());
}
template <int D, int FMT>
cudaError_t launch_one(const AttnArgs& a, const PlanDev& p, bool overlap, cudaStream_t s) {
  return launch(rows_kernel<D, FMT>, p.row_ctas, kRowWarps * 32, smem_bytes<D, FMT>(), 1, overlap, s, a, p);
}

}  // namespace

cudaError_t prepare_rows(int D, int fmt) {
  if (D == 128)
    return fmt == PS_KV_BF16   ? prepare_one<128, PS_KV_BF16>()
           : fmt == PS_KV_FP16 ? prepare_one<128, PS_KV_FP16>()
                               : prepare_one<128, PS_KV_FP8>();
  return fmt == PS_KV_BF16   ? prepare_one<64, PS_KV_BF16>()
         : fmt == PS_KV_FP16 ? prepare_one<64, PS_KV_FP16>()
                             : prepare_one<64, PS_KV_FP8>();
}

cudaError_t launch_rows(int D, int fmt, const AttnArgs& a, const PlanDev& p, bool overlap, cudaStream_t s) {
  if (D == 128)
    return fmt == PS_KV_BF16   ? launch_one<128, PS_KV_BF16>(a, p, overlap, s)
           : fmt == PS_KV_FP16 ? launch_one<128, PS_KV_FP16>(a, p, overlap, s)
                               : launch_one<128, PS_KV_FP8>(a, p, overlap, s);
  return fmt == PS_KV_BF16   ? launch_one<64, PS_KV_BF16>(a, p, overlap, s)
         : fmt == PS_KV_FP16 ? launch_one<64, PS_KV_FP16>(a, p, overlap, s)
                             : launch_one<64, PS_KV_FP8>(a, p, overlap, s);
}

}  // namespace pskv
