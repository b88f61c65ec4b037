// Attention over a paged cache in 4 bits: one row exactly, and what its two kernels offer.  Work is divided as in attn_paged.cuh.
#pragma once

#include <cmath>

#include "attn_paged.cuh"
#include "fp4.cuh"

namespace w8a8 {

w8a8_status launch_attn_fp4_tokens(const Fp4Pages& pc, const PagedBatch& pb, const AttnCall& a, void* ws, int sms,
                                   cudaStream_t st);

w8a8_status launch_attn_fp4_chunks(const Fp4Pages& pc, const PagedBatch& pb, const AttnCall& a, void* ws, int sms,
                                   cudaStream_t st);

// The scale in powers of two for the exponentials, without its own power of two, 2^ilogb(scale): times log2 e a scale need be no fp32 number,
// or has fewer bits than it had.
inline float score_significand(float scale) { return std::ldexp(scale, -std::ilogb(scale)) * kLog2e; }

// attend_row (attn_paged.cuh) with the values a 4-bit cache stands for: one row by one warp, key by key in the order of the formula.  The
// query is brought to 1 first, and the powers of two are applied last, so that a score that fp32 holds is one whatever its factors are.
template <bool kBf16, int kDim>
__device__ __noinline__ void attend_row_fp4(const Fp4Pages& c, const PagedBatch& b, const AttnCall& a, int s, int pos,
                                            int64_t row, int head, int lane, uint32_t* beat) {
  const uint16_t* q = a.q + row * a.q_row + head * a.q_head;
  const int kvh = head / (a.n_q / c.p.n_kv);
  const int lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
  uint32_t top = 0;
  for (int i = lane; i < kDim; i += 32) top = max(top, __float_as_uint(unpack2<kBf16>(q[i]).x) & 0x7fffffffu);
  top = __reduce_max_sync(0xffffffffu, top);
  const int e = top == 0 || top >= 0x7f800000u ? 0 : min((int)(top >> 23) - 127, 126);
  const float up = e < -126 ? two_to(126) : two_to(-e);
  const int se = ilogbf(a.scale), powers = se + max(e, -126) + c.k_exp;  // within 3 x 126
  const float scale = ldexpf(a.scale, -se), p0 = two_to(powers / 3), p1 = two_to((powers - powers / 3) / 2),
              p2 = two_to(powers - powers / 3 - (powers - powers / 3) / 2);
  float m = -INFINITY, l = 0.0f, acc[kDim / 32];
  bool any = false;
#pragma unroll
  for (int i = 0; i < kDim / 32; ++i) acc[i] = 0.0f;
  for (int j0 = lo; j0 <= pos; j0 += 32) {
    if (beat && lane == 0 && ((j0 - lo) & 8191) == 0) atomicAdd(beat, 1u);
    const int j = j0 + lane;
    int64_t sat = 0;
    const int64_t at = j <= pos ? fp4_key_offset(b, c, s, j, kvh, sat) : -1;
    float sc = -INFINITY;
    if (at >= 0) {
      float d = 0.0f;
      for (int i = 0; i < kDim / 16; ++i) {
        const uint2 kw = *reinterpret_cast<const uint2*>(c.k + at + 8 * i);
        const float unit = e4m3_value(c.ks[sat + i]);
        const uint4 q0 = *reinterpret_cast<const uint4*>(q + 16 * i), q1 = *reinterpret_cast<const uint4*>(q + 16 * i + 8);
        const uint32_t qa[8] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
        uint32_t h[8];
        e2m1x8_to_f16(kw.x, *reinterpret_cast<uint32_t(*)[4]>(h));
        e2m1x8_to_f16(kw.y, *reinterpret_cast<uint32_t(*)[4]>(h + 4));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 x = unpack2<false>(h[j]), y = unpack2<kBf16>(qa[j]);
          d = fmaf(x.x * unit, y.x * up, d);
          d = fmaf(x.y * unit, y.y * up, d);
        }
      }
      sc = d * scale * p0 * p1 * p2;
    }
    const uint32_t there = __ballot_sync(0xffffffffu, at >= 0);
    if (!there) continue;
    any = true;
    const float m_new = fmaxf(m, warp_max_f(sc));
    const float ref = m_new == -INFINITY ? 0.0f : m_new;
    const float corr = m == -INFINITY ? 0.0f : expf(m - ref);
    float p = at >= 0 ? expf(sc - ref) : 0.0f;
    const float before = l * corr;
    l = before + warp_sum_f(p);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // nothing but scores of -inf so far
    p *= inv;
#pragma unroll
    for (int i = 0; i < kDim / 32; ++i) acc[i] *= before * inv;
    for (int u = 0; u < 32; ++u) {
      if (!((there >> u) & 1u)) continue;
      const float pu = __shfl_sync(0xffffffffu, p, u);
      const int64_t au = __shfl_sync(0xffffffffu, (long long)at, u), su = __shfl_sync(0xffffffffu, (long long)sat, u);
#pragma unroll
      for (int i = 0; i < kDim / 32; ++i) {
        const int dim = lane + 32 * i;
        uint32_t h[4];
        e2m1x8_to_f16((uint32_t)c.v[au + (dim >> 1)] >> (4 * (dim & 1)), h);
        acc[i] = fmaf(pu, unpack2<false>(h[0]).x * e4m3_value(c.vs[su + (dim >> 4)]), acc[i]);
      }
    }
    m = m_new;
  }
  uint16_t* o = a.o + row * a.o_row + head * a.o_head;
  const float back = two_to(c.v_exp);
#pragma unroll
  for (int i = 0; i < kDim / 32; ++i)
    o[lane + 32 * i] = (uint16_t)pack2<kBf16>(!any ? 0.0f : l == 0.0f ? NAN : acc[i] * back, 0.0f);
}

}  // namespace w8a8
