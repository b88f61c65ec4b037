// Sampling of one token a row by temperature, top-k, top-p and min-p, from a given uniform number.
//
// The mathematics.  Weights are e^((l - max) / T) as multiples of 2^-42 in 64-bit integers, so that sums of up to
// 2^20 of them are exact and depend on no order: every comparison that decides a token is one of integers.  An fp32
// exponential would not do: a flat row of 262144 logits has steps of 2^-18 in the sum, and sums off by 2^-24
// a term would move the token in a noticeable share of draws.  So the exponent is formed with its rounding errors
// (two-term sum and product) and 2^f, |f| <= 1/2, by a Taylor polynomial in 32-bit fixed point.
#include <cmath>

#include "ops.cuh"

namespace w8a8 {

namespace {

typedef unsigned long long u64;

constexpr int kFrac = 42;  // weights are multiples of 2^-42 of the largest

struct RowScale {
  float mx, c_hi, c_lo;  // the row's maximum, log2(e) / temperature in two terms
};
__device__ __forceinline__ RowScale row_scale(float mx, float temperature) {
  const double c = 1.4426950408889634074 / (double)fmaxf(temperature, 1e-30f);
  RowScale r;
  r.mx = mx;
  r.c_hi = (float)c;
  r.c_lo = (float)(c - (double)r.c_hi);
  return r;
}

// 2^42 e^((l - mx) / T), rounded; 0 for NaN and -inf.  y = p + e is the exponent to about 2^-40; with n = rint(p), 2^(y - n) is
// the Taylor series of e^(2 h ln 2) in h = (y - n) / 2, a signed fraction of 2^32: terms to h^8 leave 2^-32 of the value.
__device__ __forceinline__ u64 weight_of(const RowScale& r, float l) {
  const float d = l - r.mx, t = d - l;
  const float lost = (l - (d - t)) + (-r.mx - t);
  const float p = d * r.c_hi;
  if (!(p > -(kFrac + 2.0f))) return 0;  // NaN too
  const float e = fmaf(d, r.c_hi, -p) + fmaf(d, r.c_lo, lost * r.c_hi);
  const float n = rintf(p);
  const int h = __float2int_rn((p - n) * 0x1p31f) + __float2int_rn(e * 0x1p31f);
  constexpr double k = 1.3862943611198906188;  // 2 ln 2
  constexpr double c1 = k, c2 = c1 * k / 2, c3 = c2 * k / 3, c4 = c3 * k / 4, c5 = c4 * k / 5, c6 = c5 * k / 6,
                   c7 = c6 * k / 7, c8 = c7 * k / 8, one = 1073741824.0;  // Q30
  int s = (int)(c8 * one + 0.5);
  s = (int)(c7 * one + 0.5) + __mulhi(s, h);
  s = (int)(c6 * one + 0.5) + __mulhi(s, h);
  s = (int)(c5 * one + 0.5) + __mulhi(s, h);
  s = (int)(c4 * one + 0.5) + __mulhi(s, h);
  s = (int)(c3 * one + 0.5) + __mulhi(s, h);
  s = (int)(c2 * one + 0.5) + __mulhi(s, h);
  s = (int)(c1 * one + 0.5) + __mulhi(s, h);
  const u64 v = (1ull << kFrac) + (u64)(((long long)s * h) >> (62 - kFrac));
  const int down = -(int)n;  // 0 .. 44
  return down == 0 ? v : (v + (1ull << (down - 1))) >> down;
}

// ceil(f x) and floor(f x) for 0 <= f < 1: f = m 2^-s exactly
__device__ __forceinline__ u64 scaled(float f, u64 x, bool up) {
  if (!(f > 0.0f)) return 0;
  const uint32_t bits = __float_as_uint(f), ex = bits >> 23;
  const uint32_t m = ex ? (bits & 0x7fffffu) | 0x800000u : bits;
  const int s = 150 - (int)(ex ? ex : 1u);  // 24 .. 149
  const unsigned __int128 y = (unsigned __int128)m * x;
  if (s >= 96) return up && x > 0 ? 1 : 0;  // m x < 2^88
  const u64 q = (u64)(y >> s);
  return up && ((unsigned __int128)q << s) != y ? q + 1 : q;
}

template <int kType>
__device__ __forceinline__ float logit_at(const void* p, int64_t i) {
  if constexpr (kType == W8A8_TYPE_F32) return reinterpret_cast<const float*>(p)[i];
  if constexpr (kType == W8A8_TYPE_BF16) return bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p)[i]);
  return __half2float(reinterpret_cast<const __half*>(p)[i]);
}
// order of logits as integers; NaN below everything
__device__ __forceinline__ uint32_t logit_key(float l) { return isnan(l) ? 0u : float_order_key(l); }
__device__ __forceinline__ float key_logit(uint32_t k) {
  return k == 0u ? -INFINITY : __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}

constexpr int kT = 1024;

__device__ __forceinline__ u64 block_sum(u64 v, u64* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  v = sh[threadIdx.x & 31];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// One block a row.  Thresholds are found bit by bit in the order keys, each bit one pass over the row.
template <int kType>
__global__ void __launch_bounds__(kT) sample_kernel(const void* logits, int64_t row_stride, int V, w8a8_sampling sp,
                                                    const float* __restrict__ u, int32_t* __restrict__ tokens,
                                                    float* __restrict__ probs) {
  __shared__ u64 sh[32], scan[kT];
  pdl_wait();
  pdl_trigger();
  const int row = blockIdx.x, tid = threadIdx.x;
  const int64_t base = (int64_t)row * row_stride;
  const float temp = sp.temperature ? sp.temperature[row] : 1.0f;
  const int k = sp.top_k ? sp.top_k[row] : 0;
  const float top_p = sp.top_p ? sp.top_p[row] : 1.0f, min_p = sp.min_p ? sp.min_p[row] : 0.0f;
  const int per = (V + kT - 1) / kT, i0 = min(V, tid * per), i1 = min(V, i0 + per);  // this thread's indices, in order
  auto key_at = [&](int i) { return logit_key(logit_at<kType>(logits, base + i)); };
  u64 best = 0;
  for (int i = i0; i < i1; ++i) best = max(best, ((u64)key_at(i) << 32) | (uint32_t)~i);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
  if ((tid & 31) == 0) sh[tid >> 5] = best;
  __syncthreads();
  for (int i = 0; i < 32; ++i) best = max(best, sh[i]);
  const uint32_t kmax = (uint32_t)(best >> 32);
  const float mx = key_logit(kmax);
  if (mx == -INFINITY || !(temp > 0.0f)) {
    if (tid == 0) {
      tokens[row] = mx == -INFINITY ? -1 : (int32_t)~(uint32_t)best;
      if (probs) probs[row] = mx == -INFINITY ? 0.0f : 1.0f;
    }
    return;
  }
  const RowScale rs = row_scale(mx, temp);
  auto weight = [&](uint32_t key) {
    if (mx == INFINITY) return key == kmax ? 1ull << kFrac : 0ull;
    return weight_of(rs, key_logit(key));
  };
  // the kept set: keys above cut, and the first `ties` (in index order) of those equal to it
  uint32_t cut = 0;
  u64 ties = ~0ull;
  auto sum_from = [&](uint32_t x, bool weigh) {  // over keys >= x of the set so far, `cut` itself not limited to its ties
    u64 s = 0;
    for (int i = i0; i < i1; ++i) {
      const uint32_t key = key_at(i);
      if (key >= x) s += weigh ? weight(key) : 1ull;
    }
    return block_sum(s, sh);
  };
  if (k > 0 && k < V) {
    uint32_t x = 0;
    for (int bit = 31; bit >= 0; --bit)
      if (sum_from(x | (1u << bit), false) >= (u64)k) x |= 1u << bit;
    cut = x;
    ties = (u64)k - (x == 0xffffffffu ? 0 : sum_from(x + 1, false));
  }
  if (top_p < 1.0f) {
    const u64 wc = weight(cut), above = sum_from(cut + 1, true), at_cut = sum_from(cut, true) - above;
    const u64 all = above + (ties == ~0ull ? at_cut : ties * wc);
    const u64 target = max(scaled(top_p, all, true), 1ull);
    if (above >= target) {
      uint32_t x = 0;
      for (int bit = 31; bit >= 0; --bit)
        if (sum_from(x | (1u << bit), true) >= target) x |= 1u << bit;
      cut = x;
      ties = ~0ull;
    }
    const u64 over = sum_from(cut + 1, true), w = weight(cut);
    if (w > 0) ties = min(ties, (target - over + w - 1) / w);
  }
  const u64 least = min_p > 0.0f ? (min_p >= 1.0f ? 1ull << kFrac : scaled(min_p, 1ull << kFrac, true)) : 0;
  // this thread's equals of the cut before and within its indices, in order
  u64 eq = 0;
  for (int i = i0; i < i1; ++i) eq += key_at(i) == cut;
  scan[tid] = eq;
  __syncthreads();
  u64 before = 0;
  for (int i = 0; i < tid; ++i) before += scan[i];
  auto kept = [&](int i, u64& seen) {  // its weight in the kept set
    const uint32_t key = key_at(i);
    if (key < cut) return 0ull;
    if (key == cut && seen++ >= ties) return 0ull;
    const u64 w = weight(key);
    return w >= least || key == kmax ? w : 0ull;
  };
  u64 mine = 0, seen = before;
  for (int i = i0; i < i1; ++i) mine += kept(i, seen);
  __syncthreads();
  scan[tid] = mine;
  __syncthreads();
  u64 total = 0, pre = 0;
  for (int i = 0; i < kT; ++i) {
    if (i < tid) pre += scan[i];
    total += scan[i];
  }
  float uu = u[row];
  uu = uu >= 0.0f ? fminf(uu, 0x1.fffffep-1f) : 0.0f;
  const u64 target = scaled(uu, total, false);
  if (target >= pre && target < pre + mine) {
    seen = before;
    for (int i = i0; i < i1; ++i) {
      const u64 w = kept(i, seen);
      pre += w;
      if (pre > target) {
        tokens[row] = i;
        if (probs) probs[row] = (float)((double)w / (double)total);
        break;
      }
    }
  }
}

}  // namespace

w8a8_status launch_sample(int dtype, const void* logits, int64_t row_stride, int M, int V, const w8a8_sampling& sp,
                          const float* u, int32_t* tokens, float* probs, cudaStream_t st) {
  auto go = [&](auto kernel) {
    return launch_pdl(kernel, dim3((unsigned)M), dim3(kT), 0, st, logits, row_stride, V, sp, u, tokens, probs);
  };
  W8A8_CUDA(dtype == W8A8_TYPE_F32    ? go(sample_kernel<W8A8_TYPE_F32>)
            : dtype == W8A8_TYPE_BF16 ? go(sample_kernel<W8A8_TYPE_BF16>)
                                      : go(sample_kernel<W8A8_TYPE_F16>));
  return W8A8_OK;
}

}  // namespace w8a8

using namespace w8a8;

extern "C" w8a8_status w8a8_sample(int dtype, const void* logits, int64_t row_stride, int M, int V,
                                   const w8a8_sampling* sampling, const float* u, int32_t* tokens, float* probs,
                                   void* stream) {
  const char* who = "w8a8_sample";
  W8A8_CHECK_ARG(M >= 0 && V >= 1, W8A8_ERR_INVALID_ARG, "%s: M=%d, V=%d", who, M, V);
  W8A8_CHECK_ARG(dtype >= W8A8_TYPE_BF16 && dtype <= W8A8_TYPE_F32, W8A8_ERR_INVALID_ARG, "%s: type %d", who, dtype);
  W8A8_CHECK_ARG(V <= W8A8_MAX_SAMPLE_VOCAB, W8A8_ERR_SHAPE, "%s: V=%d exceeds %d", who, V, W8A8_MAX_SAMPLE_VOCAB);
  W8A8_CHECK_ARG(sampling != nullptr, W8A8_ERR_INVALID_ARG, "%s: null parameters", who);
  if (M == 0) return W8A8_OK;
  W8A8_CHECK_ARG(logits && u && tokens, W8A8_ERR_INVALID_ARG, "%s: null pointer", who);
  const int64_t unit = dtype == W8A8_TYPE_F32 ? 4 : 8;
  W8A8_CHECK_ARG(row_stride >= 0 && row_stride <= (1ll << 40) && (M == 1 || row_stride % unit == 0), W8A8_ERR_SHAPE,
                 "%s: row stride %lld must be a multiple of 16 bytes", who, (long long)row_stride);
  W8A8_CHECK_ARG(aligned16(logits), W8A8_ERR_ALIGN, "%s: logits must be 16-byte aligned", who);
  const void* words[] = {sampling->temperature, sampling->top_k, sampling->top_p, sampling->min_p, u, tokens, probs};
  for (const void* p : words)
    W8A8_CHECK_ARG((reinterpret_cast<uintptr_t>(p) & 3u) == 0, W8A8_ERR_ALIGN, "%s: arrays must be 4-byte aligned", who);
  W8A8_TRY(check_device());
  return launch_sample(dtype, logits, row_stride, M, V, *sampling, u, tokens, probs, as_stream(stream));
}
