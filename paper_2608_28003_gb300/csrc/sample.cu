// Sampling of one token a row by temperature, top-k, top-p and min-p, from a given uniform number.
//
// The mathematics.  Weights are e^((l - max) / T) as multiples of 2^-43 in 64-bit integers, so that sums of up to
// 2^20 of them are exact and depend on no order: every comparison that decides a token is one of integers.  A plain fp32
// exponential would not do: a flat row of 262144 logits has steps of 2^-18 in the sum, and weights off by 2^-24
// or, far from the maximum, by 2^-19 would move the token in a noticeable share of draws.  So the exponent is kept with its
// rounding errors (two-term difference and product) and 2^y comes from a table of 128 values and a cubic whose small part alone is
// rounded in fp32: off by one to two steps of 2^-29 of the weight, within the 2^-27 that is promised, in about 25 instructions (two logits at a time in packed fp32; the same
// in 32-bit integer products took three times as long).
//
// The work.  A cluster of up to 16 CTAs takes a row: the maximum; then, where a filter needs it, a histogram with a bin per 1/64
// of the exponent: counts, and for a cut by weight the exact sums of the bins' weights, as two 16-bit digits of the 30-bit
// significands (a bin's weights share their exponent), so that three 32-bit additions to shared memory take a logit (a 64-bit
// one costs more than the three).  The crossing bin holds the cut: its tokens, up to kSmall, are collected and
// sorted by one CTA; more (flat or tied rows) are divided by the order of their floats until one value is left, whose
// equals are cut by index.  The last pass sums the kept weights and finds the token in index order.  Slices of up to 64 KB
// (few rows) stay in shared memory between the passes; longer ones are read again from L2.
//
// Measured, 262144 logits a row: 1 row with every filter 22 us (floor 0.15: eight cluster barriers and the steps between them,
// each a latency chain; 36 with 8 CTAs instead of 16, 27.4 with the slices read again from L2); 64 rows with a nucleus of 0.9
// 134 us (floor 9.9): 127 instructions a logit of each warp, of which the weights' two passes are 94, at half of the issue
// rate.  The next logits loaded ahead of a step's work: 138 (spills).
#include <cmath>
#include <type_traits>

#include "ops.cuh"
#include "paged.cuh"

namespace w8a8 {

namespace {

typedef unsigned long long u64;

constexpr int kT = 512, kWarps = kT / 32;
constexpr int kFrac = 43;     // weights are multiples of 2^-43 of the largest
constexpr int kBins = 2880;    // one per 1/64 of the exponent, 44.5 of which weigh anything (0 .. 2849); a multiple of 16 CTAs
constexpr int kMostSteps = 2 * 2849;  // of 1 / 128 of the exponent, that a logit with a bin lies below the maximum
constexpr int kFine = 2048;    // and of the divisions of a crowded range
constexpr int kMostSlice = 65536;  // 16-bit digits of that many weights add up in 32 bits
constexpr int kSmall = 1024;
constexpr int kMaxCluster = 16;
constexpr int kUnit = 4 * 32 * kWarps;      // a CTA's slice is a multiple: 128 logits a warp and step
constexpr int kHeldSlice = 8 * kUnit;       // slices up to 64 KB stay in shared memory (up to 48 two CTAs fit an SM)

// ------------------------------------------------------------------------------------ weights
struct RowScale {
  float mx, low;     // the maximum; logits below `low` weigh nothing
  float c_hi, c_lo;  // log2(e) / T in two terms
};
constexpr float kRound = 98304.0f;  // 1.5 2^16 (bits 0x47c00000): added to p, rounds it to multiples of 1 / 128
// the exponent of l - mx rounded to steps of 1 / 128, and kRound: falls with l; and -128 times it
__device__ __forceinline__ float rounded(const RowScale& r, float l) {
  return __fadd_rn(__fmul_rn(l - r.mx, r.c_hi), kRound);
}
__device__ __forceinline__ int steps_of(const RowScale& r, float l) {
  return __float_as_int(kRound) - __float_as_int(rounded(r, l));
}
__device__ __forceinline__ RowScale row_scale(float mx, float least, float temperature) {
  RowScale r;
  const float t = fminf(fmaxf(temperature, 1e-30f), 1e30f);
  constexpr double log2e = 1.4426950408889634074;
  constexpr float k_hi = (float)log2e, k_lo = (float)(log2e - (double)k_hi);
  r.mx = mx;
  r.c_hi = k_hi / t;
  r.c_lo = (fmaf(-r.c_hi, t, k_hi) + k_lo) / t;
  r.low = fmaxf(fmaxf(mx - (kFrac + 1.5f) / r.c_hi, least), mx - 3e38f);
  // At a temperature of a few of mx's last places the difference rounds to a logit up to twice as far below, whose bin
  // would lie beyond the last: a place or two up is one within them, which still weighs nothing.
  while (steps_of(r, r.low) > kMostSteps) r.low = nextafterf(r.low, mx);
  return r;
}
// `table`: 2^(j / 128) as a float, and 2^(29 + j / 128) as an integer less the bits of kMagic.
struct Entry {
  float t;
  uint32_t i;
};
constexpr float kMagic = 12582912.0f;  // 1.5 2^23
// Of two logits: v, 2^29 to 2^30, and i, so that e^((l - mx) / T) = v 2^(-29 - n), n = (kRoundBits + 127 - i) >> 7; for l >= low.
// nz: f2_neg_zero.
constexpr uint32_t kRoundBits = 0x47c00000u;
__device__ __forceinline__ void parts_of(const RowScale& r, const Entry* table, f32x2 nz, float l0, float l1, uint32_t& v0,
                                         uint32_t& v1, uint32_t& i0, uint32_t& i1) {
  const f32x2 minus1 = f2_both(0xbf800000u), l = f2_pack(l0, l1), nm = f2_pack(-r.mx, -r.mx);
  const f32x2 ch = f2_pack(r.c_hi, r.c_hi), cl = f2_pack(r.c_lo, r.c_lo);
  const f32x2 d = f2_add(l, nm), bb = f2_fma(l, minus1, d);                                 // d + lost = l - mx
  const f32x2 lost = f2_add(f2_fma(f2_fma(bb, minus1, d), minus1, l), f2_fma(bb, minus1, nm));
  const f32x2 np = f2_mul(d, f2_pack(-r.c_hi, -r.c_hi), nz);                                // -p
  const f32x2 e = f2_fma(lost, ch, f2_fma(d, cl, f2_fma(d, ch, np)));                       // p + e = y
  const f32x2 round = f2_pack(kRound, kRound), s = f2_fma(np, minus1, round);               // multiples of 1 / 128 of p
  const f32x2 g = f2_add(f2_fma(np, minus1, f2_fma(s, minus1, round)), e);                  // what they leave of y
  constexpr double ln2 = 0.69314718055994530942, q29 = 536870912.0;
  constexpr float c1 = (float)(ln2 * q29), c2 = (float)(ln2 * ln2 / 2 * q29), c3 = (float)(ln2 * ln2 * ln2 / 6 * q29);
  const f32x2 q = f2_mul(g, f2_fma(g, f2_fma(g, f2_pack(c3, c3), f2_pack(c2, c2)), f2_pack(c1, c1)), nz);  // 2^29 (2^g - 1)
  float s0, s1;
  f2_unpack(s, s0, s1);
  i0 = __float_as_uint(s0);  // 128 times the rounded exponent, and the bits of kRound
  i1 = __float_as_uint(s1);
  const Entry t0 = table[i0 & 127], t1 = table[i1 & 127];
  float m0, m1;
  f2_unpack(f2_fma(f2_pack(t0.t, t1.t), q, f2_pack(kMagic, kMagic)), m0, m1);
  v0 = __float_as_uint(m0) + t0.i;  // 2^(29 + fraction of y)
  v1 = __float_as_uint(m1) + t1.i;
}
// 2^43 e^((l - mx) / T) of two logits, truncated; 0 below `low` (and for NaN)
__device__ __forceinline__ void weights_of(const RowScale& r, const Entry* table, f32x2 nz, float l0, float l1, u64& w0, u64& w1) {
  uint32_t v0, v1, i0, i1;
  parts_of(r, table, nz, l0, l1, v0, v1, i0, i1);
  constexpr uint32_t n = 61 - kFrac + (kRoundBits >> 7);
  w0 = l0 >= r.low ? ((u64)v0 << 32) >> min(n - (i0 >> 7), 63u) : 0ull;
  w1 = l1 >= r.low ? ((u64)v1 << 32) >> min(n - (i1 >> 7), 63u) : 0ull;
}
// bins: two of the 128 steps an exponent has, both of one n
__device__ __forceinline__ uint32_t bin_of_steps(uint32_t steps) { return (steps + 1) >> 1; }
__device__ __forceinline__ int bin_exponent(int bin) { return (2 * bin + 127) >> 7; }

struct Table {
  Entry e[128];
  // 2^(j / 128) by repeated multiplication with 2^(1/128), whose series to the sixth power is exact to 2^-52 here
  constexpr Table() : e() {
    constexpr double h = 0.69314718055994530942 / 128;
    constexpr double step = 1 + h * (1 + h / 2 * (1 + h / 3 * (1 + h / 4 * (1 + h / 5 * (1 + h / 6)))));
    double v = 1.0;
    for (int j = 0; j < 128; ++j, v *= step) {
      e[j].t = (float)v;
      e[j].i = (uint32_t)(v * 536870912.0 + 0.5) - 0x4b400000u;  // the bits of kMagic
    }
  }
};
__constant__ constexpr Table kTable{};

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

// ----------------------------------------------------------------------------------- the cluster
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void st_remote(uint32_t addr, u64 v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;\n" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ uint32_t ld_remote(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];\n" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t add_remote(uint32_t addr, uint32_t v) {
  uint32_t old;
  asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;\n" : "=r"(old) : "r"(addr), "r"(v) : "memory");
  return old;
}
__device__ __forceinline__ u64 warp_sum(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ u64 warp_scan(u64 v, int lane) {  // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}
__device__ __forceinline__ float order_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key);
}

struct Shared {
  // the histogram: counts, and the sums of the low 16 and the high bits of the weights' significands
  uint32_t count[kBins], lo[kBins], hi[kBins];
  u64 mine[kSmall], list[kSmall];               // candidates: this CTA's, all (rank 0)
  Entry table[128];
  u64 ex[2][kMaxCluster][2];                    // what the CTAs tell one another: a pair of numbers each
  u64 res[6];
  u64 red[kWarps][2];
  uint32_t listed, n_mine, n_before;
};

// What the tokens kept so far are: those above `value`, and its equals up to index `last`.
struct Cut {
  float value;
  uint32_t last;
  __device__ __forceinline__ bool has(float x, uint32_t i) const { return x >= value && !(x == value && i > last); }
};

template <int kType, bool kHeld>
struct Row {
  Shared* sh;
  const char* src;     // this CTA's logits in global memory ..
  const float* x;      // .. and, where they are held, in shared memory
  int slice, n;        // their number, rounded up to whole steps, and as it is
  uint32_t base, rank, size;
  RowScale rs;
  f32x2 nz;
  bool infinite;       // the row's maximum is infinite: it is read as 0, all else as -inf
  int buf;
  int lo;              // elements of the first four that lie before the row (see sample_kernel)

  static constexpr int kElem = kType == W8A8_TYPE_F32 ? 4 : 2;
  // logits i .. i + 3 of the slice, -inf before the row and behind its end (no comparison below takes a NaN, and -0 is equal to 0 in all of
  // them)
  __device__ __forceinline__ float4 raw4(int i) const {
    float f[4];
    if (i >= lo && i + 4 <= n) {
      if constexpr (kType == W8A8_TYPE_F32) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(src) + i / 4);
        f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
      } else {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(src) + i / 4);
        const float2 a = unpack2<kType == W8A8_TYPE_BF16>(w.x), b = unpack2<kType == W8A8_TYPE_BF16>(w.y);
        f[0] = a.x, f[1] = a.y, f[2] = b.x, f[3] = b.y;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[e] = -INFINITY;
        if (i + e >= lo && i + e < n) {
          if constexpr (kType == W8A8_TYPE_F32)
            f[e] = __ldg(reinterpret_cast<const float*>(src) + i + e);
          else
            f[e] = unpack2<kType == W8A8_TYPE_BF16>(__ldg(reinterpret_cast<const uint16_t*>(src) + i + e)).x;
        }
      }
    }
    return make_float4(f[0], f[1], f[2], f[3]);
  }
  __device__ __forceinline__ float4 at4(int i) const {
    if constexpr (kHeld) return *reinterpret_cast<const float4*>(x + i);
    float4 v = raw4(i);
    if (infinite)
      v = make_float4(v.x == INFINITY ? 0.0f : -INFINITY, v.y == INFINITY ? 0.0f : -INFINITY,
                      v.z == INFINITY ? 0.0f : -INFINITY, v.w == INFINITY ? 0.0f : -INFINITY);
    return v;
  }

  __device__ __forceinline__ float at(int i) const {
    const float4 v = at4(i & ~3);
    return (i & 2) ? (i & 1) ? v.w : v.z : (i & 1) ? v.y : v.x;
  }

  // (a, b) of every CTA, given by thread 0 .. size - 1 of each; one cluster barrier
  __device__ __forceinline__ const u64 (*tell(u64 a, u64 b))[2] {
    u64(*slot)[2] = sh->ex[buf];
    buf ^= 1;
    if (threadIdx.x < size) {
      const uint32_t to = map_to_rank(smem_u32(&slot[rank][0]), threadIdx.x);
      st_remote(to, a);
      st_remote(to + 8, b);
    }
    cluster_sync_all();
    return slot;
  }
  // the block's sum, for every thread
  __device__ __forceinline__ u64 block_sum(u64 a) {
    a = warp_sum(a);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh->red[threadIdx.x >> 5][0] = a;
    __syncthreads();
    a = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) a += sh->red[w][0];
    return a;
  }
  // f(value, index) over the slice, each warp over a stretch of its own
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = slice / kWarps;
#pragma unroll 4
    for (int i = warp * part + 4 * lane; i < (warp + 1) * part; i += 128) {
      const float4 v = at4(i);
      f(v.x, base + i);
      f(v.y, base + i + 1);
      f(v.z, base + i + 2);
      f(v.w, base + i + 3);
    }
  }
  // f(value, index, weight) for those that pred(value, index) takes and that weigh anything
  template <class P, class F>
  __device__ __forceinline__ void each_weight(P pred, F f) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = slice / kWarps;
#pragma unroll 2
    for (int i = warp * part + 4 * lane; i < (warp + 1) * part; i += 128) {
      const float4 v = at4(i);
      const float l[4] = {v.x, v.y, v.z, v.w};
      bool in[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) in[e] = l[e] >= rs.low && pred(l[e], base + i + e);
      if (!(in[0] || in[1] || in[2] || in[3])) continue;
      u64 w[4];
      weights_of(rs, sh->table, nz, l[0], l[1], w[0], w[1]);
      weights_of(rs, sh->table, nz, l[2], l[3], w[2], w[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (in[e]) f(l[e], base + i + e, w[e]);
    }
  }
  __device__ __forceinline__ u64 weight(float l) const {
    u64 a, b;
    weights_of(rs, sh->table, nz, l, l, a, b);
    return a;
  }
  __device__ __forceinline__ u64 significand(float l) const {
    uint32_t v, v1, i0, i1;
    parts_of(rs, sh->table, nz, l, l, v, v1, i0, i1);
    return v;
  }
  __device__ __forceinline__ void clear() {
    for (int i = threadIdx.x; i < kBins; i += kT) sh->count[i] = sh->lo[i] = sh->hi[i] = 0;
    __syncthreads();
  }
  __device__ __forceinline__ uint32_t bin_of(float x) const { return bin_of_steps((uint32_t)steps_of(rs, x)); }
  // the logits that pred takes, and that may weigh anything, with their weights into the histogram
  template <class P>
  __device__ __forceinline__ void add_weights(P pred) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = slice / kWarps;
#pragma unroll 2
    for (int i = warp * part + 4 * lane; i < (warp + 1) * part; i += 128) {
      const float4 v = at4(i);
      const float l[4] = {v.x, v.y, v.z, v.w};
      uint32_t s[4], b[4];
      parts_of(rs, sh->table, nz, l[0], l[1], s[0], s[1], b[0], b[1]);
      parts_of(rs, sh->table, nz, l[2], l[3], s[2], s[3], b[2], b[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (!(l[e] >= rs.low) || !pred(l[e], base + i + e)) continue;
        const uint32_t bin = bin_of_steps(kRoundBits - b[e]);
        atomicAdd(&sh->count[bin], 1u);
        atomicAdd(&sh->lo[bin], s[e] & 0xffffu);
        atomicAdd(&sh->hi[bin], s[e] >> 16);
      }
    }
  }
  // a bin of the divided range
  __device__ __forceinline__ void add_fine(uint32_t bin, uint32_t v) {
    atomicAdd(&sh->count[bin], 1u);
    atomicAdd(&sh->lo[bin], v & 0xffffu);
    atomicAdd(&sh->hi[bin], v >> 16);
  }
  // significands of a bin's weights, summed, as a weight
  __device__ __forceinline__ u64 significant(u64 v, int bin) const {
    const int up = kFrac - 29 - bin_exponent(bin);
    return up >= 0 ? v << up : v >> -up;
  }
  // The bin of the cluster's histogram at which counts (or weights), c0 and w0 before the first bin, reach goal(all of the
  // weight), or what there is.  The CTAs add up a share of the bins each.  Three cluster barriers; then the histogram may be changed.
  struct Cross {
    uint32_t bin;
    u64 c_above, w_above, c_in, c_all;
  };
  template <bool kFineBins, class Goal>
  __device__ __forceinline__ Cross cross(bool by_weight, u64 c0, u64 w0, Goal goal) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int seg = (kFineBins ? kFine : kBins) / (int)size, first = (int)rank * seg;
    const int parts = 4 * seg <= kT ? 4 : 2 * seg <= kT ? 2 : 1, per = parts > 1 ? 1 : (seg + kT - 1) / kT;  // threads a bin, bins a thread
    auto load = [&](int bin, int part, int n_parts, u64& c, u64& w) {
      u64 lo = 0, hi = 0;
      c = 0;
      for (int r0 = part; r0 < (int)size; r0 += 8 * n_parts) {  // eight CTAs' loads ahead of their first use
        uint32_t got[8][3];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t r = min((uint32_t)(r0 + k * n_parts), size - 1);
          got[k][0] = ld_remote(map_to_rank(smem_u32(&sh->count[bin]), r));
          got[k][1] = by_weight ? ld_remote(map_to_rank(smem_u32(&sh->lo[bin]), r)) : 0u;
          got[k][2] = by_weight ? ld_remote(map_to_rank(smem_u32(&sh->hi[bin]), r)) : 0u;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (r0 + k * n_parts < (int)size) {
            c += got[k][0];
            lo += got[k][1];
            hi += got[k][2];
          }
      }
      w = (hi << 16) + lo;
    };
    cluster_sync_all();  // every CTA's histogram is complete
    const int mine = tid / parts * per;
    const uint32_t lanes = __ballot_sync(0xffffffffu, mine < seg);  // that share bins below (one bin a thread where they do)
    u64 cs = 0, ws = 0;
    if (mine < seg)
      for (int i = 0; i < per && mine + i < seg; ++i) {
        u64 c, w;
        load(first + mine + i, tid % parts, parts, c, w);
        for (int o = 1; o < parts; o <<= 1) {
          c += __shfl_xor_sync(lanes, c, o);
          w += __shfl_xor_sync(lanes, w, o);
        }
        if (tid % parts) continue;
        cs += c;
        ws += kFineBins ? w : significant(w, first + mine + i);
      }
    u64 cu = warp_scan(cs, lane), wu = warp_scan(ws, lane), ct = 0, wt = 0;
    __syncthreads();
    if (lane == 31) {
      sh->red[warp][0] = cu;
      sh->red[warp][1] = wu;
    }
    __syncthreads();
    cu -= cs;
    wu -= ws;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      if (i < warp) {
        cu += sh->red[i][0];
        wu += sh->red[i][1];
      }
      ct += sh->red[i][0];
      wt += sh->red[i][1];
    }
    const u64(*all)[2] = tell(ct, wt);
    cu += c0;
    wu += w0;
    ct = c0;
    wt = w0;
    for (uint32_t r = 0; r < size; ++r) {
      if (r < rank) {
        cu += all[r][0];
        wu += all[r][1];
      }
      ct += all[r][0];
      wt += all[r][1];
    }
    const u64 g = min(goal(wt), by_weight ? wt : ct);
    if (by_weight ? wu < g && wu + ws >= g : cu < g && cu + cs >= g) {  // within this thread's bins
      u64 c = 0, w = 0;
      int bin = first + mine;
      for (;; ++bin) {
        load(bin, 0, 1, c, w);
        if (!kFineBins) w = significant(w, bin);
        if (by_weight ? wu + w >= g : cu + c >= g) break;
        cu += c;
        wu += w;
      }
      const u64 v[4] = {(u64)bin, cu, wu, c};
      for (uint32_t r = 0; r < size; ++r)
#pragma unroll
        for (int k = 0; k < 4; ++k) st_remote(map_to_rank(smem_u32(&sh->res[k]), r), v[k]);
    }
    cluster_sync_all();
    return Cross{(uint32_t)sh->res[0], sh->res[1], sh->res[2], sh->res[3], ct};
  }

  // The index of the slice at which the sum of f(value, index), `before` ahead of the slice and red[w][0] over warp w's stretch,
  // passes `target`, and f there; for the CTA that has it.  The warps divide the stretch once more, then a warp's lanes.
  template <class F>
  __device__ __forceinline__ void find(u64 before, u64 target, F f, int& index, u64& value) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = slice / kWarps, sub = part / kWarps;
    int w = 0;
    for (; w < kWarps - 1 && before + sh->red[w][0] <= target; ++w) before += sh->red[w][0];
    u64 sum = 0;
    const int start = w * part + warp * sub;
    for (int i = lane; i < sub; i += 32) sum += f(at(start + i), base + start + i);
    sum = warp_sum(sum);
    if (lane == 0) sh->red[warp][1] = sum;
    __syncthreads();
    int v = 0;
    for (; v < kWarps - 1 && before + sh->red[v][1] <= target; ++v) before += sh->red[v][1];
    if (warp != v) return;
    const int per = (sub + 31) / 32;
    sum = 0;
    for (int i = lane * per; i < min(sub, lane * per + per); ++i) sum += f(at(start + i), base + start + i);
    u64 upto = before + warp_scan(sum, lane);
    if (upto <= target || upto - sum > target) return;
    upto -= sum;
    for (int i = lane * per; i < min(sub, lane * per + per); ++i) {
      value = f(at(start + i), base + start + i);
      upto += value;
      if (upto > target) {
        index = start + i;
        return;
      }
    }
  }

};

struct Found {
  Cut cut;
  bool done;  // the cut by weight is in it
};

// Where the kept tokens end, among those of `in`: the first k (by_weight false), or the shortest prefix that weighs p of them.
// Where the candidates of a cut by count are few, the cut by weight is made with it.
template <int kType, bool kHeld>
__device__ __forceinline__ Found find_cut(Row<kType, kHeld>& row, const Cut in, bool by_weight, int k, float p) {
  Shared* sh = row.sh;
  const RowScale& rs = row.rs;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  u64 want = 0;
  row.clear();
  if (by_weight)
    row.add_weights([&](float x, uint32_t i) { return in.has(x, i); });
  else
    row.each([&](float x, uint32_t) {
      if (x >= rs.low) atomicAdd(&sh->count[row.bin_of(x)], 1u);
    });
  typename Row<kType, kHeld>::Cross c = row.template cross<false>(
      by_weight, 0, 0, [&](u64 w_all) { return want = by_weight ? max(scaled(p, w_all, true), 1ull) : (u64)k; });
  if (!by_weight && c.c_all <= want) return Found{in, false};  // no more than k weigh anything
  const uint32_t bin = c.bin;
  u64 c_above = c.c_above, v_above = 0;
  if (by_weight) {  // from here on in sums of the bin's significands: the least whose weight reaches the rest
    const int up = kFrac - 29 - bin_exponent((int)bin);
    const u64 rest = want - c.w_above;
    want = up >= 0 ? (rest + (1ull << up) - 1) >> up : rest << -up;
  }

  // with few tokens down to the bin's end, all of them are sorted, and both cuts made
  const bool both = !by_weight && c_above + c.c_in <= kSmall;
  if (both || c.c_in <= kSmall) {
    // ---- few: one CTA sorts them (largest logit first, then lowest index) and cuts exactly.  Each CTA's in its own shared
    // memory first, then in one go behind the others'
    const float from = __uint_as_float(kRoundBits - 2 * bin);  // the bin's two steps
    const float to = both || bin == 0 ? kRound : __uint_as_float(kRoundBits - 2 * bin + 1);
    row.each([&](float x, uint32_t i) {
      const float s = rounded(rs, x);
      if (s >= from && s <= to && x >= rs.low && in.has(x, i))
        sh->mine[atomicAdd(&sh->n_mine, 1u)] = ((u64)float_order_key(x) << 32) | (uint32_t)~i;
    });
    __syncthreads();
    const uint32_t n_mine = sh->n_mine;
    if (tid == 0 && n_mine) sh->n_before = add_remote(map_to_rank(smem_u32(&sh->listed), 0), n_mine);
    __syncthreads();
    const uint32_t list0 = map_to_rank(smem_u32(sh->list), 0) + 8 * sh->n_before;
    for (uint32_t i = tid; i < n_mine; i += kT) st_remote(list0 + 8 * i, sh->mine[i]);
    if (tid == 0) sh->n_mine = 0;
    cluster_sync_all();
    if (row.rank == 0) {
      u64* list = sh->list;
      const int n = (int)sh->listed;
      if (n <= kT / 2) {  // each token's place is the number of greater ones: two threads a token
        const int i = tid >> 1;
        const u64 v = i < n ? list[i] : 0;
        int place = 0;
        for (int j = tid & 1; j < n; j += 2) place += list[j] > v;
        place += __shfl_xor_sync(0xffffffffu, place, 1);
        if (i < n && (tid & 1) == 0) sh->mine[place] = v;
        list = sh->mine;
        __syncthreads();
      } else {
        int n2 = kT;
        while (n2 < n) n2 <<= 1;
        for (int i = n + tid; i < n2; i += kT) list[i] = 0;
        __syncthreads();
        for (int len = 2; len <= n2; len <<= 1)
          for (int j = len >> 1; j > 0; j >>= 1) {
            for (int i = tid; i < n2 / 2; i += kT) {
              const int a = 2 * i - (i & (j - 1)), b = a + j;
              const u64 u = list[a], v = list[b];
              if ((u < v) == ((a & len) == 0)) {
                list[a] = v;
                list[b] = u;
              }
            }
            __syncthreads();
          }
      }
      if (tid == 0) sh->listed = 0;
      if (!by_weight && !both) {
        if (tid == 0) sh->res[0] = list[want - c_above - 1];
      } else {
        // by weight: the significands of the one bin; else weights
        const int m = by_weight || k > n ? n : k;
        u64 w[2], mine = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          w[i] = 0;
          if (2 * tid + i < m) {
            const float l = order_value((uint32_t)(list[2 * tid + i] >> 32));
            w[i] = by_weight ? row.significand(l) : row.weight(l);
          }
          mine += w[i];
        }
        u64 before = warp_scan(mine, lane);
        if (lane == 31) sh->red[warp][0] = before;
        __syncthreads();
        before -= mine;
        u64 total = 0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
          if (i < warp) before += sh->red[i][0];
          total += sh->red[i][0];
        }
        const u64 target = by_weight ? want : p < 1.0f ? max(scaled(p, total, true), 1ull) : ~0ull;
#pragma unroll
        for (int i = 0; i < 2; ++i) {  // the last one kept: where the sum reaches the target, or the last of the m
          const int at = 2 * tid + i;
          if (at < m && before < target && (before + w[i] >= target || at == m - 1)) sh->res[0] = list[at];
          before += w[i];
        }
      }
      __syncthreads();
    }
    const u64(*told)[2] = row.tell(sh->res[0], 0);
    return Found{Cut{order_value((uint32_t)(told[0][0] >> 32)), ~(uint32_t)told[0][0]}, by_weight || both};
  }

  // ---- many: divide the range by the order of its floats
  uint32_t kmin = 0xffffffffu, kmax = 0;
  row.each([&](float x, uint32_t i) {
    if (x >= rs.low && row.bin_of(x) == bin && in.has(x, i)) {
      kmin = min(kmin, float_order_key(x));
      kmax = max(kmax, float_order_key(x));
    }
  });
  kmin = __reduce_min_sync(0xffffffffu, kmin);
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  __syncthreads();
  if (lane == 0) sh->red[warp][1] = ((u64)kmin << 32) | kmax;
  __syncthreads();
  auto fold = [&](u64 v) {
    kmin = min(kmin, (uint32_t)(v >> 32));
    kmax = max(kmax, (uint32_t)v);
  };
  for (int i = 0; i < kWarps; ++i) fold(sh->red[i][1]);
  const u64(*ends)[2] = row.tell(((u64)kmin << 32) | kmax, 0);
  for (uint32_t r = 0; r < row.size; ++r) fold(ends[r][0]);
  do {
    const int s = max(0, 32 - __clz((int)(kmax - kmin)) - 11);
    row.clear();
    row.each([&](float x, uint32_t i) {
      const uint32_t key = float_order_key(x);
      if (x >= rs.low && key >= kmin && key <= kmax && in.has(x, i)) row.add_fine((kmax - key) >> s, by_weight ? (uint32_t)row.significand(x) : 0u);
    });
    c = row.template cross<true>(by_weight, c_above, v_above, [&](u64) { return want; });
    c_above = c.c_above;
    v_above = c.w_above;
    const uint32_t top = kmax - (c.bin << s);
    kmin = (1u << s) - 1u >= top - kmin ? kmin : top - ((1u << s) - 1u);
    kmax = top;
  } while (kmin < kmax);
  // ---- one value is left: as many of its equals as it takes, the lower indices first
  const float value = order_value(kmax);
  const u64 one = row.significand(value);
  const u64 ties = min(by_weight ? (want - v_above + one - 1) / one : want - c_above, c.c_in);
  Found f{Cut{value, in.value == value ? in.last : 0xffffffffu}, by_weight};
  if (ties == c.c_in) return f;
  u64 eq = 0;
  row.each([&](float x, uint32_t) { eq += x == value; });
  const u64 csum = row.block_sum(eq);
  const u64(*counts)[2] = row.tell(csum, 0);
  u64 before = 0;
  for (uint32_t r = 0; r < row.rank; ++r) before += counts[r][0];
  if (before < ties && before + csum >= ties) {  // this CTA holds the last of them
    int index = -1;
    u64 v;
    row.find(before, ties - 1, [&](float x, uint32_t) -> u64 { return x == value; }, index, v);
    if (index >= 0)
      for (uint32_t r = 0; r < row.size; ++r) st_remote(map_to_rank(smem_u32(&sh->res[5]), r), row.base + index);
  }
  cluster_sync_all();
  f.cut.last = (uint32_t)sh->res[5];
  return f;
}

template <int kType, bool kHeld>
__global__ void __launch_bounds__(kT, 2) sample_kernel(const void* logits, int64_t row_stride, int V, int slice, w8a8_sampling sp,
                                                       const float* __restrict__ u, int32_t* __restrict__ tokens,
                                                       float* __restrict__ probs) {
  extern __shared__ __align__(16) float xs[];
  __shared__ Shared sh;
  uint32_t rank, size;
  asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;\n" : "=r"(size));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / size;
  asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");  // waited for after the load
  if (tid < 128) sh.table[tid] = kTable.e[tid];
  if (tid == 0) sh.listed = sh.n_mine = 0;
  pdl_wait();
  pdl_trigger();
  const uint32_t base = rank * (uint32_t)slice;
  // A row may begin anywhere: its logits are counted from the four-element boundary at or before it, `skew` elements on (whose
  // values are not read), so that all loads but those at the ends are of four.
  constexpr int kElem = Row<kType, kHeld>::kElem;
  const char* from = static_cast<const char*>(logits) + (int64_t)row * row_stride * kElem;
  const int skew = (int)(reinterpret_cast<uintptr_t>(from) / kElem & 3u);
  Row<kType, kHeld> rw{&sh, from + ((int64_t)base - skew) * kElem, xs, slice, min(slice, max(0, V + skew - (int)base)), base, rank,
                       size, {}, f2_neg_zero(), false, 0, rank == 0 ? skew : 0};
  const float temp = sp.temperature ? sp.temperature[row] : 1.0f;
  const int k = sp.top_k ? sp.top_k[row] : 0;
  const float top_p = sp.top_p ? sp.top_p[row] : 1.0f, min_p = sp.min_p ? sp.min_p[row] : 0.0f;

  // ---- the slice's maximum and least finite value
  float mx = -INFINITY, mn = INFINITY;
  uint32_t at = 0;
#pragma unroll 8
  for (int i = 4 * tid; i < slice; i += 4 * kT) {
    const float4 v = rw.raw4(i);
    const float f[4] = {v.x, v.y, v.z, v.w};
    if constexpr (kHeld) *reinterpret_cast<float4*>(xs + i) = v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (f[e] > mx) {  // indices ascend: the first of equals stays
        mx = f[e];
        at = base + i + e;
      }
      if (f[e] > -INFINITY) mn = fminf(mn, f[e]);
    }
  }
  u64 best = ((u64)float_order_key(mx) << 32) | (uint32_t)~at;
  uint32_t least_key = float_order_key(mn);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
  least_key = __reduce_min_sync(0xffffffffu, least_key);
  if (lane == 0) {
    sh.red[warp][0] = best;
    sh.red[warp][1] = least_key;
  }
  __syncthreads();
  for (int i = 0; i < kWarps; ++i) {
    best = max(best, sh.red[i][0]);
    least_key = min(least_key, (uint32_t)sh.red[i][1]);
  }
  // the peers run: their shared memory may be written
  asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
  const u64(*tops)[2] = rw.tell(best, least_key);
  for (uint32_t r = 0; r < size; ++r) {
    best = max(best, tops[r][0]);
    least_key = min(least_key, (uint32_t)tops[r][1]);
  }
  mx = order_value((uint32_t)(best >> 32));
  mn = order_value(least_key);
  if (mx == -INFINITY || !(temp > 0.0f)) {
    if (rank == 0 && tid == 0) {
      tokens[row] = mx == -INFINITY ? -1 : (int32_t)(~(uint32_t)best - (uint32_t)skew);
      if (probs) probs[row] = mx == -INFINITY ? 0.0f : 1.0f;
    }
    return;
  }
  if (mx == INFINITY) {  // infinities share the weight: a row of zeros in their places
    rw.infinite = true;
    if constexpr (kHeld) {
      for (int i = tid; i < slice; i += kT) xs[i] = xs[i] == INFINITY ? 0.0f : -INFINITY;
      __syncthreads();
    }
    mx = mn = 0.0f;
  }
  rw.rs = row_scale(mx, mn, temp);
  Cut cut{-INFINITY, 0xffffffffu};
  // by count, then by weight (one call in a loop, so that it is compiled once, in place)
  for (int by_weight = k > 0 && k < V ? 0 : 1; by_weight < (top_p < 1.0f ? 2 : 1); ++by_weight) {
    const Found f = find_cut(rw, cut, by_weight != 0, k, top_p);
    cut = f.cut;
    if (f.done) break;
  }

  // ---- the kept weights, and the token
  const u64 least = !(min_p > 0.0f) ? 0ull : min_p >= 1.0f ? 1ull << kFrac : scaled(min_p, 1ull << kFrac, true);
  u64 mine = 0;
  if (least)
    rw.each_weight([&](float x, uint32_t i) { return cut.has(x, i); },
                   [&](float x, uint32_t, u64 w) { mine += w >= least || x == mx ? w : 0ull; });
  else
    rw.each_weight([&](float x, uint32_t i) { return cut.has(x, i); }, [&](float, uint32_t, u64 w) { mine += w; });
  mine = rw.block_sum(mine);
  const u64(*sums)[2] = rw.tell(mine, 0);
  u64 total = 0, before = 0;
  for (uint32_t r = 0; r < size; ++r) {
    if (r < rank) before += sums[r][0];
    total += sums[r][0];
  }
  float uu = u[row];
  uu = uu >= 0.0f ? fminf(uu, 0x1.fffffep-1f) : 0.0f;
  const u64 target = scaled(uu, total, false);
  if (!(target >= before && target < before + mine)) return;  // another CTA's
  int index = -1;
  u64 w;
  rw.find(before, target,
          [&](float x, uint32_t i) -> u64 {
            if (!(x >= rw.rs.low) || !cut.has(x, i)) return 0;
            const u64 v = rw.weight(x);
            return v >= least || x == mx ? v : 0;
          },
          index, w);
  if (index >= 0) {
    tokens[row] = (int32_t)(base + index) - skew;
    if (probs) probs[row] = (float)((double)w / (double)total);
  }
}

template <int kType, bool kHeld>
w8a8_status launch(int size, int slice, const void* logits, int64_t row_stride, int M, int V, const w8a8_sampling& sp,
                   const float* u, int32_t* tokens, float* probs, cudaStream_t st) {
  static bool attr_set[64] = {};
  int dev = 0;
  W8A8_CUDA(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64 && !attr_set[dev]) {
    if (kHeld)
      W8A8_CUDA(cudaFuncSetAttribute(sample_kernel<kType, kHeld>, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeldSlice * 4));
    W8A8_CUDA(cudaFuncSetAttribute(sample_kernel<kType, kHeld>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    attr_set[dev] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(M * size));
  cfg.blockDim = dim3(kT);
  cfg.dynamicSmemBytes = kHeld ? (size_t)slice * 4 : 0;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)size;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  W8A8_CUDA(cudaLaunchKernelEx(&cfg, sample_kernel<kType, kHeld>, logits, row_stride, V, slice, sp, u, tokens, probs));
  return W8A8_OK;
}

}  // namespace

w8a8_status launch_sample(int dtype, const void* logits, int64_t row_stride, int M, int V, const w8a8_sampling& sp,
                          const float* u, int32_t* tokens, float* probs, int sms, cudaStream_t st) {
  // CTAs a row: as many as all rows' clusters can run at once (two CTAs an SM; clusters of 16 and 8 leave some SMs of a GPC
  // unused, and with a slice in shared memory one CTA fills an SM), down to one step a warp and up to the longest slice
  int size = kMaxCluster;
  const int elem = dtype == W8A8_TYPE_F32 ? 4 : 2;
  const int all = V + (reinterpret_cast<uintptr_t>(logits) / elem % 4 || (M > 1 && row_stride % 4) ? 3 : 0);  // rows that begin anywhere
  auto slice_of = [&](int n) { return (((all + n - 1) / n) + kUnit - 1) / kUnit * kUnit; };
  auto room = [&](int n) { return n == 16 ? 3 * sms / 4 : n == 8 ? 15 * sms / 8 : 2 * sms; };
  while (size > 1 && ((long long)M * size > room(size) || slice_of(size) == slice_of(size / 2)) &&
         slice_of(size / 2) <= kMostSlice)
    size /= 2;
  const int slice = slice_of(size);
  auto go = [&](auto type) {
    constexpr int kType = decltype(type)::value;
    const bool held = slice <= kHeldSlice && (4 * slice <= 3 * kHeldSlice || (long long)M * size <= room(16));
    return held ? launch<kType, true>(size, slice, logits, row_stride, M, V, sp, u, tokens, probs, st)
                               : launch<kType, false>(size, slice, logits, row_stride, M, V, sp, u, tokens, probs, st);
  };
  return dtype == W8A8_TYPE_F32    ? go(std::integral_constant<int, W8A8_TYPE_F32>())
         : dtype == W8A8_TYPE_BF16 ? go(std::integral_constant<int, W8A8_TYPE_BF16>())
                                   : go(std::integral_constant<int, W8A8_TYPE_F16>());
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
  const uintptr_t elem = dtype == W8A8_TYPE_F32 ? 4 : 2, at = reinterpret_cast<uintptr_t>(logits);
  W8A8_CHECK_ARG(row_stride >= 0 && row_stride <= (1ll << 40), W8A8_ERR_SHAPE, "%s: row stride %lld", who, (long long)row_stride);
  W8A8_CHECK_ARG(at % elem == 0, W8A8_ERR_ALIGN, "%s: logits must be aligned to their type", who);
  W8A8_CHECK_ARG(V <= W8A8_MAX_SAMPLE_VOCAB - 3 || (at / elem % 4 == 0 && (M == 1 || row_stride % 4 == 0)), W8A8_ERR_SHAPE,
                 "%s: V=%d exceeds %d, the most where rows do not begin at multiples of four elements", who, V,
                 W8A8_MAX_SAMPLE_VOCAB - 3);
  const void* words[] = {sampling->temperature, sampling->top_k, sampling->top_p, sampling->min_p, u, tokens, probs};
  for (const void* p : words)
    W8A8_CHECK_ARG((reinterpret_cast<uintptr_t>(p) & 3u) == 0, W8A8_ERR_ALIGN, "%s: arrays must be 4-byte aligned", who);
  W8A8_CHECK_ARG(M <= 1 << 24, W8A8_ERR_SHAPE, "%s: M=%d rows", who, M);
  DevInfo d;
  W8A8_TRY(dev_info(&d));
  return launch_sample(dtype, logits, row_stride, M, V, *sampling, u, tokens, probs, d.sms, as_stream(stream));
}
