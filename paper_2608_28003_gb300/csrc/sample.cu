// Sampling of one token a row by temperature, top-k, top-p and min-p, from a given uniform number.
//
// The mathematics.  Weights are e^((l - max) / T) as multiples of 2^-43 in 64-bit integers, so that sums of up to
// 2^20 of them are exact and depend on no order: every comparison that decides a token is one of integers.  An fp32
// exponential would not do: a flat row of 262144 logits has steps of 2^-18 in the sum, and weights off by 2^-24
// or, far from the maximum, by 2^-19 would move the token in a noticeable share of draws.  So logits become 32-bit fixed-point
// numbers over the range that has any weight (exact for all but those near zero), their distance D to the maximum is
// multiplied by log2(e) / T in 64 bits, and 2^-y comes from a table of 128 values and a cubic, all in integers: about 2^-28 of the
// weight at worst, and 23 instructions.
//
// The work.  A cluster of up to 16 CTAs holds a row in shared memory (one read of HBM) and goes over it there: the maximum;
// then, where a filter needs it, a histogram of counts and weights over 2048 bins of D, whose crossing bin bounds the cut.
// If at most kSmall tokens lie above the bin's end, one CTA sorts them and finds the cut; else the bin is divided again, by the
// order of its floats, until one value is left, whose equals are cut by index.  The last pass sums the kept weights and finds
// the token in index order.  A row of 262144 in fp32 is 64 KB a CTA, two CTAs an SM.
#include <cmath>

#include "ops.cuh"

namespace w8a8 {

namespace {

typedef unsigned long long u64;

constexpr int kT = 512, kWarps = kT / 32;
constexpr int kFrac = 43;     // weights are multiples of 2^-43 of the largest
constexpr int kBins = 2048, kSmall = 1024;
constexpr int kMaxCluster = 16;
constexpr int kUnit = 4 * 32 * kWarps;      // a CTA's slice is a multiple: 128 logits a warp and step
constexpr int kMaxSlice = 24 * kUnit;       // 192 KB of shared memory
static_assert(kMaxSlice * kMaxCluster >= W8A8_MAX_SAMPLE_VOCAB, "a cluster holds the largest row");

// ------------------------------------------------------------------------------------ weights
struct RowScale {
  float low;         // logits below weigh nothing
  float scale;       // 2^(31 - e): logits as 32-bit integers
  int top;           // the maximum's
  u64 c;             // log2(e) / T per unit of them, times 2^(64 + shift)
  int shift;         // 0 .. 31
};
__device__ __forceinline__ RowScale row_scale(float mx, float least, float temperature) {
  RowScale r;
  const double c = 1.4426950408889634074 / (double)fmaxf(temperature, 1e-30f);
  r.low = mx == INFINITY ? INFINITY : fmaxf(__double2float_rd((double)mx - (kFrac + 1) / c), least);
  const float a = fmaxf(fabsf(mx), fabsf(r.low));
  int e = a == INFINITY ? 31 : max(ilogbf(fmaxf(a, 1e-37f)) + 1, -95);
  r.scale = scalbnf(1.0f, 31 - e);
  r.top = __float2int_rn(mx * r.scale);
  int k;
  const double m = frexp(ldexp(c, e - 31), &k);
  r.c = (u64)(m * 18446744073709551616.0);
  if (k > 0) {  // one unit is more than the whole range: only the maximum weighs
    r.c = ~0ull;
    k = 0;
  }
  if (k < -31) {
    r.c = -31 - k > 63 ? 0ull : r.c >> (-31 - k);
    k = -31;
  }
  if (mx == INFINITY) r.c = 0;
  r.shift = -k;
  return r;
}
// Distance to the maximum in the row's units (l >= low).
__device__ __forceinline__ uint32_t distance(const RowScale& r, float l) {
  return (uint32_t)r.top - (uint32_t)__float2int_rn(l * r.scale);
}
// 2^43 e^((l - max) / T) truncated; 0 below `low` (and for NaN).  `table`: 2^(31 - j / 128).
__device__ __forceinline__ u64 weight_of(const RowScale& r, const uint32_t* table, float l) {
  const uint32_t d = distance(r, l);
  const u64 y = (u64)d * (uint32_t)(r.c >> 32) + __umulhi(d, (uint32_t)r.c);  // exponent, 32 + shift fraction bits
  const uint32_t n = (uint32_t)(y >> 32) >> r.shift, f = __funnelshift_r((uint32_t)y, (uint32_t)(y >> 32), r.shift);
  const uint32_t t = table[f >> 25], x = f & 0x1ffffffu;  // 2^-f = 2^-(j / 128) 2^-x, x < 1/128 in units of 2^-32
  constexpr double ln2 = 0.69314718055994530942, one = 4294967296.0;
  constexpr uint32_t c1 = (uint32_t)(ln2 * one), c2 = (uint32_t)(ln2 * ln2 / 2 * one), c3 = (uint32_t)(ln2 * ln2 * ln2 / 6 * one);
  // 1 - 2^-x = x ln2 - (x ln2)^2 / 2 + (x ln2)^3 / 6 - .. (the next term is below 2^-34)
  const uint32_t q = __umulhi(x, c1 - __umulhi(x, c2 - __umulhi(x, c3)));
  const uint32_t v = t - __umulhi(t, q);
  return l >= r.low && n <= kFrac ? ((u64)v << 32) >> (63 - kFrac + n) : 0ull;
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
  uint32_t count[kBins], lo[kBins], hi[kBins];  // the histogram; at other times the list of candidates
  uint32_t table[128];
  u64 ex[2][kMaxCluster][2];                    // what the CTAs tell one another: a pair of numbers each
  u64 res[6];                                   // and what one of them found
  u64 red[kWarps][2];
  uint32_t listed;
};

// What the tokens kept so far are: those above `value`, and its equals up to index `last`.
struct Cut {
  float value;
  uint32_t last;
  __device__ __forceinline__ bool has(float x, uint32_t i) const { return x > value || (x == value && i <= last); }
};

struct Row {
  Shared* sh;
  const float* x;      // this CTA's slice
  int slice;
  uint32_t base, rank, size;
  int buf = 0;

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
  // the block's sums of a and b, for every thread
  __device__ __forceinline__ void block_sum(u64& a, u64& b) {
    a = warp_sum(a);
    b = warp_sum(b);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) {
      sh->red[threadIdx.x >> 5][0] = a;
      sh->red[threadIdx.x >> 5][1] = b;
    }
    __syncthreads();
    a = b = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      a += sh->red[w][0];
      b += sh->red[w][1];
    }
  }
  // f(value, index) over the slice, each warp over a stretch of its own
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = slice / kWarps;
    for (int i = warp * part + 4 * lane; i < (warp + 1) * part; i += 128) {
      const float4 v = *reinterpret_cast<const float4*>(x + i);
      f(v.x, base + i);
      f(v.y, base + i + 1);
      f(v.z, base + i + 2);
      f(v.w, base + i + 3);
    }
  }
  __device__ __forceinline__ void clear() {
    for (int i = threadIdx.x; i < kBins; i += kT) sh->count[i] = sh->lo[i] = sh->hi[i] = 0;
    __syncthreads();
  }
  __device__ __forceinline__ void add(uint32_t bin, u64 w) {
    atomicAdd(&sh->count[bin], 1u);
    const uint32_t lo = (uint32_t)w, old = atomicAdd(&sh->lo[bin], lo);
    const uint32_t up = (uint32_t)(w >> 32) + (old + lo < lo ? 1u : 0u);
    if (up) atomicAdd(&sh->hi[bin], up);
  }

  // The bin of the cluster's histogram at which counts (or weights) above it, `c0` and `w0` before the first bin, reach the
  // goal.  goal(total count, total weight) gives it.  Three cluster barriers.
  struct Cross {
    uint32_t bin;
    u64 c_above, w_above, c_in, w_in, c_all, w_all;
  };
  template <class Goal>
  __device__ __forceinline__ Cross cross(bool by_weight, u64 c0, u64 w0, Goal goal) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int seg = kBins / (int)size, per = (seg + kT - 1) / kT, first = (int)rank * seg;
    cluster_sync_all();  // every CTA's histogram is complete
    u64 c[4], w[4], cs = 0, ws = 0;  // this thread's bins (up to 4 where one CTA has them all)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      c[i] = w[i] = 0;
      const int b = tid * per + i;
      if (i < per && b < seg)
        for (uint32_t r = 0; r < size; ++r) {
          const uint32_t at = map_to_rank(smem_u32(sh->count) + 4u * (uint32_t)(first + b), r);
          c[i] += ld_remote(at);
          w[i] += ((u64)ld_remote(at + 8 * kBins) << 32) + ld_remote(at + 4 * kBins);
        }
      cs += c[i];
      ws += w[i];
    }
    u64 cb = warp_scan(cs, lane), wb = warp_scan(ws, lane);
    __syncthreads();
    if (lane == 31) {
      sh->red[warp][0] = cb;
      sh->red[warp][1] = wb;
    }
    __syncthreads();
    cb -= cs;
    wb -= ws;
    u64 cseg = 0, wseg = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      if (i < warp) {
        cb += sh->red[i][0];
        wb += sh->red[i][1];
      }
      cseg += sh->red[i][0];
      wseg += sh->red[i][1];
    }
    const u64(*all)[2] = tell(cseg, wseg);
    u64 ct = c0, wt = w0;
    cb += c0;
    wb += w0;
    for (uint32_t r = 0; r < size; ++r) {
      if (r < rank) {
        cb += all[r][0];
        wb += all[r][1];
      }
      ct += all[r][0];
      wt += all[r][1];
    }
    const u64 g = goal(ct, wt);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (by_weight ? wb < g && wb + w[i] >= g : cb < g && cb + c[i] >= g) {
        const u64 v[5] = {(u64)(first + tid * per + i), cb, wb, c[i], w[i]};
        for (uint32_t r = 0; r < size; ++r)
#pragma unroll
          for (int k = 0; k < 5; ++k) st_remote(map_to_rank(smem_u32(&sh->res[k]), r), v[k]);
      }
      cb += c[i];
      wb += w[i];
    }
    cluster_sync_all();
    return Cross{(uint32_t)sh->res[0], sh->res[1], sh->res[2], sh->res[3], sh->res[4], ct, wt};
  }
};

struct Found {
  Cut cut;
  u64 weight;  // of the kept tokens
};

// Where the kept tokens end, among those of `in`: the first top_k (by_weight false: goal tokens), or the shortest prefix that
// weighs share of the weight of `in` (`all`, or with all == 0 what the first histogram finds).  With `both`, a cut by count is
// followed by the one by weight where the candidates are few.
struct Filters {
  int k;
  float p;
};

template <class Weight>
__device__ Found find_cut(Row& row, const RowScale& rs, const Weight& weight, const Cut in, bool by_weight, u64 known_all,
                          const Filters fl, bool& done) {
  Shared* sh = row.sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t far = distance(rs, rs.low);
  const int sh1 = max(0, 32 - __clz((int)(far | 1u)) - 11);  // far >> sh1 < 2048; the last bin is for what weighs nothing
  auto bin_of = [&](float x) { return x >= rs.low ? min(distance(rs, x) >> sh1, (uint32_t)kBins - 2) : (uint32_t)kBins - 1; };
  auto goal = [&](u64, u64 w_all) {
    return by_weight ? max(scaled(fl.p, known_all ? known_all : w_all, true), 1ull) : (u64)fl.k;
  };
  row.clear();
  row.each([&](float x, uint32_t i) {
    if (in.has(x, i) && (!by_weight || x >= rs.low)) row.add(bin_of(x), weight(x));
  });
  Row::Cross c = row.cross(by_weight, 0, 0, goal);
  const u64 all = known_all ? known_all : c.w_all, want = goal(0, all);
  if (!by_weight && c.bin == kBins - 1) return Found{in, c.w_all};  // all that weighs anything is among the first k
  const uint32_t bin = c.bin;

  if (c.c_above + c.c_in <= kSmall) {
    // ---- few: one CTA sorts them (largest logit first, then lowest index) and cuts exactly
    u64* list = reinterpret_cast<u64*>(sh->count);  // free since the last barrier
    static_assert(sizeof(u64) * kSmall <= sizeof(uint32_t) * kBins, "the list fits over the counts");
    if (tid == 0) sh->listed = 0;
    cluster_sync_all();
    const uint32_t list0 = map_to_rank(smem_u32(list), 0), n0 = map_to_rank(smem_u32(&sh->listed), 0);
    row.each([&](float x, uint32_t i) {
      if (in.has(x, i) && (!by_weight || x >= rs.low) && bin_of(x) <= bin)
        st_remote(list0 + 8 * add_remote(n0, 1), ((u64)float_order_key(x) << 32) | (uint32_t)~i);
    });
    cluster_sync_all();
    if (row.rank == 0) {
      const int n = (int)(c.c_above + c.c_in);
      int n2 = 32;
      while (n2 < n) n2 <<= 1;
      for (int i = n + tid; i < n2; i += kT) list[i] = 0;
      __syncthreads();
      for (int k = 2; k <= n2; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
          for (int i = tid; i < n2 / 2; i += kT) {
            const int a = 2 * i - (i & (j - 1)), b = a + j;
            const u64 u = list[a], v = list[b];
            if ((u < v) == ((a & k) == 0)) {
              list[a] = v;
              list[b] = u;
            }
          }
          __syncthreads();
        }
      const int m = by_weight || fl.k > n ? n : fl.k;
      u64 w[2], mine = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        w[i] = 2 * tid + i < m ? weight(order_value((uint32_t)(list[2 * tid + i] >> 32))) : 0ull;
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
      const bool cut_weight = by_weight || fl.p < 1.0f;
      const u64 target = !cut_weight ? ~0ull : by_weight ? want : max(scaled(fl.p, total, true), 1ull);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int at = 2 * tid + i;
        // the last one kept: the first at which the sum reaches the target, or the last of the m
        if (at < m && before < target && (before + w[i] >= target || at == m - 1)) {
          sh->res[0] = list[at];
          sh->res[1] = before + w[i];
        }
        before += w[i];
      }
      __syncthreads();
    }
    const u64(*told)[2] = row.tell(sh->res[0], sh->res[1]);
    done = true;
    return Found{Cut{order_value((uint32_t)(told[0][0] >> 32)), ~(uint32_t)told[0][0]}, told[0][1]};
  }

  // ---- many: divide the bin by the order of its floats
  uint32_t kmin = 0xffffffffu, kmax = 0;
  row.each([&](float x, uint32_t i) {
    if (in.has(x, i) && bin_of(x) == bin) {
      kmin = min(kmin, float_order_key(x));
      kmax = max(kmax, float_order_key(x));
    }
  });
  kmin = __reduce_min_sync(0xffffffffu, kmin);
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  __syncthreads();
  if (lane == 0) sh->red[warp][0] = ((u64)kmin << 32) | kmax;
  __syncthreads();
  auto fold = [&](u64 v) {
    kmin = min(kmin, (uint32_t)(v >> 32));
    kmax = max(kmax, (uint32_t)v);
  };
  for (int i = 0; i < kWarps; ++i) fold(sh->red[i][0]);
  const u64(*ends)[2] = row.tell(((u64)kmin << 32) | kmax, 0);
  for (uint32_t r = 0; r < row.size; ++r) fold(ends[r][0]);
  u64 c_above = c.c_above, w_above = c.w_above, c_in = c.c_in;
  while (kmin < kmax) {
    const int s = max(0, 32 - __clz((int)(kmax - kmin)) - 11);
    row.clear();
    row.each([&](float x, uint32_t i) {
      const uint32_t key = float_order_key(x);
      if (key >= kmin && key <= kmax && in.has(x, i)) row.add((kmax - key) >> s, weight(x));
    });
    c = row.cross(by_weight, c_above, w_above, [&](u64, u64) { return want; });
    c_above = c.c_above;
    w_above = c.w_above;
    c_in = c.c_in;
    const uint32_t top = kmax - (c.bin << s);
    kmin = (1u << s) - 1u >= top - kmin ? kmin : top - ((1u << s) - 1u);
    kmax = top;
  }
  // ---- one value is left: as many of its equals as it takes, the lower indices first
  const float value = order_value(kmax);
  const u64 each_w = weight(value);
  const u64 ties = min(by_weight ? (want - w_above + each_w - 1) / each_w : want - c_above, c_in);
  Found f{Cut{value, in.value == value ? in.last : 0xffffffffu}, w_above + ties * each_w};
  if (ties == c_in) return f;
  u64 eq = 0, none = 0;
  row.each([&](float x, uint32_t) { eq += x == value; });
  const u64 wsum = warp_sum(eq);
  u64 csum = eq;
  row.block_sum(csum, none);
  const u64(*counts)[2] = row.tell(csum, 0);
  u64 before = 0;
  for (uint32_t r = 0; r < row.rank; ++r) before += counts[r][0];
  __syncthreads();
  if (lane == 0) sh->red[warp][0] = wsum;
  __syncthreads();
  for (int i = 0; i < warp; ++i) before += sh->red[i][0];
  if (before < ties && before + wsum >= ties) {  // this warp holds the last of them
    const int part = row.slice / kWarps;
    for (int i = warp * part; i < (warp + 1) * part; i += 32) {
      const bool hit = row.x[i + lane] == value;
      const uint32_t hits = __ballot_sync(0xffffffffu, hit);
      if (hit && before + __popc(hits & ((2u << lane) - 1u)) == ties) {
        for (uint32_t r = 0; r < row.size; ++r) st_remote(map_to_rank(smem_u32(&sh->res[0]), r), row.base + i + lane);
      }
      before += __popc(hits);
    }
  }
  cluster_sync_all();
  f.cut.last = (uint32_t)sh->res[0];
  return f;
}

template <int kType>
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
  if (tid < 128) sh.table[tid] = (uint32_t)rint(exp2(31.0 - tid / 128.0));
  pdl_wait();
  pdl_trigger();
  Row rw{&sh, xs, slice, rank * (uint32_t)slice, rank, size};
  const float temp = sp.temperature ? sp.temperature[row] : 1.0f;
  const int k = sp.top_k ? sp.top_k[row] : 0;
  const float top_p = sp.top_p ? sp.top_p[row] : 1.0f, min_p = sp.min_p ? sp.min_p[row] : 0.0f;

  // ---- the slice into shared memory (NaN as -inf, -0 as 0), its maximum and least finite value
  float mx = -INFINITY, mn = INFINITY;
  uint32_t at = 0;
  auto take = [&](float l, uint32_t i) {
    l = isnan(l) ? -INFINITY : l + 0.0f;
    if (l > mx) {  // indices ascend: the first of equals stays
      mx = l;
      at = i;
    }
    if (l > -INFINITY) mn = fminf(mn, l);
    return l;
  };
  {
    constexpr int kEach = kType == W8A8_TYPE_F32 ? 4 : 8, kAhead = kType == W8A8_TYPE_F32 ? 8 : 4;
    constexpr int kElem = kType == W8A8_TYPE_F32 ? 4 : 2;
    const char* src = static_cast<const char*>(logits) + (int64_t)row * row_stride * kElem;
    const int n = min(slice, max(0, V - (int)rw.base));  // logits of this CTA
    for (int i0 = 0; i0 < slice; i0 += kT * kEach * kAhead) {
      uint4 v[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = i0 + (j * kT + tid) * kEach;
        if (i + kEach <= n) v[j] = ldg_stream(src + (int64_t)(rw.base + i) * kElem);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = i0 + (j * kT + tid) * kEach;
        if (i >= slice) continue;
        float f[kEach];
        if (i + kEach <= n) {
          const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
          if constexpr (kType == W8A8_TYPE_F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(w[e]);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if constexpr (kType == W8A8_TYPE_BF16) {
                f[2 * e] = bf16_lo(w[e]);
                f[2 * e + 1] = bf16_hi(w[e]);
              } else {
                const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w[e]));
                f[2 * e] = h.x;
                f[2 * e + 1] = h.y;
              }
            }
          }
        } else {  // the row's ragged end
#pragma unroll
          for (int e = 0; e < kEach; ++e) {
            f[e] = -INFINITY;
            if (i + e < n) {
              const char* p = src + (int64_t)(rw.base + i + e) * kElem;
              if constexpr (kType == W8A8_TYPE_F32) f[e] = *reinterpret_cast<const float*>(p);
              if constexpr (kType == W8A8_TYPE_BF16) f[e] = bf16_bits_to_f32(*reinterpret_cast<const uint16_t*>(p));
              if constexpr (kType == W8A8_TYPE_F16) f[e] = __half2float(*reinterpret_cast<const __half*>(p));
            }
          }
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) f[e] = take(f[e], rw.base + i + e);
#pragma unroll
        for (int e = 0; e < kEach; e += 4)
          *reinterpret_cast<float4*>(xs + i + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
      }
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
  cluster_sync_all();
  const u64(*tops)[2] = rw.tell(best, least_key);
  for (uint32_t r = 0; r < size; ++r) {
    best = max(best, tops[r][0]);
    least_key = min(least_key, (uint32_t)tops[r][1]);
  }
  mx = order_value((uint32_t)(best >> 32));
  if (mx == -INFINITY || !(temp > 0.0f)) {
    if (rank == 0 && tid == 0) {
      tokens[row] = mx == -INFINITY ? -1 : (int32_t)~(uint32_t)best;
      if (probs) probs[row] = mx == -INFINITY ? 0.0f : 1.0f;
    }
    return;
  }

  const RowScale rs = row_scale(mx, order_value(least_key), temp);
  auto weight = [&](float l) { return weight_of(rs, sh.table, l); };
  Cut cut{-INFINITY, 0xffffffffu};
  const Filters fl{k, top_p};
  bool done = false;
  if (k > 0 && k < V) {
    const Found f = find_cut(rw, rs, weight, cut, false, 0, fl, done);
    cut = f.cut;
    if (!done && top_p < 1.0f) cut = find_cut(rw, rs, weight, cut, true, f.weight, fl, done).cut;
  } else if (top_p < 1.0f) {
    cut = find_cut(rw, rs, weight, cut, true, 0, fl, done).cut;
  }

  // ---- the kept weights, and the token
  const u64 least = !(min_p > 0.0f) ? 0ull : min_p >= 1.0f ? 1ull << kFrac : scaled(min_p, 1ull << kFrac, true);
  auto kept = [&](float x, uint32_t i) -> u64 {
    if (!cut.has(x, i)) return 0ull;
    const u64 w = weight(x);
    return w >= least || x == mx ? w : 0ull;
  };
  u64 mine = 0, none = 0;
  rw.each([&](float x, uint32_t i) { mine += kept(x, i); });
  const u64 wsum = warp_sum(mine);
  rw.block_sum(mine, none);
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
  __syncthreads();
  if (lane == 0) sh.red[warp][0] = wsum;
  __syncthreads();
  for (int i = 0; i < warp; ++i) before += sh.red[i][0];
  if (!(target >= before && target < before + wsum)) return;  // another warp's
  const int part = slice / kWarps;
  for (int i = warp * part; i < (warp + 1) * part; i += 32) {
    const u64 w = kept(xs[i + lane], rw.base + i + lane);
    const u64 upto = before + warp_scan(w, lane);
    if (upto > target && upto - w <= target) {
      tokens[row] = (int32_t)(rw.base + i + lane);
      if (probs) probs[row] = (float)((double)w / (double)total);
    }
    before = __shfl_sync(0xffffffffu, upto, 31);
    if (before > target) break;
  }
}

template <int kType>
w8a8_status launch(const void* logits, int64_t row_stride, int M, int V, const w8a8_sampling& sp, const float* u, int32_t* tokens,
                   float* probs, int sms, cudaStream_t st) {
  // CTAs a row: enough that a slice is 16384 logits at most (64 KB, two CTAs an SM), more for few rows, whose latency is
  // that of a pass over a slice
  int size = 1;
  auto slice_of = [&](int n) { return (((V + n - 1) / n) + kUnit - 1) / kUnit * kUnit; };
  while (size < kMaxCluster &&
         (slice_of(size) > 16384 || (slice_of(size) > kUnit && (long long)M * size * 2 <= 2 * sms)))
    size *= 2;
  const int slice = slice_of(size);
  static bool attr_set[64] = {};
  int dev = 0;
  W8A8_CUDA(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64 && !attr_set[dev]) {
    W8A8_CUDA(cudaFuncSetAttribute(sample_kernel<kType>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlice * 4));
    W8A8_CUDA(cudaFuncSetAttribute(sample_kernel<kType>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    attr_set[dev] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(M * size));
  cfg.blockDim = dim3(kT);
  cfg.dynamicSmemBytes = (size_t)slice * 4;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)size;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  W8A8_CUDA(cudaLaunchKernelEx(&cfg, sample_kernel<kType>, logits, row_stride, V, slice, sp, u, tokens, probs));
  return W8A8_OK;
}

}  // namespace

w8a8_status launch_sample(int dtype, const void* logits, int64_t row_stride, int M, int V, const w8a8_sampling& sp,
                          const float* u, int32_t* tokens, float* probs, int sms, cudaStream_t st) {
  return dtype == W8A8_TYPE_F32    ? launch<W8A8_TYPE_F32>(logits, row_stride, M, V, sp, u, tokens, probs, sms, st)
         : dtype == W8A8_TYPE_BF16 ? launch<W8A8_TYPE_BF16>(logits, row_stride, M, V, sp, u, tokens, probs, sms, st)
                                   : launch<W8A8_TYPE_F16>(logits, row_stride, M, V, sp, u, tokens, probs, sms, st);
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
  W8A8_CHECK_ARG(M <= 1 << 24, W8A8_ERR_SHAPE, "%s: M=%d rows", who, M);
  DevInfo d;
  W8A8_TRY(dev_info(&d));
  return launch_sample(dtype, logits, row_stride, M, V, *sampling, u, tokens, probs, d.sms, as_stream(stream));
}
