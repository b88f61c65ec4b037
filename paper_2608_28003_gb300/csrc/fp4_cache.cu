// A paged cache in 4 bits: the append of a projection's rows to it, and its pages' values.
//
// Append.  Queries are turned by blocks of their own, as rope_append does it.  For keys and values a warp takes a row and walks its
// heads with a fixed step, so that the row's sines and cosines are computed once for all of them; a lane holds 8, 4 or 2
// neighbouring dims (head dim 256, 128, 64) and reaches the other dim of a pair by a shuffle.  A block of 16 dims is 2, 4 or 8
// lanes.  Little is moved (a key's 144 bytes at head dim 256), so latency bounds it: launch, sequence, length, page, store.
// 5 chunks of up to 811 tokens, 16 query and 4 key/value heads of 128: 13.0 us, half of the issue slots used (the 16-bit append: 7.5);
// 23 with the queries by warps too and every dim of an open block in 64 bits, 33 with a head's load behind the one before.  48
// single tokens 4.8.
//
// Codes are decided as in exact arithmetic: the rotation and the norm are computed in fp32 with a bound on what they are off by, and where
// that leaves a code or a scale open (both ends of the bound are rounded and compared; a few heads in a thousand), or fp32's range does not
// hold the norm or the rotation, the value is computed again in 64 bits.
#include <cmath>

#include "fp4.cuh"
#include "ops.cuh"
#include "rope.cuh"

namespace w8a8 {

namespace {

constexpr int kThreads = 256;

// What the fp32 values are off by, in units of 2^-24 of |x| + |its partner|: 3.6 for cos and sin (their argument to 2^-25 half
// turns, 1 unit in the last place, the factor), 2 for the two products, and with a norm 11 (13 additions' halves, the square root, the
// quotient, two products).
constexpr float kOff = 8.0f * 0x1p-24f, kOffNorm = 20.0f * 0x1p-24f;

// The code of x / unit in 64 bits.
__device__ __forceinline__ uint32_t code_of(double x, double unit) {
  const double a = fabs(x);
  const uint32_t c = (a > 0.25 * unit) + (a >= 0.75 * unit) + (a > 1.25 * unit) + (a >= 1.75 * unit) + (a > 2.5 * unit) +
                     (a >= 3.5 * unit) + (a > 5.0 * unit);
  return unit > 0.0 ? c | (x < 0.0 ? 8u : 0u) : 0u;
}
// The e4m3 byte of t >= 0 in 64 bits (448 above it).
__device__ __forceinline__ uint32_t e4m3_of_double(double t) {
  t = fmin(t, 448.0);
  const int e = max(t > 0.0 ? ilogb(t) : -6, -6);
  return e4m3_of((float)(rint(ldexp(t, 3 - e)) * ldexp(1.0, e - 3)));
}

template <int kE>
struct Raw;  // kE values as loaded
template <>
struct Raw<8> {
  uint4 w;
};
template <>
struct Raw<4> {
  uint2 w;
};
template <>
struct Raw<2> {
  uint32_t w;
};
template <bool kBf16, int kE>
__device__ __forceinline__ void raw_floats(const Raw<kE>& r, float (&x)[kE]) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
  for (int i = 0; i < kE / 2; ++i) {
    const float2 f = unpack2<kBf16>(w[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}

// The largest over a block's lanes.
template <int kLanes>
__device__ __forceinline__ float block_max(float x) {
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
// Codes to their place, kE / 2 bytes a lane, and the scale by the block's first lane.
template <int kE>
__device__ __forceinline__ void put_codes(uint8_t* codes, uint8_t* scales, uint32_t w, uint32_t byte, int lane) {
  if constexpr (kE == 8)
    *reinterpret_cast<uint32_t*>(codes + 4 * lane) = w;
  else if constexpr (kE == 4)
    *reinterpret_cast<uint16_t*>(codes + 2 * lane) = (uint16_t)w;
  else
    codes[lane] = (uint8_t)w;
  if (lane % (16 / kE) == 0) scales[lane / (16 / kE)] = (uint8_t)byte;
}

// A row's queries, by units of 16 dims as in rope_append: thread i of all.  Every lane of a warp makes the same number of trips, so
// that the shuffles of the norm's sum are whole.
template <bool kBf16, int kUnits>
__device__ __forceinline__ void turn_queries(const RopeArgs& r, const PagedCache& c, const PagedBatch& batch, int64_t i,
                                             const uint16_t* q, int64_t q_row, int n_q, const float* __restrict__ q_norm, float eps,
                                             uint16_t* q_out, int64_t q_out_row, int step) {
  const int unit = (int)(i % kUnits), h0 = (int)((i / kUnits) % step);
  const int64_t row64 = i / kUnits / step;
  const int row = (int)min(row64, (int64_t)batch.n_rows - 1), s = seq_of_row(batch, row);
  const SeqShape q0 = seq_shape(batch, s, c.page_shift);
  const bool live = row64 < batch.n_rows && row >= q0.row0 && row < q0.row0 + q0.rows;
  bool rotated;
  int at0, at1;
  unit_place(r, unit, rotated, at0, at1);
  float co[8], si[8], x[16];
  const int trips = (n_q + step - 1) / step;
  for (int t0 = 0; t0 < trips; t0 += kAhead) {
    Unit u[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int h = h0 + (t0 + j) * step;
      if (live && h < n_q) u[j] = unit_load(q + (int64_t)row * q_row + (int64_t)h * (16 * kUnits), at0, at1);
    }
    if (t0 == 0 && rotated && live) unit_angles(r, unit, q0.pos0 + (row - q0.row0), co, si);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int h = h0 + (t0 + j) * step;
      if (t0 + j >= trips) break;
      const bool work = live && h < n_q;
      float ss = 0.0f;
      if (work) {
        unit_values<kBf16>(u[j], x);
#pragma unroll
        for (int e = 0; e < 16; ++e) ss = fmaf(x[e], x[e], ss);
      }
      if (q_norm)
#pragma unroll
        for (int o = kUnits / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (!work) continue;
      if (q_norm) {
        const float inv = 1.0f / sqrtf(ss / (float)(16 * kUnits) + eps);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = x[e] * inv * q_norm[e < 8 ? at0 + e : at1 + e - 8];
      }
      if (rotated) unit_rotate(r.inter, co, si, x);
      unit_store<kBf16>(q_out + (int64_t)row * q_out_row + (int64_t)h * (16 * kUnits), at0, at1, x);
    }
  }
}

template <bool kBf16, int kDim>
__global__ void __launch_bounds__(kThreads)
    fp4_append_kernel(RopeArgs t, Fp4Pages cache, PagedBatch batch, const uint16_t* q, int64_t q_row, int n_q, const uint16_t* k,
                      int64_t k_row, const uint16_t* v, int64_t v_row, const float* __restrict__ q_norm,
                      const float* __restrict__ k_norm, float eps, uint16_t* q_out, int64_t q_out_row, int step, int q_step,
                      unsigned kv_blocks) {
  constexpr int kE = kDim / 32, kLanes = 16 / kE;
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x >= kv_blocks) {
    turn_queries<kBf16, kDim / 16>(t, cache.p, batch, (int64_t)(blockIdx.x - kv_blocks) * kThreads + threadIdx.x, q, q_row, n_q,
                                   q_norm, eps, q_out, q_out_row, q_step);
    return;
  }
  const int lane = threadIdx.x & 31;
  const int64_t wid = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int h0 = (int)(wid % step);
  const int64_t row64 = wid / step;
  if (row64 >= batch.n_rows) return;
  const int row = (int)row64, n_kv = cache.p.n_kv, heads = 2 * n_kv;
  auto source = [&](int h) {
    return h < n_kv ? k + row64 * k_row + (int64_t)h * kDim : v + row64 * v_row + (int64_t)(h - n_kv) * kDim;
  };
  Raw<kE> next[kAhead];  // the heads ahead (rows of no sequence are the caller's memory too)
#pragma unroll
  for (int j = 0; j < kAhead; ++j)
    if (h0 + j * step < heads) next[j] = *(reinterpret_cast<const Raw<kE>*>(source(h0 + j * step)) + lane);
  const int s = seq_of_row(batch, row);
  const SeqShape sq = seq_shape(batch, s, cache.p.page_shift);
  if (row < sq.row0 || row >= sq.row0 + sq.rows) return;
  const int pos = sq.pos0 + (row - sq.row0);
  int64_t scale_at = 0;
  const int64_t code_at = fp4_key_offset(batch, cache, s, pos, 0, scale_at);
  if (code_at < 0) return;

  // this lane's angles: dim d of a pair with the other one `mate` lanes on (half layout) or beside it
  const int d0 = lane * kE, half = t.rot / 2;
  const bool turned = d0 < t.rot, first = d0 < half;
  const int mate = t.inter ? lane : turned ? (first ? lane + half / kE : lane - half / kE) : lane;
  auto pair_of = [&](int e) { return t.inter ? (d0 + e) >> 1 : (first ? d0 : d0 - half) + e; };
  auto minus = [&](int e) { return t.inter ? (e & 1) == 0 : first; };  // whether the partner's part is subtracted
  float c[kE], sn[kE];
  if (turned) {
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      const uint64_t turn = (uint64_t)(int64_t)pos * t.turns[pair_of(e)];
      sincospif((float)(int64_t)turn * 0x1p-63f, &sn[e], &c[e]);
      c[e] *= t.scale;
      sn[e] *= minus(e) ? -t.scale : t.scale;
    }
  }

  for (int h = h0; h < heads; h += step) {
    const Raw<kE> raw = next[0];
#pragma unroll
    for (int j = 0; j + 1 < kAhead; ++j) next[j] = next[j + 1];
    if (h + kAhead * step < heads) next[kAhead - 1] = *(reinterpret_cast<const Raw<kE>*>(source(h + kAhead * step)) + lane);
    const bool is_v = h >= n_kv;
    float x[kE], y[kE], off[kE];  // as they come, turned, the bound on what y is off by
    raw_floats<kBf16, kE>(raw, x);
    const float* nw = is_v ? nullptr : k_norm;
    bool far = false;  // the sum of squares left fp32's range
    if (!is_v) {
#pragma unroll
      for (int e = 0; e < kE; ++e) y[e] = x[e];
      if (nw) {
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < kE; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        far = ss > 0x1p120f || (ss < 0x1p-80f && eps < 0x1p-60f);
        const float inv = 1.0f / sqrtf(ss / (float)kDim + eps);
#pragma unroll
        for (int e = 0; e < kE; ++e) y[e] = x[e] * inv * nw[d0 + e];
      }
      float p[kE];
#pragma unroll
      for (int e = 0; e < kE; ++e) p[e] = t.inter ? y[e ^ 1] : __shfl_sync(0xffffffffu, y[e], mate);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        off[e] = (nw ? kOffNorm : turned ? kOff : 0.0f) * (fabsf(y[e]) + (turned ? fabsf(p[e]) : 0.0f));
        if (turned) y[e] = fmaf(p[e], sn[e], y[e] * c[e]);
      }
      if (turned)  // cos and sin are up to the table's factor
#pragma unroll
        for (int e = 0; e < kE; ++e) off[e] *= fmaxf(1.0f, fabsf(t.scale));
    } else {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        y[e] = x[e];
        off[e] = 0.0f;
      }
    }
    // A key's dim e of this lane in 64 bits (all lanes take part in the exchange; `mine`: those that want it).
    auto exact_norm = [&] {
      double ss = 0.0;
#pragma unroll 1
      for (int e = 0; e < kE; ++e) ss += (double)x[e] * (double)x[e];
#pragma unroll 1
      for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      return 1.0 / sqrt(ss / kDim + (double)eps);
    };
    auto exact = [&](int e, double inv, bool mine) {
      float xe = 0.0f, we = 1.0f, pe = 0.0f, wp = 1.0f;
#pragma unroll
      for (int j = 0; j < kE; ++j)
        if (j == e) {
          xe = x[j];
          pe = t.inter ? x[j ^ 1] : 0.0f;
        }
      const float other = __shfl_sync(0xffffffffu, xe, mate);
      if (!t.inter) pe = other;
      if (!mine) return 0.0;
      if (nw) {
        we = nw[d0 + e];
        wp = t.inter ? nw[d0 + (e ^ 1)] : nw[mate * kE + e];
      }
      double z = (double)xe * inv * (double)we;
      if (turned) {
        const uint64_t turn = (uint64_t)(int64_t)pos * t.turns[pair_of(e)];
        double cd, sd;
        sincospi((double)(int64_t)turn * 0x1p-63, &sd, &cd);
        const double zp = (double)pe * inv * (double)wp;
        z = (z * cd + (minus(e) ? -zp : zp) * sd) * (double)t.scale;
      }
      return z;
    };
    const int kv_head = is_v ? h - n_kv : h, exponent = is_v ? cache.v_exp : cache.k_exp;
    const float s2 = two_to(-exponent);
    bool finite = true;
#pragma unroll
    for (int e = 0; e < kE; ++e) finite = finite && fabsf(y[e]) < INFINITY;
    uint32_t unsound = __ballot_sync(0xffffffffu, !finite || far);
    if (unsound != 0 && !is_v) {  // fp32 left its range: the key in 64 bits, what is beyond fp32 at its end (far above the cut-off)
      const double inv = nw ? exact_norm() : 1.0;
      finite = true;
#pragma unroll 1
      for (int e = 0; e < kE; ++e) {
        const double z = exact(e, inv, true);
        finite = finite && fabs(z) < (double)INFINITY;
        const float f = (float)fmax(fmin(z, 0x1.fffffep127), -0x1.fffffep127);
#pragma unroll
        for (int j = 0; j < kE; ++j)
          if (j == e) {
            y[j] = f;
            off[j] = 0x1p-23f * fabsf(f);
          }
      }
      unsound = __ballot_sync(0xffffffffu, !finite);
    }
    const bool nan = (unsound >> (lane & ~(kLanes - 1)) & ((1u << kLanes) - 1u)) != 0;
    float top = 0.0f, wide = 0.0f;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      top = fmaxf(top, fabsf(y[e]));
      wide = fmaxf(wide, off[e]);
    }
    top = block_max<kLanes>(top);
    wide = block_max<kLanes>(wide);
    Block16 b;
    b.unit(__float_as_uint(nan ? INFINITY : top), s2);
    // both ends of the bound
    bool open_unit = false, open[kE] = {};
    if (!nan && wide > 0.0f)
      open_unit = e4m3_of(sixth((top - wide) * s2)) != e4m3_of(sixth((top + wide) * s2));
    uint32_t w = 0;
    auto encode = [&] {
      w = 0;
#pragma unroll
      for (int i = 0; i < kE / 2; ++i) {
        float g[2], o[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          // (what is beyond the cut-off is 6 of any unit, but an infinite product has no quotient)
          g[e] = b.over(fminf(fmaxf(y[2 * i + e] * s2, -0x1p20f), 0x1p20f));
          o[e] = off[2 * i + e] * s2 * b.hi;
        }
        if (!nan) {
          w |= e2m1x2_of(g[0], g[1]) << (8 * i);
          const uint32_t apart = e2m1x2_of(g[0] - o[0], g[1] - o[1]) ^ e2m1x2_of(g[0] + o[0], g[1] + o[1]);
          open[2 * i] = (apart & 15u) != 0;
          open[2 * i + 1] = (apart >> 4) != 0;
        }
      }
    };
    encode();
    bool any = open_unit;
#pragma unroll
    for (int e = 0; e < kE; ++e) any = any || open[e];
    if (__any_sync(0xffffffffu, any) && !is_v) {
      const double inv = nw ? exact_norm() : 1.0;
      double top64 = 0.0, unit = (double)b.scale / (double)s2;
      // first the scales that are open, for which the dims that can be their blocks' largest are looked at; then the codes that are
#pragma unroll 1
      for (int pass = __any_sync(0xffffffffu, open_unit) ? 0 : 1; pass < 2; ++pass) {
#pragma unroll 1
        for (int e = 0; e < kE; ++e) {
          bool mine = false;
#pragma unroll
          for (int j = 0; j < kE; ++j)
            if (j == e) mine = pass == 0 ? open_unit && fabsf(y[j]) + off[j] >= top - wide : open[j];
          const double z = exact(e, inv, mine);
          if (!mine) continue;
          if (pass == 0) {
            top64 = fmax(top64, fabs(z));
          } else {
            const uint32_t code = code_of(z, unit);
            w = (w & ~(15u << (4 * e))) | code << (4 * e);
          }
        }
        __syncwarp();
        if (pass == 0) {
#pragma unroll 1
          for (int o = kLanes / 2; o > 0; o >>= 1) top64 = fmax(top64, __shfl_xor_sync(0xffffffffu, top64, o));
          if (open_unit) {
            b.byte = e4m3_of_double(top64 * (double)s2 / 6.0);
            b.of_byte();
            unit = (double)b.scale / (double)s2;
            encode();
          }
          __syncwarp();
        }
      }
    }
    uint8_t* codes = (is_v ? cache.v : cache.k) + code_at + (int64_t)kv_head * cache.p.head_stride;
    uint8_t* scales = (is_v ? cache.vs : cache.ks) + scale_at + (int64_t)kv_head * cache.s_head;
    put_codes<kE>(codes, scales, w, b.byte, lane);
  }
}

// A thread has eight dims of (page, slot, head), so that a warp's stores are contiguous; blockIdx.y: keys or values.
template <int kType>
__global__ void __launch_bounds__(kThreads) fp4_values_kernel(Fp4Pages c, const int32_t* __restrict__ pages, int64_t total,
                                                              int eighths_shift, void* k_out, void* v_out) {
  pdl_wait();
  pdl_trigger();
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const bool is_v = blockIdx.y == 1 || k_out == nullptr;
  char* out = static_cast<char*>(is_v ? v_out : k_out);
  if (i >= total) return;
  const int d = (int)i & ((1 << eighths_shift) - 1);
  const int64_t r = i >> eighths_shift;
  const int64_t rh = r < (1ll << 32) ? (int64_t)((uint32_t)r / (uint32_t)c.p.n_kv) : r / c.p.n_kv;  // page and slot
  const int h = (int)(r - rh * c.p.n_kv), slot = (int)(rh & ((1 << c.p.page_shift) - 1));
  const int64_t n = rh >> c.p.page_shift;
  const int64_t page = pages ? pages[n] : n;
  uint32_t w = 0;
  float unit = 0.0f;
  if (page >= 0 && page < c.p.n_pages) {
    w = *reinterpret_cast<const uint32_t*>((is_v ? c.v : c.k) + page * c.p.page_stride + slot * c.p.slot_stride +
                                           h * c.p.head_stride + 4 * d);
    unit = e4m3_value((is_v ? c.vs : c.ks)[page * c.s_page + slot * c.s_slot + h * c.s_head + (d >> 1)]) *
           two_to(is_v ? c.v_exp : c.k_exp);
  }
  uint32_t a[4];
  e2m1x8_to_f16(w, a);
  float v[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = unpack2<false>(a[e]);
    v[2 * e] = f.x * unit;
    v[2 * e + 1] = f.y * unit;
  }
  if constexpr (kType == W8A8_TYPE_F32) {
    uint4* to = reinterpret_cast<uint4*>(out + i * 32);
    to[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    to[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
  } else {
    constexpr bool kBf = kType == W8A8_TYPE_BF16;
    *reinterpret_cast<uint4*>(out + i * 16) =
        make_uint4(pack2<kBf>(v[0], v[1]), pack2<kBf>(v[2], v[3]), pack2<kBf>(v[4], v[5]), pack2<kBf>(v[6], v[7]));
  }
}

}  // namespace

w8a8_status check_fp4_paged(const char* who, const w8a8_paged_cache_fp4* c, const w8a8_paged_batch* b, Fp4Pages* pc,
                            PagedBatch* pb) {
  W8A8_CHECK_ARG(c && b, W8A8_ERR_INVALID_ARG, "%s: null cache or batch", who);
  const int dim = c->head_dim;
  const w8a8_paged_cache shape{W8A8_TYPE_BF16, c->n_pages, c->page_size, c->n_kv, dim, dim, dim, dim,
                               reinterpret_cast<uint16_t*>(c->k), reinterpret_cast<uint16_t*>(c->v)};
  W8A8_TRY(check_paged(who, &shape, b, &pc->p, pb));
  const int64_t str[3] = {c->page_stride, c->slot_stride, c->head_stride},
                s_str[3] = {c->s_page_stride, c->s_slot_stride, c->s_head_stride};
  for (int i = 0; i < 3; ++i)
    W8A8_CHECK_ARG(str[i] >= dim / 2 && str[i] % 16 == 0 && str[i] <= (1ll << 38) && s_str[i] >= dim / 16 &&
                       s_str[i] % (dim / 16) == 0 && s_str[i] <= (1ll << 38),
                   W8A8_ERR_SHAPE, "%s: the codes' strides must be multiples of 16 bytes from head_dim / 2 on, the scales' of "
                   "head_dim / 16 bytes", who);
  W8A8_CHECK_ARG(c->k_exp >= -100 && c->k_exp <= 100 && c->v_exp >= -100 && c->v_exp <= 100, W8A8_ERR_INVALID_ARG,
                 "%s: exponents %d and %d must lie within [-100, 100]", who, c->k_exp, c->v_exp);
  W8A8_CHECK_ARG(b->n_seqs == 0 || b->n_rows == 0 || (c->k_scales && c->v_scales), W8A8_ERR_INVALID_ARG, "%s: null pointer", who);
  W8A8_CHECK_ARG(aligned16(c->k_scales) && aligned16(c->v_scales), W8A8_ERR_ALIGN, "%s: the scales must be 16-byte aligned", who);
  pc->p.page_stride = c->page_stride;
  pc->p.slot_stride = c->slot_stride;
  pc->p.head_stride = c->head_stride;
  pc->p.k = pc->p.v = nullptr;
  pc->s_page = c->s_page_stride;
  pc->s_slot = c->s_slot_stride;
  pc->s_head = c->s_head_stride;
  pc->k = c->k;
  pc->v = c->v;
  pc->ks = c->k_scales;
  pc->vs = c->v_scales;
  pc->k_exp = c->k_exp;
  pc->v_exp = c->v_exp;
  return W8A8_OK;
}

}  // namespace w8a8

using namespace w8a8;

extern "C" w8a8_status w8a8_fp4_rope_append(const w8a8_rope_table* rope, const w8a8_paged_cache_fp4* cache,
                                            const w8a8_paged_batch* batch, int dtype, const uint16_t* q, int64_t q_row, int n_q,
                                            const uint16_t* k, int64_t k_row, const uint16_t* v, int64_t v_row,
                                            const float* q_norm, const float* k_norm, float eps, uint16_t* q_out,
                                            int64_t q_out_row, void* stream) {
  const char* who = "w8a8_fp4_rope_append";
  Fp4Pages pc;
  PagedBatch pb;
  W8A8_TRY(check_fp4_paged(who, cache, batch, &pc, &pb));
  const int dim = cache->head_dim;
  W8A8_TRY(check_rope(who, rope, dim));
  W8A8_CHECK_ARG(dtype == W8A8_TYPE_BF16 || dtype == W8A8_TYPE_F16, W8A8_ERR_INVALID_ARG, "%s: type %d must be bf16 or fp16",
                 who, dtype);
  W8A8_TRY(check_append(who, pb, dim, q, q_row, n_q, k, k_row, v, v_row, q_norm, k_norm, eps, q_out, q_out_row));
  if (pb.n_seqs == 0 || pb.n_rows == 0) return W8A8_OK;
  DevInfo d;
  W8A8_TRY(dev_info(&d));
  const RopeArgs t{rope->turns, rope->scale, rope->rotary_dim, rope->interleaved};
  // few rows spread over their heads, many compute their angles once: up to 16 warps an SM, one wave (2400 rows, 4 key/value heads of 128:
  // 13.0 us; 14.2 with 32 warps, 16.5 with 48)
  const int64_t want = (int64_t)d.sms * 16 / pb.n_rows;
  const int step = (int)(want < 1 ? 1 : want > 2 * pc.p.n_kv ? 2 * pc.p.n_kv : want), units = dim / 16;
  const int q_step = head_step(pb.n_rows, units, n_q, d.sms);
  const int64_t kv_blocks = ((int64_t)pb.n_rows * step * 32 + kThreads - 1) / kThreads;
  const int64_t q_blocks = ((int64_t)pb.n_rows * units * q_step + kThreads - 1) / kThreads;
  W8A8_CHECK_ARG(kv_blocks + q_blocks <= 0x7fffffffll, W8A8_ERR_SHAPE, "%s: n_rows=%d is too large", who, pb.n_rows);
  const dim3 grid((unsigned)(kv_blocks + q_blocks));
  auto go = [&](auto kernel) {
    return launch_pdl(kernel, grid, dim3(kThreads), 0, as_stream(stream), t, pc, pb, q, q_row, n_q, k, k_row, v, v_row, q_norm,
                      k_norm, eps, q_out, q_out_row, step, q_step, (unsigned)kv_blocks);
  };
  W8A8_CUDA(dtype == W8A8_TYPE_BF16 ? (dim == 256   ? go(fp4_append_kernel<true, 256>)
                                       : dim == 128 ? go(fp4_append_kernel<true, 128>)
                                                    : go(fp4_append_kernel<true, 64>))
                                    : (dim == 256   ? go(fp4_append_kernel<false, 256>)
                                       : dim == 128 ? go(fp4_append_kernel<false, 128>)
                                                    : go(fp4_append_kernel<false, 64>)));
  return W8A8_OK;
}

extern "C" w8a8_status w8a8_fp4_paged_values(const w8a8_paged_cache_fp4* cache, const int32_t* pages, int n, int dtype,
                                             void* k_out, void* v_out, void* stream) {
  const char* who = "w8a8_fp4_paged_values";
  Fp4Pages pc;
  PagedBatch pb;
  int32_t dummy = 0;
  const w8a8_paged_batch one{1, 1, 1, 1, &dummy, &dummy, &dummy};  // for the checks of the cache
  W8A8_TRY(check_fp4_paged(who, cache, &one, &pc, &pb));
  W8A8_CHECK_ARG(dtype >= W8A8_TYPE_BF16 && dtype <= W8A8_TYPE_F32, W8A8_ERR_INVALID_ARG, "%s: type %d", who, dtype);
  W8A8_CHECK_ARG(n >= 0 && (pages || n == 0 || n == pc.p.n_pages), W8A8_ERR_INVALID_ARG, "%s: n=%d, the cache has %d pages", who, n,
                 pc.p.n_pages);
  if (n == 0 || (!k_out && !v_out)) return W8A8_OK;
  W8A8_CHECK_ARG(aligned16(k_out) && aligned16(v_out) && (reinterpret_cast<uintptr_t>(pages) & 3u) == 0, W8A8_ERR_ALIGN,
                 "%s: outputs must be 16-byte aligned, pages 4-byte", who);
  W8A8_TRY(check_device());
  const int shift = cache->head_dim == 256 ? 5 : cache->head_dim == 128 ? 4 : 3;  // eight dims a thread
  const int64_t total = (((int64_t)n << pc.p.page_shift) * pc.p.n_kv) << shift, grid = (total + kThreads - 1) / kThreads;
  W8A8_CHECK_ARG(grid <= 0x7fffffffll, W8A8_ERR_SHAPE, "%s: %d pages are too many for one call", who, n);
  auto go = [&](auto kernel) {
    return launch_pdl(kernel, dim3((unsigned)grid, k_out && v_out ? 2u : 1u), dim3(kThreads), 0, as_stream(stream), pc, pages,
                      total, shift, k_out, v_out);
  };
  W8A8_CUDA(dtype == W8A8_TYPE_BF16  ? go(fp4_values_kernel<W8A8_TYPE_BF16>)
            : dtype == W8A8_TYPE_F16 ? go(fp4_values_kernel<W8A8_TYPE_F16>)
                                     : go(fp4_values_kernel<W8A8_TYPE_F32>));
  return W8A8_OK;
}
