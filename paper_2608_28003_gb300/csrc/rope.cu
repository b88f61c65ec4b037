// Rotary positions, and the append of a projection's rows to a paged cache.
//
// The mathematics: pair i of a head turns by p f_i radians at position p.  With g_i = f_i / (2 pi) held as a
// 64-bit fraction, the product p g_i in wrapping 64-bit arithmetic is that angle in turns with the whole turns
// gone: no reduction of a large argument, and nothing lost beside what g_i itself is off by.  That is a double's power and
// quotient, about g_i 2^-50 for bases up to 10^6: p 2^-52 turns for the fastest pairs, 2^-32 at position 2^20 and 2^-21 at
// the farthest ones.  The signed upper bits then give half-turns in [-1, 1) for sincospif.
//
// Both kernels only move data (a few operations a byte), so HBM or, for few rows, latency bounds them.  A thread
// holds one unit of 16 dims (8 pairs: two 16-byte loads) and walks the heads of one row with a fixed step, so
// that the 8 sines and cosines are computed once for all of its heads; the loads of four heads fly over the sines.
// Measured: 8192 rows, half of every head rotated (134 MB) 23.9 us, 5.6 TB/s (0.83 of the measured copy; floor 19.8); the
// append of 2400 rows of 16 + 8 heads of 128 (30 MB, floor 4.4) 11.4 to 14 us from one machine to the next: one wave of threads, of which
// the wait for a row's sequence, length and page, one after the other, is a third (the rows' loads, which need none of them, come
// after it); 16 and 48 rows 7 to 9 and 10.5 to 12 us, the launch and its arguments.
#include <cmath>

#include "ops.cuh"
#include "paged.cuh"
#include "rope.cuh"

namespace w8a8 {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxDim = 256;

// Thread = (row, first head, unit), units fastest so that neighbours read on.
template <bool kBf16>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs r, const uint16_t* x, int64_t x_row, int64_t x_head, int T,
                                                        int heads, int units, int step,
                                                        const int32_t* __restrict__ positions, uint16_t* y, int64_t y_row,
                                                        int64_t y_head) {
  pdl_wait();
  pdl_trigger();
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int unit = (int)(i % units);
  const int64_t rest = i / units;
  const int h0 = (int)(rest % step);
  const int64_t row = rest / step;
  if (row >= T) return;
  bool rotated;
  int at0, at1;
  unit_place(r, unit, rotated, at0, at1);
  float c[8], s[8], v[16];
  for (int h = h0, first = 1; h < heads; h += kAhead * step, first = 0) {
    Unit u[kAhead];  // the loads of a few heads ahead of the first use, and of the angles
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (h + j * step < heads) u[j] = unit_load(x + row * x_row + (h + j * step) * x_head, at0, at1);
    if (rotated && first) unit_angles(r, unit, positions[row], c, s);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (h + j * step >= heads) break;
      unit_values<kBf16>(u[j], v);
      if (rotated) unit_rotate(r.inter, c, s, v);
      unit_store<kBf16>(y + row * y_row + (h + j * step) * y_head, at0, at1, v);
    }
  }
}

// The same units over the heads q, k, v of a row.  kUnits lanes share a head: the RMSNorm's sum is a shuffle
// among them.  Every lane of a warp makes the same number of trips, so that the shuffles are whole.
template <bool kBf16, int kUnits>
__global__ void __launch_bounds__(kThreads)
    rope_append_kernel(RopeArgs r, PagedCache cache, PagedBatch batch, const uint16_t* q, int64_t q_row, int n_q,
                       const uint16_t* k, int64_t k_row, const uint16_t* v, int64_t v_row,
                       const float* __restrict__ q_norm, const float* __restrict__ k_norm, float eps, uint16_t* q_out,
                       int64_t q_out_row, int step) {
  constexpr int kDim = 16 * kUnits;
  pdl_wait();
  pdl_trigger();
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int unit = (int)(i % kUnits);
  const int h0 = (int)((i / kUnits) % step);
  const int64_t row64 = i / kUnits / step;
  const int row = (int)min(row64, (int64_t)batch.n_rows - 1);
  const int s = seq_of_row(batch, row);
  const SeqShape q0 = seq_shape(batch, s, cache.page_shift);
  const bool live = row64 < batch.n_rows && row >= q0.row0 && row < q0.row0 + q0.rows;
  const int pos = q0.pos0 + (row - q0.row0);
  const int64_t slot = live ? key_offset(batch, cache, s, pos, 0) : -1;
  bool rotated;
  int at0, at1;
  unit_place(r, unit, rotated, at0, at1);
  float c[8], sn[8], x[16];
  const int heads = n_q + 2 * cache.n_kv, trips = (heads + step - 1) / step;
  for (int t0 = 0; t0 < trips; t0 += kAhead) {
    Unit u[kAhead];  // the loads of a few heads ahead of the first use, and of the angles
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int h = h0 + (t0 + j) * step;
      if (!live || h >= heads) continue;
      const uint16_t* src = h < n_q                ? q + (int64_t)row * q_row + (int64_t)h * kDim
                            : h < n_q + cache.n_kv ? k + (int64_t)row * k_row + (int64_t)(h - n_q) * kDim
                                                   : v + (int64_t)row * v_row + (int64_t)(h - n_q - cache.n_kv) * kDim;
      u[j] = unit_load(src, at0, at1);
    }
    if (t0 == 0 && rotated && live) unit_angles(r, unit, pos, c, sn);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int h = h0 + (t0 + j) * step;
      if (t0 + j >= trips) break;
      const bool is_q = h < n_q, is_k = !is_q && h < n_q + cache.n_kv, here = live && h < heads;
      const bool work = here && (is_q || is_k);
      if (here && !work && slot >= 0) {  // v: its bits as they are
        uint16_t* dst = cache.v + slot + (int64_t)(h - n_q - cache.n_kv) * cache.head_stride;
        *reinterpret_cast<uint4*>(dst + at0) = u[j].a;
        *reinterpret_cast<uint4*>(dst + at1) = u[j].b;
      }
      if (work) unit_values<kBf16>(u[j], x);
      const float* nw = is_q ? q_norm : k_norm;
      float ss = 0.0f;
      if (work) {
#pragma unroll
        for (int e = 0; e < 16; ++e) ss = fmaf(x[e], x[e], ss);
      }
#pragma unroll
      for (int o = kUnits / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (work) {
        if (nw) {
          const float inv = 1.0f / sqrtf(ss / (float)kDim + eps);
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] = x[e] * inv * nw[e < 8 ? at0 + e : at1 + e - 8];
        }
        if (rotated) unit_rotate(r.inter, c, sn, x);
        if (is_q)
          unit_store<kBf16>(q_out + (int64_t)row * q_out_row + (int64_t)h * kDim, at0, at1, x);
        else if (slot >= 0)
          unit_store<kBf16>(cache.k + slot + (int64_t)(h - n_q) * cache.head_stride, at0, at1, x);
      }
    }
  }
}

}  // namespace

w8a8_status check_rope(const char* who, const w8a8_rope_table* r, int dim) {
  W8A8_CHECK_ARG(r != nullptr && r->turns != nullptr, W8A8_ERR_INVALID_ARG, "%s: null rope table", who);
  W8A8_CHECK_ARG(r->rotary_dim >= 16 && r->rotary_dim % 16 == 0 && r->rotary_dim <= dim, W8A8_ERR_SHAPE,
                 "%s: rotary_dim %d must be a multiple of 16 in [16, %d]", who, r->rotary_dim, dim);
  W8A8_CHECK_ARG(aligned16(r->turns), W8A8_ERR_ALIGN, "%s: turns must be 16-byte aligned", who);
  return W8A8_OK;
}

w8a8_status check_append(const char* who, const PagedBatch& pb, int dim, const uint16_t* q, int64_t q_row, int n_q,
                         const uint16_t* k, int64_t k_row, const uint16_t* v, int64_t v_row, const float* q_norm,
                         const float* k_norm, float eps, const uint16_t* q_out, int64_t q_out_row) {
  W8A8_CHECK_ARG(n_q > 0 && n_q <= 65536 / dim, W8A8_ERR_SHAPE, "%s: n_q=%d", who, n_q);
  W8A8_CHECK_ARG(q_norm == nullptr && k_norm == nullptr || (eps >= 0.0f && std::isfinite(eps)), W8A8_ERR_INVALID_ARG,
                 "%s: eps %g", who, (double)eps);
  if (pb.n_seqs == 0 || pb.n_rows == 0) return W8A8_OK;
  W8A8_CHECK_ARG(q && k && v && q_out, W8A8_ERR_INVALID_ARG, "%s: null pointer", who);
  W8A8_CHECK_ARG(aligned16(q) && aligned16(k) && aligned16(v) && aligned16(q_out) && aligned16(q_norm) && aligned16(k_norm),
                 W8A8_ERR_ALIGN, "%s: pointers must be 16-byte aligned", who);
  const int64_t big = 1ll << 40, rows[4] = {q_row, k_row, v_row, q_out_row};
  for (int64_t s : rows) W8A8_CHECK_ARG(s >= 0 && s % 8 == 0 && s <= big, W8A8_ERR_SHAPE, "%s: row strides must be multiples of 8", who);
  W8A8_CHECK_ARG(pb.n_rows == 1 || q_out_row >= (int64_t)n_q * dim, W8A8_ERR_SHAPE, "%s: q_out's rows overlap", who);
  W8A8_CHECK_ARG(q != q_out || q_row == q_out_row || pb.n_rows == 1, W8A8_ERR_SHAPE, "%s: in place needs the same row stride",
                 who);
  return W8A8_OK;
}

w8a8_status launch_rope_append(const w8a8_rope_table& rt, const PagedCache& pc, const PagedBatch& pb, int dim, bool bf16,
                               const uint16_t* q, int64_t q_row, int n_q, const uint16_t* k, int64_t k_row,
                               const uint16_t* v, int64_t v_row, const float* q_norm, const float* k_norm, float eps,
                               uint16_t* q_out, int64_t q_out_row, int sms, cudaStream_t st) {
  const RopeArgs r{rt.turns, rt.scale, rt.rotary_dim, rt.interleaved};
  const int units = dim / 16, step = head_step(pb.n_rows, units, n_q + 2 * pc.n_kv, sms);
  const int64_t threads = (int64_t)pb.n_rows * units * step;
  const dim3 grid((unsigned)((threads + kThreads - 1) / kThreads));
  auto go = [&](auto kernel) {
    return launch_pdl(kernel, grid, dim3(kThreads), 0, st, r, pc, pb, q, q_row, n_q, k, k_row, v, v_row, q_norm, k_norm, eps,
                      q_out, q_out_row, step);
  };
  W8A8_CUDA(bf16 ? (units == 16  ? go(rope_append_kernel<true, 16>)
                    : units == 8 ? go(rope_append_kernel<true, 8>)
                                 : go(rope_append_kernel<true, 4>))
                 : (units == 16  ? go(rope_append_kernel<false, 16>)
                    : units == 8 ? go(rope_append_kernel<false, 8>)
                                 : go(rope_append_kernel<false, 4>)));
  return W8A8_OK;
}

w8a8_status check_paged(const char* who, const w8a8_paged_cache* c, const w8a8_paged_batch* b, PagedCache* pc,
                        PagedBatch* pb) {
  W8A8_CHECK_ARG(c && b, W8A8_ERR_INVALID_ARG, "%s: null cache or batch", who);
  W8A8_CHECK_ARG(c->dtype == W8A8_TYPE_BF16 || c->dtype == W8A8_TYPE_F16, W8A8_ERR_INVALID_ARG,
                 "%s: the cache's type must be bf16 or fp16", who);
  W8A8_CHECK_ARG(c->n_pages > 0 && c->n_kv > 0 && b->n_seqs >= 0 && b->n_rows >= 0 && b->max_new >= 1 && b->max_pages >= 0,
                 W8A8_ERR_INVALID_ARG, "%s: n_pages %d, n_kv %d, n_seqs %d, n_rows %d, max_new %d, max_pages %d", who,
                 c->n_pages, c->n_kv, b->n_seqs, b->n_rows, b->max_new, b->max_pages);
  W8A8_CHECK_ARG(c->head_dim == 64 || c->head_dim == 128 || c->head_dim == 256, W8A8_ERR_SHAPE,
                 "%s: head_dim %d must be 64, 128 or 256", who, c->head_dim);
  int shift = 4;
  while (shift < 8 && (1 << shift) < c->page_size) ++shift;
  W8A8_CHECK_ARG((1 << shift) == c->page_size, W8A8_ERR_SHAPE, "%s: page_size %d must be 16, 32, 64, 128 or 256", who,
                 c->page_size);
  W8A8_CHECK_ARG((long long)b->max_pages << shift <= (1ll << 30) && b->n_rows <= (1 << 28) && b->n_seqs <= (1 << 28) &&
                     (long long)c->n_kv * c->head_dim <= 65536,
                 W8A8_ERR_SHAPE, "%s: more than 2^30 positions a sequence, 2^28 rows or sequences, or n_kv * head_dim above 65536",
                 who);
  const int64_t str[3] = {c->page_stride, c->slot_stride, c->head_stride};
  for (int64_t s : str)
    W8A8_CHECK_ARG(s >= c->head_dim && s % 8 == 0 && s <= (1ll << 38), W8A8_ERR_SHAPE,
                   "%s: cache strides must be multiples of 8 from head_dim on", who);
  W8A8_CHECK_ARG(b->n_seqs == 0 || b->n_rows == 0 ||
                     (c->k && c->v && b->row_start && b->kv_len && (b->pages || b->max_pages == 0)),
                 W8A8_ERR_INVALID_ARG, "%s: null pointer", who);
  W8A8_CHECK_ARG(aligned16(c->k) && aligned16(c->v), W8A8_ERR_ALIGN, "%s: the cache must be 16-byte aligned", who);
  W8A8_CHECK_ARG((reinterpret_cast<uintptr_t>(b->row_start) & 3u) == 0 && (reinterpret_cast<uintptr_t>(b->kv_len) & 3u) == 0 &&
                     (reinterpret_cast<uintptr_t>(b->pages) & 3u) == 0,
                 W8A8_ERR_ALIGN, "%s: the batch's arrays must be 4-byte aligned", who);
  *pc = PagedCache{c->n_pages, shift, c->n_kv, c->page_stride, c->slot_stride, c->head_stride, c->k, c->v};
  *pb = PagedBatch{b->n_seqs, b->n_rows, b->max_pages, b->row_start, b->kv_len, b->pages};
  return W8A8_OK;
}

}  // namespace w8a8

using namespace w8a8;

extern "C" w8a8_status w8a8_rope_frequencies(const w8a8_rope_cfg* c, uint64_t* turns, float* scale) {
  const char* who = "w8a8_rope_frequencies";
  W8A8_CHECK_ARG(c && turns && scale, W8A8_ERR_INVALID_ARG, "%s: null argument", who);
  W8A8_CHECK_ARG(c->rotary_dim >= 16 && c->rotary_dim % 16 == 0 && c->rotary_dim <= kMaxDim, W8A8_ERR_SHAPE,
                 "%s: rotary_dim %d must be a multiple of 16 in [16, %d]", who, c->rotary_dim, kMaxDim);
  W8A8_CHECK_ARG(c->base > 1.0 && std::isfinite(c->base) && c->scaling >= W8A8_ROPE_NONE && c->scaling <= W8A8_ROPE_PARTS &&
                     c->attn_factor >= 0.0 && std::isfinite(c->attn_factor),
                 W8A8_ERR_INVALID_ARG, "%s: base %g, scaling %d, attn_factor %g", who, c->base, c->scaling, c->attn_factor);
  const bool banded = c->scaling >= W8A8_ROPE_WAVELENGTH;
  W8A8_CHECK_ARG(c->scaling == W8A8_ROPE_NONE || (c->factor > 0.0 && std::isfinite(c->factor)), W8A8_ERR_INVALID_ARG,
                 "%s: factor %g", who, c->factor);
  W8A8_CHECK_ARG(!banded || (c->low > 0.0 && c->high > c->low && std::isfinite(c->high) && c->original_len > 0),
                 W8A8_ERR_INVALID_ARG, "%s: low %g, high %g, original_len %d", who, c->low, c->high, c->original_len);
  const double two_pi = 6.283185307179586476925286766559;
  const int half = c->rotary_dim / 2;
  double a = 0.0, b = 0.0;
  if (c->scaling == W8A8_ROPE_PARTS) {
    auto at = [&](double x) { return c->rotary_dim * std::log(c->original_len / (two_pi * x)) / (2.0 * std::log(c->base)); };
    a = std::fmax(0.0, std::floor(at(c->high)));
    b = std::fmin((double)(c->rotary_dim - 1), std::ceil(at(c->low)));
  }
  for (int i = 0; i < half; ++i) {
    double f = std::pow(c->base, -2.0 * i / c->rotary_dim);
    if (c->scaling == W8A8_ROPE_LINEAR) f /= c->factor;
    if (c->scaling == W8A8_ROPE_WAVELENGTH) {
      const double m = std::fmin(1.0, std::fmax(0.0, (c->original_len * f / two_pi - c->low) / (c->high - c->low)));
      f *= m + (1.0 - m) / c->factor;
    }
    if (c->scaling == W8A8_ROPE_PARTS) {
      const double r = std::fmin(1.0, std::fmax(0.0, (i - a) / std::fmax(b - a, 0.001)));
      f *= (1.0 - r) + r / c->factor;
    }
    const double turn = f / two_pi - std::floor(f / two_pi);  // whole turns a position change nothing
    turns[i] = turn >= 1.0 ? 0ull : (uint64_t)std::ldexp(turn, 64);
  }
  const double def = c->scaling == W8A8_ROPE_PARTS && c->factor > 1.0 ? 0.1 * std::log(c->factor) + 1.0 : 1.0;
  *scale = (float)(c->attn_factor > 0.0 ? c->attn_factor : def);
  return W8A8_OK;
}

extern "C" w8a8_status w8a8_rope(const w8a8_rope_table* rope, int dtype, const uint16_t* x, int64_t x_row, int64_t x_head,
                                 int T, int heads, int dim, const int32_t* positions, uint16_t* y, int64_t y_row,
                                 int64_t y_head, void* stream) {
  const char* who = "w8a8_rope";
  W8A8_CHECK_ARG(T >= 0 && heads >= 0, W8A8_ERR_INVALID_ARG, "%s: T=%d, heads=%d", who, T, heads);
  W8A8_CHECK_ARG(dtype == W8A8_TYPE_BF16 || dtype == W8A8_TYPE_F16, W8A8_ERR_INVALID_ARG, "%s: type %d must be bf16 or fp16",
                 who, dtype);
  W8A8_CHECK_ARG(dim >= 16 && dim % 16 == 0 && dim <= kMaxDim, W8A8_ERR_SHAPE, "%s: dim %d must be a multiple of 16 in [16, %d]",
                 who, dim, kMaxDim);
  W8A8_TRY(check_rope(who, rope, dim));
  if (T == 0 || heads == 0) return W8A8_OK;
  W8A8_CHECK_ARG(heads <= 1 << 30, W8A8_ERR_SHAPE, "%s: more than 2^30 heads", who);  // a thread's steps over them fit in 32 bits
  W8A8_CHECK_ARG(x && y && positions, W8A8_ERR_INVALID_ARG, "%s: null pointer", who);
  W8A8_CHECK_ARG(aligned16(x) && aligned16(y) && (reinterpret_cast<uintptr_t>(positions) & 3u) == 0, W8A8_ERR_ALIGN,
                 "%s: x and y must be 16-byte aligned, positions 4-byte", who);
  const int64_t big = 1ll << 40;
  W8A8_CHECK_ARG(x_row % 8 == 0 && x_head % 8 == 0 && y_row % 8 == 0 && y_head % 8 == 0 && x_row >= 0 && x_head >= 0 &&
                     x_row <= big && x_head <= big && y_row <= big && y_head <= big,
                 W8A8_ERR_SHAPE, "%s: strides must be multiples of 8", who);
  // y's rows and heads apart, whichever of the two is the outer one
  W8A8_CHECK_ARG((heads == 1 || y_head >= dim) && (T == 1 || y_row >= dim) &&
                     (heads == 1 || T == 1 || y_row >= (heads - 1) * y_head + dim || y_head >= (T - 1) * y_row + dim),
                 W8A8_ERR_SHAPE, "%s: y's rows overlap (strides %lld, %lld)", who, (long long)y_row, (long long)y_head);
  W8A8_CHECK_ARG(x != y || (x_row == y_row || T == 1) && (x_head == y_head || heads == 1), W8A8_ERR_SHAPE,
                 "%s: in place needs the same strides", who);
  DevInfo d;
  W8A8_TRY(dev_info(&d));
  const RopeArgs r{rope->turns, rope->scale, rope->rotary_dim, rope->interleaved};
  const int units = dim / 16, step = head_step(T, units, heads, d.sms);
  const int64_t blocks = ((int64_t)T * units * step + kThreads - 1) / kThreads;
  W8A8_CHECK_ARG(blocks <= 0x7fffffffll, W8A8_ERR_SHAPE, "%s: T=%d with %d heads of %d is too large", who, T, heads, dim);
  auto go = [&](auto kernel) {
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3(kThreads), 0, as_stream(stream), r, x, x_row, x_head, T, heads,
                      units, step, positions, y, y_row, y_head);
  };
  W8A8_CUDA(dtype == W8A8_TYPE_BF16 ? go(rope_kernel<true>) : go(rope_kernel<false>));
  return W8A8_OK;
}

extern "C" w8a8_status w8a8_rope_append(const w8a8_rope_table* rope, const w8a8_paged_cache* cache,
                                        const w8a8_paged_batch* batch, const uint16_t* q, int64_t q_row, int n_q,
                                        const uint16_t* k, int64_t k_row, const uint16_t* v, int64_t v_row,
                                        const float* q_norm, const float* k_norm, float eps, uint16_t* q_out,
                                        int64_t q_out_row, void* stream) {
  const char* who = "w8a8_rope_append";
  PagedCache pc;
  PagedBatch pb;
  W8A8_TRY(check_paged(who, cache, batch, &pc, &pb));
  W8A8_TRY(check_rope(who, rope, cache->head_dim));
  const int dim = cache->head_dim;
  W8A8_TRY(check_append(who, pb, dim, q, q_row, n_q, k, k_row, v, v_row, q_norm, k_norm, eps, q_out, q_out_row));
  if (pb.n_seqs == 0 || pb.n_rows == 0) return W8A8_OK;
  DevInfo d;
  W8A8_TRY(dev_info(&d));
  return launch_rope_append(*rope, pc, pb, dim, cache->dtype == W8A8_TYPE_BF16, q, q_row, n_q, k, k_row, v, v_row, q_norm,
                            k_norm, eps, q_out, q_out_row, d.sms, as_stream(stream));
}
