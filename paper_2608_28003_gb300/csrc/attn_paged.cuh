// Attention over a paged cache: what its two kernels share.
//
// Work.  An item is (sequence, key/value head, tile of rows); its rows are the tokens of the tile times the query
// heads of the group, so that a group reads its keys once.  Its cost is the number of key tiles any of its
// rows sees.  All items, one after the other, make a line of key tiles, which the CTAs of the grid divide into equal
// stretches: whatever the lengths, the CTAs finish together.  An item that a stretch border cuts leaves fp32
// partials (output, reference, sum) in the workspace, and the last of its pieces to arrive joins them in the order of the
// pieces: a fixed order, so results do not depend on who was last.  Lengths are read on the device, so a captured call follows
// them.
#pragma once

#include "attn_common.cuh"
#include "paged.cuh"

namespace w8a8 {

// Tensor maps of a call: keys and values as [page][head][slot][dim] boxes of 64 dims x kBoxSlots slots (or a page's),
// and, for the chunk kernel, q as [row][head][dim].
constexpr int kBoxSlots = 32;
w8a8_status launch_attn_tokens(const PagedCache& pc, const PagedBatch& pb, const AttnCall& a, void* ws, int sms, cudaStream_t st);
w8a8_status launch_attn_chunks(const PagedCache& pc, const PagedBatch& pb, const AttnCall& a, void* ws, int sms, cudaStream_t st);
// bytes of the partials behind the workspace's reserved part
size_t attn_tokens_ws(int dim, int sms);
size_t attn_chunks_ws(int dim, int sms);

constexpr float kGrowth = 8.0f;  // a row's reference moves when its maximum grew by 2^8: weights stay within 2^8
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(x));
  return r;
}

// ------------------------------------------------------------------------------------ the line
// The key tiles rows [t tt, t tt + tt) of a sequence see: `first` of them and their number; a tile of rows without keys counts
// one, so that someone writes its zeros.
__device__ __forceinline__ int tiles_seen(const SeqShape& q, int window, int tt, int bk_shift, int t, int& first) {
  const int hi = q.pos0 + min(q.rows, (t + 1) * tt) - 1, lo = window > 0 ? max(0, q.pos0 + t * tt - window + 1) : 0;
  first = hi < 0 ? 0 : lo >> bk_shift;
  return hi < 0 ? 1 : (hi >> bk_shift) - first + 1;
}

// A CTA's place on the line.
struct LineStart {
  long long total, begin, end;  // key tiles in all; this CTA's stretch
  long long head_cost;          // key tiles of one head of sequence s
  long long rest;               // key tiles of sequence s before `begin`
  int s, ctas;
  SeqShape q;                   // of sequence s
};

// Key tiles of one head of each lane's sequence (0 rows: none).  Sequences of many row tiles are summed by the whole warp, so
// that one long prompt does not leave a single thread counting.
__device__ __forceinline__ long long head_cost(const SeqShape& q, int window, int tt, int bk_shift, int lane) {
  const int tiles = (q.rows + tt - 1) / tt;
  long long cost = 0;
  int first;
  if (tiles <= 4)
    for (int t = 0; t < tiles; ++t) cost += tiles_seen(q, window, tt, bk_shift, t, first);
  for (uint32_t many = __ballot_sync(0xffffffffu, tiles > 4); many; many &= many - 1) {
    const int src = __ffs(many) - 1;
    SeqShape p;
    p.row0 = 0;
    p.rows = __shfl_sync(0xffffffffu, q.rows, src);
    p.keys = 0;
    p.pos0 = __shfl_sync(0xffffffffu, q.pos0, src);
    const int n = (p.rows + tt - 1) / tt;
    long long sum = 0;
    for (int t = lane; t < n; t += 32) sum += tiles_seen(p, window, tt, bk_shift, t, first);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == src) cost = sum;
  }
  return cost;
}

// All of the block's kT threads; `out` and `scan` (kT / 32 words) in shared memory.  Each thread takes `per` neighbouring sequences; up
// to 32 of them are one warp's alone.  A stretch has at least `least` key tiles (but the line's last).
template <int kT>
__device__ __forceinline__ void find_start(const PagedBatch& b, int page_shift, int n_kv, int window, int tt, int bk_shift,
                                           int least, LineStart* out, long long* scan) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool one_warp = b.n_seqs <= 32;
  if (one_warp && warp > 0) {
    __syncthreads();
    return;
  }
  const int per = one_warp ? 1 : (b.n_seqs + kT - 1) / kT;
  SeqShape q{0, 0, 0, 0};
  auto cost_of = [&](int s) {
    q = SeqShape{0, 0, 0, 0};
    if (s < b.n_seqs) q = seq_shape(b, s, page_shift);
    return head_cost(q, window, tt, bk_shift, lane);
  };
  long long mine = 0;
  for (int i = 0; i < per; ++i) mine += cost_of(tid * per + i);
  const long long one = mine;
  mine *= n_kv;
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  long long total = 0;
  if (one_warp) {
    total = __shfl_sync(0xffffffffu, upto, 31);
  } else {
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    for (int w = 0; w < kT / 32; ++w) {
      if (w < warp) upto += scan[w];
      total += scan[w];
    }
  }
  const int ctas = (int)min((long long)gridDim.x, (total + least - 1) / least), cta = blockIdx.x;
  if (cta >= ctas) {
    if (tid == 0) *out = LineStart{total, 0, 0, 1, 0, 0, ctas, q};
    __syncthreads();
    return;
  }
  const long long begin = total * cta / ctas, end = total * (cta + 1) / ctas;
  const bool owner = begin >= upto - mine && begin < upto;
  if (per == 1) {
    if (owner) *out = LineStart{total, begin, end, one, begin - (upto - mine), tid, ctas, q};
  } else if (__any_sync(0xffffffffu, owner)) {  // the owner's warp walks its sequences again
    long long at = upto - mine;
    for (int i = 0; i < per; ++i) {
      const long long c = cost_of(tid * per + i);
      if (begin >= at && begin < at + c * n_kv) *out = LineStart{total, begin, end, c, begin - at, tid * per + i, ctas, q};
      at += c * n_kv;
    }
  }
  __syncthreads();
}

// One item of a CTA's stretch and this CTA's piece of it; a warp walks the same items as the others.
struct Walk {
  long long off, at, end;   // line offsets: the item's first key tile, the piece's, the stretch's end
  SeqShape q;
  int s, h, t, row_tiles;
  int first, n;             // the item's key tiles: first, first + 1, ..
  int k0, cnt;              // the piece: tiles k0 .. k0 + cnt - 1 of them

  __device__ __forceinline__ void piece() {
    k0 = (int)(at - off);
    cnt = (int)min((long long)(n - k0), end - at);
  }
  // the whole warp
  __device__ __forceinline__ void start(const LineStart& ls, const PagedBatch& b, int page_shift, int window, int tt,
                                        int bk_shift, int lane) {
    s = ls.s;
    q = ls.q;
    row_tiles = (q.rows + tt - 1) / tt;
    h = ls.rest < ls.head_cost ? 0
        : ((ls.rest | ls.head_cost) >> 31) == 0 ? (int)((uint32_t)ls.rest / (uint32_t)ls.head_cost)
                                                 : (int)(ls.rest / ls.head_cost);
    long long left = ls.rest - h * ls.head_cost;  // key tiles of this head before the stretch
    at = ls.begin;
    end = ls.end;
    for (int t0 = 0;; t0 += 32) {
      int f;
      const int c = t0 + lane < row_tiles ? tiles_seen(q, window, tt, bk_shift, t0 + lane, f) : 0;
      int upto = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
      }
      const uint32_t hit = __ballot_sync(0xffffffffu, left < upto);
      if (hit) {
        const int src = __ffs(hit) - 1;
        t = t0 + src;
        off = at - (left - __shfl_sync(0xffffffffu, upto - c, src));
        break;
      }
      left -= __shfl_sync(0xffffffffu, upto, 31);
      if (t0 + 32 >= row_tiles) {  // the arrays changed under the call: nothing of it is defined, but it ends
        t = 0;
        off = at;
        end = at;
        break;
      }
    }
    n = tiles_seen(q, window, tt, bk_shift, t, first);
    piece();
  }
  __device__ __forceinline__ bool more() const { return at < end; }
  __device__ __forceinline__ void next(const PagedBatch& b, int page_shift, int n_kv, int window, int tt, int bk_shift) {
    at += cnt;
    if (at >= end) return;
    off += n;
    if (++t == row_tiles) {
      t = 0;
      if (++h == n_kv) {
        h = 0;
        do {
          if (++s >= b.n_seqs) {  // as above
            end = at;
            return;
          }
          q = seq_shape(b, s, page_shift);
        } while (q.rows == 0);
        row_tiles = (q.rows + tt - 1) / tt;
      }
    }
    n = tiles_seen(q, window, tt, bk_shift, t, first);
    piece();
  }
  __device__ __forceinline__ bool whole() const { return cnt == n; }
  // the range of keys any row of the item sees
  __device__ __forceinline__ int lo(int window, int tt) const {
    return window > 0 ? max(0, q.pos0 + t * tt - window + 1) : 0;
  }
  __device__ __forceinline__ int hi(int tt) const { return q.pos0 + min(q.rows, (t + 1) * tt) - 1; }
};

// The pages of 32 consecutive 16-key groups, one a lane (-1: none, or none of its box of `box` keys in lo .. hi), beginning with
// position p0 of sequence s.
__device__ __forceinline__ int group_page(const PagedBatch& b, const PagedCache& c, int s, int p0, int lo, int hi, int box, int lane) {
  const int p = p0 + 16 * lane, col = p >> c.page_shift;
  int page = -1;
  if (p <= hi && (p | (box - 1)) >= lo && col < b.max_pages) page = b.pages[(int64_t)s * b.max_pages + col];
  return page < 0 || page >= c.n_pages ? -1 : page;
}

// The CTA whose stretch holds line offset x: the last i with floor(total i / ctas) <= x.
__device__ __forceinline__ int cta_of(long long x, const LineStart& ls) {
  return (int)(((x + 1) * ls.ctas - 1) / ls.total);
}

// Partials.  A CTA cuts at most two items: the one its stretch begins within (slot 0) and the one it ends within and began
// itself (slot 1); an item's pieces lie in slot 1 of its first CTA and slot 0 of the following ones.  Arrivals are counted
// at the first CTA's index in the workspace's counters.
struct Pieces {
  int first, count;  // CTAs
};
__device__ __forceinline__ Pieces pieces_of(const Walk& w, const LineStart& ls) {
  Pieces p;
  p.first = cta_of(w.off, ls);
  p.count = cta_of(w.off + w.n - 1, ls) - p.first + 1;
  return p;
}

// ------------------------------------------------------------------------------- one row exactly
// One row's attention by one warp, key by key in the order of the formula: NaN and infinities travel as they do
// in it, and nothing outside the row's range is read.  The kernels run it for rows whose result is not finite (a value
// that only other rows of the tile may see can make it so).  Lane l scores key j0 + l, then holds dims l, l + 32, ...
template <bool kBf16, int kDim>
__device__ __noinline__ void attend_row(const PagedCache& c, const PagedBatch& b, const AttnCall& a, int s, int pos,
                                        int64_t row, int head, int lane) {
  const uint16_t* q = a.q + row * a.q_row + head * a.q_head;
  const int kvh = head / (a.n_q / c.n_kv);
  const int lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
  float m = -INFINITY, l = 0.0f, acc[kDim / 32];
  bool any = false;
#pragma unroll
  for (int i = 0; i < kDim / 32; ++i) acc[i] = 0.0f;
  for (int j0 = lo; j0 <= pos; j0 += 32) {
    const int j = j0 + lane;
    const int64_t at = j <= pos ? key_offset(b, c, s, j, kvh) : -1;
    float sc = -INFINITY;
    if (at >= 0) {
      float d = 0.0f;
      for (int i = 0; i < kDim / 8; ++i) {
        const uint4 kw = *reinterpret_cast<const uint4*>(c.k + at + 8 * i), qw = *reinterpret_cast<const uint4*>(q + 8 * i);
        const uint32_t ka[4] = {kw.x, kw.y, kw.z, kw.w}, qa[4] = {qw.x, qw.y, qw.z, qw.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 x = unpack2<kBf16>(ka[e]), y = unpack2<kBf16>(qa[e]);
          d = fmaf(x.x, y.x, d);
          d = fmaf(x.y, y.y, d);
        }
      }
      sc = d * a.scale;
    }
    const uint32_t there = __ballot_sync(0xffffffffu, at >= 0);
    if (!there) continue;
    any = true;
    const float m_new = fmaxf(m, warp_max_f(sc));
    const float ref = m_new == -INFINITY ? 0.0f : m_new;
    const float corr = m == -INFINITY ? 0.0f : expf(m - ref);
    const float p = at >= 0 ? expf(sc - ref) : 0.0f;
    l = l * corr + warp_sum_f(p);
#pragma unroll
    for (int i = 0; i < kDim / 32; ++i) acc[i] *= corr;
    for (int u = 0; u < 32; ++u) {
      if (!((there >> u) & 1u)) continue;
      const float pu = __shfl_sync(0xffffffffu, p, u);
      const int64_t au = __shfl_sync(0xffffffffu, (long long)at, u);
#pragma unroll
      for (int i = 0; i < kDim / 32; ++i) {
        const float2 v = unpack2<kBf16>((uint32_t)c.v[au + lane + 32 * i]);
        acc[i] = fmaf(pu, v.x, acc[i]);
      }
    }
    m = m_new;
  }
  uint16_t* o = a.o + row * a.o_row + head * a.o_head;
#pragma unroll
  for (int i = 0; i < kDim / 32; ++i) o[lane + 32 * i] = (uint16_t)pack2<kBf16>(any ? acc[i] / l : 0.0f, 0.0f);
}

}  // namespace w8a8
