// Attention over a paged cache: what its two kernels share.
//
// Work.  An item is (sequence, key/value head, tile of rows); its rows are the tokens of the tile times the query
// heads of the group, so that a group reads its keys once.  Its cost is the number of key tiles any of its rows sees.  All
// items, one after the other, make a line of key tiles, which the workers of the grid (its CTAs) divide into
// equal stretches: whatever the lengths, they finish together.  An item that a stretch border cuts leaves fp32
// partials (output, reference, sum) in the workspace, and the last of its pieces to arrive joins them in the order of the
// pieces: a fixed order, so results do not depend on who was last.  Where stretches are short (kShort tiles), two cut items
// a worker would cost more than the balance gains: if items cut into pieces of at most `unit` tiles, for a unit of up to twice the
// even share, make no more pieces than there are workers, each worker takes one piece.  A prompt of 2048 tokens at head
// dim 256 (4 tiles a worker) takes 28.5 us so, and 37.7 in equal stretches; 32 single tokens in a window of 1024 (4) 16.6
// and 19.6; 160 items of 10 tiles (11) 40.2 and 39.9, which is where kShort comes from.  Lengths are read on the device, so
// a captured call follows them.
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
// the device's word of waits that gave up
w8a8_status gave_up_word(unsigned int** word);
// what a call's heads, rows, strides and workspace have to be
w8a8_status check_heads(const char* who, int n_kv, int dim, int n_q);
w8a8_status check_attention(const char* who, const PagedBatch& pb, const uint16_t* q, int64_t q_row, int64_t q_head, int n_q,
                            int dim, float scale, int window, const uint16_t* o, int64_t o_row, int64_t o_head);
w8a8_status check_attention_ws(const char* who, int dim, int sms, const void* workspace, size_t ws_bytes);

// A wait that gave up, in the workspace's error word and in the device's: a decoder's workspace and a captured call's are out of
// the caller's reach.
__device__ __forceinline__ void give_up(unsigned int* err, const AttnCall& a, unsigned int bits) {
  atomicOr(err, bits);
  atomicOr(a.gave_up, bits);
}

// mbar_wait_warp, whose limit begins again whenever `beat`, in shared memory, has moved: while a warp computes rows again exactly
// (11 us a key for a warp's 32 rows at head dim 256, 3 s at 260000 keys), the others' copies and products wait for it.
__device__ __forceinline__ bool wait_beat(uint32_t bar, uint32_t parity, const uint32_t* beat) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  long long t0 = clock64();
  uint32_t seen = *reinterpret_cast<const volatile uint32_t*>(beat);
  while (!__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) {
    const uint32_t now = *reinterpret_cast<const volatile uint32_t*>(beat);
    if (__any_sync(0xffffffffu, now != seen)) {
      seen = now;
      t0 = clock64();
    } else if (__any_sync(0xffffffffu, clock64() - t0 > kWaitBudgetCycles)) {
      return false;
    }
  }
  return true;
}

// A row's reference moves when its maximum grew by 2^kGrowth, and weights are 2^kLift times what they are against it, so that they
// stay within 2^8 in bf16 and 2^15 in fp16, where the largest are put near the type's end: weights down to 2^-26 of the
// reference are normal numbers and those down to 2^-37 are counted (unlifted, 2^-14 and 2^-25: a tail of 40000 keys at
// 2^-25.5 vanished, which is 8e-4 of the output).
template <bool kBf16>
constexpr float kGrowth = kBf16 ? 8.0f : 3.0f;
template <bool kBf16>
constexpr float kLift = kBf16 ? 0.0f : 12.0f;
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

constexpr int kShort = 12;

// A worker's place on the line, in its units: key tiles, or pieces of up to `unit` of them.
struct LineStart {
  long long total, begin, end;  // units in all; this worker's stretch
  long long head_cost;          // units of one head of sequence s
  long long rest;               // units of sequence s before `begin`
  int s, workers, unit;         // unit 0: key tiles
  SeqShape q;                   // of sequence s
  int extra;                    // units ahead of an item's tiles that stand for what an item costs beside them; nobody's work
};
__device__ __forceinline__ int units_of(int n, int unit) { return unit ? (n + unit - 1) / unit : n; }

// The sum of f(key tiles) over the row tiles of each lane's sequence, for one head (0 rows: 0).  Sequences of many row tiles are
// summed by the whole warp, so that one long prompt does not leave a single thread counting.
template <class F>
__device__ __forceinline__ long long sum_tiles(const SeqShape& q, int window, int tt, int bk_shift, int lane, F f) {
  const int tiles = (q.rows + tt - 1) / tt;
  long long cost = 0;
  int first;
  if (tiles <= 4)
    for (int t = 0; t < tiles; ++t) cost += f(tiles_seen(q, window, tt, bk_shift, t, first));
  for (uint32_t many = __ballot_sync(0xffffffffu, tiles > 4); many; many &= many - 1) {
    const int src = __ffs(many) - 1;
    SeqShape p;
    p.row0 = 0;
    p.rows = __shfl_sync(0xffffffffu, q.rows, src);
    p.keys = 0;
    p.pos0 = __shfl_sync(0xffffffffu, q.pos0, src);
    const int n = (p.rows + tt - 1) / tt;
    unsigned long long sum = 0;
    for (int t = lane; t < n; t += 32) sum += (unsigned long long)f(tiles_seen(p, window, tt, bk_shift, t, first));
    // the warp's sum in three digits of 24 bits
    const uint32_t a = __reduce_add_sync(0xffffffffu, (uint32_t)(sum & 0xffffffu)),
                   b = __reduce_add_sync(0xffffffffu, (uint32_t)((sum >> 24) & 0xffffffu)),
                   c = __reduce_add_sync(0xffffffffu, (uint32_t)(sum >> 48));
    if (lane == src) cost = (long long)(a + ((unsigned long long)b << 24) + ((unsigned long long)c << 48));
  }
  return cost;
}

// All of the block's kT threads; `out` and `scan` (kT / 32 words) in shared memory.  Each thread takes `per` neighbouring
// sequences; up to 32 of them are one warp's alone.
template <int kT>
__device__ __forceinline__ void find_start(const PagedBatch& b, int page_shift, int n_kv, int window, int tt, int bk_shift,
                                           int worker, int workers, LineStart* out, long long* scan, int extra = 0,
                                           float per_unit = 0.0f) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool one_warp = b.n_seqs <= 32;
  if (one_warp && warp > 0) {
    __syncthreads();
    return;
  }
  const int per = one_warp ? 1 : (b.n_seqs + kT - 1) / kT;
  SeqShape q{0, 0, 0, 0};
  auto sum_of = [&](int s, auto f) {
    if (per > 1 || s < 0) {
      s = s < 0 ? ~s : s;
      q = SeqShape{0, 0, 0, 0};
      if (s < b.n_seqs) q = seq_shape(b, s, page_shift);
    }
    return sum_tiles(q, window, tt, bk_shift, lane, f);
  };
  // the running sum over the block's threads, and its total
  auto run = [&](long long mine, long long& total) {
    if (b.n_seqs == 1) {
      total = __shfl_sync(0xffffffffu, mine, 0);
      return total;
    }
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    if (one_warp) {
      total = __shfl_sync(0xffffffffu, upto, 31);
      return upto;
    }
    __syncthreads();
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    total = 0;
    for (int w = 0; w < kT / 32; ++w) {
      if (w < warp) upto += scan[w];
      total += scan[w];
    }
    return upto;
  };
  long long one = 0, total = 0;
  for (int i = 0; i < per; ++i) one += sum_of(~(tid * per + i), [&](int n) { return (long long)(n + extra); });
  long long upto = run(one * n_kv, total);
  int unit = 0;
  // A piece costs its item's last one a join: of n tiles in pieces of u they take u tiles' time and n / u joins', least at the
  // square root of n times a join over a tile.  per_unit: that quotient over the items there can be (0: pieces of any size).
  const int few = (int)min((float)kShort, sqrtf(per_unit * (float)total));
  if ((total > workers || few > 1) && total <= (long long)kShort * workers) {
    // pieces for four units, 16 bits each (no more of them than tiles, 12 x 152)
    const int least = max((int)((total + workers - 1) / workers), few), step = max(1, (least + 2) / 4);
    uint32_t inv[4];  // quotients by a product: exact for the 12 x 152 tiles and units up to 21 there are
#pragma unroll
    for (int j = 0; j < 4; ++j) inv[j] = (uint32_t)ceilf(__fdividef(65536.0f, (float)(least + j * step)) + 0.001f);
    auto pieces = [&](int n) {
      uint32_t p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = (uint32_t)(n + least + j * step - 1) * inv[j] >> 16;
      return (long long)(((unsigned long long)(p[3] << 16 | p[2]) << 32) | (p[1] << 16 | p[0]));
    };
    long long some = 0, sums = 0;
    for (int i = 0; i < per; ++i) some += sum_of(tid * per + i, pieces);
    const long long upto4 = run(some * n_kv, sums);
#pragma unroll
    for (int j = 3; j >= 0; --j)
      if ((int)((sums >> (16 * j)) & 0xffff) <= workers) {
        unit = least + j * step;
        total = (sums >> (16 * j)) & 0xffff;
        upto = (upto4 >> (16 * j)) & 0xffff;
        one = (some >> (16 * j)) & 0xffff;
      }
  }
  if (unit) extra = 0;
  const long long mine = one * n_kv;
  const int used = (int)min((long long)workers, total);
  if (worker >= used) {
    if (tid == 0) *out = LineStart{total, 0, 0, 1, 0, 0, used, unit, q, 0};
    __syncthreads();
    return;
  }
  const long long begin = total * worker / used, end = total * (worker + 1) / used;
  const bool owner = begin >= upto - mine && begin < upto;
  if (per == 1) {
    if (owner) *out = LineStart{total, begin, end, one, begin - (upto - mine), tid, used, unit, q, extra};
  } else if (__any_sync(0xffffffffu, owner)) {  // the owner's warp walks its sequences again
    long long at = upto - mine;
    for (int i = 0; i < per; ++i) {
      const long long c = sum_of(tid * per + i, [&](int n) { return (long long)(units_of(n, unit) + extra); });
      if (begin >= at && begin < at + c * n_kv) *out = LineStart{total, begin, end, c, begin - at, tid * per + i, used, unit, q, extra};
      at += c * n_kv;
    }
  }
  __syncthreads();
}

// One item of a worker's stretch and this worker's piece of it; a warp walks the same items as the others.
struct Walk {
  long long off, at, end;   // line offsets: the item's first unit, the piece's, the stretch's end
  SeqShape q;
  int s, h, t, row_tiles, unit, extra;
  int first, n;             // the item's key tiles: first, first + 1, ..
  int k0, cnt;              // the piece: tiles k0 .. k0 + cnt - 1 of them

  __device__ __forceinline__ void piece() {
    if (unit) {  // one unit: as even a share of the tiles as it goes
      const int of = units_of(n, unit), j = (int)(at - off);
      k0 = n * j / of;
      cnt = n * (j + 1) / of - k0;
    } else {
      k0 = (int)(at - off);
      cnt = (int)min((long long)(n - k0), end - at);
    }
  }
  // the whole warp
  __device__ __forceinline__ void start(const LineStart& ls, const PagedBatch& b, int page_shift, int window, int tt,
                                        int bk_shift, int lane) {
    s = ls.s;
    q = ls.q;
    unit = ls.unit;
    extra = ls.extra;
    row_tiles = (q.rows + tt - 1) / tt;
    h = ls.rest < ls.head_cost ? 0
        : ((ls.rest | ls.head_cost) >> 31) == 0 ? (int)((uint32_t)ls.rest / (uint32_t)ls.head_cost)
                                                 : (int)(ls.rest / ls.head_cost);
    long long left = ls.rest - h * ls.head_cost;  // units of this head before the stretch
    at = ls.begin;
    end = ls.end;
    for (int t0 = 0;; t0 += 32) {
      int f;
      const int c = t0 + lane < row_tiles ? units_of(tiles_seen(q, window, tt, bk_shift, t0 + lane, f), unit) + extra : 0;
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
        off = at - (left - __shfl_sync(0xffffffffu, upto - c, src)) + extra;  // the first tile's
        if (at < off) at = off;
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
    at += (unit ? 1 : cnt) + extra;
    if (at >= end) return;
    off += units_of(n, unit) + extra;
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

// The worker whose stretch holds line offset x: the last i with floor(total i / workers) <= x.
__device__ __forceinline__ int worker_of(long long x, const LineStart& ls) {
  return (int)(((x + 1) * ls.workers - 1) / ls.total);
}

// Partials.  A worker cuts at most two items: the one its stretch begins within (slot 0) and the one it ends within and began
// itself (slot 1); an item's pieces lie in slot 1 of its first worker and slot 0 of the following ones.  Arrivals are counted
// at the first worker's index in the workspace's counters.
struct Pieces {
  int first, count;  // workers
};
// One thread, after a barrier of the block: counts the block's piece in, its writes ahead of the count; what other blocks
// wrote ahead of theirs is visible to the block after its next barrier.  Returns whether it is the last of `of`.
__device__ __forceinline__ bool last_piece(unsigned int* counter, int of) {
  unsigned int before;
  asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;\n" : "=r"(before) : "l"(counter) : "memory");
  const bool last = before + 1 == (unsigned int)of;
  if (last) *counter = 0;
  return last;
}
__device__ __forceinline__ Pieces pieces_of(const Walk& w, const LineStart& ls) {
  Pieces p;
  p.first = worker_of(w.off, ls);
  p.count = worker_of(w.off + units_of(w.n, w.unit) - 1, ls) - p.first + 1;
  return p;
}

constexpr int kTokenRows = 16;    // rows of a partial of the kernels for tokens: [row][dim] outputs, then the rows' m and l
constexpr int kMaxPieces = 192;   // of an item: no more than CTAs

// The pieces of an item of up to 16 rows, joined in their order, by the consumer warps (threads 0 .. 32 kWarps - 1; barrier 1):
// outputs, times `back`, to o (row r at (r / group) o_row + (r % group) o_head).
// What another SM has just written takes a microsecond to read, so few loads follow one another: the statistics of all
// pieces (a warp a row, lane = piece), then every thread's part of the output with up to kAhead pieces in flight.  Rows whose
// result is not finite, or without weight, are marked in *bad.  Not inline: its registers are not the main loop's.
template <bool kBf16, int kDim, int kWarps>
__device__ __noinline__ void join_pieces(const float* part, int first, int count, int rows, int group, uint16_t* o, int64_t o_row,
                                         int64_t o_head, float* fac, uint32_t* bad, float back = 1.0f) {
  constexpr int kRows = kTokenRows, kPart = kRows * kDim + 2 * kRows, kConsumers = 32 * kWarps, kAhead = 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto slot = [&](int i) { return part + (size_t)(2 * (first + i) + (i == 0 ? 1 : 0)) * kPart; };
  float* sums = fac + kMaxPieces * kRows;  // fac: [piece][row] 2^(m - max)
  for (int r = warp; r < rows; r += kWarps) {
    float mi[kMaxPieces / 32], li[kMaxPieces / 32], top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int j = 0; j < kMaxPieces / 32; ++j) {
      const bool there = lane + 32 * j < count;
      mi[j] = there ? __ldcg(slot(lane + 32 * j) + kRows * kDim + r) : -INFINITY;
      li[j] = there ? __ldcg(slot(lane + 32 * j) + kRows * kDim + kRows + r) : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < kMaxPieces / 32; ++j) top = fmaxf(top, mi[j]);
    top = warp_max_f(top);
#pragma unroll
    for (int j = 0; j < kMaxPieces / 32; ++j) {
      const float f = mi[j] == -INFINITY ? 0.0f : ex2(mi[j] - top);
      sum = fmaf(li[j], f, sum);
      fac[(lane + 32 * j) * kRows + r] = f;
    }
    sum = warp_sum_f(sum);
    if (lane == 0) sums[r] = sum;
  }
  named_bar_sync(1, kConsumers);
  for (int e = threadIdx.x; e < rows * (kDim / 4); e += kConsumers) {  // four dims of a row
    const int r = e / (kDim / 4);
    float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i0 = 0; i0 < count; i0 += kAhead) {
      float4 x[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i0 + i < count) x[i] = __ldcg(reinterpret_cast<const float4*>(slot(i0 + i)) + e);
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i0 + i < count) {
          const float f = fac[(i0 + i) * kRows + r];
          y.x = fmaf(x[i].x, f, y.x);
          y.y = fmaf(x[i].y, f, y.y);
          y.z = fmaf(x[i].z, f, y.z);
          y.w = fmaf(x[i].w, f, y.w);
        }
    }
    const float sum = sums[r], inv = 1.0f / sum;
    y.x = y.x * inv * back, y.y = y.y * inv * back, y.z = y.z * inv * back, y.w = y.w * inv * back;
    *reinterpret_cast<uint2*>(o + (r / group) * o_row + (r % group) * o_head + 4 * (e % (kDim / 4))) =
        make_uint2(pack2<kBf16>(y.x, y.y), pack2<kBf16>(y.z, y.w));
    if (y.x * 0.0f + y.y * 0.0f + y.z * 0.0f + y.w * 0.0f != 0.0f || !(sum > 0.0f)) atomicOr(bad, 1u << r);
  }
}

// ------------------------------------------------------------------------------- one row exactly
// One row's attention by one warp, key by key in the order of the formula: NaN and infinities travel as they do
// in it, and nothing outside the row's range is read.  The kernels run it for rows whose result is not finite (a value
// that only other rows of the tile may see can make it so, or sums of weights times values beyond fp32's range: here the
// output so far is kept as an average, which stays within the values).  Lane l scores key j0 + l, then holds dims l, l + 32, ...
// It counts `beat` up as it goes (see wait_beat).
template <bool kBf16, int kDim>
__device__ __noinline__ void attend_row(const PagedCache& c, const PagedBatch& b, const AttnCall& a, int s, int pos,
                                        int64_t row, int head, int lane, uint32_t* beat) {
  const uint16_t* q = a.q + row * a.q_row + head * a.q_head;
  const int kvh = head / (a.n_q / c.n_kv);
  const int lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
  float m = -INFINITY, l = 0.0f, acc[kDim / 32];
  bool any = false;
#pragma unroll
  for (int i = 0; i < kDim / 32; ++i) acc[i] = 0.0f;
  for (int j0 = lo; j0 <= pos; j0 += 32) {
    if (lane == 0 && ((j0 - lo) & 8191) == 0) atomicAdd(beat, 1u);
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
  for (int i = 0; i < kDim / 32; ++i) o[lane + 32 * i] = (uint16_t)pack2<kBf16>(!any ? 0.0f : l == 0.0f ? NAN : acc[i], 0.0f);
}

}  // namespace w8a8
