// Attention over a paged cache for single tokens and a few drafted ones: items of up to 16 rows (tokens times the query heads
// of a group).
//
// The cache is read once and little is computed with it, so HBM bounds the kernel; everything is arranged to keep copies in
// flight.  One CTA per SM walks its stretch of the line of key tiles (attn_paged.cuh).  A loader warp copies K and V tiles,
// page by page, into a ring of three stages of 64 KB by TMA (64, 128, 256 keys at head dims 256, 128, 64); kWarps consumer
// warps take 16 keys of a tile each (32 at head dim 64, where the chain of a step would not keep up with the copies: 51.8 ->
// 40.4 us below), on their own from scores to output: no barrier inside the loop but the ring's.  The products are mma.sync
// m16n8k16 (16 rows are one operand's height: tcgen05's 128 would be mostly padding, and at the rate HBM feeds an SM this
// takes a third of the legacy tensor rate); K is read by ldmatrix, V by its transposing form, and a score fragment is the
// next product's operand as it is.  A warp keeps its own reference, sum and output; they are joined in shared memory when
// the item ends.
//
// Measured: 64 sequences of up to 30000 keys at head dim 256 (934 MB) 147-151 us, 6.2-6.4 TB/s (0.91-0.94 of the measured
// copy); 20 sequences of 4 drafted tokens behind up to 5000 keys, 8 heads of 64 in pages of 16 (98 MB, 160 items of about 10
// tiles) 40.3 us: 5 until the first tile is there, 15 of copies, and an item's end costs 2 to 3 (the warps' join, and for a cut
// item the partial, its arrival and the join of the pieces), twice a CTA; the rest, a third, is not accounted for.  One
// sequence of 700 keys 11 to 12 us, latency alone.
#include "attn_paged.cuh"
#include "ops.cuh"
#include "tmap.cuh"

namespace w8a8 {

namespace {

constexpr int kRows = 16;
constexpr int kMaxPieces = 192;  // of an item: no more than CTAs

template <int kDim>
struct Cfg {
  static constexpr int kWarps = kDim == 256 ? 4 : 8;          // consumers
  static constexpr int kBlocks = kDim == 64 ? 2 : 1;          // of 16 keys, that a warp has of a tile
  static constexpr int kBk = 16 * kBlocks * kWarps, kBkShift = kDim == 256 ? 6 : kDim == 128 ? 7 : 8;
  static constexpr int kChunks = kDim / 64;                   // 128-byte columns of a tile
  static constexpr int kSub = kBk * 128, kTile = kChunks * kSub, kStage = 2 * kTile;
  static constexpr int kStages = 196608 / kStage;             // 3
  static constexpr int kJoin = kWarps * 8 * kDim * 4;         // 8 rows' outputs of every warp
  static constexpr int kPer = kDim / 8 / kWarps;              // groups of 8 dims that a warp joins
  static constexpr int kSmem = kStages * kStage + kJoin + 1024;
  static constexpr int kThreads = 32 * (kWarps + 1);
  // floats of a partial: [16 rows][dim] outputs, then m and l of the rows
  static constexpr int kPart = kRows * kDim + 2 * kRows;
};

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
template <bool kBf16>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (kBf16)
    mma_bf16_16816(c, a[0], a[1], a[2], a[3], b0, b1);
  else
    mma_f16_16816(c, a[0], a[1], a[2], a[3], b0, b1);
}

// The pieces of an item, joined in their order, by the consumer warps: outputs to o (row r at (r / group) o_row + (r % group) o_head).
// What another SM has just written takes a microsecond to read, so few loads follow one another: the statistics of all
// pieces (a warp a row, lane = piece), then every thread's part of the output with up to kAhead pieces in flight.  Rows whose
// result is not finite, or without weight, are marked in *bad.  Not inline: its registers are not the main loop's.
template <bool kBf16, int kDim>
__device__ __noinline__ void join_pieces(const float* part, int first, int count, int rows, int group, uint16_t* o, int64_t o_row,
                                         int64_t o_head, float* fac, uint32_t* bad) {
  using C = Cfg<kDim>;
  constexpr int kConsumers = 32 * C::kWarps, kAhead = 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto slot = [&](int i) { return part + (size_t)(2 * (first + i) + (i == 0 ? 1 : 0)) * C::kPart; };
  float* sums = fac + kMaxPieces * kRows;  // fac: [piece][row] 2^(m - max)
  static_assert(C::kJoin >= (kMaxPieces + 1) * kRows * (int)sizeof(float), "the factors fit over the join buffer");
  for (int r = warp; r < rows; r += C::kWarps) {
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
    y.x *= inv, y.y *= inv, y.z *= inv, y.w *= inv;
    *reinterpret_cast<uint2*>(o + (r / group) * o_row + (r % group) * o_head + 4 * (e % (kDim / 4))) =
        make_uint2(pack2<kBf16>(y.x, y.y), pack2<kBf16>(y.z, y.w));
    if (y.x * 0.0f + y.y * 0.0f + y.z * 0.0f + y.w * 0.0f != 0.0f || !(sum > 0.0f)) atomicOr(bad, 1u << r);
  }
}

template <bool kBf16, int kDim>
__global__ void __launch_bounds__(Cfg<kDim>::kThreads, 1)
    attn_tokens_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, PagedCache c,
                       PagedBatch b, AttnCall a, int tt, float* __restrict__ part, unsigned int* __restrict__ counters,
                       unsigned int* __restrict__ err) {
  using C = Cfg<kDim>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ uint64_t bars[2 * C::kStages];
  __shared__ LineStart ls;
  __shared__ long long scan[C::kThreads / 32];
  __shared__ uint32_t held[C::kStages];                    // 16-key groups of a stage's tile that lie in a page
  __shared__ float s_m[C::kWarps][kRows], s_l[C::kWarps][kRows];
  __shared__ uint32_t s_last, s_bad, s_beat;
  const uint32_t raw = smem_u32(smem_raw), ring = (raw + 1023u) & ~1023u;
  float2* join = reinterpret_cast<float2*>(smem_raw + (ring - raw) + C::kStages * C::kStage);
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  auto empty = [&](int i) { return bar0 + 8u * (uint32_t)(C::kStages + i); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), C::kWarps);
    }
    fence_mbar_init();
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
    s_bad = s_beat = 0;
  }
  pdl_wait();
  pdl_trigger();
  find_start<C::kThreads>(b, c.page_shift, c.n_kv, a.window, tt, C::kBkShift, (int)blockIdx.x, (int)gridDim.x, &ls, scan);
  if (ls.begin >= ls.end) return;
  Walk w;
  w.start(ls, b, c.page_shift, a.window, tt, C::kBkShift, lane);
  int g = 0;  // tiles of this CTA so far
  bool ok = true;

  if (warp == C::kWarps) {
    // -------------------------------------------------------------------------- loader
    const int box = min(kBoxSlots, 1 << c.page_shift), boxes = C::kBk / box;  // per tile and column
    const int n_ops = 2 * C::kChunks * boxes;
    for (; ok && w.more(); w.next(b, c.page_shift, c.n_kv, a.window, tt, C::kBkShift)) {
      const int lo = w.lo(a.window, tt), hi = w.hi(tt);
      constexpr int kGroups = C::kBk / 16, kBatch = 32 / kGroups;  // tiles whose pages are read at once, ahead of their use
      int page = group_page(b, c, w.s, (w.first + w.k0) << C::kBkShift, lo, hi, box, lane), ahead = -1;
      for (int i = 0; i < w.cnt; ++i, ++g) {
        const int st = g % C::kStages, tile0 = (w.first + w.k0 + i) << C::kBkShift, in_batch = i % kBatch;
        if (in_batch == 0) {
          if (i > 0) page = ahead;
          if (i + kBatch < w.cnt) ahead = group_page(b, c, w.s, tile0 + (kBatch << C::kBkShift), lo, hi, box, lane);
        }
        const uint32_t there = (__ballot_sync(0xffffffffu, page >= 0) >> (in_batch * kGroups)) & ((1u << kGroups) - 1u);
        if (g >= C::kStages && !wait_beat(empty(st), (uint32_t)(g / C::kStages - 1) & 1u, &s_beat)) {
          ok = false;
          break;
        }
        if (lane == 0) {
          held[st] = there;
          mbar_arrive_expect_tx(full(st), C::kStage);
        }
        __syncwarp();
        const uint32_t dst = ring + (uint32_t)(st * C::kStage);
        for (int o0 = 0; o0 < n_ops; o0 += 32) {
          const int o = o0 + lane, bx = o % boxes, ch = o / boxes % C::kChunks, kv = o / boxes / C::kChunks;
          const int pg = __shfl_sync(0xffffffffu, page, (in_batch * kGroups + bx * (box / 16)) & 31);
          if (o < n_ops) {
            const int slot = (tile0 + bx * box) & ((1 << c.page_shift) - 1);
            // a page that holds nothing: a coordinate outside the tensor, which fills zeros
            tma_load_4d(dst + (uint32_t)(kv * C::kTile + ch * C::kSub + bx * box * 128), kv ? &tmV : &tmK, 64 * ch, slot, w.h,
                        pg < 0 ? c.n_pages : pg, full(st));
          }
        }
      }
    }
    // the last copies land before the CTA may end
    if (!ok && lane == 0) give_up(err, a, DEVERR_PRODUCER_WAIT);
    for (int k = max(0, g - C::kStages); k < g; ++k)
      if (!wait_beat(full(k % C::kStages), (uint32_t)(k / C::kStages) & 1u, &s_beat) && lane == 0)
        give_up(err, a, DEVERR_DRAIN_WAIT);
    return;
  }

  // -------------------------------------------------------------------------- consumers
  constexpr int kBar = 1, kConsumers = 32 * C::kWarps;
  const int group = a.n_q / c.n_kv;
  const float sc = a.scale * kLog2e;
  const int r0 = lane >> 2, quad = lane & 3;  // this lane's fragment rows r0, r0 + 8 and columns 2 quad, 2 quad + 1
  for (; w.more(); w.next(b, c.page_shift, c.n_kv, a.window, tt, C::kBkShift)) {
    const int tok0 = w.t * tt, n_tok = min(w.q.rows - tok0, tt), rows = n_tok * group;
    const int lo = w.lo(a.window, tt), hi = w.hi(tt);
    // where every row of the item sees everything: between the last row's first key and the first row's position
    const int all_lo = a.window > 0 ? max(0, hi - a.window + 1) : 0, all_hi = w.q.pos0 + tok0;
    // the queries as the first product's left operand, a lane's four words a k step, over this warp's part of the join buffer
    // (as registers they would crowd the outputs out)
    uint4* qf = reinterpret_cast<uint4*>(join + warp * (kDim * 4)) + lane;
    int pos[2], from[2];
    {
      const uint16_t* qp[2];
      bool live[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = r0 + 8 * i;
        live[i] = r < rows;
        const int tok = live[i] ? tok0 + r / group : tok0;
        pos[i] = w.q.pos0 + tok;
        from[i] = a.window > 0 ? pos[i] - a.window + 1 : 0;
        qp[i] = a.q + (int64_t)(w.q.row0 + tok) * a.q_row + (int64_t)(w.h * group + (live[i] ? r % group : 0)) * a.q_head + 2 * quad;
      }
#pragma unroll
      for (int k = 0; k < kDim / 16; ++k) {
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          v[i] = live[i] ? *reinterpret_cast<const uint32_t*>(qp[i] + 16 * k) : 0u;
          v[2 + i] = live[i] ? *reinterpret_cast<const uint32_t*>(qp[i] + 16 * k + 8) : 0u;
        }
        qf[32 * k] = make_uint4(v[0], v[1], v[2], v[3]);
      }
    }
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f}, acc[kDim / 8][4];
#pragma unroll
    for (int i = 0; i < kDim / 8; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.0f;

    for (int i = 0; i < w.cnt; ++i, ++g) {
      constexpr int kBlocks = C::kBlocks;
      const int st = g % C::kStages, j0 = ((w.first + w.k0 + i) << C::kBkShift) + 16 * kBlocks * warp;
      if (ok && !wait_beat(full(st), (uint32_t)(g / C::kStages) & 1u, &s_beat)) ok = false;
      if (!ok) continue;
      const uint32_t there = held[st] >> (kBlocks * warp) & ((1u << kBlocks) - 1u);
      if (there != 0 && j0 <= hi && j0 + 16 * kBlocks - 1 >= lo) {
        const uint32_t kt = ring + (uint32_t)(st * C::kStage), vt = kt + C::kTile;
        float s[kBlocks][2][4];  // [block][keys 0-7, 8-15]
        {
          float z[kBlocks][2][2][4] = {};  // [even, odd k steps]
          const int row = 16 * kBlocks * warp + ((lane >> 4) << 3) + (lane & 7), half = (lane >> 3) & 1;
#pragma unroll
          for (int k = 0; k < kDim / 16; ++k) {
            const int col = 2 * (k & 3) + half;
            const uint4 q4 = qf[32 * k];
            const uint32_t qa[4] = {q4.x, q4.y, q4.z, q4.w};
#pragma unroll
            for (int u = 0; u < kBlocks; ++u) {
              uint32_t kb[4];
              ldsm4(kt + (uint32_t)((k >> 2) * C::kSub + (row + 16 * u) * 128 + ((col ^ (row & 7)) << 4)), kb);
              mma16<kBf16>(z[u][k & 1][0], qa, kb[0], kb[1]);
              mma16<kBf16>(z[u][k & 1][1], qa, kb[2], kb[3]);
            }
          }
#pragma unroll
          for (int u = 0; u < kBlocks; ++u)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) s[u][n][e] = z[u][0][n][e] + z[u][1][n][e];
        }
        if (j0 < all_lo || j0 + 16 * kBlocks - 1 > all_hi || there != (1u << kBlocks) - 1u) {
#pragma unroll
          for (int u = 0; u < kBlocks; ++u)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int j = j0 + 16 * u + 8 * n + 2 * quad + (e & 1);
                if (j > pos[e >> 1] || j < from[e >> 1] || !((there >> u) & 1u)) s[u][n][e] = -INFINITY;
              }
        }
        float up[2], ref[2];
        bool grown = false;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float top = -INFINITY;
#pragma unroll
          for (int u = 0; u < kBlocks; ++u)
            top = fmaxf(top, fmaxf(fmaxf(s[u][0][2 * r], s[u][0][2 * r + 1]), fmaxf(s[u][1][2 * r], s[u][1][2 * r + 1])));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)) * sc;
          up[r] = 1.0f;
          if (top > m[r] + kGrowth<kBf16>) {  // m = -inf: any visible key
            up[r] = m[r] == -INFINITY ? 0.0f : ex2(m[r] - top);
            m[r] = top;
            grown = true;
          }
          ref[r] = m[r] == -INFINITY ? 0.0f : m[r] - kLift<kBf16>;
        }
        if (__any_sync(0xffffffffu, grown)) {
          l[0] *= up[0];
          l[1] *= up[1];
#pragma unroll
          for (int d = 0; d < kDim / 8; ++d) {
            acc[d][0] *= up[0];
            acc[d][1] *= up[0];
            acc[d][2] *= up[1];
            acc[d][3] *= up[1];
          }
        }
        // the weights as the second product's left operand: rows r0 / r0 + 8, keys 0-7 then 8-15
        uint32_t p[kBlocks][4];
#pragma unroll
        for (int u = 0; u < kBlocks; ++u)
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              p[u][2 * n + r] = pack2<kBf16>(ex2(fmaf(s[u][n][2 * r], sc, -ref[r])), ex2(fmaf(s[u][n][2 * r + 1], sc, -ref[r])));
              const float2 as_used = unpack2<kBf16>(p[u][2 * n + r]);
              l[r] += as_used.x + as_used.y;
            }
        // values of keys outside the item's range (another sequence's, or nobody's) must not meet a weight of zero
        const bool cut = j0 < lo || j0 + 16 * kBlocks - 1 > hi;
        const int key = 16 * kBlocks * warp + (((lane >> 3) & 1) << 3) + (lane & 7);
#pragma unroll
        for (int d = 0; d < kDim / 16; ++d) {
          const int col = 2 * (d & 3) + (lane >> 4);
#pragma unroll
          for (int u = 0; u < kBlocks; ++u) {
            uint32_t vb[4];
            ldsm4t(vt + (uint32_t)((d >> 2) * C::kSub + (key + 16 * u) * 128 + ((col ^ (key & 7)) << 4)), vb);
            if (cut) {
#pragma unroll
              for (int n = 0; n < 2; ++n) {
                const int j = j0 + 16 * u + 8 * n + 2 * quad;
                const uint32_t keep = (j >= lo && j <= hi ? 0xffffu : 0u) | (j + 1 >= lo && j + 1 <= hi ? 0xffff0000u : 0u);
                vb[n] &= keep;
                vb[2 + n] &= keep;
              }
            }
            mma16<kBf16>(acc[2 * d], p[u], vb[0], vb[1]);
            mma16<kBf16>(acc[2 * d + 1], p[u], vb[2], vb[3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(st));
    }
    if (!ok && lane == 0) give_up(err, a, DEVERR_CONSUMER_WAIT);

    // ---- the warps' outputs of the item, on a common reference
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
      if (quad == 0) {
        s_m[warp][r0 + 8 * r] = m[r];
        s_l[warp][r0 + 8 * r] = l[r];
      }
    }
    named_bar_sync(kBar, kConsumers);
    float M[2], L[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      M[r] = -INFINITY;
      L[r] = 0.0f;
      for (int i = 0; i < C::kWarps; ++i) M[r] = fmaxf(M[r], s_m[i][r0 + 8 * r]);
      for (int i = 0; i < C::kWarps; ++i) {
        const float mi = s_m[i][r0 + 8 * r];
        L[r] += s_l[i][r0 + 8 * r] * (mi == -INFINITY ? 0.0f : ex2(mi - M[r]));
      }
      const float f = m[r] == -INFINITY ? 0.0f : ex2(m[r] - M[r]);
#pragma unroll
      for (int d = 0; d < kDim / 8; ++d) {
        acc[d][2 * r] *= f;
        acc[d][2 * r + 1] *= f;
      }
    }
    // each warp adds up its share of the dims over the warps, in their order, 8 rows at a time
    constexpr int kPer = C::kPer;
    float y[kPer][4];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      if (r == 1 && rows <= 8) break;
      if (r == 1) named_bar_sync(kBar, kConsumers);  // the first rows have been read
      float2* to = join + warp * (kDim * 4) + lane;
#pragma unroll
      for (int d = 0; d < kDim / 8; ++d) to[32 * d] = make_float2(acc[d][2 * r], acc[d][2 * r + 1]);
      named_bar_sync(kBar, kConsumers);
#pragma unroll
      for (int d = 0; d < kPer; ++d) {
        float2 sum = join[32 * (warp * kPer + d) + lane];
#pragma unroll
        for (int i = 1; i < C::kWarps; ++i) {
          const float2 x = join[i * (kDim * 4) + 32 * (warp * kPer + d) + lane];
          sum.x += x.x;
          sum.y += x.y;
        }
        y[d][2 * r] = sum.x;
        y[d][2 * r + 1] = sum.y;
      }
    }

    auto out_at = [&](int r) {
      return a.o + (int64_t)(w.q.row0 + tok0 + r / group) * a.o_row + (int64_t)(w.h * group + r % group) * a.o_head;
    };
    auto mend = [&]() {  // the marked rows, a warp each, exactly
      named_bar_sync(kBar, kConsumers);
      const uint32_t bad = s_bad;
      if (bad == 0) return;
      named_bar_sync(kBar, kConsumers);
      if (threadIdx.x == 0) s_bad = 0;
      for (int r = warp; r < rows; r += C::kWarps) {
        if (!((bad >> r) & 1u)) continue;
        const int tok = tok0 + r / group;
        attend_row<kBf16, kDim>(c, b, a, w.s, w.q.pos0 + tok, w.q.row0 + tok, w.h * group + r % group, lane, &s_beat);
      }
      named_bar_sync(kBar, kConsumers);
    };
    // this warp's dims of the output: y over the rows' sums; rows whose result is not finite, or without weight, are marked
    auto put = [&](const float (&sums)[2]) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int row = r0 + 8 * r;
        if (row >= rows) continue;
        const float inv = 1.0f / sums[r];
        float nan = 0.0f;
        uint16_t* o = out_at(row) + 2 * quad + 8 * warp * kPer;
#pragma unroll
        for (int d = 0; d < kPer; ++d) {
          const float x = y[d][2 * r] * inv, z = y[d][2 * r + 1] * inv;
          nan = fmaf(x, 0.0f, fmaf(z, 0.0f, nan));
          *reinterpret_cast<uint32_t*>(o + 8 * d) = pack2<kBf16>(x, z);
        }
        if (nan != 0.0f || !(sums[r] > 0.0f)) atomicOr(&s_bad, 1u << row);
      }
      mend();
    };
    if (w.whole()) {
      put(L);
      continue;
    }
    // ---- a piece: into the workspace, joined by the last one to arrive
    const Pieces ps = pieces_of(w, ls);
    {
      float* to = part + (size_t)(2 * blockIdx.x + (w.k0 > 0 ? 0 : 1)) * C::kPart;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int row = r0 + 8 * r;
        if (row >= rows) continue;
#pragma unroll
        for (int d = 0; d < kPer; ++d)
          __stcg(reinterpret_cast<float2*>(to + row * kDim + 8 * (warp * kPer + d) + 2 * quad),
                 make_float2(y[d][2 * r], y[d][2 * r + 1]));
        if (warp == 0 && quad == 0) {
          __stcg(to + kRows * kDim + row, M[r]);
          __stcg(to + kRows * kDim + kRows + row, L[r]);
        }
      }
      named_bar_sync(kBar, kConsumers);
      if (threadIdx.x == 0) s_last = last_piece(counters + ps.first, ps.count);
    }
    named_bar_sync(kBar, kConsumers);
    if (s_last) {
      join_pieces<kBf16, kDim>(part, ps.first, ps.count, rows, group, out_at(0), a.o_row, a.o_head,
                               reinterpret_cast<float*>(join), &s_bad);
      mend();
    }
    named_bar_sync(kBar, kConsumers);  // s_last, s_bad and the statistics are free again
  }
}

template <bool kBf16, int kDim>
w8a8_status launch(const CUtensorMap& tk, const CUtensorMap& tv, const PagedCache& pc, const PagedBatch& pb, const AttnCall& a,
                   void* ws, int sms, cudaStream_t st) {
  using C = Cfg<kDim>;
  static bool attr_set[64] = {};
  int dev = 0;
  W8A8_CUDA(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64 && !attr_set[dev]) {
    W8A8_CUDA(cudaFuncSetAttribute(attn_tokens_kernel<kBf16, kDim>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
    attr_set[dev] = true;
  }
  const int tt = kRows / (a.n_q / pc.n_kv);
  char* base = static_cast<char*>(ws);
  const dim3 grid((unsigned)(sms < kMaxPieces ? sms : kMaxPieces));
  W8A8_CUDA(launch_pdl(attn_tokens_kernel<kBf16, kDim>, grid, dim3(C::kThreads), (size_t)C::kSmem, st, tk, tv, pc, pb, a, tt,
                       reinterpret_cast<float*>(base + W8A8_WS_RESERVED), reinterpret_cast<unsigned int*>(base),
                       reinterpret_cast<unsigned int*>(base + kErrWordOffset)));
  return W8A8_OK;
}

}  // namespace

size_t attn_tokens_ws(int dim, int sms) { return (size_t)2 * sms * (kRows * dim + 2 * kRows) * sizeof(float); }

w8a8_status make_kv_maps(const PagedCache& pc, int dim, CUtensorMap* tk, CUtensorMap* tv) {
  const int page = 1 << pc.page_shift;
  const uint64_t dims[4] = {(uint64_t)dim, (uint64_t)page, (uint64_t)pc.n_kv, (uint64_t)pc.n_pages};
  const uint64_t strides[3] = {(uint64_t)pc.slot_stride * 2, (uint64_t)pc.head_stride * 2, (uint64_t)pc.page_stride * 2};
  const uint32_t box[4] = {64, (uint32_t)(page < kBoxSlots ? page : kBoxSlots), 1, 1};
  W8A8_TRY(make_tmap_16(tk, pc.k, 4, dims, strides, box));
  return make_tmap_16(tv, pc.v, 4, dims, strides, box);
}

w8a8_status launch_attn_tokens(const PagedCache& pc, const PagedBatch& pb, const AttnCall& a, void* ws, int sms,
                               cudaStream_t st) {
  CUtensorMap tk, tv;
  W8A8_TRY(make_kv_maps(pc, a.dim, &tk, &tv));
  if (a.bf16)
    return a.dim == 256   ? launch<true, 256>(tk, tv, pc, pb, a, ws, sms, st)
           : a.dim == 128 ? launch<true, 128>(tk, tv, pc, pb, a, ws, sms, st)
                          : launch<true, 64>(tk, tv, pc, pb, a, ws, sms, st);
  return a.dim == 256   ? launch<false, 256>(tk, tv, pc, pb, a, ws, sms, st)
         : a.dim == 128 ? launch<false, 128>(tk, tv, pc, pb, a, ws, sms, st)
                        : launch<false, 64>(tk, tv, pc, pb, a, ws, sms, st);
}

}  // namespace w8a8
