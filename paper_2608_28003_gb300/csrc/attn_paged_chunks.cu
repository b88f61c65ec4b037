// Attention over a paged cache for chunks of tokens, on the 5th-generation tensor cores: items of up to 256 rows (128 at head
// dim 256, whose output fills tensor memory), tokens times the query heads of a group, in two tiles (one) of 128 rows with
// one row per TMEM lane.
//
// One CTA per SM walks its stretch of the line of key tiles (attn_paged.cuh), 128 keys at a time:
//  * two warps copy by TMA, page by page: one an item's queries and the K tiles, one the V tiles (either as its tiles are
//    handed back, which one warp's order would tie together);
//  * the issue warp allocates tensor memory and issues tcgen05.mma: S = Q K^T (128 x 128 x dim) for each row tile, and
//    O += P V (128 x dim x 128), P read from tensor memory.  V lies as the cache has it, keys by dims, so it is the
//    product's MN-major operand and needs no transposition;
//  * eight softmax warps, four for each row tile (thread = row), or two threads a row, each with half of the keys and of
//    the dims, where there is one: they take the row's maximum over the scores, rescale O in tensor memory if it grew by
//    more than 2^kGrowth (m moves only then), then p = 2^(s c - m + kLift) with c = scale log2 e in chunks of 32 scores, and write P over
//    the scores they have read, where the second product finds it.  P is handed over in halves: the product of the first
//    half runs while the second is computed.
// Tensor memory holds 512 columns: two slots of 128 for S and P, and O of 2 x 64, 2 x 128 or 256.  With two row tiles each
// has a slot of its own, and the tensor cores work for one while the other's softmax runs.  At head dim 256 the slots
// alternate: S of the next key tile is issued before P of this one is awaited; one K and one V tile fill shared memory
// beside the queries, so tiles are copied and handed back in quarters (K by 64 dims, V by 32 keys), and the copies of the
// next tile follow the products through this one.
// The products of one thread run in the order of their issue, which is what frees a slot: S of a slot is issued after
// the product that read the slot's P.
//
// What bounds it.  At head dims 64 and 128 the chain S -> maximum -> exponentials -> P V of a row tile, about 3100 cycles a
// tile of keys where the products take 2048: four chunks of 1001 tokens behind up to 9000 keys, 28 heads over 4 of 128, take
// 180 to 183 us (680 TFLOP/s, 0.36 of the measured rate; 217 with P in one piece after the rescaling).  Tried and slower: a part of
// the exponentials as a polynomial (an eighth 180 us, a quarter 184, half 207: issue slots, not the special function unit,
// are short), two threads a row for both row tiles (211: 96 registers), scores loaded ahead or kept in registers (189 and
// 233: spills, at the 168 registers that all of the block's threads have; not tried with shares of different size).  A whole
// prompt of 2048 tokens at head dim 256 takes 28.5 us, four key tiles a CTA: latency from step to step, of which the parts
// that were timed (lookup 2, first tile 3, key tiles 7, partials and their join 8) make two thirds.  There every CTA copies all of its K and V from L2;
// a pair of CTAs, each copying half for both, took 27.9, and 67.2 us instead of 71.9 for a larger chunk, but a copy to several
// CTAs has no place in a library that also runs on several GPUs.
// Every wait is bounded: on timeout a bit of the error word is set, and the CTA passes its items without waiting.
#include "attn_paged.cuh"
#include "ops.cuh"
#include "tc_common.cuh"
#include "tmap.cuh"

namespace w8a8 {

w8a8_status make_kv_maps(const PagedCache& pc, int dim, CUtensorMap* tk, CUtensorMap* tv);

namespace {

constexpr int kBq = 128, kBk = 128, kBkShift = 7;
constexpr int kSub = 128 * 128;  // bytes of 128 rows of 64 dims

template <int kDim>
struct Cfg {
  static constexpr int kRt = kDim == 256 ? 1 : 2;  // row tiles of a CTA
  static constexpr int kChunks = kDim / 64;
  static constexpr int kStages = kDim == 256 ? 1 : kDim == 128 ? 2 : 4;
  static constexpr int kTile = kChunks * kSub;
  static constexpr int kOffK = kRt * kTile, kOffV = kOffK + kStages * kTile;
  static constexpr int kSmem = kOffV + kStages * kTile + 1024;
  static constexpr int kKParts = kDim == 256 ? 4 : 1, kVParts = kKParts;  // a K tile comes by 64 dims, a V tile by 32 keys
  static constexpr int kKCols = kChunks / kKParts, kVKeys = kBk / kVParts;  // columns, keys a part
  static constexpr int kSplit = 2 / kRt;           // threads a row
  static constexpr int kSoft = 8, kLoadWarp = kSoft, kIssueWarp = kSoft + 1, kLoadV = kSoft + 2, kThreads = 32 * (kSoft + 3);
  static constexpr int kRows = kBq * kRt;
  static constexpr int kPart = kRows * kDim + 2 * kRows;  // floats of a partial: [dim / 4][rows][4], m, l
  static constexpr uint32_t kOCol = 256;                  // O of row tile r: kOCol + r kDim
  static constexpr int kArrive = kSplit * kBq;            // threads of a row tile
  // barriers.  A wait tells a phase from the one before it only, so none may complete twice before a waiter looks: P_FULL counts by
  // slot and half (with one row tile, whose softmax may be a tile ahead of the products; by row tile and half with two, the same);
  // PV_DONE by row tile, its second one with one row tile for an item's last product
  static constexpr int Q_FULL = 0, Q_FREE = 1, S_FULL = 2, P_FULL = 4, PV_DONE = 8, O_FREE = 10, ALL_DONE = 12, X_FULL = 13,
                       K_FULL = 14, K_FREE = K_FULL + kStages * kKParts, V_FULL = K_FREE + kStages * kKParts,
                       V_FREE = V_FULL + kStages * kVParts, kBars = V_FREE + kStages * kVParts;
};

// Shared-memory descriptor of an MN-major tile, 128-byte swizzle: 64 elements of the MN dimension a row of 128 bytes, 8 rows
// (of the K dimension) a swizzle group, groups 1024 bytes apart (stride byte offset), the next 64 MN elements `lead` bytes on.
__device__ __forceinline__ uint64_t sdesc_mn(uint32_t saddr, uint32_t lead) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
constexpr uint32_t kIdescBMnMajor = 1u << 16;

// A from tensor memory (two 16-bit elements a column)
__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
      "%15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};\n" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
      "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
      "%15};\n" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }

template <bool kBf16, int kDim>
__global__ void __launch_bounds__(Cfg<kDim>::kThreads, 1)
    attn_chunks_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, PagedCache c, PagedBatch b, AttnCall a, int tt,
                       float* __restrict__ part, unsigned int* __restrict__ counters, unsigned int* __restrict__ err) {
  using C = Cfg<kDim>;
  constexpr int kRt = C::kRt, kThreads = C::kThreads, kIssueWarp = C::kIssueWarp;
  constexpr uint32_t kOCol = C::kOCol;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ uint64_t bars[C::kBars];
  __shared__ LineStart ls;
  __shared__ long long scan[kThreads / 32];
  __shared__ uint32_t held[8];  // 16-key groups of a tile that lie in a page
  __shared__ uint32_t tmem_slot, s_last, s_bad[4], s_beat;
  __shared__ float s_max[C::kSplit][C::kSplit][kBq], s_sum[C::kSplit][kBq];  // two threads a row: what they tell each other
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = a.n_q / c.n_kv, item_tt = kRt * tt;  // tokens of a row tile, of an item

  if (threadIdx.x < 4) s_bad[threadIdx.x] = 0;
  if (threadIdx.x == 0) {
    s_beat = 0;
    for (int i = 0; i < C::kBars; ++i)
      mbar_init(bar(i), (i >= C::P_FULL && i < C::PV_DONE) || i == C::O_FREE || i == C::O_FREE + 1 || i == C::X_FULL ? C::kArrive : 1);
    fence_mbar_init();
    prefetch_tmap(&tmQ);
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
  }
  if (warp == kIssueWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(&tmem_slot))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_wait();
  pdl_trigger();
  // (syncs the block)
  find_start<kThreads>(b, c.page_shift, c.n_kv, a.window, item_tt, kBkShift, (int)blockIdx.x, (int)gridDim.x, &ls, scan);
  bool ok = true;

  if (ls.begin < ls.end) {
    Walk w;
    w.start(ls, b, c.page_shift, a.window, item_tt, kBkShift, lane);
    int g = 0, item = 0;  // tiles and items of this CTA so far
    if (warp == C::kLoadWarp || warp == C::kLoadV) {
      // ---------------------------------------------------------------------- TMA copies
      const bool kv = warp == C::kLoadV;
      const CUtensorMap* map = kv ? &tmV : &tmK;
      const int full = kv ? C::V_FULL : C::K_FULL, free = kv ? C::V_FREE : C::K_FREE;
      const int box = min(kBoxSlots, 1 << c.page_shift), n_box = (kv ? C::kVKeys : kBk) / box;  // boxes of a part in a column
      const int n_ops = n_box * (kv ? C::kChunks : C::kKCols);
      const uint32_t q_bytes = (uint32_t)(kRt * group * tt * 128 * C::kChunks);
      int issued = 0;  // parts whose copies have been issued
      for (; ok && w.more(); w.next(b, c.page_shift, c.n_kv, a.window, item_tt, kBkShift), ++item) {
        const int lo = w.lo(a.window, item_tt), hi = w.hi(item_tt);
        constexpr int kGroups = kBk / 16, kBatch = 32 / kGroups;  // tiles whose pages are read at once, ahead of their use
        int page = group_page(b, c, w.s, (w.first + w.k0) << kBkShift, lo, hi, box, lane), ahead = -1;
        if (!kv) {
          if (item > 0 && !wait_beat(bar(C::Q_FREE), (uint32_t)(item - 1) & 1u, &s_beat)) {
            ok = false;
            break;
          }
          if (elect_one()) {
            mbar_arrive_expect_tx(bar(C::Q_FULL), q_bytes);
#pragma unroll
            for (int rt = 0; rt < kRt; ++rt)
#pragma unroll
              for (int ch = 0; ch < C::kChunks; ++ch)
                tma_load_3d(base + (uint32_t)(rt * C::kTile + ch * kSub), &tmQ, 64 * ch, w.h * group,
                            w.q.row0 + w.t * item_tt + rt * tt, bar(C::Q_FULL));
          }
          __syncwarp();
        }
        for (int i = 0; ok && i < w.cnt; ++i, ++g) {
          const int st = g % C::kStages, tile0 = (w.first + w.k0 + i) << kBkShift, in_batch = i % kBatch;
          if (in_batch == 0) {
            if (i > 0) page = ahead;
            if (i + kBatch < w.cnt) ahead = group_page(b, c, w.s, tile0 + (kBatch << kBkShift), lo, hi, box, lane);
          }
          const uint32_t there = (__ballot_sync(0xffffffffu, page >= 0) >> (in_batch * kGroups)) & ((1u << kGroups) - 1u);
          for (int pt = 0; pt < C::kKParts; ++pt) {
            const int bi = st * C::kKParts + pt;
            if (g >= C::kStages && !wait_beat(bar(free + bi), (uint32_t)(g / C::kStages - 1) & 1u, &s_beat)) {
              ok = false;
              break;
            }
            if (lane == 0) {
              if (!kv && pt == 0) held[g & 7] = there;
              mbar_arrive_expect_tx(bar(full + bi), (uint32_t)(C::kTile / C::kKParts));
            }
            __syncwarp();
            // lane = (column, box)
            const int bx = (kv ? pt * n_box : 0) + lane % n_box, ch = (kv ? 0 : pt * C::kKCols) + lane / n_box;
            const int pg = __shfl_sync(0xffffffffu, page, (in_batch * kGroups + bx * (box / 16)) & 31);
            if (lane < n_ops) {
              const uint32_t dst = base + (uint32_t)((kv ? C::kOffV : C::kOffK) + st * C::kTile + ch * kSub + bx * box * 128);
              const int slot = (tile0 + bx * box) & ((1 << c.page_shift) - 1), at = pg < 0 ? c.n_pages : pg;
              tma_load_4d(dst, map, 64 * ch, slot, w.h, at, bar(full + bi));
            }
            issued = g * C::kKParts + pt + 1;
          }
        }
      }
      // the last copies land before the CTA may end
      if (!ok && lane == 0) give_up(err, a, DEVERR_PRODUCER_WAIT);
      constexpr int kRing = C::kStages * C::kKParts;
      bool drained = kv || item == 0 || wait_beat(bar(C::Q_FULL), (uint32_t)(item - 1) & 1u, &s_beat);
      for (int k = max(0, issued - kRing); k < issued; ++k)
        drained &= wait_beat(bar(full + k % kRing), (uint32_t)(k / kRing) & 1u, &s_beat);
      if (!drained && lane == 0) give_up(err, a, DEVERR_DRAIN_WAIT);
    } else if (warp == kIssueWarp) {
      // ---------------------------------------------------------------------- MMAs
      constexpr uint32_t fmt = kBf16 ? 1u : 0u;
      constexpr uint32_t idesc_s = idesc_f16(fmt, kBk, kBq), idesc_o = idesc_f16(fmt, kDim, kBq) | kIdescBMnMajor;
      const uint64_t dq = sdesc_swz(base);
      // S of key tile i (this CTA's count) for row tile rt, into its slot; hands K back after the last row tile, Q after `last`
      auto issue_s = [&](int i, int rt, bool last) {
        const int st = i % C::kStages, slot = kRt == 2 ? rt : i & 1;
        const uint64_t dk = sdesc_swz(base + (uint32_t)(C::kOffK + st * C::kTile));
#pragma unroll 1
        for (int pt = 0; pt < C::kKParts; ++pt) {
          if (rt == 0 &&
              !wait_beat(bar(C::K_FULL + st * C::kKParts + pt), (uint32_t)(i / C::kStages) & 1u, &s_beat))
            return false;
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4 * C::kKCols; ++k) {
              const uint32_t at = (uint32_t)((pt * C::kKCols + (k >> 2)) * (kSub >> 4) + 2 * (k & 3));
              tc_mma(tmem + 128u * (uint32_t)slot, dq + (uint32_t)(rt * (C::kTile >> 4)) + at, dk + at, idesc_s, pt > 0 || k > 0);
            }
            if (rt == kRt - 1) tc_commit(bar(C::K_FREE + st * C::kKParts + pt));
          }
          __syncwarp();
        }
        if (elect_one()) {
          tc_commit(bar(C::S_FULL + slot));
          if (last && rt == kRt - 1) tc_commit(bar(C::Q_FREE));
        }
        __syncwarp();
        return true;
      };
      // O += P V of key tile i for row tile rt, in two halves as P comes; hands V back after the last row tile
      auto issue_pv = [&](int i, int rt, bool first, bool last) {
        const int st = i % C::kStages, slot = kRt == 2 ? rt : i & 1;
        if (first && item > 0 && !wait_beat(bar(C::O_FREE + rt), (uint32_t)(item - 1) & 1u, &s_beat)) return false;
        const uint64_t dv = sdesc_mn(base + (uint32_t)(C::kOffV + st * C::kTile), kSub);
        const uint32_t p = tmem + 128u * (uint32_t)slot, o = tmem + kOCol + (uint32_t)(rt * kDim);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!wait_beat(bar(C::P_FULL + 2 * slot + half), (uint32_t)(kRt == 2 ? i : i >> 1) & 1u, &s_beat))
            return false;
          if constexpr (C::kVParts == 1) {
            if (rt == 0 && half == 0 && !wait_beat(bar(C::V_FULL + st), (uint32_t)(i / C::kStages) & 1u, &s_beat))
              return false;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int kk = 4 * half + k;  // 16 keys: 8 columns of P
                tc_mma_ts(o, p + 8u * (uint32_t)kk, dv + (uint32_t)(kk * (16 * 128 >> 4)), idesc_o, !first || kk > 0);
              }
              if (half == 1 && rt == kRt - 1) tc_commit(bar(C::V_FREE + st));
              if (half == 1) tc_commit(bar(C::PV_DONE + rt));
            }
            __syncwarp();
          } else {  // two threads a row: the halves are keys 0-31 and 64-95, then the others
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int vp = half + 2 * j;  // 32 keys
              if (!wait_beat(bar(C::V_FULL + st * C::kVParts + vp), (uint32_t)(i / C::kStages) & 1u, &s_beat))
                return false;
              tc_fence_after();
              if (elect_one()) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const int kk = 2 * vp + k;  // (P over the scores that were read: the second thread's over its own)
                  tc_mma_ts(o, p + 8u * (uint32_t)kk + (kk >= 4 ? 32u : 0u), dv + (uint32_t)(kk * (16 * 128 >> 4)), idesc_o,
                            !first || kk > 0);
                }
                tc_commit(bar(C::V_FREE + st * C::kVParts + vp));
                if (vp == C::kVParts - 1) {
                  tc_commit(bar(C::PV_DONE));
                  if (last) tc_commit(bar(C::PV_DONE + 1));
                }
              }
              __syncwarp();
            }
          }
        }
        return true;
      };
      for (; ok && w.more(); w.next(b, c.page_shift, c.n_kv, a.window, item_tt, kBkShift), ++item) {
        ok = wait_beat(bar(C::Q_FULL), (uint32_t)item & 1u, &s_beat);
#pragma unroll
        for (int rt = 0; rt < kRt; ++rt) ok = ok && issue_s(g, rt, w.cnt == 1);
        for (int i = 0; ok && i < w.cnt; ++i, ++g) {
          const bool more = i + 1 < w.cnt, last = i + 2 == w.cnt;
          if constexpr (kRt == 1) {
            ok = (!more || issue_s(g + 1, 0, last)) && issue_pv(g, 0, i == 0, !more);
          } else {  // a slot's next S follows the product that has read its P
            ok = issue_pv(g, 0, i == 0, !more) && (!more || issue_s(g + 1, 0, last)) && issue_pv(g, 1, i == 0, !more) &&
                 (!more || issue_s(g + 1, 1, last));
          }
        }
      }
      if (elect_one()) {
        if (!ok) give_up(err, a, DEVERR_PRODUCER_WAIT);
        tc_commit(bar(C::ALL_DONE));  // completes once every MMA issued above has
        if (!mbar_wait_bounded(bar(C::ALL_DONE), 0u, kWaitBudgetCycles)) give_up(err, a, DEVERR_DRAIN_WAIT);
      }
      __syncwarp();
    } else {
      // ---------------------------------------------------------------------- softmax, one row per thread
      constexpr int kSplit = C::kSplit, kQ = 4 / kSplit, kCh = kDim / 32 / kSplit;  // chunks of 32 keys, of 32 dims a thread
      const int rt = kRt == 2 ? warp >> 2 : 0, r = threadIdx.x & (kBq - 1);  // row tile, row of it
      const int hf = kRt == 2 ? 0 : warp >> 2;                               // which half
      const uint32_t lanes = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
      const uint32_t otm = lanes + kOCol + (uint32_t)(rt * kDim + hf * (kDim / 2));
      const float sc = a.scale * kLog2e;
      for (; w.more(); w.next(b, c.page_shift, c.n_kv, a.window, item_tt, kBkShift), ++item) {
        const int tok0 = w.t * item_tt + rt * tt, rows = max(0, min(w.q.rows - tok0, tt)) * group;
        const int lo = w.lo(a.window, item_tt), hi = w.hi(item_tt);
        const bool live = r < rows, busy = 32 * (warp & 3) < rows;  // this row's, and any of the warp's
        const int tok = tok0 + (live ? r / group : 0), head = w.h * group + (live ? r % group : 0);
        const int pos = w.q.pos0 + tok, from = a.window > 0 ? max(0, pos - a.window + 1) : 0;
        float m = -INFINITY, l = 0.0f;
        for (int i = 0; i < w.cnt; ++i, ++g) {
          const int j0 = (w.first + w.k0 + i) << kBkShift, slot = kRt == 2 ? rt : g & 1;
          const uint32_t stm = lanes + 128u * (uint32_t)slot;
          if (ok && !wait_beat(bar(C::S_FULL + slot), (uint32_t)(kRt == 2 ? g : g >> 1) & 1u, &s_beat)) ok = false;
          if (!ok) continue;
          tc_fence_after();
          uint32_t x[32];
          float top = -INFINITY;
          const uint32_t there = held[g & 7];
          const bool cut = j0 < from || j0 + kBk - 1 > pos || there != 0xffu;  // some key is not this row's
          // the scores of 32 keys that are not this row's become -inf
          auto mask = [&](int q4) {
            const int f = from - j0 - 32 * q4, t = pos - j0 - 32 * q4;  // keys f .. t of the 32
            uint32_t keep = t < 0 || f > 31 ? 0u : 0xffffffffu;
            if (f > 0 && f <= 31) keep &= 0xffffffffu << f;
            if (t >= 0 && t < 31) keep &= (2u << t) - 1u;
            if (!((there >> (2 * q4)) & 1u)) keep &= 0xffff0000u;
            if (!((there >> (2 * q4 + 1)) & 1u)) keep &= 0x0000ffffu;
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (!((keep >> k) & 1u)) x[k] = 0xff800000u;
          };
          if (busy) {
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int q = 0; q < kQ; ++q) {
              tmem_ld32(stm + 32 * (hf * kQ + q), x);
              if (cut) mask(hf * kQ + q);
#pragma unroll
              for (int k = 0; k < 32; k += 2)
                mx[(k >> 1) & 3] = fmaxf(fmaxf(mx[(k >> 1) & 3], __uint_as_float(x[k])), __uint_as_float(x[k + 1]));
            }
            top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
          }
          if constexpr (kSplit == 2) {  // the row's other thread
            s_max[g & 1][hf][r] = top;
            mbar_arrive(bar(C::X_FULL));
            if (!wait_beat(bar(C::X_FULL), (uint32_t)g & 1u, &s_beat)) {
              ok = false;
              continue;
            }
            top = fmaxf(top, s_max[g & 1][hf ^ 1][r]);
          }
          if (busy) {
            top *= sc;
            const bool grown = top > m + kGrowth<kBf16>;  // m = -inf: any visible key
            float up = 1.0f;
            if (grown) {
              up = m == -INFINITY ? 0.0f : ex2(m - top);
              m = top;
              l *= up;
            }
            if (i > 0 && __any_sync(0xffffffffu, grown)) {
              // O is the previous products' (with two row tiles their order ahead of this S says so already)
              if (kRt == 1 && !wait_beat(bar(C::PV_DONE), (uint32_t)(g - 1) & 1u, &s_beat)) {
                ok = false;
                continue;
              }
              tc_fence_after();
#pragma unroll 1
              for (int ch = 0; ch < kCh; ++ch) {
                tmem_ld32(otm + 32 * ch, x);
#pragma unroll
                for (int k = 0; k < 32; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * up);
                tmem_st32(otm + 32 * ch, x);
              }
            }
          }
          if (rt == 0 && hf == 0 && (j0 < lo || j0 + kBk - 1 > hi)) {
            // values of keys outside the item's range (another sequence's, or nobody's) must not meet a weight of zero: row r
            // of the tile, once its copies have landed
            const int st = g % C::kStages;
            // with one row tile and stage, the values of the tile before may not have landed yet: its product has them
            bool landed = kRt == 2 || i == 0 || wait_beat(bar(C::PV_DONE), (uint32_t)(g - 1) & 1u, &s_beat);
#pragma unroll
            for (int vp = 0; vp < C::kVParts; ++vp)
              landed = landed && wait_beat(bar(C::V_FULL + st * C::kVParts + vp), (uint32_t)(g / C::kStages) & 1u, &s_beat);
            if (!landed) {
              ok = false;
              continue;
            }
            if (j0 + r < lo || j0 + r > hi) {
#pragma unroll
              for (int ch = 0; ch < C::kChunks; ++ch)
#pragma unroll
                for (int k = 0; k < 8; ++k)
                  asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};\n" ::"r"(
                                   base + (uint32_t)(C::kOffV + st * C::kTile + ch * kSub + r * 128 + 16 * k)),
                               "r"(0u)
                               : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
          }
          const float ref = m == -INFINITY ? 0.0f : m - kLift<kBf16>;
          const f32x2 sc2 = f2_pack(sc, sc), ref2 = f2_pack(-ref, -ref);
          f32x2 sum[2] = {0ull, 0ull};  // of weights before their rounding: summed as used, 188 us where it is 180 and no closer
#pragma unroll
          for (int q = 0; q < kQ; ++q) {
            if (busy) {
              tmem_ld32(stm + 32 * (hf * kQ + q), x);
              if (cut) mask(hf * kQ + q);
              uint32_t pk[16];
#pragma unroll
              for (int k = 0; k < 32; k += 2) {
                const f32x2 y = f2_fma(f2_pack(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), sc2, ref2);
                float e0, e1;
                f2_unpack(y, e0, e1);
                e0 = ex2(e0);
                e1 = ex2(e1);
                sum[(k >> 1) & 1] = f2_add(sum[(k >> 1) & 1], f2_pack(e0, e1));
                pk[k >> 1] = pack2<kBf16>(e0, e1);
              }
              tmem_st16(stm + 64 * hf + 16 * q, pk);  // over scores that have been read
            }
            if ((q + 1) % (kQ / 2) == 0) {  // half of P is there
              if (busy) tmem_wait_st();
              tc_fence_before();
              mbar_arrive(bar(C::P_FULL + 2 * slot + (q + 1) / (kQ / 2) - 1));
            }
          }
          float s0, s1;
          f2_unpack(f2_add(sum[0], sum[1]), s0, s1);
          l += s0 + s1;
        }
        // the item's last product
        if (ok && !wait_beat(bar(kRt == 2 ? C::PV_DONE + rt : C::PV_DONE + 1), (uint32_t)(kRt == 2 ? g - 1 : item) & 1u, &s_beat))
          ok = false;
        if (!ok && lane == 0) give_up(err, a, DEVERR_CONSUMER_WAIT);
        __syncwarp();
        tc_fence_after();

        // ---- the item's output
        const int64_t row = w.q.row0 + tok;
        uint16_t* orow = a.o + row * a.o_row + (int64_t)head * a.o_head + hf * (kDim / 2);
        if constexpr (kSplit == 2) {
          s_sum[hf][r] = l;
          named_bar_sync(1, 32 * C::kSoft);
          l = s_sum[0][r] + s_sum[1][r];
        }
        auto store = [&](int ch, const float (&x)[32], float inv, float& nan) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float y = x[8 * k + 2 * e] * inv, z = x[8 * k + 2 * e + 1] * inv;
              nan = fmaf(y, 0.0f, fmaf(z, 0.0f, nan));
              p[e] = pack2<kBf16>(y, z);
            }
            if (live) *reinterpret_cast<uint4*>(orow + 32 * ch + 8 * k) = make_uint4(p[0], p[1], p[2], p[3]);
          }
        };
        auto exactly = [&](bool bad) {  // rows whose result is not finite, or without weight; all softmax warps
          uint32_t rest = __ballot_sync(0xffffffffu, live && bad);
          __syncwarp();  // the lanes' stores of their rows come before the warp's below
          if constexpr (kSplit == 2) {  // in either half
            if (rest && lane == 0) atomicOr(&s_bad[warp & 3], rest);
            named_bar_sync(1, 32 * C::kSoft);
            if (hf == 1) return;
            rest = s_bad[warp & 3];
            __syncwarp();
            if (lane == 0) s_bad[warp & 3] = 0;
          }
          for (; rest; rest &= rest - 1) {
            const int src = __ffs(rest) - 1;
            attend_row<kBf16, kDim>(c, b, a, w.s, __shfl_sync(0xffffffffu, pos, src),
                                    (int64_t)w.q.row0 + __shfl_sync(0xffffffffu, tok, src), __shfl_sync(0xffffffffu, head, src),
                                    lane, &s_beat);
          }
        };
        if (w.whole()) {
          float nan = 0.0f;
          if (busy) {
            const float inv = 1.0f / l;
#pragma unroll 1
            for (int ch = 0; ch < kCh; ++ch) {
              uint32_t x[32];
              float f[32];
              tmem_ld32(otm + 32 * ch, x);
#pragma unroll
              for (int k = 0; k < 32; ++k) f[k] = __uint_as_float(x[k]);
              store(ch, f, inv, nan);
            }
          }
          tc_fence_before();
          mbar_arrive(bar(C::O_FREE + rt));
          exactly(nan != 0.0f || !(l > 0.0f));
          continue;
        }
        // ---- a piece: into the workspace, joined by the last one to arrive
        const Pieces ps = pieces_of(w, ls);
        const int pr = rt * kBq + r;  // row of the partial
        float* mine = part + (size_t)(2 * blockIdx.x + (w.k0 > 0 ? 0 : 1)) * C::kPart;
        if (busy) {
#pragma unroll 1
          for (int ch = 0; ch < kCh; ++ch) {
            uint32_t x[32];
            tmem_ld32(otm + 32 * ch, x);
            if (live) {
#pragma unroll
              for (int k = 0; k < 8; ++k)
                __stcg(reinterpret_cast<float4*>(mine) + (size_t)(8 * (hf * kCh + ch) + k) * C::kRows + pr,
                       make_float4(__uint_as_float(x[4 * k]), __uint_as_float(x[4 * k + 1]), __uint_as_float(x[4 * k + 2]),
                                   __uint_as_float(x[4 * k + 3])));
            }
          }
          if (live && hf == 0) {
            __stcg(mine + C::kRows * kDim + pr, m);
            __stcg(mine + C::kRows * kDim + C::kRows + pr, l);
          }
        }
        tc_fence_before();
        mbar_arrive(bar(C::O_FREE + rt));
        named_bar_sync(1, 32 * C::kSoft);
        if (threadIdx.x == 0) s_last = last_piece(counters + ps.first, ps.count);
        named_bar_sync(1, 32 * C::kSoft);
        if (s_last) {
          auto slot = [&](int i) { return part + (size_t)(2 * (ps.first + i) + (i == 0 ? 1 : 0)) * C::kPart; };
          float M = -INFINITY, L = 0.0f, nan = 0.0f;
          if (live) {
#pragma unroll 4
            for (int i = 0; i < ps.count; ++i) M = fmaxf(M, __ldcg(slot(i) + C::kRows * kDim + pr));
#pragma unroll 4
            for (int i = 0; i < ps.count; ++i) {
              const float mi = __ldcg(slot(i) + C::kRows * kDim + pr);
              L = fmaf(__ldcg(slot(i) + C::kRows * kDim + C::kRows + pr), mi == -INFINITY ? 0.0f : ex2(mi - M), L);
            }
          }
          const float inv = 1.0f / L;
#pragma unroll 1
          for (int ch = 0; ch < kCh; ++ch) {
            float f[32];
#pragma unroll
            for (int k = 0; k < 32; ++k) f[k] = 0.0f;
            if (live) {
#pragma unroll 2
              for (int i = 0; i < ps.count; ++i) {
                const float mi = __ldcg(slot(i) + C::kRows * kDim + pr);
                const float4* src = reinterpret_cast<const float4*>(slot(i)) + (size_t)(8 * (hf * kCh + ch)) * C::kRows + pr;
                float4 x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = __ldcg(src + k * C::kRows);
                const float e = mi == -INFINITY ? 0.0f : ex2(mi - M);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  f[4 * k] = fmaf(x[k].x, e, f[4 * k]);
                  f[4 * k + 1] = fmaf(x[k].y, e, f[4 * k + 1]);
                  f[4 * k + 2] = fmaf(x[k].z, e, f[4 * k + 2]);
                  f[4 * k + 3] = fmaf(x[k].w, e, f[4 * k + 3]);
                }
              }
            }
            store(ch, f, inv, nan);
          }
          exactly(nan != 0.0f || !(L > 0.0f));
        }
        named_bar_sync(1, 32 * C::kSoft);  // s_last is free again
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kIssueWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem) : "memory");
  }
}

template <bool kBf16, int kDim>
w8a8_status launch(const PagedCache& pc, const PagedBatch& pb, const AttnCall& a, void* ws, int sms, cudaStream_t st) {
  using C = Cfg<kDim>;
  static bool attr_set[64] = {};
  int dev = 0;
  W8A8_CUDA(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64 && !attr_set[dev]) {
    W8A8_CUDA(cudaFuncSetAttribute(attn_chunks_kernel<kBf16, kDim>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
    attr_set[dev] = true;
  }
  const int group = a.n_q / pc.n_kv, tt = kBq / group;
  CUtensorMap tq, tk, tv;
  const uint64_t dims[3] = {(uint64_t)kDim, (uint64_t)a.n_q, (uint64_t)pb.n_rows};
  const uint64_t strides[2] = {(uint64_t)a.q_head * 2, (uint64_t)a.q_row * 2};
  const uint32_t box[3] = {64, (uint32_t)group, (uint32_t)tt};
  W8A8_TRY(make_tmap_16(&tq, a.q, 3, dims, strides, box));
  W8A8_TRY(make_kv_maps(pc, kDim, &tk, &tv));
  char* base = static_cast<char*>(ws);
  W8A8_CUDA(launch_pdl(attn_chunks_kernel<kBf16, kDim>, dim3((unsigned)sms), dim3(C::kThreads), (size_t)C::kSmem, st, tq, tk, tv,
                       pc, pb, a, tt, reinterpret_cast<float*>(base + W8A8_WS_RESERVED), reinterpret_cast<unsigned int*>(base),
                       reinterpret_cast<unsigned int*>(base + kErrWordOffset)));
  return W8A8_OK;
}

}  // namespace

size_t attn_chunks_ws(int dim, int sms) {
  const int part = dim == 256 ? Cfg<256>::kPart : dim == 128 ? Cfg<128>::kPart : Cfg<64>::kPart;
  return (size_t)2 * sms * part * sizeof(float);
}

w8a8_status launch_attn_chunks(const PagedCache& pc, const PagedBatch& pb, const AttnCall& a, void* ws, int sms,
                               cudaStream_t st) {
  if (a.bf16)
    return a.dim == 256   ? launch<true, 256>(pc, pb, a, ws, sms, st)
           : a.dim == 128 ? launch<true, 128>(pc, pb, a, ws, sms, st)
                          : launch<true, 64>(pc, pb, a, ws, sms, st);
  return a.dim == 256   ? launch<false, 256>(pc, pb, a, ws, sms, st)
         : a.dim == 128 ? launch<false, 128>(pc, pb, a, ws, sms, st)
                        : launch<false, 64>(pc, pb, a, ws, sms, st);
}

}  // namespace w8a8
