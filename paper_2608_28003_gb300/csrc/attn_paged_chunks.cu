// Attention over a paged cache for chunks of tokens, on the 5th-generation tensor cores: items of up to 128 rows (tokens times
// the query heads of a group, one row per TMEM lane).
//
// One CTA per SM walks its stretch of the line of key tiles (attn_paged.cuh), 128 keys at a time:
//  * warp 4 copies by TMA: an item's queries, and K and V tiles page by page;
//  * warp 5 allocates tensor memory and issues tcgen05.mma: S = Q K^T (128 x 128 x dim) into one of two 128-column slots, and
//    O += P V (128 x dim x 128).  V lies as the cache has it, keys by dims, so it is the product's MN-major operand and needs
//    no transposition.  S of the next tile is issued before P of this one is awaited;
//  * warps 0-3: thread = row.  It reads its 128 scores, masks them, p = 2^(s c - m) with c = scale log2 e, adds the rounded
//    weights and writes them into the swizzled tile that the second product reads.  m moves when the maximum grew by more than
//    2^8 only: O is then rescaled in tensor memory.
// At head dim 256 one K and one V tile fill shared memory beside the queries and P, so tiles are copied and handed
// back in quarters (K by 64 dims, V by 32 keys): the copies of the next tile follow the products through this one.  At
// head dims 128 and 64 two and four tiles fit.
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
constexpr int kLoadWarp = 4, kIssueWarp = 5, kThreads = 192;
constexpr uint32_t kOCol = 256;  // tensor memory: two S slots of 128 columns, then O

template <int kDim>
struct Cfg {
  static constexpr int kChunks = kDim / 64;
  static constexpr int kStages = kDim == 256 ? 1 : kDim == 128 ? 2 : 4;
  static constexpr int kTile = kChunks * kSub;
  static constexpr int kOffK = kTile, kOffV = kOffK + kStages * kTile, kOffP = kOffV + kStages * kTile;
  static constexpr int kSmem = kOffP + 2 * kSub + 1024;
  static constexpr int kKParts = kChunks, kVParts = 4;  // a K tile comes by 64 dims, a V tile by 32 keys
  static constexpr int kPart = kBq * kDim + 2 * kBq;    // floats of a partial: [dim / 4][128 rows][4], m, l
  // barriers
  static constexpr int Q_FULL = 0, Q_FREE = 1, S_FULL = 2, S_FREE = 4, P_FULL = 6, PV_DONE = 7, O_FREE = 8, ALL_DONE = 9,
                       K_FULL = 10, K_FREE = K_FULL + kStages * kKParts, V_FULL = K_FREE + kStages * kKParts,
                       V_FREE = V_FULL + kStages * kVParts, kBars = V_FREE + kStages * kVParts;
};

// Shared-memory descriptor of an MN-major tile, 128-byte swizzle: 64 elements of the MN dimension a row of 128 bytes, 8 rows
// (of the K dimension) a swizzle group, groups 1024 bytes apart (stride byte offset), the next 64 MN elements `lead` bytes on.
__device__ __forceinline__ uint64_t sdesc_mn(uint32_t saddr, uint32_t lead) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
constexpr uint32_t kIdescBMnMajor = 1u << 16;

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

template <bool kBf16, int kDim>
__global__ void __launch_bounds__(kThreads, 1)
    attn_chunks_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, PagedCache c, PagedBatch b, AttnCall a, int tt,
                       float* __restrict__ part, unsigned int* __restrict__ counters, unsigned int* __restrict__ err) {
  using C = Cfg<kDim>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ uint64_t bars[C::kBars];
  __shared__ LineStart ls;
  __shared__ long long scan[kThreads / 32];
  __shared__ uint32_t held[8];  // 16-key groups of a tile that lie in a page
  __shared__ uint32_t tmem_slot, s_last;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = a.n_q / c.n_kv;

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kBars; ++i)
      mbar_init(bar(i), i == C::S_FREE || i == C::S_FREE + 1 || i == C::P_FULL || i == C::O_FREE ? kBq : 1);
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
  pdl_wait();
  pdl_trigger();
  find_start<kThreads>(b, c.page_shift, c.n_kv, a.window, tt, kBkShift, &ls, scan);  // syncs the block
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  bool ok = true;

  if (ls.begin < ls.end) {
    Walk w;
    w.start(ls, b, c.page_shift, a.window, tt, kBkShift, lane);
    int g = 0, item = 0;  // tiles and items of this CTA so far
    if (warp == kLoadWarp) {
      // ---------------------------------------------------------------------- TMA copies
      const int box = min(kBoxSlots, 1 << c.page_shift);
      const uint32_t q_bytes = (uint32_t)(group * tt * 128 * C::kChunks);
      int nk = 0, nv = 0;  // tiles whose copies have been issued
      for (; ok && w.more(); w.next(b, c.page_shift, c.n_kv, a.window, tt, kBkShift), ++item) {
        const int lo = w.lo(a.window, tt), hi = w.hi(tt);
        if (item > 0 && !mbar_wait_warp(bar(C::Q_FREE), (uint32_t)(item - 1) & 1u, kWaitBudgetCycles)) {
          ok = false;
          break;
        }
        if (elect_one()) {
          mbar_arrive_expect_tx(bar(C::Q_FULL), q_bytes);
#pragma unroll
          for (int ch = 0; ch < C::kChunks; ++ch)
            tma_load_3d(base + (uint32_t)(ch * kSub), &tmQ, 64 * ch, w.h * group, w.q.row0 + w.t * tt, bar(C::Q_FULL));
        }
        __syncwarp();
        for (int i = 0; ok && i < w.cnt; ++i, ++g) {
          const int st = g % C::kStages, tile0 = (w.first + w.k0 + i) << kBkShift;
          int page = -1;
          if (lane < kBk / 16) {
            const int p = tile0 + 16 * lane, col = p >> c.page_shift;
            if (p <= hi && (p | (box - 1)) >= lo && col < b.max_pages) page = b.pages[(int64_t)w.s * b.max_pages + col];
            if (page < 0 || page >= c.n_pages) page = -1;
          }
          const uint32_t there = __ballot_sync(0xffffffffu, page >= 0);
          // K by 64 dims, V by 32 keys: 128 / box boxes a column of K, 32 / box a column of a part of V
          const uint32_t ph = (uint32_t)(g / C::kStages - 1) & 1u;
          const int kbox = kBk / box;
          for (int ch = 0; ch < C::kKParts; ++ch) {
            const int bi = st * C::kKParts + ch;
            if (g >= C::kStages && !mbar_wait_warp(bar(C::K_FREE + bi), ph, kWaitBudgetCycles)) {
              ok = false;
              break;
            }
            if (lane == 0) {
              if (ch == 0) held[g & 7] = there;
              mbar_arrive_expect_tx(bar(C::K_FULL + bi), kSub);
            }
            __syncwarp();
            const int pg = __shfl_sync(0xffffffffu, page, lane * (box / 16) & 31);
            if (lane < kbox)
              tma_load_4d(base + (uint32_t)(C::kOffK + st * C::kTile + ch * kSub + lane * box * 128), &tmK, 64 * ch,
                          (tile0 + lane * box) & ((1 << c.page_shift) - 1), w.h, pg < 0 ? c.n_pages : pg, bar(C::K_FULL + bi));
            nk = g * C::kKParts + ch + 1;
          }
          const int vbox = 32 / box, v_ops = C::kChunks * vbox;
          for (int vp = 0; ok && vp < C::kVParts; ++vp) {
            const int bi = st * C::kVParts + vp;
            if (g >= C::kStages && !mbar_wait_warp(bar(C::V_FREE + bi), ph, kWaitBudgetCycles)) {
              ok = false;
              break;
            }
            if (lane == 0) mbar_arrive_expect_tx(bar(C::V_FULL + bi), (uint32_t)(C::kChunks * 32 * 128));
            __syncwarp();
            const int bx = vp * vbox + lane % vbox, ch = lane / vbox;  // box of the tile, column
            const int pg = __shfl_sync(0xffffffffu, page, bx * (box / 16) & 31);
            if (lane < v_ops)
              tma_load_4d(base + (uint32_t)(C::kOffV + st * C::kTile + ch * kSub + bx * box * 128), &tmV, 64 * ch,
                          (tile0 + bx * box) & ((1 << c.page_shift) - 1), w.h, pg < 0 ? c.n_pages : pg, bar(C::V_FULL + bi));
            nv = g * C::kVParts + vp + 1;
          }
        }
      }
      // the last copies land before the CTA may end
      if (!ok && lane == 0) atomicOr(err, DEVERR_PRODUCER_WAIT);
      bool drained = item == 0 || mbar_wait_warp(bar(C::Q_FULL), (uint32_t)(item - 1) & 1u, kWaitBudgetCycles);
      for (int k = max(0, nk - C::kStages * C::kKParts); k < nk; ++k)
        drained &= mbar_wait_warp(bar(C::K_FULL + k % (C::kStages * C::kKParts)), (uint32_t)(k / (C::kStages * C::kKParts)) & 1u,
                                  kWaitBudgetCycles);
      for (int k = max(0, nv - C::kStages * C::kVParts); k < nv; ++k)
        drained &= mbar_wait_warp(bar(C::V_FULL + k % (C::kStages * C::kVParts)), (uint32_t)(k / (C::kStages * C::kVParts)) & 1u,
                                  kWaitBudgetCycles);
      if (!drained && lane == 0) atomicOr(err, DEVERR_DRAIN_WAIT);
    } else if (warp == kIssueWarp) {
      // ---------------------------------------------------------------------- MMAs
      constexpr uint32_t fmt = kBf16 ? 1u : 0u;
      constexpr uint32_t idesc_s = idesc_f16(fmt, kBk, kBq), idesc_o = idesc_f16(fmt, kDim, kBq) | kIdescBMnMajor;
      const uint64_t dq = sdesc_swz(base), dp = sdesc_swz(base + C::kOffP);
      // S of tile i (this CTA's count) of an item whose last tile is `last`
      auto issue_s = [&](int i, bool last) {
        const int st = i % C::kStages;
        const uint32_t ph = (uint32_t)(i / C::kStages) & 1u;
        if (i >= 2 && !mbar_wait_warp(bar(C::S_FREE + (i & 1)), (uint32_t)((i >> 1) - 1) & 1u, kWaitBudgetCycles)) return false;
        const uint64_t dk = sdesc_swz(base + (uint32_t)(C::kOffK + st * C::kTile));
        for (int ch = 0; ch < C::kChunks; ++ch) {
          if (!mbar_wait_warp(bar(C::K_FULL + st * C::kKParts + ch), ph, kWaitBudgetCycles)) return false;
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t at = (uint32_t)(ch * (kSub >> 4) + 2 * k);
              tc_mma(tmem + 128u * (uint32_t)(i & 1), dq + at, dk + at, idesc_s, ch > 0 || k > 0);
            }
            tc_commit(bar(C::K_FREE + st * C::kKParts + ch));
          }
          __syncwarp();
        }
        if (elect_one()) {
          tc_commit(bar(C::S_FULL + (i & 1)));
          if (last) tc_commit(bar(C::Q_FREE));
        }
        __syncwarp();
        return true;
      };
      for (; ok && w.more(); w.next(b, c.page_shift, c.n_kv, a.window, tt, kBkShift), ++item) {
        ok = mbar_wait_warp(bar(C::Q_FULL), (uint32_t)item & 1u, kWaitBudgetCycles) && issue_s(g, w.cnt == 1);
        for (int i = 0; ok && i < w.cnt; ++i, ++g) {
          if (i + 1 < w.cnt && !issue_s(g + 1, i + 2 == w.cnt)) {
            ok = false;
            break;
          }
          if (!mbar_wait_warp(bar(C::P_FULL), (uint32_t)g & 1u, kWaitBudgetCycles) ||
              (i == 0 && item > 0 && !mbar_wait_warp(bar(C::O_FREE), (uint32_t)(item - 1) & 1u, kWaitBudgetCycles))) {
            ok = false;
            break;
          }
          const int st = g % C::kStages;
          const uint64_t dv = sdesc_mn(base + (uint32_t)(C::kOffV + st * C::kTile), kSub);
          for (int vp = 0; vp < C::kVParts; ++vp) {  // O += P V, 32 keys at a time
            if (!mbar_wait_warp(bar(C::V_FULL + st * C::kVParts + vp), (uint32_t)(g / C::kStages) & 1u, kWaitBudgetCycles)) {
              ok = false;
              break;
            }
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const int kk = 2 * vp + k;  // 16 keys
                tc_mma(tmem + kOCol, dp + (uint32_t)((kk >> 2) * (kSub >> 4) + 2 * (kk & 3)), dv + (uint32_t)(kk * (16 * 128 >> 4)),
                       idesc_o, i > 0 || kk > 0);
              }
              tc_commit(bar(C::V_FREE + st * C::kVParts + vp));
              if (vp == C::kVParts - 1) tc_commit(bar(C::PV_DONE));
            }
            __syncwarp();
          }
        }
      }
      if (elect_one()) {
        if (!ok) atomicOr(err, DEVERR_PRODUCER_WAIT);
        tc_commit(bar(C::ALL_DONE));  // completes once every MMA issued above has
        if (!mbar_wait_bounded(bar(C::ALL_DONE), 0u, kWaitBudgetCycles)) atomicOr(err, DEVERR_DRAIN_WAIT);
      }
      __syncwarp();
    } else {
      // ---------------------------------------------------------------------- softmax, one row per thread
      const int r = threadIdx.x;
      const uint32_t lanes = tmem + ((uint32_t)(32 * warp) << 16);
      const uint32_t prow = base + C::kOffP + (uint32_t)(r * 128);
      const float sc = a.scale * kLog2e;
      for (; w.more(); w.next(b, c.page_shift, c.n_kv, a.window, tt, kBkShift), ++item) {
        const int tok0 = w.t * tt, rows = min(w.q.rows - tok0, tt) * group;
        const int lo = w.lo(a.window, tt), hi = w.hi(tt);
        const bool live = r < rows, busy = 32 * warp < rows;  // this row's, and any of the warp's
        const int tok = tok0 + (live ? r / group : 0), head = w.h * group + (live ? r % group : 0);
        const int pos = w.q.pos0 + tok, from = a.window > 0 ? max(0, pos - a.window + 1) : 0;
        float m = -INFINITY, l = 0.0f;
        for (int i = 0; i < w.cnt; ++i, ++g) {
          const int j0 = (w.first + w.k0 + i) << kBkShift;
          if (ok && !mbar_wait_warp(bar(C::S_FULL + (g & 1)), (uint32_t)(g >> 1) & 1u, kWaitBudgetCycles)) ok = false;
          if (!ok) continue;
          tc_fence_after();
          uint32_t pk[kBk / 2];
          bool grown = false;
          float up = 1.0f;
          if (busy) {
            float v[kBk];
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
              uint32_t x[32];
              tmem_ld32(lanes + 128u * (uint32_t)(g & 1) + 32 * q4, x);
#pragma unroll
              for (int k = 0; k < 32; ++k) v[32 * q4 + k] = __uint_as_float(x[k]);
            }
            tc_fence_before();
            mbar_arrive(bar(C::S_FREE + (g & 1)));
            const uint32_t there = held[g & 7];
            if (j0 < from || j0 + kBk - 1 > pos) {
#pragma unroll
              for (int k = 0; k < kBk; ++k)
                if (j0 + k < from || j0 + k > pos) v[k] = -INFINITY;
            }
            if (there != 0xffu) {  // groups of 16 keys in no page
#pragma unroll
              for (int k = 0; k < kBk; ++k)
                if (!((there >> (k >> 4)) & 1u)) v[k] = -INFINITY;
            }
            float mx[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) mx[k] = v[k];
#pragma unroll
            for (int k = 8; k < kBk; ++k) mx[k & 7] = fmaxf(mx[k & 7], v[k]);
            const float top = sc * fmaxf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])),
                                         fmaxf(fmaxf(mx[4], mx[5]), fmaxf(mx[6], mx[7])));
            grown = top > m + kGrowth;  // m = -inf: any visible key
            if (grown) {
              up = m == -INFINITY ? 0.0f : ex2(m - top);
              m = top;
              l *= up;
            }
            const float ref = m == -INFINITY ? 0.0f : m;
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < kBk; k += 2) {
              pk[k >> 1] = pack2<kBf16>(ex2(fmaf(v[k], sc, -ref)), ex2(fmaf(v[k + 1], sc, -ref)));
              const float2 as_used = unpack2<kBf16>(pk[k >> 1]);
              sum[(k >> 1) & 3] += as_used.x + as_used.y;
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
          } else {
            tc_fence_before();
            mbar_arrive(bar(C::S_FREE + (g & 1)));
          }
          // the P tile and O are free once the previous tile's product has completed
          if (g > 0 && !mbar_wait_warp(bar(C::PV_DONE), (uint32_t)(g - 1) & 1u, kWaitBudgetCycles)) {
            ok = false;
            continue;
          }
          if (i > 0 && __any_sync(0xffffffffu, grown)) {
            tc_fence_after();
#pragma unroll 1
            for (int ch = 0; ch < kDim / 32; ++ch) {
              uint32_t x[32];
              tmem_ld32(lanes + kOCol + 32 * ch, x);
#pragma unroll
              for (int k = 0; k < 32; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * up);
              tmem_st32(lanes + kOCol + 32 * ch, x);
            }
            asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory");
            tc_fence_before();
          }
          if (busy) {
#pragma unroll
            for (int k = 0; k < kBk / 8; ++k)
              asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};\n" ::"r"(prow + (uint32_t)((k >> 3) * kSub) +
                                                                              (uint32_t)(((k & 7) ^ (r & 7)) << 4)),
                           "r"(pk[4 * k]), "r"(pk[4 * k + 1]), "r"(pk[4 * k + 2]), "r"(pk[4 * k + 3])
                           : "memory");
          }
          if (j0 < lo || j0 + kBk - 1 > hi) {
            // values of keys outside the item's range (another sequence's, or nobody's) must not meet a weight of zero: row r
            // of the tile, once its copies have landed
            const int st = g % C::kStages;
            bool landed = true;
#pragma unroll
            for (int vp = 0; vp < C::kVParts; ++vp)
              landed = landed && mbar_wait_warp(bar(C::V_FULL + st * C::kVParts + vp), (uint32_t)(g / C::kStages) & 1u,
                                                kWaitBudgetCycles);
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
          }
          asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
          mbar_arrive(bar(C::P_FULL));
        }
        if (ok && !mbar_wait_warp(bar(C::PV_DONE), (uint32_t)(g - 1) & 1u, kWaitBudgetCycles)) ok = false;
        if (!ok && lane == 0) atomicOr(err, DEVERR_CONSUMER_WAIT);
        __syncwarp();
        tc_fence_after();

        // ---- the item's output
        const int64_t row = w.q.row0 + tok;
        uint16_t* orow = a.o + row * a.o_row + (int64_t)head * a.o_head;
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
        auto exactly = [&](bool bad) {  // rows whose result is not finite, or without weight
          __syncwarp();
          for (uint32_t rest = __ballot_sync(0xffffffffu, live && bad); rest; rest &= rest - 1) {
            const int src = __ffs(rest) - 1;
            attend_row<kBf16, kDim>(c, b, a, w.s, __shfl_sync(0xffffffffu, pos, src),
                                    (int64_t)w.q.row0 + __shfl_sync(0xffffffffu, tok, src), __shfl_sync(0xffffffffu, head, src),
                                    lane);
          }
        };
        if (w.whole()) {
          if (busy) {
            float nan = 0.0f;
            const float inv = 1.0f / l;
#pragma unroll 1
            for (int ch = 0; ch < kDim / 32; ++ch) {
              uint32_t x[32];
              float f[32];
              tmem_ld32(lanes + kOCol + 32 * ch, x);
#pragma unroll
              for (int k = 0; k < 32; ++k) f[k] = __uint_as_float(x[k]);
              store(ch, f, inv, nan);
            }
            tc_fence_before();
            mbar_arrive(bar(C::O_FREE));
            exactly(nan != 0.0f || !(l > 0.0f));
          } else {
            tc_fence_before();
            mbar_arrive(bar(C::O_FREE));
          }
          continue;
        }
        // ---- a piece: into the workspace, joined by the last one to arrive
        const Pieces ps = pieces_of(w, ls);
        float* mine = part + (size_t)(2 * blockIdx.x + (w.k0 > 0 ? 0 : 1)) * C::kPart;
        if (busy) {
#pragma unroll 1
          for (int ch = 0; ch < kDim / 32; ++ch) {
            uint32_t x[32];
            tmem_ld32(lanes + kOCol + 32 * ch, x);
            if (live) {
#pragma unroll
              for (int k = 0; k < 8; ++k)
                __stcg(reinterpret_cast<float4*>(mine) + (size_t)(8 * ch + k) * kBq + r,
                       make_float4(__uint_as_float(x[4 * k]), __uint_as_float(x[4 * k + 1]), __uint_as_float(x[4 * k + 2]),
                                   __uint_as_float(x[4 * k + 3])));
            }
          }
          if (live) {
            __stcg(mine + kBq * kDim + r, m);
            __stcg(mine + kBq * kDim + kBq + r, l);
          }
        }
        tc_fence_before();
        mbar_arrive(bar(C::O_FREE));
        __threadfence();
        named_bar_sync(1, kBq);
        if (r == 0) {
          const unsigned int before = atomicAdd(counters + ps.first, 1u);
          s_last = before + 1 == (unsigned int)ps.count;
          if (s_last) counters[ps.first] = 0;
          __threadfence();
        }
        named_bar_sync(1, kBq);
        if (s_last && busy) {
          auto slot = [&](int i) { return part + (size_t)(2 * (ps.first + i) + (i == 0 ? 1 : 0)) * C::kPart; };
          float M = -INFINITY, L = 0.0f, nan = 0.0f;
          if (live) {
            for (int i = 0; i < ps.count; ++i) M = fmaxf(M, __ldcg(slot(i) + kBq * kDim + r));
            for (int i = 0; i < ps.count; ++i) {
              const float mi = __ldcg(slot(i) + kBq * kDim + r);
              L = fmaf(__ldcg(slot(i) + kBq * kDim + kBq + r), mi == -INFINITY ? 0.0f : ex2(mi - M), L);
            }
          }
          const float inv = 1.0f / L;
#pragma unroll 1
          for (int ch = 0; ch < kDim / 32; ++ch) {
            float f[32];
#pragma unroll
            for (int k = 0; k < 32; ++k) f[k] = 0.0f;
            if (live) {
#pragma unroll 1
              for (int i = 0; i < ps.count; ++i) {
                const float mi = __ldcg(slot(i) + kBq * kDim + r), e = mi == -INFINITY ? 0.0f : ex2(mi - M);
                const float4* src = reinterpret_cast<const float4*>(slot(i)) + (size_t)(8 * ch) * kBq + r;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                  const float4 x = __ldcg(src + k * kBq);
                  f[4 * k] = fmaf(x.x, e, f[4 * k]);
                  f[4 * k + 1] = fmaf(x.y, e, f[4 * k + 1]);
                  f[4 * k + 2] = fmaf(x.z, e, f[4 * k + 2]);
                  f[4 * k + 3] = fmaf(x.w, e, f[4 * k + 3]);
                }
              }
            }
            store(ch, f, inv, nan);
          }
          exactly(nan != 0.0f || !(L > 0.0f));
        }
        named_bar_sync(1, kBq);  // s_last is free again
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
  W8A8_CUDA(launch_pdl(attn_chunks_kernel<kBf16, kDim>, dim3((unsigned)sms), dim3(kThreads), (size_t)C::kSmem, st, tq, tk, tv,
                       pc, pb, a, tt, reinterpret_cast<float*>(base + W8A8_WS_RESERVED), reinterpret_cast<unsigned int*>(base),
                       reinterpret_cast<unsigned int*>(base + kErrWordOffset)));
  return W8A8_OK;
}

}  // namespace

size_t attn_chunks_ws(int dim, int sms) { return (size_t)2 * sms * (kBq * dim + 2 * kBq) * sizeof(float); }

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
