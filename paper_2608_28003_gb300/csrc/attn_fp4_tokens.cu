// Attention over a paged cache in 4 bits for single tokens and a few drafted ones: items of up to 16 rows (tokens times the query
// heads of a group).
//
// The cache is read once, at 4.5 bits a value, so HBM bounds the kernel as long as turning codes into operands keeps up: at the
// measured copy rate an SM gets 47 codes a cycle, for which it has 128 lanes.  So the cache is the left operand of both products
// (mma.sync m16n8k16: 16 keys by 8 rows, then 16 dims by 8 rows; rows of at most 8 or 16), and which lane holds which dims is
// chosen so that codes need no shuffles:
//  * scores: lane (g, q) = (lane / 4, lane % 4) has keys g and g + 8 and a quarter of their dims, whole blocks of them, 32, 16 or 8
//    bytes as they lie; a product's k index is 4 dims of each of the quarters, the queries laid out alike;
//  * values: lane (g, q) has an eighth of the dims of keys 2q, 2q + 1, 2q + 8, 2q + 9; the codes of two keys are
//    interleaved by masks and a shift, so that a byte is a dim's two keys.
// A code is converted (two an instruction) and multiplied by its block's scale in fp16, which is exact: six significant bits between
// 2^-10 and 2688.  2^k_exp and 2^v_exp are applied to scores and outputs.
// Queries are fp16 too: a row is brought to [2^14, 2^15) by a power of two, which is exact for fp16 and for all of a bf16 row's dims
// down to 2^-29 of its largest (smaller ones are off by at most 2^-40 of it, less than fp32 sums are).  Weights are
// fp16 lifted to 2^15 (attn_paged.cuh), whatever the type.
//
// One CTA per SM walks its stretch of the line of key tiles (attn_paged.cuh).  Four loader warps, one each for the codes and the
// scales of keys and values, fill a ring of tiles of 36 KB (128, 256, 512 keys at head dims 256, 128, 64): codes page by page by
// TMA (an operation costs its warp some 70 cycles, which one warp for all of them could not afford), scales 16 bytes a lane where a
// page's follow one another, else key by key; 8 consumer warps take 16, 32 or 64 keys of a tile each, on their own from scores to output.
// A warp's reference moves when one of its lanes sees a score that outgrew it, so a step has no reduction over lanes; sums stay
// in the lanes until the item ends.
//
// Measured: 64 sequences of up to 30000 keys at head dim 256 (263 MB) 63.5 us, 4.1 TB/s and 0.61 of the copy rate; the loaders alone
// would take 41 (6.4 TB/s), then 6 until the first tile is there, 2.5 to 5 an item's end, and the consumers, of whose
// issue slots half are taken, two warps a scheduler (three, with a block of keys each and fewer stages, spill: 97.7 us).  20 sequences
// with 4 drafted tokens, fp16, head dim 64 (28 MB) 30.2 us: latency from step to step, a fifth of it waits for instructions that
// run for the first time.  With one loader warp, one block of keys at a time and the
// queries read as they are needed the first took 105 us.  Rows of 16 at head dim 256, whose accumulators alone are 128 registers, spill (916
// bytes of stores; 284 at head dim 128; rows of 8 at 256 28): 40 sequences of 3000 keys, 4 drafted tokens of 4 heads on 1 of 256, 40 us.
#include "attn_fp4.cuh"
#include "ops.cuh"
#include "tmap.cuh"

namespace w8a8 {

namespace {

constexpr int kWarps = 8;     // consumers
// What an item costs beside its key tiles, in key tiles (0, 2, 4, 6: 64 long sequences 73.0, 67.5, 65.3, 65.0 us, 20 with drafts 42.4,
// 31.4, 31.2, 33.4).
constexpr int kItemCost = 4;

template <int kDim, int kNt>
struct Cfg {
  static constexpr int kTeams = kDim == 256 ? 2 : 1;          // of warps, that take tiles in turn
  static constexpr int kTeam = kWarps / kTeams;               // warps of a team
  static constexpr int kBlocks = kDim == 64 ? 4 : 2;          // of 16 keys, that a warp has of a tile, two at a time
  static constexpr int kBk = 16 * kBlocks * kTeam, kBkShift = kDim == 256 ? 7 : kDim == 128 ? 8 : 9;
  static constexpr int kRow = kDim / 2, kSRow = kDim / 16;    // bytes of a key's codes, scales
  static constexpr int kCodes = kBk * kRow, kScales = kBk * kSRow;
  static constexpr int kStage = 2 * (kCodes + kScales);       // K codes, V codes, K scales, V scales
  static constexpr int kJoin = kWarps * 8 * kDim * 4;         // 8 rows' outputs of every warp
  static constexpr int kQRow = 2 * kDim + 16;                 // bytes between the rows of an item's queries
  static constexpr int kQ = 2 * 8 * kNt * kQRow;              // of two items
  static constexpr int kStages = (kDim == 256 ? 5 : 6) - kNt;
  static constexpr int kSmem = kStages * kStage + kJoin + kQ + 1024;
  static constexpr int kThreads = 384;                        // consumers and four loaders
  static constexpr int kTiles = kDim / 16;                    // of 16 dims
  static constexpr int kPer = kTiles < kWarps ? 1 : kTiles / kWarps;  // tiles that a warp joins
  static_assert(kSmem + 16 * kNt * kDim <= 227 * 1024 - 2048, "shared memory");
};

// Where byte `byte` of a key's codes lies in a tile: rows of 128 bytes swizzled over 128, of 64 over 64, of 32 as they are.
template <int kDim>
__device__ __forceinline__ uint32_t code_at(int key, int byte) {
  const int swz = kDim == 256 ? (key & 7) << 4 : kDim == 128 ? ((key >> 1) & 3) << 4 : 0;
  return (uint32_t)(key * (kDim / 2) + (byte ^ swz));
}
__device__ __forceinline__ uint32_t lds8(uint32_t a) {
  uint16_t v;
  asm volatile("{\n .reg .u8 t;\n ld.shared.u8 t, [%1];\n cvt.u16.u8 %0, t;\n}\n" : "=h"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];\n" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {  // of an 8 x 8 matrix of 16-bit elements
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
  return y;
}
// Up to four scale bytes as fp16 pairs, each twice.
template <int kN>
__device__ __forceinline__ void scale_pairs(uint32_t bytes, uint32_t (&s)[kN]) {
#pragma unroll
  for (int i = 0; i < kN; i += 2) {
    const uint32_t h = e4m3x2_to_f16x2(bytes >> (8 * i));
    s[i] = __byte_perm(h, h, 0x1010);
    if (i + 1 < kN) s[i + 1] = __byte_perm(h, h, 0x3232);
  }
}

struct LoadPlan {
  int contiguous;  // a page's scales of a head are one piece, 16-byte aligned
};

template <bool kBf16, int kDim, int kNt>
__global__ void __launch_bounds__(Cfg<kDim, kNt>::kThreads, 1)
    attn_fp4_tokens_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, Fp4Pages c,
                           PagedBatch b, AttnCall a, LoadPlan plan, int tt, float* __restrict__ part,
                           unsigned int* __restrict__ counters, unsigned int* __restrict__ err) {
  using C = Cfg<kDim, kNt>;
  constexpr int kRows = 8 * kNt, kPart = kTokenRows * kDim + 2 * kTokenRows;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ uint64_t bars[2 * C::kStages + 4];
  __shared__ LineStart ls;
  __shared__ long long scan[C::kThreads / 32];
  __shared__ uint32_t held[C::kStages];  // 16-key groups of a stage's tile that lie in a page
  __shared__ __align__(16) float s_m[kRows][kWarps], s_l[kRows][kWarps];
  __shared__ uint2 qs[kNt][kDim / 16][32];  // the queries as the first product's right operand, a lane's words of a k step
  __shared__ uint32_t s_last, s_bad, s_beat;
  const uint32_t raw = smem_u32(smem_raw), ring = (raw + 1023u) & ~1023u;
  uint8_t* behind = smem_raw + (ring - raw) + C::kStages * C::kStage;
  float4* join = reinterpret_cast<float4*>(behind);
  const uint32_t qring = ring + (uint32_t)(C::kStages * C::kStage + C::kJoin);  // the queries of two items as they come
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  auto empty = [&](int i) { return bar0 + 8u * (uint32_t)(C::kStages + i); };
  auto q_full = [&](int i) { return bar0 + 8u * (uint32_t)(2 * C::kStages + i); };
  auto q_free = [&](int i) { return bar0 + 8u * (uint32_t)(2 * C::kStages + 2 + i); };
  const int group = a.n_q / c.p.n_kv;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, shift = c.p.page_shift, n_kv = c.p.n_kv;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(full(i), 2 + 64);  // two counts of bytes, two warps of lanes
      mbar_init(empty(i), C::kTeam);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full(i), 32);
      mbar_init(q_free(i), kWarps);
    }
    fence_mbar_init();
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
    s_bad = s_beat = 0;
  }
  pdl_wait();
  pdl_trigger();
  find_start<C::kThreads>(b, shift, n_kv, a.window, tt, C::kBkShift, (int)blockIdx.x, (int)gridDim.x, &ls, scan,
                          kItemCost);
  if (ls.begin >= ls.end) return;
  Walk w;
  w.start(ls, b, shift, a.window, tt, C::kBkShift, lane);
  int g = 0, item = 0;  // tiles and items of this CTA so far
  bool ok = true;

  // registers: 384 threads of 168 are shared out as 256 of 200 and 128 of 104
  if (warp >= kWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;\n");
    // ------------------------------------------ loaders: K codes, V codes, K scales, V scales and queries
    const int what = warp - kWarps, kv = what & 1;
    const int box = min(1 << shift, C::kBk), boxes = C::kBk / box;  // per tile
    const uint8_t* scales = kv ? c.vs : c.ks;
    for (; ok && w.more(); w.next(b, shift, n_kv, a.window, tt, C::kBkShift), ++item) {
      const int lo = w.lo(a.window, tt), hi = w.hi(tt);
      if (what == 3) {  // the item's queries
        if (item >= 2 && !wait_beat(q_free(item & 1), (uint32_t)(item / 2 - 1) & 1u, &s_beat)) {
          ok = false;
          break;
        }
        const int tok0 = w.t * tt, rows = min(w.q.rows - tok0, tt) * group;
        for (int e = lane; e < rows * (kDim / 8); e += 32) {
          const int r = e / (kDim / 8), at = e % (kDim / 8);
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(
                           qring + (uint32_t)(((item & 1) * kRows + r) * C::kQRow + 16 * at)),
                       "l"(a.q + (int64_t)(w.q.row0 + tok0 + r / group) * a.q_row + (int64_t)(w.h * group + r % group) * a.q_head + 8 * at)
                       : "memory");
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];\n" ::"r"(q_full(item & 1)) : "memory");
      }
      constexpr int kGroups = C::kBk / 16, kBatch = 32 / kGroups;  // tiles whose pages are read at once, ahead of their use
      int page = group_page(b, c.p, w.s, (w.first + w.k0) << C::kBkShift, lo, hi, box, lane), ahead = -1;
      for (int i = 0; i < w.cnt; ++i, ++g) {
        const int st = g % C::kStages, tile0 = (w.first + w.k0 + i) << C::kBkShift, in_batch = i % kBatch;
        if (in_batch == 0) {
          if (i > 0) page = ahead;
          if (i + kBatch < w.cnt) ahead = group_page(b, c.p, w.s, tile0 + (kBatch << C::kBkShift), lo, hi, box, lane);
        }
        const uint32_t there = (__ballot_sync(0xffffffffu, page >= 0) >> (in_batch * kGroups)) &
                               (kGroups == 32 ? 0xffffffffu : (1u << (kGroups & 31)) - 1u);
        if (g >= C::kStages && !wait_beat(empty(st), (uint32_t)(g / C::kStages - 1) & 1u, &s_beat)) {
          ok = false;
          break;
        }
        const uint32_t dst = ring + (uint32_t)(st * C::kStage + kv * C::kCodes),
                       sdst = ring + (uint32_t)(st * C::kStage + 2 * C::kCodes + kv * C::kScales);
        if (what < 2) {
          if (lane == 0) {
            if (kv == 0) held[st] = there;
            mbar_arrive_expect_tx(full(st), (uint32_t)C::kCodes);
          }
          __syncwarp();
          const int pg = __shfl_sync(0xffffffffu, page, (in_batch * kGroups + lane * (box / 16)) & 31);
          if (lane < boxes)  // a page that holds nothing: a coordinate outside the tensor, which fills zeros
            tma_load_4d(dst + (uint32_t)(lane * box * C::kRow), kv ? &tmV : &tmK, 0, (tile0 + lane * box) & ((1 << shift) - 1), w.h,
                        pg < 0 ? c.p.n_pages : pg, full(st));
        } else {
          // 16 bytes a lane where a page's scales follow one another, else a key's
          const int per = plan.contiguous ? 16 / C::kSRow : 1;
          for (int k0 = 0; k0 < C::kBk; k0 += 32 * per) {
            const int key = k0 + lane * per, pg = __shfl_sync(0xffffffffu, page, (in_batch * kGroups + key / 16) & 31);
            if (pg >= 0) {
              const uint8_t* from = scales + (int64_t)pg * c.s_page + (int64_t)((tile0 + key) & ((1 << shift) - 1)) * c.s_slot +
                                    (int64_t)w.h * c.s_head;
              if (plan.contiguous)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(sdst + (uint32_t)(key * C::kSRow)), "l"(from)
                             : "memory");
              else
                asm volatile("cp.async.ca.shared.global [%0], [%1], %2;\n" ::"r"(sdst + (uint32_t)(key * C::kSRow)), "l"(from),
                             "n"(C::kSRow)
                             : "memory");
            }
          }
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];\n" ::"r"(full(st)) : "memory");
        }
      }
    }
    // the last copies land before the CTA may end
    if (!ok && lane == 0) give_up(err, a, DEVERR_PRODUCER_WAIT);
    if (what >= 2)
      asm volatile("cp.async.wait_all;\n" ::: "memory");
    else
      for (int k = max(0, g - C::kStages); k < g; ++k)
        if (!wait_beat(full(k % C::kStages), (uint32_t)(k / C::kStages) & 1u, &s_beat) && lane == 0)
          give_up(err, a, DEVERR_DRAIN_WAIT);
    return;
  }

  // -------------------------------------------------------------------------- consumers
  asm volatile("setmaxnreg.inc.sync.aligned.u32 200;\n");
  constexpr int kBar = 1, kConsumers = 32 * kWarps, kChains = 2;
  const int gq = lane >> 2, quad = lane & 3;
  const float back = two_to(c.v_exp);
  const int team = warp / C::kTeam, in_team = warp % C::kTeam;
  for (; w.more(); w.next(b, shift, n_kv, a.window, tt, C::kBkShift), ++item) {
    const int tok0 = w.t * tt, n_tok = min(w.q.rows - tok0, tt), rows = n_tok * group;
    const int lo = w.lo(a.window, tt), hi = w.hi(tt);
    // where every row of the item sees everything: between the last row's first key and the first row's position
    const int all_lo = a.window > 0 ? max(0, hi - a.window + 1) : 0, all_hi = w.q.pos0 + tok0;
    // the queries as the first product's right operand: row 8 n + gq, dims of quarter `quad`, four a k step; a warp turns the
    // slices of 32 dims that are its own, after every warp has the rows' largest magnitudes
    float fac[kNt][2];  // of rows 8 n + 2 quad + {0, 1}: scores in powers of two
    int pos[kNt][2], from[kNt][2];
    if (ok && !wait_beat(q_full(item & 1), (uint32_t)(item / 2) & 1u, &s_beat)) ok = false;
#pragma unroll
    for (int n = 0; n < kNt; ++n) {
      const int r = 8 * n + gq;
      const bool live = r < rows;
      const uint32_t qat = qring + (uint32_t)(((item & 1) * kRows + (live ? r : 0)) * C::kQRow + quad * (kDim / 2));
      uint32_t tops = 0;  // of both halves, as integers
#pragma unroll
      for (int i = 0; i < kDim / 32; ++i) {
        const uint4 x = lds128(qat + 16 * i);
        tops = __vmaxu2(__vmaxu2(tops, __vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu)),
                        __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu));
      }
      tops = __vmaxu2(tops, __shfl_xor_sync(0xffffffffu, tops, 1));
      tops = __vmaxu2(tops, __shfl_xor_sync(0xffffffffu, tops, 2));
      const uint32_t top16 = live ? max(tops & 0xffffu, tops >> 16) : 0u, top = __float_as_uint(unpack2<kBf16>(top16).x);
      // the row in units of 2^e: its largest in [2^14, 2^15) (a row that is not finite is NaN, and its result too)
      const int e = top == 0 ? 0 : max((int)(top >> 23) - 127, -126) - 14;
      const float up0 = top >= 0x7f800000u ? NAN : two_to(-e / 2), up1 = two_to(-e - (-e / 2));
#pragma unroll
      for (int i = 0; i < kDim / 32; ++i) {
        if (i % kWarps != warp) continue;
        const uint4 x = live ? lds128(qat + 16 * i) : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t v[4] = {x.x, x.y, x.z, x.w};
        uint32_t h[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 f = unpack2<kBf16>(v[k]);
          h[k] = pack2<false>(f.x * up0 * up1, f.y * up0 * up1);
        }
        qs[n][2 * i][lane] = make_uint2(h[0], h[1]);
        qs[n][2 * i + 1][lane] = make_uint2(h[2], h[3]);
      }
      const float f = ldexpf(c.score, e + c.k_exp + ilogbf(a.scale));  // of row 8 n + gq, which lane 4 gq has
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fac[n][i] = __shfl_sync(0xffffffffu, f, 4 * (2 * quad + i));
        const int rr = 8 * n + 2 * quad + i, tok = rr < rows ? tok0 + rr / group : tok0;
        pos[n][i] = w.q.pos0 + tok;
        from[n][i] = a.window > 0 ? pos[n][i] - a.window + 1 : 0;
      }
    }
    named_bar_sync(kBar, kConsumers);
    if (lane == 0) mbar_arrive(q_free(item & 1));
    float m[kNt][2], l[kNt][2], acc[kNt][C::kTiles][4];
#pragma unroll
    for (int n = 0; n < kNt; ++n) {
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.0f;
#pragma unroll
      for (int i = 0; i < C::kTiles; ++i) acc[n][i][0] = acc[n][i][1] = acc[n][i][2] = acc[n][i][3] = 0.0f;
    }

    for (int it = 0; it < w.cnt; ++it, ++g) {
      if (C::kTeams > 1 && (g & 1) != team) continue;
      const int st = g % C::kStages, k0 = 16 * C::kBlocks * in_team, j00 = ((w.first + w.k0 + it) << C::kBkShift) + k0;
      if (ok && !wait_beat(full(st), (uint32_t)(g / C::kStages) & 1u, &s_beat)) ok = false;
      if (!ok) continue;
      const uint32_t mine = held[st] >> (C::kBlocks * in_team);
      const uint32_t kt = ring + (uint32_t)(st * C::kStage), vt = kt + C::kCodes, ksc = vt + C::kCodes, vsc = ksc + C::kScales;
#pragma unroll 1
      for (int u0 = 0; u0 < C::kBlocks; u0 += 2) {  // two blocks of 16 keys
        const int jj = j00 + 16 * u0;
        const uint32_t both = (mine >> u0) & 3u;
        if (both == 0 || jj > hi || jj + 31 < lo) continue;
        float s[2][kNt][4];
        {
          float z[2][kNt][kChains][4] = {};  // k steps in turn
          uint32_t sp[2][2][kDim / 64];
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const uint32_t at = ksc + (uint32_t)((k0 + 16 * (u0 + u) + gq + 8 * r) * C::kSRow + quad * (kDim / 64));
              scale_pairs(kDim == 256 ? lds32(at) : kDim == 128 ? lds16(at) : lds8(at), sp[u][r]);
            }
#pragma unroll
          for (int t4 = 0; t4 < (kDim == 256 ? 2 : 1); ++t4) {
            uint32_t cw[2][2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int r = 0; r < 2; ++r) {
                const uint32_t at = kt + code_at<kDim>(k0 + 16 * (u0 + u) + gq + 8 * r, quad * (kDim / 8) + 16 * t4);
                if constexpr (kDim == 64) {
                  const uint2 v = lds64(at);
                  cw[u][r][0] = v.x, cw[u][r][1] = v.y, cw[u][r][2] = cw[u][r][3] = 0;
                } else {
                  const uint4 v = lds128(at);
                  cw[u][r][0] = v.x, cw[u][r][1] = v.y, cw[u][r][2] = v.z, cw[u][r][3] = v.w;
                }
              }
#pragma unroll
            for (int x = 0; x < (kDim == 64 ? 2 : 4); ++x) {  // 8 dims: two k steps
              uint2 qv[2][kNt];
#pragma unroll
              for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int n = 0; n < kNt; ++n) qv[y][n] = qs[n][8 * t4 + 2 * x + y][lane];
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                uint32_t h[2][4];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                  e2m1x8_to_f16(cw[u][r][x], h[r]);
#pragma unroll
                  for (int e = 0; e < 4; ++e) h[r][e] = hmul2_bits(h[r][e], sp[u][r][2 * t4 + x / 2]);
                }
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                  for (int n = 0; n < kNt; ++n)
                    mma_f16_16816(z[u][n][(2 * x + y) % kChains], h[0][2 * y], h[1][2 * y], h[0][2 * y + 1], h[1][2 * y + 1],
                                  qv[y][n].x, qv[y][n].y);
              }
            }
          }
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int n = 0; n < kNt; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) s[u][n][e] = (z[u][n][0][e] + z[u][n][1][e]) * fac[n][e & 1];
        }
        if (jj < all_lo || jj + 31 > all_hi || both != 3u) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int n = 0; n < kNt; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int j = jj + 16 * u + gq + 8 * (e >> 1);
                if (j > pos[n][e & 1] || j < from[n][e & 1] || !((both >> u) & 1u)) s[u][n][e] = -INFINITY;
              }
        }
        // ---- the references
        bool grown = false;
        float top[kNt][2];
#pragma unroll
        for (int n = 0; n < kNt; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            top[n][i] = fmaxf(fmaxf(s[0][n][i], s[0][n][2 + i]), fmaxf(s[1][n][i], s[1][n][2 + i]));
            grown = grown || top[n][i] > m[n][i] + kGrowth<false>;
          }
        if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
          for (int n = 0; n < kNt; ++n) {
            float up[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float t = top[n][i];
              t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
              t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
              t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
              up[i] = 1.0f;
              if (t > m[n][i] + kGrowth<false>) {  // m = -inf: any visible key
                up[i] = m[n][i] == -INFINITY ? 0.0f : ex2(m[n][i] - t);
                m[n][i] = t;
              }
              l[n][i] *= up[i];
            }
#pragma unroll
            for (int i = 0; i < C::kTiles; ++i) {
              acc[n][i][0] *= up[0];
              acc[n][i][1] *= up[1];
              acc[n][i][2] *= up[0];
              acc[n][i][3] *= up[1];
            }
          }
        }
        // ---- the weights, keys by rows, turned into the second product's right operand, rows by keys
        uint32_t p[2][kNt][2];
#pragma unroll
        for (int n = 0; n < kNt; ++n) {
          const float r0 = m[n][0] == -INFINITY ? 0.0f : m[n][0] - kLift<false>, r1 = m[n][1] == -INFINITY ? 0.0f : m[n][1] - kLift<false>;
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t x = pack2<false>(ex2(s[u][n][2 * h] - r0), ex2(s[u][n][2 * h + 1] - r1));
              const float2 as_used = unpack2<false>(x);
              l[n][0] += as_used.x;
              l[n][1] += as_used.y;
              p[u][n][h] = transposed(x);
            }
        }
#pragma unroll 1
        for (int u = 0; u < 2; ++u) {  // (rolled: the code of both stays in the instruction cache)
        const int key0 = k0 + 16 * (u0 + u), j0 = jj + 16 * u;
        uint32_t pu[kNt][2];
#pragma unroll
        for (int n = 0; n < kNt; ++n) {
          pu[n][0] = u ? p[1][n][0] : p[0][n][0];
          pu[n][1] = u ? p[1][n][1] : p[0][n][1];
        }
        // ---- values: keys 2 quad + {0, 1, 8, 9}, an eighth of the dims
        // values of keys outside the item's range, or in no page, must not meet a weight of 0
        const bool none = !((both >> u) & 1u), cut = j0 < lo || j0 + 15 > hi || none;
        uint32_t sv[2][kDim == 256 ? 2 : 1], sb[4];  // scales of the pairs of keys
        uint32_t vw[4][kDim / 64];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int key = key0 + 2 * quad + (x & 1) + 8 * (x >> 1), j = j0 + key - key0;
          const uint32_t at = vsc + (uint32_t)(key * C::kSRow);
          sb[x] = kDim == 256 ? lds16(at + 2 * gq) : kDim == 128 ? lds8(at + gq) : lds8(at + (gq >> 1));
          if (cut && (j < lo || j > hi || none)) sb[x] = 0;
          const uint32_t from_at = vt + code_at<kDim>(key, gq * (kDim / 16));
          if constexpr (kDim == 256) {
            const uint4 v = lds128(from_at);
            vw[x][0] = v.x, vw[x][1] = v.y, vw[x][2] = v.z, vw[x][3] = v.w;
          } else if constexpr (kDim == 128) {
            const uint2 v = lds64(from_at);
            vw[x][0] = v.x, vw[x][1] = v.y;
          } else {
            vw[x][0] = lds32(from_at);
          }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          sv[x][0] = e4m3x2_to_f16x2(__byte_perm(sb[2 * x], sb[2 * x + 1], 0x0040));
          if constexpr (kDim == 256) sv[x][1] = e4m3x2_to_f16x2(__byte_perm(sb[2 * x], sb[2 * x + 1], 0x0051));
        }
#pragma unroll
        for (int y = 0; y < kDim / 64; ++y) {  // 8 dims of the lane: four tiles of two dims
          uint32_t h[2][2][4];                 // [pair of keys][even, odd dims][]: a dim's two keys
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t w0 = vw[2 * x][y], w1 = vw[2 * x + 1][y];
            e2m1x8_to_f16((w0 & 0x0f0f0f0fu) | ((w1 << 4) & 0xf0f0f0f0u), h[x][0]);
            e2m1x8_to_f16(((w0 >> 4) & 0x0f0f0f0fu) | (w1 & 0xf0f0f0f0u), h[x][1]);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[x][e >> 2][e & 3] = hmul2_bits(h[x][e >> 2][e & 3], sv[x][kDim == 256 ? y / 2 : 0]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int n = 0; n < kNt; ++n)
              mma_f16_16816(acc[n][4 * y + e], h[0][0][e], h[0][1][e], h[1][0][e], h[1][1][e], pu[n][0], pu[n][1]);
        }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(st));
    }
    if (!ok && lane == 0) give_up(err, a, DEVERR_CONSUMER_WAIT);

    // ---- the warps' outputs of the item, on a common reference
#pragma unroll
    for (int n = 0; n < kNt; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], 4);
        l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], 8);
        l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], 16);
        if (gq == 0) {
          s_m[8 * n + 2 * quad + i][warp] = m[n][i];
          s_l[8 * n + 2 * quad + i][warp] = l[n][i];
        }
      }
    named_bar_sync(kBar, kConsumers);
    float M[kNt][2], L[kNt][2], y[kNt][C::kPer][4];
#pragma unroll
    for (int n = 0; n < kNt; ++n) {
      float f[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = 8 * n + 2 * quad + i;
        float mk[kWarps], lk[kWarps];
#pragma unroll
        for (int k = 0; k < kWarps; k += 4) {
          *reinterpret_cast<float4*>(mk + k) = *reinterpret_cast<const float4*>(&s_m[r][k]);
          *reinterpret_cast<float4*>(lk + k) = *reinterpret_cast<const float4*>(&s_l[r][k]);
        }
        M[n][i] = fmaxf(fmaxf(fmaxf(mk[0], mk[1]), fmaxf(mk[2], mk[3])), fmaxf(fmaxf(mk[4], mk[5]), fmaxf(mk[6], mk[7])));
        L[n][i] = 0.0f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) L[n][i] += lk[k] * (mk[k] == -INFINITY ? 0.0f : ex2(mk[k] - M[n][i]));
        f[i] = m[n][i] == -INFINITY ? 0.0f : ex2(m[n][i] - M[n][i]);
      }
      // each warp adds up its tiles over the warps, in their order, 8 rows at a time
      if (n > 0) named_bar_sync(kBar, kConsumers);  // the first rows have been read
      const bool used = 8 * n + 2 * quad < rows;  // any of the lane's two rows
      if (used)
#pragma unroll
      for (int i = 0; i < C::kTiles; ++i)
        join[(warp * C::kTiles + i) * 32 + lane] =
            make_float4(acc[n][i][0] * f[0], acc[n][i][1] * f[1], acc[n][i][2] * f[0], acc[n][i][3] * f[1]);
      named_bar_sync(kBar, kConsumers);
#pragma unroll
      for (int i = 0; i < C::kPer; ++i) {
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (used && warp * C::kPer + i < C::kTiles) {
#pragma unroll
          for (int k = 0; k < kWarps; ++k) {
            const float4 x = join[(k * C::kTiles + warp * C::kPer + i) * 32 + lane];
            sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
          }
        }
        y[n][i][0] = sum.x, y[n][i][1] = sum.y, y[n][i][2] = sum.z, y[n][i][3] = sum.w;
      }
    }
    const bool has = warp * C::kPer < C::kTiles;
    auto dim_of = [&](int i) { return gq * (kDim / 8) + 2 * (warp * C::kPer + i); };  // the first of the lane's two dims of a tile
    auto out_at = [&](int r) {
      return a.o + (int64_t)(w.q.row0 + tok0 + r / group) * a.o_row + (int64_t)(w.h * group + r % group) * a.o_head;
    };
    auto mend = [&]() {  // the marked rows, a warp each, exactly
      named_bar_sync(kBar, kConsumers);
      const uint32_t bad = s_bad;
      if (bad == 0) return;
      named_bar_sync(kBar, kConsumers);
      if (threadIdx.x == 0) s_bad = 0;
      for (int r = warp; r < rows; r += kWarps) {
        if (!((bad >> r) & 1u)) continue;
        const int tok = tok0 + r / group;
        attend_row_fp4<kBf16, kDim>(c, b, a, w.s, w.q.pos0 + tok, w.q.row0 + tok, w.h * group + r % group, lane, &s_beat);
      }
      named_bar_sync(kBar, kConsumers);
    };
    if (w.whole()) {  // rows whose result is not finite, or without weight, are marked
#pragma unroll
      for (int n = 0; n < kNt; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = 8 * n + 2 * quad + i;
          if (r >= rows || !has) continue;
          const float inv = 1.0f / L[n][i];
          float nan = 0.0f;
          uint16_t* o = out_at(r);
#pragma unroll
          for (int k = 0; k < C::kPer; ++k) {
            const float x = y[n][k][i] * inv * back, z = y[n][k][2 + i] * inv * back;
            nan = fmaf(x, 0.0f, fmaf(z, 0.0f, nan));
            *reinterpret_cast<uint32_t*>(o + dim_of(k)) = pack2<kBf16>(x, z);
          }
          if (nan != 0.0f || !(L[n][i] > 0.0f)) atomicOr(&s_bad, 1u << r);
        }
      mend();
      continue;
    }
    // ---- a piece: into the workspace, joined by the last one to arrive
    const Pieces ps = pieces_of(w, ls);
    {
      float* to = part + (size_t)(2 * blockIdx.x + (w.k0 > 0 ? 0 : 1)) * kPart;
#pragma unroll
      for (int n = 0; n < kNt; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = 8 * n + 2 * quad + i;
          if (r >= rows || !has) continue;
#pragma unroll
          for (int k = 0; k < C::kPer; ++k)
            __stcg(reinterpret_cast<float2*>(to + r * kDim + dim_of(k)), make_float2(y[n][k][i], y[n][k][2 + i]));
          if (warp == 0 && gq == 0) {
            __stcg(to + kTokenRows * kDim + r, M[n][i]);
            __stcg(to + kTokenRows * kDim + kTokenRows + r, L[n][i]);
          }
        }
      named_bar_sync(kBar, kConsumers);
      if (threadIdx.x == 0) s_last = last_piece(counters + ps.first, ps.count);
    }
    named_bar_sync(kBar, kConsumers);
    if (s_last) {
      join_pieces<kBf16, kDim, kWarps>(part, ps.first, ps.count, rows, group, out_at(0), a.o_row, a.o_head,
                                       reinterpret_cast<float*>(join), &s_bad, back);
      mend();
    }
    named_bar_sync(kBar, kConsumers);  // s_last, s_bad and the statistics are free again
  }
}

template <bool kBf16, int kDim, int kNt>
w8a8_status launch(const Fp4Pages& pc, const PagedBatch& pb, const AttnCall& a, void* ws, int sms, cudaStream_t st) {
  using C = Cfg<kDim, kNt>;
  static bool attr_set[64] = {};
  int dev = 0;
  W8A8_CUDA(cudaGetDevice(&dev));
  auto kernel = attn_fp4_tokens_kernel<kBf16, kDim, kNt>;
  if (dev >= 0 && dev < 64 && !attr_set[dev]) {
    W8A8_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
    attr_set[dev] = true;
  }
  CUtensorMap tk, tv;
  const int page = 1 << pc.p.page_shift;
  const uint64_t dims[4] = {(uint64_t)C::kRow, (uint64_t)page, (uint64_t)pc.p.n_kv, (uint64_t)pc.p.n_pages};
  const uint64_t strides[3] = {(uint64_t)pc.p.slot_stride, (uint64_t)pc.p.head_stride, (uint64_t)pc.p.page_stride};
  const uint32_t box[4] = {(uint32_t)C::kRow, (uint32_t)(page < C::kBk ? page : C::kBk), 1, 1};
  const int swizzle = kDim == 256 ? 128 : kDim == 128 ? 64 : 0;
  W8A8_TRY(make_tmap_8(&tk, pc.k, 4, dims, strides, box, swizzle));
  W8A8_TRY(make_tmap_8(&tv, pc.v, 4, dims, strides, box, swizzle));
  const LoadPlan plan{pc.s_slot == C::kSRow && pc.s_page % 16 == 0 && pc.s_head % 16 == 0};
  const int tt = 8 * kNt / (a.n_q / pc.p.n_kv);
  char* base = static_cast<char*>(ws);
  const dim3 grid((unsigned)(sms < kMaxPieces ? sms : kMaxPieces));
  W8A8_CUDA(launch_pdl(kernel, grid, dim3(C::kThreads), (size_t)C::kSmem, st, tk, tv, pc, pb, a, plan, tt,
                       reinterpret_cast<float*>(base + W8A8_WS_RESERVED), reinterpret_cast<unsigned int*>(base),
                       reinterpret_cast<unsigned int*>(base + kErrWordOffset)));
  return W8A8_OK;
}

}  // namespace

w8a8_status launch_attn_fp4_tokens(const Fp4Pages& cache, const PagedBatch& pb, const AttnCall& a, void* ws, int sms,
                                   cudaStream_t st) {
  Fp4Pages pc = cache;
  pc.score = score_significand(a.scale);
  const bool wide = (long long)a.max_new * (a.n_q / pc.p.n_kv) > 8;
  auto of = [&](auto bf) {
    constexpr bool kBf = decltype(bf)::value;
    if (wide)
      return a.dim == 256   ? launch<kBf, 256, 2>(pc, pb, a, ws, sms, st)
             : a.dim == 128 ? launch<kBf, 128, 2>(pc, pb, a, ws, sms, st)
                            : launch<kBf, 64, 2>(pc, pb, a, ws, sms, st);
    return a.dim == 256   ? launch<kBf, 256, 1>(pc, pb, a, ws, sms, st)
           : a.dim == 128 ? launch<kBf, 128, 1>(pc, pb, a, ws, sms, st)
                          : launch<kBf, 64, 1>(pc, pb, a, ws, sms, st);
  };
  return a.bf16 ? of(std::true_type()) : of(std::false_type());
}

}  // namespace w8a8
