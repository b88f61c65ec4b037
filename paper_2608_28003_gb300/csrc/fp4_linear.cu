// The linear in floating point of 4 bits, on the 5th-generation tensor cores' block-scaled products.
//
// y_ti = sx_t sw_i sum_b ux_tb uw_ib sum_j x_tj w_ij: tcgen05.mma kind::mxf4nvf4 takes 64 columns of codes of both operands and the
// units of their blocks (four bytes a row with blocks of 16, two with blocks of 32) and adds the scaled sums into fp32 accumulators in
// tensor memory; the row scales are applied to the accumulators.  One kernel computes D [A's rows, B's rows] = A B^T:
//  * up to 48 tokens (kSwap): A are 128 output channels, B the tokens, so that few tokens do not pad 128 lanes.  The weights
//    are read once, which HBM bounds (or, for a single layer's few megabytes, latency);
//  * more tokens: A are 128 or 256 tokens, B 128 or 192 channels.
// Codes come by TMA, 256 columns (128 bytes, swizzled) a stage; a stage's scales are one contiguous copy per 128 rows in the order
// that they have in memory (w8a8_fp4), from where tcgen05.cp spreads them over tensor memory, 32 rows a column, ahead of the
// products on the same pipe.
// A warp copies, a warp issues, 4 to 16 epilogue warps (a thread per lane of tensor memory) turn accumulators into outputs: through
// swizzled shared memory and TMA stores where D's lanes are tokens, directly where they are channels, which neighbouring lanes
// hold.  Units are walked by one CTA an SM, copies running ahead over unit borders, accumulators in two slots where they fit: not in the
// 256 x 192 tile of long prompts (384 columns of 512, and three stages of copies), whose next products wait until its accumulators are
// read.
// Long rows of few tiles are split over a cluster of up to 8 CTAs, which add up their accumulators through distributed shared memory in
// the order of their ranks: the same bits every time.
//
// Measured, with the quantisation of the tokens ahead of it (2.5 us for few tokens, 5 for 2048): 1 token 1152 -> 6912 6.6 us, 37 tokens
// 6912 -> 1152 8.1 (5.4 and 7.0 in a chain of captured calls, whose starts and ends overlap), both latency (two launches, five to eight
// dependent steps of a microsecond or so); 16 tokens 1152 -> 262144 34.3, 170 MB at 5.0 TB/s and 0.73 of the copy rate; 2048 tokens
// 1152 -> 13824 27 us, 22 of them in the product, where 167 MB of operands from L2, 57 MB of outputs and the accumulators' one slot bound
// it, not the tensor cores (8.4 us at four times the bf16 rate).
//
// Every wait is bounded: on timeout a bit is set in the workspace's error word and in the device's, as the stream's own scratch and a
// captured call's are out of the caller's reach, and the CTA passes its units without waiting.
#include <algorithm>
#include <atomic>

#include "fp4.cuh"
#include "ops.cuh"
#include "tc_common.cuh"
#include "tmap.cuh"

namespace w8a8 {

namespace {

__device__ unsigned int g_gave_up;  // DevErr bits of any call on this device since the last check

constexpr int kKStage = 256;  // columns of a stage

template <int kMT, int kBN, bool kSwap, int kBlock>
struct Cfg {
  static constexpr int kChunks = kKStage / (4 * kBlock);         // 512-byte pieces of scales a stage and 128 rows
  static constexpr int kBBlocks = kBN > 128 ? 2 : 1;             // 128-row blocks of scales that B's rows touch
  static constexpr int kARows = 128 * kMT;
  static constexpr int kCodes = (kARows + kBN) * 128, kScales = (kMT + kBBlocks) * kChunks * 512;
  static constexpr int kStage = (kCodes + kScales + 1023) / 1024 * 1024;
  static constexpr int kHalves = kSwap ? 1 : 2;                  // of a tile's columns, a warp each
  static constexpr int kEpi = 4 * kMT * kHalves;                 // epilogue warps
  static constexpr int kEpiCols = kBN / kHalves;
  static constexpr int kStaging = kSwap ? 0 : kEpi * 2048;       // 32 rows of 64 bytes a warp
  static constexpr int kRoom = 224 * 1024 - kStaging;
  static constexpr int kStages = kRoom / kStage < 8 ? kRoom / kStage : 8;
  static constexpr int kSmem = kStages * kStage + kStaging + 1024;
  static constexpr int kThreads = 64 + 32 * kEpi;
  static constexpr int kAccCols = kMT * kBN, kSfCols = (kMT + kBBlocks) * kChunks * 4;
  static constexpr int kAccs = 2 * kAccCols + 2 * kSfCols <= 512 ? 2 : 1;
  static constexpr int kCols = kAccs * kAccCols + 2 * kSfCols;
  static constexpr int kTmem = kCols <= 32 ? 32 : kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
  static_assert(kCols <= 512 && kStages >= 3, "tensor memory and a ring");
  static_assert(128 * kBN * 4 <= kStages * kStage || kMT == 2, "a cluster's accumulators fit over the ring");
};

struct Fp4Args {
  const uint8_t *a_scales, *b_scales;
  const float *x_scale, *w_scale, *bias;  // row scales: tokens', channels'
  char* y;
  int64_t y_row;  // elements
  unsigned int *err, *gave_up;  // the workspace's word of waits that gave up, the device's
  int M, N, K;              // tokens, channels
  int a_tiles, b_tiles;     // of A's and B's rows
  int a_blocks, b_blocks;   // 128-row blocks of their scales
  int groups;               // 512-byte pieces a block
  int split;                // CTAs of a cluster, parts of k
  int out;                  // W8A8_TYPE_*
  int tma_out;              // y by TMA stores: 1 but for a row's last columns, 2 those too
};

// Instruction descriptor of kind::mxf4nvf4: both operands e2m1 (1 at bits 7 and 10), N >> 3 at bit 17, scales e4m3 (0) or
// e8m0 (1) at bit 23, M >> 7 at bit 27; with blocks of 32, which half of a row's word holds the units (0 or 2) at bits 4 (B) and
// 29 (A).  64 columns (bit 31 clear).
template <int kBlock>
__device__ constexpr uint32_t idesc_fp4(int n, int half) {
  return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (kBlock == 32 ? 1u << 23 : 0u) | (1u << 27) |
         (kBlock == 32 ? (uint32_t)half << 5 | (uint32_t)half << 30 : 0u);
}
template <int kBlock>
__device__ __forceinline__ void tc_mma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                           uint32_t accumulate) {
  if constexpr (kBlock == 16)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%5], [%6], p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb)
        : "memory");
}
// 512 bytes of scales, 32 rows of 16 bytes as they lie, to 4 columns of tensor memory, the same in all four lane quarters.
__device__ __forceinline__ void tc_copy_scales(uint32_t tmem, uint32_t smem) {
  // no swizzle: 8-row groups of 128 bytes (stride byte offset), descriptor version 1
  const uint64_t d = (uint64_t)((smem & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n" ::"r"(tmem), "l"(d) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n"
      "tcgen05.wait::ld.sync.aligned;\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tma_store_2d(const void* tmap, uint32_t src, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];\n" ::"l"(
                   reinterpret_cast<uint64_t>(tmap)),
               "r"(src), "r"(c0), "r"(c1)
               : "memory");
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(at) : "r"(addr), "r"(rank));
  return at;
}
__device__ __forceinline__ float ld_peer(uint32_t at) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};\n" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void give_up(const Fp4Args& a, unsigned int bits) {
  atomicOr(a.err, bits);
  atomicOr(a.gave_up, bits);
}
__device__ __forceinline__ void put_one(const Fp4Args& a, int64_t at, float v) {
  if (a.out == W8A8_TYPE_F32)
    reinterpret_cast<float*>(a.y)[at] = v;
  else
    reinterpret_cast<uint16_t*>(a.y)[at] = (uint16_t)(a.out == W8A8_TYPE_BF16 ? pack2<true>(v, 0.0f) : pack2<false>(v, 0.0f));
}

// This CTA's share of the columns (a row a thread), added up over its cluster's accumulators in the order of the ranks, to y.  kFly loads of
// distributed shared memory are in flight: a column at a time, 64 of 6912 -> 1152 at 37 tokens in parts of two took 19.5 us, more than
// whole ones (15.2).
constexpr int kFly = 32;
template <int kS, int kBN, bool kSwap, int kBlock, int kHalves>
__device__ __forceinline__ void add_up(const Fp4Args& a, uint32_t ring, int rank, int tile, int warp, int lane, const float* s_scale,
                                       const float* s_bias) {
  constexpr int kShare = kBN / kS / kHalves, kC = kFly / kS < kShare ? kFly / kS : kShare;  // columns of a warp, together
  static_assert(kShare >= 1 && kShare % kC == 0, "whole groups of columns");
  const int quarter = warp & 3, half = (warp - 2) >> 2, at = tile % a.a_tiles, b0 = tile / a.a_tiles * kBN;
  const int arow = at * 128 + 32 * quarter + lane, b_end = kSwap ? a.M : a.N, a_end = kSwap ? a.N : a.M;
  const float mine = kBlock == 16 && arow < a_end ? (kSwap ? a.w_scale : a.x_scale)[arow] : 1.0f;
  const float mine_bias = kSwap && a.bias && arow < a_end ? a.bias[arow] : 0.0f;
  uint32_t from[kS];
#pragma unroll
  for (int r = 0; r < kS; ++r) from[r] = peer_addr(ring + (uint32_t)((32 * quarter + lane) * 4), (uint32_t)r);
  const int c_end = (rank * kHalves + half + 1) * kShare;
  for (int c = c_end - kShare; c < c_end && b0 + c < b_end; c += kC) {
    float p[kS][kC];
#pragma unroll
    for (int r = 0; r < kS; ++r)
#pragma unroll
      for (int j = 0; j < kC; ++j) p[r][j] = ld_peer(from[r] + (uint32_t)((c + j) * 512));
    float v[kC];
#pragma unroll
    for (int j = 0; j < kC; ++j) {
      v[j] = p[0][j];
#pragma unroll
      for (int r = 1; r < kS; ++r) v[j] += p[r][j];
      if constexpr (kBlock == 16) v[j] = kSwap ? v[j] * mine * s_scale[c + j] : v[j] * s_scale[c + j] * mine;
      v[j] += kSwap ? mine_bias : s_bias[c + j];
    }
    if (arow >= a_end) continue;
    if constexpr (!kSwap && kC % 4 == 0) {
      if (a.tma_out && b0 + c + kC <= b_end) {  // rows 16-byte aligned, so are four columns
        char* to = a.y + ((int64_t)arow * a.y_row + b0 + c) * (a.out == W8A8_TYPE_F32 ? 4 : 2);
#pragma unroll
        for (int j = 0; j < kC; j += 4) {
          if (a.out == W8A8_TYPE_F32)
            *reinterpret_cast<float4*>(to + 4 * j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
          else if (a.out == W8A8_TYPE_BF16)
            *reinterpret_cast<uint2*>(to + 2 * j) = make_uint2(pack2<true>(v[j], v[j + 1]), pack2<true>(v[j + 2], v[j + 3]));
          else
            *reinterpret_cast<uint2*>(to + 2 * j) = make_uint2(pack2<false>(v[j], v[j + 1]), pack2<false>(v[j + 2], v[j + 3]));
        }
        continue;
      }
    }
#pragma unroll
    for (int j = 0; j < kC; ++j)
      if (b0 + c + j < b_end) put_one(a, kSwap ? (int64_t)(b0 + c + j) * a.y_row + arow : (int64_t)arow * a.y_row + b0 + c + j, v[j]);
  }
}

template <int kMT, int kBN, bool kSwap, int kBlock>
__global__ void __launch_bounds__(Cfg<kMT, kBN, kSwap, kBlock>::kThreads, 1)
    fp4_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                    const __grid_constant__ CUtensorMap tmY, Fp4Args a) {
  using C = Cfg<kMT, kBN, kSwap, kBlock>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ uint64_t bars[2 * C::kStages + 4];
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(16) float s_scale[kBN], s_bias[kBN];  // of B's rows
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u, staging = ring + C::kStages * C::kStage;
  const uint32_t bar0 = smem_u32(bars);
  auto full = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  auto empty = [&](int i) { return bar0 + 8u * (uint32_t)(C::kStages + i); };
  auto acc_full = [&](int i) { return bar0 + 8u * (uint32_t)(2 * C::kStages + i); };
  auto acc_free = [&](int i) { return bar0 + 8u * (uint32_t)(2 * C::kStages + 2 + i); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(acc_full(i), 1);
      mbar_init(acc_free(i), 32 * C::kEpi);
    }
    fence_mbar_init();
    prefetch_tmap(&tmA);
    prefetch_tmap(&tmB);
    if (!kSwap) prefetch_tmap(&tmY);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_slot)),
                 "n"(C::kTmem)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();  // after the allocation: a kernel behind this one that wants tensor memory too comes second
  const uint32_t tmem = tmem_slot;

  const int split = a.split, rank = split > 1 ? (int)(blockIdx.x % (unsigned)split) : 0;
  const int tiles = a.a_tiles * a.b_tiles, first = (int)(blockIdx.x / (unsigned)split), step = (int)(gridDim.x / (unsigned)split);
  const int all = (a.K + kKStage - 1) / kKStage;
  const int s0 = all * rank / split, s1 = all * (rank + 1) / split;  // this CTA's stages of k
  bool ok = true;

  if (warp == 0) {
    // -------------------------------------------------------------------------- copies
    int g = 0;
    // codes and scales of one operand's rows for a stage
    auto bytes_of = [&](int s, int block0, int blocks, int of) {
      const int pieces = min(C::kChunks, a.groups - s * C::kChunks);
      return (uint32_t)(min(blocks, of - block0) * pieces * 512);
    };
    auto load = [&](bool is_b, int tile, int s, int st) {
      const uint32_t at = ring + (uint32_t)(st * C::kStage);
      const int rows = is_b ? kBN : C::kARows, r0 = tile * rows, block0 = r0 >> 7;
      const int blocks = is_b ? C::kBBlocks : kMT, of = is_b ? a.b_blocks : a.a_blocks;
      const int pieces = min(C::kChunks, a.groups - s * C::kChunks);
      tma_load_2d(at + (is_b ? C::kARows * 128 : 0), is_b ? &tmB : &tmA, s * 128, r0, full(st));
      for (int i = 0; i < blocks && block0 + i < of; ++i)
        bulk_g2s(at + (uint32_t)(C::kCodes + ((is_b ? kMT : 0) + i) * C::kChunks * 512),
                 (is_b ? a.b_scales : a.a_scales) + ((size_t)(block0 + i) * a.groups + (size_t)s * C::kChunks) * 512,
                 (uint32_t)pieces * 512u, full(st));
    };
    // The weights do not wait for the launch before this one, the tokens' codes do: the first stages' weights are on their way.
    constexpr bool kWeightsA = kSwap;
    int ahead = 0;
    if (first < tiles) {
      const int at = first % a.a_tiles, bt = first / a.a_tiles;
      ahead = min(C::kStages, s1 - s0);
      if (elect_one())
        for (int i = 0; i < ahead; ++i) {
          const int s = s0 + i;
          mbar_arrive_expect_tx(full(i), (uint32_t)C::kCodes + bytes_of(s, at * C::kARows >> 7, kMT, a.a_blocks) +
                                             bytes_of(s, bt * kBN >> 7, C::kBBlocks, a.b_blocks));
          load(!kWeightsA, kWeightsA ? at : bt, s, i);
        }
      __syncwarp();
    }
    pdl_wait();
    for (int u = first; ok && u < tiles; u += step) {
      const int at = u % a.a_tiles, bt = u / a.a_tiles;
      for (int s = s0; s < s1; ++s, ++g) {
        const int st = g % C::kStages;
        if (g >= C::kStages && !mbar_wait_warp(empty(st), (uint32_t)(g / C::kStages - 1) & 1u, kWaitBudgetCycles)) {
          ok = false;
          break;
        }
        if (elect_one()) {
          if (g >= ahead) {
            mbar_arrive_expect_tx(full(st), (uint32_t)C::kCodes + bytes_of(s, at * C::kARows >> 7, kMT, a.a_blocks) +
                                                bytes_of(s, bt * kBN >> 7, C::kBBlocks, a.b_blocks));
            load(!kWeightsA, kWeightsA ? at : bt, s, st);
          }
          load(kWeightsA, kWeightsA ? bt : at, s, st);
        }
        __syncwarp();
      }
    }
    if (!ok && lane == 0) give_up(a, DEVERR_PRODUCER_WAIT);
    for (int i = max(0, g - C::kStages); i < g; ++i)  // the last copies land before the CTA may end
      if (!mbar_wait_warp(full(i % C::kStages), (uint32_t)(i / C::kStages) & 1u, kWaitBudgetCycles) && lane == 0)
        give_up(a, DEVERR_DRAIN_WAIT);
  } else if (warp == 1) {
    // -------------------------------------------------------------------------- products
    int g = 0, n = 0;
    for (int u = first; ok && u < tiles; u += step, ++n) {
      const int slot = n % C::kAccs, bt = u / a.a_tiles;
      const uint32_t shift = (uint32_t)((bt * kBN & 127) >> 5);  // B's first row within its block of scales
      if (n >= C::kAccs && !mbar_wait_warp(acc_free(slot), (uint32_t)(n / C::kAccs - 1) & 1u, kWaitBudgetCycles)) {
        ok = false;
        break;
      }
      tc_fence_after();
      for (int s = s0; s < s1; ++s, ++g) {
        const int st = g % C::kStages;
        if (!mbar_wait_warp(full(st), (uint32_t)(g / C::kStages) & 1u, kWaitBudgetCycles)) {
          ok = false;
          break;
        }
        tc_fence_after();
        if (elect_one()) {
          const uint32_t at = ring + (uint32_t)(st * C::kStage);
          const uint32_t sf = tmem + (uint32_t)(C::kAccs * C::kAccCols + (g & 1) * C::kSfCols);
          const int pieces = min(C::kChunks, a.groups - s * C::kChunks);
          for (int j = 0; j < pieces; ++j)
#pragma unroll
            for (int i = 0; i < kMT + C::kBBlocks; ++i)
              tc_copy_scales(sf + 4u * (uint32_t)(i < kMT ? i * C::kChunks + j : kMT * C::kChunks + j * C::kBBlocks + i - kMT),
                             at + (uint32_t)(C::kCodes + (i * C::kChunks + j) * 512));
          const uint64_t da = sdesc_swz(at), db = sdesc_swz(at + C::kARows * 128);
          const int steps = min(kKStage / 64, (a.K - s * kKStage + 63) / 64);
          for (int k = 0; k < steps; ++k) {
            const int piece = kBlock == 16 ? k : k >> 1, half = kBlock == 16 ? 0 : k & 1;
            const uint32_t idesc = half ? idesc_fp4<kBlock>(kBN, 1) : idesc_fp4<kBlock>(kBN, 0);
            const uint32_t sfb = sf + (uint32_t)(4 * (kMT * C::kChunks + piece * C::kBBlocks)) + shift;
#pragma unroll
            for (int i = 0; i < kMT; ++i)
              tc_mma_fp4<kBlock>(tmem + (uint32_t)(slot * C::kAccCols + i * kBN), da + (uint64_t)(i * (128 * 128 >> 4) + 2 * k),
                                 db + (uint64_t)(2 * k), idesc, sf + (uint32_t)(4 * (i * C::kChunks + piece)), sfb,
                                 s > s0 || k > 0);
          }
          tc_commit(empty(st));
          if (s == s1 - 1) tc_commit(acc_full(slot));
        }
        __syncwarp();
      }
    }
    if (!ok && lane == 0) give_up(a, DEVERR_PRODUCER_WAIT);
    // every product issued ends before the accumulators go: the last stage's commit says so
    if (g > 0 && !mbar_wait_warp(empty((g - 1) % C::kStages), (uint32_t)((g - 1) / C::kStages) & 1u, kWaitBudgetCycles) &&
        lane == 0)
      give_up(a, DEVERR_DRAIN_WAIT);
  } else {
    // -------------------------------------------------------------------------- outputs
    pdl_wait();
    const int e = warp - 2, quarter = warp & 3, mt = (e >> 2) / C::kHalves, half = (e >> 2) % C::kHalves, tid = threadIdx.x - 64;
    const int col0 = half * C::kEpiCols;
    const uint32_t lanes = tmem + ((uint32_t)(32 * quarter) << 16);
    constexpr int kT = 32 * C::kEpi;
    int n = 0;
    for (int u = first; u < tiles; u += step, ++n) {
      const int slot = n % C::kAccs, at = u % a.a_tiles, bt = u / a.a_tiles;
      const int arow = at * C::kARows + 128 * mt + 32 * quarter + lane, b0 = bt * kBN;  // this thread's row of A
      // scales and bias of B's rows in shared memory, of A's row here
      const float* bs = kSwap ? a.x_scale : a.w_scale;
      const int b_end = kSwap ? a.M : a.N, a_end = kSwap ? a.N : a.M;
      named_bar_sync(1, kT);  // the tile before has read them
      for (int i = tid; i < kBN; i += kT) {
        s_scale[i] = kBlock == 16 && b0 + i < b_end ? bs[b0 + i] : 1.0f;
        s_bias[i] = !kSwap && a.bias && b0 + i < b_end ? a.bias[b0 + i] : 0.0f;
      }
      const float mine = kBlock == 16 && arow < a_end ? (kSwap ? a.w_scale : a.x_scale)[arow] : 1.0f;
      const float mine_bias = kSwap && a.bias && arow < a_end ? a.bias[arow] : 0.0f;
      named_bar_sync(1, kT);
      // the channel's scale first: the token's is a power of two
      auto value = [&](float acc, int c) {
        float v = acc;
        if constexpr (kBlock == 16) v = kSwap ? v * mine * s_scale[c] : v * s_scale[c] * mine;
        return v + (kSwap ? mine_bias : s_bias[c]);
      };
      if (ok && !mbar_wait_warp(acc_full(slot), (uint32_t)(n / C::kAccs) & 1u, kWaitBudgetCycles)) ok = false;
      tc_fence_after();
      const uint32_t acc = lanes + (uint32_t)(slot * C::kAccCols + mt * kBN);
      if (split > 1) {  // (one unit a CTA; the accumulators leave over the ring, which every product has read)
        if constexpr (kMT == 1) {
          if (ok)
            for (int c = col0; c < col0 + C::kEpiCols; c += 8) {
              uint32_t r[8];
              tmem_ld8(acc + c, r);
#pragma unroll
              for (int j = 0; j < 8; ++j)
                asm volatile("st.shared.u32 [%0], %1;\n" ::"r"(ring + (uint32_t)(((c + j) * 128 + 32 * quarter + lane) * 4)),
                             "r"(r[j])
                             : "memory");
            }
        }
      } else if constexpr (kSwap) {
        for (int c = 0; ok && c < kBN && b0 + c < b_end; c += 8) {
          uint32_t r[8];
          tmem_ld8(acc + c, r);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (b0 + c + j < b_end && arow < a_end)
              put_one(a, (int64_t)(b0 + c + j) * a.y_row + arow, value(__uint_as_float(r[j]), c + j));
        }
        tc_fence_before();
        mbar_arrive(acc_free(slot));
      } else {
        // 32 columns at a time, which leave in groups of 64 bytes of a row: all of them, or 16 of fp32.  16-bit outputs are all held
        // first, so that the accumulators are free before the first store: 1.8 + 0.7 us a tile were theirs otherwise
        const uint32_t stage = staging + (uint32_t)(e * 2048), to = stage + (uint32_t)(lane * 64), swz = (uint32_t)((lane >> 1) & 3);
        const bool f32 = a.out == W8A8_TYPE_F32;
        const int row0 = at * C::kARows + 128 * mt + 32 * quarter;
        const f32x2 mine2 = f2_pack(mine, mine);
        auto read = [&](int c, uint32_t (&r)[32]) {
          tmem_ld32(acc + c, r);
          // pairs of columns: the channel's scale, then the token's (a power of two, so that the sum with the bias rounds as two steps)
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            const float4 sc = kBlock == 16 ? *reinterpret_cast<const float4*>(&s_scale[c + j]) : make_float4(1.f, 1.f, 1.f, 1.f);
            const float4 bi = a.bias ? *reinterpret_cast<const float4*>(&s_bias[c + j]) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              f32x2 v = f2_pack(__uint_as_float(r[j + 2 * q]), __uint_as_float(r[j + 2 * q + 1]));
              const f32x2 b2 = q ? f2_pack(bi.z, bi.w) : f2_pack(bi.x, bi.y);
              if constexpr (kBlock == 16)
                v = f2_fma(f2_fma(v, q ? f2_pack(sc.z, sc.w) : f2_pack(sc.x, sc.y), 0ull), mine2, b2);
              else
                v = f2_add(v, b2);
              float lo, hi;
              f2_unpack(v, lo, hi);
              r[j + 2 * q] = __float_as_uint(lo);
              r[j + 2 * q + 1] = __float_as_uint(hi);
            }
          }
        };
        // 64 bytes of each of the warp's rows, from column c0 on
        auto put_group = [&](int c0, uint32_t (&w)[16]) {
          if (c0 >= b_end || row0 >= a_end) return;
          // a store is of whole 16 bytes, those that cross the row's end too: columns beside y are not its to write
          const bool by_tma = a.tma_out > (c0 + (f32 ? 16 : 32) > b_end ? 1 : 0);
          if (a.tma_out) {
            if (elect_one()) asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory");
            __syncwarp();
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) sts128(to + ((j ^ swz) << 4), w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
          if (by_tma) {
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            __syncwarp();
            if (elect_one()) {
              tma_store_2d(&tmY, stage, c0, row0);
              asm volatile("cp.async.bulk.commit_group;\n" ::: "memory");
            }
            __syncwarp();
            return;
          }
          __syncwarp();  // rows that begin or end anywhere: a row at a time
          const int rows = min(32, a_end - row0), here = min(f32 ? 16 : 32, b_end - c0);
          for (int q = 0; q < rows; ++q)
            if (lane < here) {
              const uint32_t byte = (uint32_t)(lane * (f32 ? 4 : 2));
              const uint32_t from = stage + (uint32_t)(q * 64) + ((((byte >> 4) ^ (uint32_t)((q >> 1) & 3)) << 4) | (byte & 15u));
              const int64_t at_y = (int64_t)(row0 + q) * a.y_row + c0 + lane;
              if (f32) {
                float v;
                asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(v) : "r"(from) : "memory");
                reinterpret_cast<float*>(a.y)[at_y] = v;
              } else {
                uint16_t v;
                asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(v) : "r"(from) : "memory");
                reinterpret_cast<uint16_t*>(a.y)[at_y] = v;
              }
            }
          __syncwarp();
        };
        if (f32) {
          for (int c = col0; ok && c < col0 + C::kEpiCols; c += 32) {
            uint32_t r[32];
            read(c, r);
#pragma unroll
            for (int h = 0; h < 2; ++h) put_group(b0 + c + 16 * h, *reinterpret_cast<uint32_t(*)[16]>(r + 16 * h));
          }
          tc_fence_before();
          mbar_arrive(acc_free(slot));
        } else {
          uint32_t w[C::kEpiCols / 32][16];
#pragma unroll
          for (int i = 0; i < C::kEpiCols / 32; ++i) {
            uint32_t r[32];
            read(col0 + 32 * i, r);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float lo = __uint_as_float(r[2 * j]), hi = __uint_as_float(r[2 * j + 1]);
              w[i][j] = a.out == W8A8_TYPE_BF16 ? pack2<true>(lo, hi) : pack2<false>(lo, hi);
            }
          }
          tc_fence_before();
          mbar_arrive(acc_free(slot));
#pragma unroll
          for (int i = 0; i < C::kEpiCols / 32; ++i)
            if (ok) put_group(b0 + col0 + 32 * i, w[i]);
        }
      }
    }
    if (!kSwap && a.tma_out && elect_one()) asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory");
    if (!ok && lane == 0) give_up(a, DEVERR_CONSUMER_WAIT);
    __syncwarp();
  }
  if constexpr (kMT == 1) {
    if (split > 1) {  // each CTA adds up a share of the columns of all of its cluster's accumulators
      cluster_sync_all();
      if (warp >= 2 && first < tiles) {
        if (split == 2)
          add_up<2, kBN, kSwap, kBlock, C::kHalves>(a, ring, rank, first, warp, lane, s_scale, s_bias);
        else if (split == 4)
          add_up<4, kBN, kSwap, kBlock, C::kHalves>(a, ring, rank, first, warp, lane, s_scale, s_bias);
        else
          add_up<8, kBN, kSwap, kBlock, C::kHalves>(a, ring, rank, first, warp, lane, s_scale, s_bias);
      }
      cluster_sync_all();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "n"(C::kTmem) : "memory");
  }
}

cudaLaunchConfig_t config(unsigned grid, int threads, int smem, int split, cudaStream_t st, cudaLaunchAttribute (&attr)[2]) {
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = split > 1 ? 2 : 1;
  return cfg;
}

// least: stages from which on k is divided.
template <int kMT, int kBN, bool kSwap, int kBlock>
w8a8_status launch(const w8a8_fp4& x, const w8a8_fp4& w, Fp4Args a, int least, int sms, cudaStream_t st) {
  using C = Cfg<kMT, kBN, kSwap, kBlock>;
  static std::atomic<bool> known[64] = {};  // whether the attribute is set and at_once filled in, for threads to see in this order
  static int at_once[64][4] = {};           // clusters of 1, 2, 4, 8 that the GPU holds: a call's sums are split by it
  int dev = 0;
  W8A8_CUDA(cudaGetDevice(&dev));
  W8A8_CHECK_ARG(dev >= 0 && dev < 64, W8A8_ERR_CUDA, "w8a8_fp4_linear: device %d", dev);
  auto kernel = fp4_gemm_kernel<kMT, kBN, kSwap, kBlock>;
  cudaLaunchAttribute attr[2];
  if (!known[dev].load(std::memory_order_acquire)) {
    W8A8_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
    for (int i = 1; i < 4 && kMT == 1; ++i) {
      const cudaLaunchConfig_t one = config(1u << i, C::kThreads, C::kSmem, 1 << i, st, attr);
      W8A8_CUDA(cudaOccupancyMaxActiveClusters(&at_once[dev][i], kernel, &one));
    }
    known[dev].store(true, std::memory_order_release);
  }
  const w8a8_fp4 &fa = kSwap ? w : x, &fb = kSwap ? x : w;
  a.a_scales = fa.scales;
  a.b_scales = fb.scales;
  a.a_tiles = (fa.rows + C::kARows - 1) / C::kARows;
  a.b_tiles = (fb.rows + kBN - 1) / kBN;
  a.a_blocks = (fa.rows + 127) / 128;
  a.b_blocks = (fb.rows + 127) / 128;
  const int64_t tiles = (int64_t)a.a_tiles * a.b_tiles;
  const int stages = (a.K + kKStage - 1) / kKStage;
  int split = 1;
  for (int i = 1; i < 4 && kMT == 1; ++i)
    if (tiles <= at_once[dev][i] && stages >= std::max(2 << i, least)) split = 1 << i;
  a.split = split;
  CUtensorMap ta, tb, ty;
  const uint64_t bytes = (uint64_t)a.K / 2;
  W8A8_TRY(make_tmap_2d(&ta, fa.codes, 1, bytes, (uint64_t)fa.rows, bytes, 128, C::kARows));
  W8A8_TRY(make_tmap_2d(&tb, fb.codes, 1, bytes, (uint64_t)fb.rows, bytes, 128, kBN));
  const int e = type_bytes(a.out);
  a.tma_out = kSwap || a.y_row * e % 16 != 0 ? 0 : (int64_t)a.N * e % 16 != 0 ? 1 : 2;
  ty = ta;
  if (a.tma_out)
    W8A8_TRY(make_tmap_2d(&ty, a.y, e, (uint64_t)a.N, (uint64_t)a.M, (uint64_t)a.y_row * e, 64 / e, 32, 64));
  const unsigned grid = (unsigned)(split > 1 ? tiles * split : std::min<int64_t>(tiles, sms));
  const cudaLaunchConfig_t cfg = config(grid, C::kThreads, C::kSmem, split, st, attr);
  W8A8_CUDA(cudaLaunchKernelEx(&cfg, kernel, ta, tb, ty, a));
  return W8A8_OK;
}

// How a call is cut up.
// Up to 48 tokens: as many columns of tokens as there are, 128 channels a tile (1152 -> 262144 at 16 tokens: 34.3 us, 55 with the tiles
// for more; at 37: 42.4 and 55.3).  From there on those (64 tokens: 50.2, 53.8 with channels as the lanes, whose stores are 16 bits each;
// 128: 43.2 and 90.8).
// More: 256 x 192, whose operands are read less often, or 128 x 128, whichever has its waves over the SMs done first, at 2.4 times
// the time for a larger tile (2048 tokens 1152 -> 13824: 27.2 and 32.2; 8192 tokens 1152 -> 1152: 24.0 and 22.4).
// Parts of k: while a CTA has two stages (6912 -> 1152 at 1 token: 14.0, 10.5, 7.9, 7.0 us in 1, 2, 4, 8 parts; 2304 -> 1152 at 16: 8.4, 7.5,
// 6.8 in 1, 2, 4) and the GPU holds all clusters at once, which are as many as its groups of SMs have room for, not its SMs divided by
// the parts (6912 -> 2048 at 16 tokens, 16 tiles, in 8 parts 12.4 us, 8.6 in 4; 4096 -> 4608 and 4736, 36 and 37 tiles, in 4: 8.6 and
// 12.9); tiles of 128 tokens, whose sums are 64 KB a part, from 16 stages on (1152 -> 6912, 5 stages, at 128 tokens: 7.7 whole, 9.9 in two).
template <int kBlock>
w8a8_status run_gemm(const w8a8_fp4& x, const w8a8_fp4& w, const Fp4Args& a, int sms, cudaStream_t st) {
  if (a.M <= 16) return launch<1, 16, true, kBlock>(x, w, a, 0, sms, st);
  if (a.M <= 32) return launch<1, 32, true, kBlock>(x, w, a, 0, sms, st);
  if (a.M <= 48) return launch<1, 64, true, kBlock>(x, w, a, 0, sms, st);
  auto waves = [&](int64_t tiles) { return (tiles + sms - 1) / sms; };
  const int64_t big = (int64_t)((a.M + 255) / 256) * (((int64_t)a.N + 191) / 192),
                small = (int64_t)((a.M + 127) / 128) * ((a.N + 127) / 128);
  if (12 * waves(big) <= 5 * waves(small)) return launch<2, 192, false, kBlock>(x, w, a, 0, sms, st);
  return launch<1, 128, false, kBlock>(x, w, a, 16, sms, st);
}

w8a8_status gave_up_word(unsigned int** word) {
  static unsigned int* known[64] = {};
  return device_word(&g_gave_up, known, word);
}

struct LinearFp4Ws {
  size_t codes, scales, row_scale, total;
};
LinearFp4Ws linear_fp4_ws(int M, int K, int block) {
  LinearFp4Ws w;
  w.codes = W8A8_WS_RESERVED;
  w.scales = w.codes + round_up((size_t)M * (K / 2), 1024);
  w.row_scale = w.scales + round_up((size_t)M, 128) / 128 * (size_t)fp4_groups(K, block) * 512;
  w.total = w.row_scale + round_up((size_t)M * 4, 1024);
  return w;
}

}  // namespace

}  // namespace w8a8

using namespace w8a8;

extern "C" w8a8_status w8a8_fp4_linear_workspace_size(int M, int N, int K, int block, size_t* bytes) {
  const char* who = "w8a8_fp4_linear_workspace_size";
  W8A8_CHECK_ARG(bytes != nullptr && (block == 16 || block == 32), W8A8_ERR_INVALID_ARG, "%s: null pointer, or block %d", who,
                 block);
  W8A8_CHECK_ARG(M >= 0 && M <= kMaxFp4Rows && N >= 0 && N <= kMaxFp4Rows && K > 0 && K % 32 == 0 && K <= W8A8_MAX_K,
                 W8A8_ERR_SHAPE, "%s: M=%d N=%d K=%d", who, M, N, K);
  *bytes = linear_fp4_ws(M, K, block).total;
  return W8A8_OK;
}

extern "C" w8a8_status w8a8_fp4_linear(const w8a8_fp4* w, int dtype, const void* X, int64_t x_row, int M, const float* bias,
                                       int out_dtype, void* Y, int64_t y_row, void* workspace, size_t ws_bytes, void* stream) {
  const char* who = "w8a8_fp4_linear";
  W8A8_TRY(check_fp4(who, w));
  W8A8_CHECK_ARG(M >= 0, W8A8_ERR_INVALID_ARG, "%s: M=%d is negative", who, M);
  W8A8_CHECK_ARG(M <= kMaxFp4Rows, W8A8_ERR_SHAPE, "%s: M=%d is too large", who, M);
  W8A8_CHECK_ARG(dtype >= W8A8_TYPE_BF16 && dtype <= W8A8_TYPE_F32 && out_dtype >= W8A8_TYPE_BF16 &&
                     out_dtype <= W8A8_TYPE_F32,
                 W8A8_ERR_INVALID_ARG, "%s: types %d, %d", who, dtype, out_dtype);
  W8A8_CHECK_ARG(x_row >= 0 && x_row <= (1ll << 40) && x_row * type_bytes(dtype) % 16 == 0, W8A8_ERR_SHAPE,
                 "%s: X's row stride of %lld elements is not a multiple of 16 bytes", who, (long long)x_row);
  W8A8_CHECK_ARG((M <= 1 || y_row >= w->rows) && y_row >= 0 && y_row <= (1ll << 40), W8A8_ERR_SHAPE,
                 "%s: Y's row stride %lld is below N=%d", who, (long long)y_row, w->rows);
  if (M == 0 || w->rows == 0) return W8A8_OK;
  W8A8_CHECK_ARG(X && Y, W8A8_ERR_INVALID_ARG, "%s: null X or Y", who);
  W8A8_CHECK_ARG(aligned16(X) && aligned16(Y) && aligned16(bias), W8A8_ERR_ALIGN, "%s: X, Y and bias must be 16-byte aligned",
                 who);
  W8A8_CHECK_ARG(X != Y, W8A8_ERR_INVALID_ARG, "%s: Y must not be X", who);
  DevInfo d;
  W8A8_TRY(dev_info(&d));
  const int N = w->rows, K = w->k;
  const LinearFp4Ws L = linear_fp4_ws(M, K, w->block);
  W8A8_CHECK_ARG(workspace != nullptr && ws_bytes >= L.total, W8A8_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who,
                 workspace ? ws_bytes : 0, L.total);
  W8A8_CHECK_ARG(aligned16(workspace), W8A8_ERR_ALIGN, "%s: workspace must be 16-byte aligned", who);
  char* base = static_cast<char*>(workspace);
  w8a8_fp4 x{M, K, w->block, reinterpret_cast<uint8_t*>(base + L.codes), reinterpret_cast<uint8_t*>(base + L.scales),
             reinterpret_cast<float*>(base + L.row_scale)};
  cudaStream_t st = as_stream(stream);
  Fp4Args a{};
  a.x_scale = x.row_scale;
  a.w_scale = w->row_scale;
  a.bias = bias;
  a.y = static_cast<char*>(Y);
  a.y_row = M > 1 ? y_row : round_up((size_t)N, 8);  // one row has no stride
  a.err = reinterpret_cast<unsigned int*>(base + kErrWordOffset);
  W8A8_TRY(gave_up_word(&a.gave_up));
  W8A8_TRY(launch_fp4_quantize(dtype, X, x_row, x, false, st));
  a.M = M;
  a.N = N;
  a.K = K;
  a.groups = fp4_groups(K, w->block);
  a.out = out_dtype;
  return w->block == 16 ? run_gemm<16>(x, *w, a, d.sms, st) : run_gemm<32>(x, *w, a, d.sms, st);
}

extern "C" w8a8_status w8a8_fp4_linear_error_word(uint32_t** word) {
  W8A8_CHECK_ARG(word != nullptr, W8A8_ERR_INVALID_ARG, "w8a8_fp4_linear_error_word: null argument");
  W8A8_TRY(check_device());
  return gave_up_word(word);
}

extern "C" w8a8_status w8a8_fp4_linear_check(void* stream) {
  unsigned int* word = nullptr;
  W8A8_TRY(w8a8_fp4_linear_error_word(&word));
  return take_error_word(word, as_stream(stream));
}
