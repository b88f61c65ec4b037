// Attention of a ragged batch over a paged cache.
#include <cmath>

#include "attn_common.cuh"
#include "ops.cuh"
#include "paged.cuh"

namespace w8a8 {

namespace {

// One row's attention by one warp, key by key in the order of the formula: NaN and infinities travel as they do
// in it, and nothing outside the row's range is read.  Lane l scores key j0 + l, then holds dims l, l + 32, ...
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

template <bool kBf16, int kDim>
__global__ void __launch_bounds__(128) attn_rows_kernel(PagedCache c, PagedBatch b, AttnCall a) {
  pdl_wait();
  pdl_trigger();
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int row = (int)(w / a.n_q), head = (int)(w % a.n_q);
  if (row >= b.n_rows) return;
  const int s = seq_of_row(b, row);
  const SeqShape q = seq_shape(b, s, c.page_shift);
  if (row < q.row0 || row >= q.row0 + q.rows) return;
  attend_row<kBf16, kDim>(c, b, a, s, q.pos0 + row - q.row0, row, head, threadIdx.x & 31);
}

}  // namespace

size_t paged_attention_ws(int, int, int, int) { return W8A8_WS_RESERVED; }

w8a8_status launch_paged_attention(const PagedCache& pc, const PagedBatch& pb, const AttnCall& a, void*, int,
                                   cudaStream_t st) {
  const dim3 grid((unsigned)(((int64_t)pb.n_rows * a.n_q + 3) / 4));
  auto go = [&](auto kernel) { return launch_pdl(kernel, grid, dim3(128), 0, st, pc, pb, a); };
  W8A8_CUDA(a.bf16 ? (a.dim == 256   ? go(attn_rows_kernel<true, 256>)
                      : a.dim == 128 ? go(attn_rows_kernel<true, 128>)
                                     : go(attn_rows_kernel<true, 64>))
                   : (a.dim == 256   ? go(attn_rows_kernel<false, 256>)
                      : a.dim == 128 ? go(attn_rows_kernel<false, 128>)
                                     : go(attn_rows_kernel<false, 64>)));
  return W8A8_OK;
}

namespace {

w8a8_status check_heads(const char* who, const w8a8_paged_cache* c, int n_q) {
  W8A8_CHECK_ARG(n_q > 0 && n_q % c->n_kv == 0 && n_q / c->n_kv <= 128 && n_q <= 65536 / c->head_dim, W8A8_ERR_SHAPE,
                 "%s: n_q=%d must be a multiple of n_kv=%d, at most 128 times it and 65536 / head_dim", who, n_q, c->n_kv);
  return W8A8_OK;
}

}  // namespace

}  // namespace w8a8

using namespace w8a8;

extern "C" w8a8_status w8a8_paged_attention_workspace_size(const w8a8_paged_cache* cache, int n_q, size_t* bytes) {
  const char* who = "w8a8_paged_attention_workspace_size";
  W8A8_CHECK_ARG(cache && bytes, W8A8_ERR_INVALID_ARG, "%s: null argument", who);
  W8A8_CHECK_ARG(cache->n_kv > 0 && (cache->head_dim == 64 || cache->head_dim == 128 || cache->head_dim == 256),
                 W8A8_ERR_SHAPE, "%s: n_kv %d, head_dim %d", who, cache->n_kv, cache->head_dim);
  W8A8_TRY(check_heads(who, cache, n_q));
  *bytes = paged_attention_ws(cache->head_dim, n_q, cache->n_kv, device_sms());
  return W8A8_OK;
}

extern "C" w8a8_status w8a8_paged_attention(const w8a8_paged_cache* cache, const w8a8_paged_batch* batch, const uint16_t* q,
                                            int64_t q_row, int64_t q_head, int n_q, float scale, int window, uint16_t* o,
                                            int64_t o_row, int64_t o_head, void* workspace, size_t ws_bytes, void* stream) {
  const char* who = "w8a8_paged_attention";
  PagedCache pc;
  PagedBatch pb;
  W8A8_TRY(check_paged(who, cache, batch, &pc, &pb));
  W8A8_TRY(check_heads(who, cache, n_q));
  const int dim = cache->head_dim;
  W8A8_CHECK_ARG(window >= 0 && std::isfinite(scale) && scale > 0.0f, W8A8_ERR_INVALID_ARG, "%s: window %d, scale %g", who,
                 window, (double)scale);
  if (pb.n_seqs == 0 || pb.n_rows == 0) return W8A8_OK;
  W8A8_CHECK_ARG(q && o, W8A8_ERR_INVALID_ARG, "%s: null pointer", who);
  W8A8_CHECK_ARG(aligned16(q) && aligned16(o), W8A8_ERR_ALIGN, "%s: q and o must be 16-byte aligned", who);
  const int64_t big = 1ll << 38, str[4] = {q_row, q_head, o_row, o_head};
  for (int64_t s : str)
    W8A8_CHECK_ARG(s % 8 == 0 && s >= dim && s <= big, W8A8_ERR_SHAPE, "%s: strides must be multiples of 8 from head_dim on",
                   who);
  W8A8_CHECK_ARG(o_row >= (n_q - 1) * o_head + dim || o_head >= (pb.n_rows - 1) * o_row + dim, W8A8_ERR_SHAPE,
                 "%s: o's rows overlap (strides %lld, %lld)", who, (long long)o_row, (long long)o_head);
  DevInfo d;
  W8A8_TRY(dev_info(&d));
  const size_t need = paged_attention_ws(dim, n_q, cache->n_kv, d.sms);
  W8A8_CHECK_ARG(workspace != nullptr && ws_bytes >= need, W8A8_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who,
                 workspace ? ws_bytes : 0, need);
  W8A8_CHECK_ARG(aligned16(workspace), W8A8_ERR_ALIGN, "%s: workspace must be 16-byte aligned", who);
  const AttnCall a{q, q_row, q_head, o, o_row, o_head, n_q, dim, window, batch->max_new, scale,
                   cache->dtype == W8A8_TYPE_BF16};
  return launch_paged_attention(pc, pb, a, workspace, d.sms, as_stream(stream));
}
