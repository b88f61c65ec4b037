// Attention of a ragged batch over a paged cache in 4 bits: checks and choice of the kernel.
#include <cmath>

#include "attn_fp4.cuh"
#include "ops.cuh"

using namespace w8a8;

extern "C" w8a8_status w8a8_fp4_paged_attention_workspace_size(const w8a8_paged_cache_fp4* cache, int n_q, size_t* bytes) {
  const char* who = "w8a8_fp4_paged_attention_workspace_size";
  W8A8_CHECK_ARG(cache && bytes, W8A8_ERR_INVALID_ARG, "%s: null argument", who);
  W8A8_CHECK_ARG(cache->n_kv > 0 && (cache->head_dim == 64 || cache->head_dim == 128 || cache->head_dim == 256),
                 W8A8_ERR_SHAPE, "%s: n_kv %d, head_dim %d", who, cache->n_kv, cache->head_dim);
  W8A8_TRY(check_heads(who, cache->n_kv, cache->head_dim, n_q));
  *bytes = paged_attention_ws(cache->head_dim, device_sms());
  return W8A8_OK;
}

extern "C" w8a8_status w8a8_fp4_paged_attention(const w8a8_paged_cache_fp4* cache, const w8a8_paged_batch* batch, int dtype,
                                                const uint16_t* q, int64_t q_row, int64_t q_head, int n_q, float scale,
                                                int window, uint16_t* o, int64_t o_row, int64_t o_head, void* workspace,
                                                size_t ws_bytes, void* stream) {
  const char* who = "w8a8_fp4_paged_attention";
  Fp4Pages pc;
  PagedBatch pb;
  W8A8_TRY(check_fp4_paged(who, cache, batch, &pc, &pb));
  W8A8_CHECK_ARG(dtype == W8A8_TYPE_BF16 || dtype == W8A8_TYPE_F16, W8A8_ERR_INVALID_ARG, "%s: type %d must be bf16 or fp16",
                 who, dtype);
  const int dim = cache->head_dim;
  W8A8_TRY(check_heads(who, cache->n_kv, dim, n_q));
  W8A8_TRY(check_attention(who, pb, q, q_row, q_head, n_q, dim, scale, window, o, o_row, o_head));
  if (pb.n_seqs == 0 || pb.n_rows == 0) return W8A8_OK;
  DevInfo d;
  W8A8_TRY(dev_info(&d));
  W8A8_TRY(check_attention_ws(who, dim, d.sms, workspace, ws_bytes));
  AttnCall a{q, q_row, q_head, o, o_row, o_head, n_q, dim, window, batch->max_new, scale, dtype == W8A8_TYPE_BF16};
  if (a.window >= 1 << 30) a.window = 0;  // beyond every position
  W8A8_TRY(gave_up_word(&a.gave_up));
  // Up to 16 rows an item: 64 tokens of 4 rows behind 8000 keys at head dim 256 43.5 us, 130 by the chunk kernel, whose row tiles are 128.
  // At 16 rows still 98 and 127 (the 64 with 4 drafted tokens), 66 and 143 (32 x 2 tokens of 8 heads on each of 4 of 128 behind 8000 keys), 47
  // and 121 (64 x 4 of 4 heads on each of 2 of 64); nearest 24.1 and 26.4 (one sequence of 700 keys, 4 drafted tokens, head dim 256).
  return (long long)a.max_new * (n_q / pc.p.n_kv) <= 16 ? launch_attn_fp4_tokens(pc, pb, a, workspace, d.sms, as_stream(stream))
                                                        : launch_attn_fp4_chunks(pc, pb, a, workspace, d.sms, as_stream(stream));
}
