// Attention of a ragged batch over a paged cache: checks and choice of the kernel.
#include <algorithm>
#include <cmath>

#include "attn_paged.cuh"
#include "ops.cuh"
#include "paged.cuh"

namespace w8a8 {

size_t paged_attention_ws(int dim, int sms) {
  return W8A8_WS_RESERVED + std::max(attn_tokens_ws(dim, sms), attn_chunks_ws(dim, sms));
}

namespace {

__device__ unsigned int g_gave_up;  // DevErr bits of any call on this device since the last check

}  // namespace

w8a8_status gave_up_word(unsigned int** word) {
  static unsigned int* known[64] = {};
  return device_word(&g_gave_up, known, word);
}

// Up to 16 rows a sequence and key/value head go to the kernel for tokens, more to the one for chunks (a longer sequence in
// the batch is right in either): 64 sequences of 4000 keys, 1 head of 256, take 54.5, 63.6 and 95.4 us for 4, 16 and 32 rows
// there and 60 here; 40 sequences of 4 heads of 128 69.5 and 121 us for 16 and 32 rows there, 71 here; of 8
// heads of 64 67.4 and 121 us for 15 and 30 rows there, 115 here.
w8a8_status launch_paged_attention(const PagedCache& pc, const PagedBatch& pb, const AttnCall& call, void* ws, int sms,
                                   cudaStream_t st) {
  const int group = call.n_q / pc.n_kv;
  AttnCall a = call;
  if (a.window >= 1 << 30) a.window = 0;  // beyond every position, and negative ones less it would not fit in 32 bits
  W8A8_TRY(gave_up_word(&a.gave_up));
  return (long long)a.max_new * group <= 16 ? launch_attn_tokens(pc, pb, a, ws, sms, st)
                                            : launch_attn_chunks(pc, pb, a, ws, sms, st);
}

w8a8_status check_heads(const char* who, int n_kv, int dim, int n_q) {
  W8A8_CHECK_ARG(n_q > 0 && n_q % n_kv == 0 && n_q / n_kv <= 128 && n_q <= 65536 / dim, W8A8_ERR_SHAPE,
                 "%s: n_q=%d must be a multiple of n_kv=%d, at most 128 times it and 65536 / head_dim", who, n_q, n_kv);
  return W8A8_OK;
}

w8a8_status check_attention(const char* who, const PagedBatch& pb, const uint16_t* q, int64_t q_row, int64_t q_head, int n_q,
                            int dim, float scale, int window, const uint16_t* o, int64_t o_row, int64_t o_head) {
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
  W8A8_CHECK_ARG(o != q, W8A8_ERR_INVALID_ARG, "%s: o must not be q: other rows' pieces still read it", who);
  return W8A8_OK;
}

w8a8_status check_attention_ws(const char* who, int dim, int sms, const void* workspace, size_t ws_bytes) {
  const size_t need = paged_attention_ws(dim, sms);
  W8A8_CHECK_ARG(workspace != nullptr && ws_bytes >= need, W8A8_ERR_WORKSPACE, "%s: workspace %zu bytes, need %zu", who,
                 workspace ? ws_bytes : 0, need);
  W8A8_CHECK_ARG(aligned16(workspace), W8A8_ERR_ALIGN, "%s: workspace must be 16-byte aligned", who);
  return W8A8_OK;
}

}  // namespace w8a8

using namespace w8a8;

extern "C" w8a8_status w8a8_paged_attention_workspace_size(const w8a8_paged_cache* cache, int n_q, size_t* bytes) {
  const char* who = "w8a8_paged_attention_workspace_size";
  W8A8_CHECK_ARG(cache && bytes, W8A8_ERR_INVALID_ARG, "%s: null argument", who);
  W8A8_CHECK_ARG(cache->n_kv > 0 && (cache->head_dim == 64 || cache->head_dim == 128 || cache->head_dim == 256),
                 W8A8_ERR_SHAPE, "%s: n_kv %d, head_dim %d", who, cache->n_kv, cache->head_dim);
  W8A8_TRY(check_heads(who, cache->n_kv, cache->head_dim, n_q));
  *bytes = paged_attention_ws(cache->head_dim, device_sms());
  return W8A8_OK;
}

extern "C" w8a8_status w8a8_paged_attention(const w8a8_paged_cache* cache, const w8a8_paged_batch* batch, const uint16_t* q,
                                            int64_t q_row, int64_t q_head, int n_q, float scale, int window, uint16_t* o,
                                            int64_t o_row, int64_t o_head, void* workspace, size_t ws_bytes, void* stream) {
  const char* who = "w8a8_paged_attention";
  PagedCache pc;
  PagedBatch pb;
  W8A8_TRY(check_paged(who, cache, batch, &pc, &pb));
  W8A8_TRY(check_heads(who, cache->n_kv, cache->head_dim, n_q));
  const int dim = cache->head_dim;
  W8A8_TRY(check_attention(who, pb, q, q_row, q_head, n_q, dim, scale, window, o, o_row, o_head));
  if (pb.n_seqs == 0 || pb.n_rows == 0) return W8A8_OK;
  DevInfo d;
  W8A8_TRY(dev_info(&d));
  W8A8_TRY(check_attention_ws(who, dim, d.sms, workspace, ws_bytes));
  const AttnCall a{q, q_row, q_head, o, o_row, o_head, n_q, dim, window, batch->max_new, scale,
                   cache->dtype == W8A8_TYPE_BF16};
  return launch_paged_attention(pc, pb, a, workspace, d.sms, as_stream(stream));
}

extern "C" w8a8_status w8a8_paged_attention_error_word(uint32_t** word) {
  W8A8_CHECK_ARG(word != nullptr, W8A8_ERR_INVALID_ARG, "w8a8_paged_attention_error_word: null argument");
  W8A8_TRY(check_device());
  return gave_up_word(word);
}

extern "C" w8a8_status w8a8_paged_attention_check(void* stream) {
  unsigned int* word = nullptr;
  W8A8_TRY(w8a8_paged_attention_error_word(&word));
  return take_error_word(word, as_stream(stream));
}
