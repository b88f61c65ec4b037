// Shared by the kernels over a paged cache: the ragged batch and the cache as kernels see them, the
// sequence and position of a row, the place of a key, and the types' conversions.
#pragma once

#include "common.cuh"

namespace w8a8 {

// (p, s): a batch's three arrays and their bounds, w8a8_paged_batch without the hints
struct PagedBatch {
  int n_seqs, n_rows, max_pages;
  const int32_t *row_start, *kv_len, *pages;
};
struct PagedCache {
  int n_pages, page_shift, n_kv;
  int64_t page_stride, slot_stride, head_stride;
  uint16_t *k, *v;
};

w8a8_status check_paged(const char* who, const w8a8_paged_cache* c, const w8a8_paged_batch* b, PagedCache* pc,
                        PagedBatch* pb);
w8a8_status check_rope(const char* who, const w8a8_rope_table* r, int dim);
// what an append's rows, norms and strides have to be
w8a8_status check_append(const char* who, const PagedBatch& pb, int dim, const uint16_t* q, int64_t q_row, int n_q,
                         const uint16_t* k, int64_t k_row, const uint16_t* v, int64_t v_row, const float* q_norm,
                         const float* k_norm, float eps, const uint16_t* q_out, int64_t q_out_row);

// (no argument checks; n_rows and n_seqs at least 1)
w8a8_status launch_rope_append(const w8a8_rope_table& rt, const PagedCache& pc, const PagedBatch& pb, int dim, bool bf16,
                               const uint16_t* q, int64_t q_row, int n_q, const uint16_t* k, int64_t k_row,
                               const uint16_t* v, int64_t v_row, const float* q_norm, const float* k_norm, float eps,
                               uint16_t* q_out, int64_t q_out_row, int sms, cudaStream_t st);

// What one call of attention reads and writes beside the cache and the batch.
struct AttnCall {
  const uint16_t* q;
  int64_t q_row, q_head;
  uint16_t* o;
  int64_t o_row, o_head;
  int n_q, dim, window, max_new;
  float scale;
  bool bf16;
  unsigned int* gave_up = nullptr;  // the device's word of waits that gave up, beside the workspace's (launch_paged_attention's)
};
w8a8_status launch_paged_attention(const PagedCache& pc, const PagedBatch& pb, const AttnCall& a, void* ws, int sms,
                                   cudaStream_t st);
size_t paged_attention_ws(int dim, int sms);

// Rows and keys of sequence s, held within the call's bounds whatever the arrays say.
struct SeqShape {
  int row0, rows;  // first row and row count
  int keys;        // cached keys, the rows' own included
  int pos0;        // position of row0 (negative where there are more rows than keys)
};
__device__ __forceinline__ SeqShape seq_shape(const PagedBatch& b, int s, int page_shift) {
  SeqShape q;
  const int r0 = b.row_start[s], r1 = b.row_start[s + 1], len = b.kv_len[s];
  q.row0 = min(max(r0, 0), b.n_rows);
  q.rows = max(min(max(r1, 0), b.n_rows) - q.row0, 0);
  const long long most = (long long)b.max_pages << page_shift;
  q.keys = (int)min((long long)max(len, 0), most);
  q.pos0 = q.keys - q.rows;
  return q;
}
// The last sequence that begins at or before `row`: the only one that can own it (row_start does not decrease).
__device__ __forceinline__ int seq_of_row(const PagedBatch& b, int row) {
  int lo = 0, hi = b.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (b.row_start[mid] <= row)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}
// Element offset of (sequence s, position p, head h); -1 where the page holds nothing.
__device__ __forceinline__ int64_t key_offset(const PagedBatch& b, const PagedCache& c, int s, int p, int h) {
  const int col = p >> c.page_shift;
  if (p < 0 || col >= b.max_pages) return -1;
  const int page = b.pages[(int64_t)s * b.max_pages + col];
  if (page < 0 || page >= c.n_pages) return -1;
  return (int64_t)page * c.page_stride + (int64_t)(p & ((1 << c.page_shift) - 1)) * c.slot_stride +
         (int64_t)h * c.head_stride;
}

// Two 16-bit values of a type <-> fp32 (lo in the low half); rounding to nearest even.
template <bool kBf16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (kBf16) return make_float2(bf16_lo(w), bf16_hi(w));
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <bool kBf16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if constexpr (kBf16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

}  // namespace w8a8
