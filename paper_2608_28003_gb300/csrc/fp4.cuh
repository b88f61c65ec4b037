// Floating point of 4 bits: conversions, the choice of a block's unit, and what the kernels over a 4-bit cache share.
#pragma once

#include "common.cuh"
#include "paged.cuh"

namespace w8a8 {

// ------------------------------------------------------------------------------- conversions
// Two fp32 values -> two e2m1 codes (lo in the low half): nearest, ties to the even code, saturating at +-6.
__device__ __forceinline__ uint32_t e2m1x2_of(float lo, float hi) {
  uint16_t r;
  asm("{\n .reg .b8 t;\n cvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n cvt.u16.u8 %0, t;\n}\n" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Four packed pairs -> eight codes, in order.
__device__ __forceinline__ uint32_t e2m1x8_of(f32x2 a, f32x2 b, f32x2 c, f32x2 d) {
  uint32_t r;
  asm("{\n .reg .b8 p, q, r, s;\n .reg .f32 l, h;\n mov.b64 {l, h}, %1;\n cvt.rn.satfinite.e2m1x2.f32 p, h, l;\n"
      " mov.b64 {l, h}, %2;\n cvt.rn.satfinite.e2m1x2.f32 q, h, l;\n mov.b64 {l, h}, %3;\n cvt.rn.satfinite.e2m1x2.f32 r, h, l;\n"
      " mov.b64 {l, h}, %4;\n cvt.rn.satfinite.e2m1x2.f32 s, h, l;\n mov.b32 %0, {p, q, r, s};\n}\n"
      : "=r"(r)
      : "l"(a), "l"(b), "l"(c), "l"(d));
  return r;
}
// Eight codes -> their values as four fp16 pairs, in order (exact).
__device__ __forceinline__ void e2m1x8_to_f16(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
      " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}\n"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
}
__device__ __forceinline__ uint32_t e4m3_of(float x) {
  return (uint32_t)__nv_cvt_float_to_fp8(x, __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float e4m3_value(uint32_t byte) {
  const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3);
  return __half2float(__half(h));
}
__device__ __forceinline__ uint32_t hmul2_bits(uint32_t a, uint32_t b) {
  const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&y);
}
__device__ __forceinline__ uint32_t bmul2_bits(uint32_t a, uint32_t b) {  // bf16
  const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&y);
}
// 2^e for -126 <= e <= 127
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

constexpr uint32_t kE8m0NaN = 255, kE4m3NaN = 127;

// The exponent of a row's scale: the smallest p >= -126 with `top` (the bits of a finite fp32 value above 0) <= 21 2^7 2^p.
// top = f 2^e with f in [1, 2), 21 2^7 = 1.3125 2^11.
__device__ __forceinline__ int row_exponent(uint32_t top) {
  const int e = (int)(top >> 23) - 127;
  const int p = e - 11 + ((top & 0x7fffffu) > 0x280000u ? 1 : 0);  // a subnormal top has e = -127: below the clamp anyway
  return p < -126 ? -126 : p;
}

// How x is quantised in a block of 16: x s2 / scale, s2 the reciprocal of the row's scale (a power of two).
// An fp32 quotient that is rounded correctly lies on the same side of every border of the codes, and of the e4m3 scales, as the exact
// one, and on a border only with it: a border b has few bits, and x (24 bits) over a scale of 4 bits, or m over 6, that
// differs from b does so by more than half a unit in the last place of b (with f and g the significands of b and of
// b times the divisor: by 2 g^-1 of that, relative to f^-1, and g < 2 f).
// The quotient is x hi + fl(x lo) with hi + lo the reciprocal to 2^-43 (hi to 2^-22, lo from its exact remainder): exact where the
// quotient is a border, within 2^-19 of a unit in the last place of correctly rounded elsewhere, where the nearest border is 2^-5 of
// one further off than half of it (g is at most 1.875 where f is 1).
__device__ __forceinline__ float sixth(float x) {  // x / 6; what is above every scale as the largest of them has it
  x = fminf(x, 0x1p20f);
  return fmaf(x, 0x1.555556p-3f, x * -0x1.555556p-28f);
}
struct Block16 {
  float scale, hi, lo;
  uint32_t byte;
  __device__ __forceinline__ void unit(uint32_t top_bits, float s2) {  // top_bits: of the block's largest magnitude
    byte = top_bits >= 0x7f800000u ? kE4m3NaN : e4m3_of(sixth(__uint_as_float(top_bits) * s2));
    of_byte();
  }
  __device__ __forceinline__ void of_byte() {
    scale = byte == kE4m3NaN ? 0.0f : e4m3_value(byte);
    asm("rcp.approx.f32 %0, %1;\n" : "=f"(hi) : "f"(scale));
    lo = fmaf(-scale, hi, 1.0f) * hi;
    if (scale == 0.0f) hi = lo = 0.0f;
  }
  // x s2 / scale (x already times s2)
  __device__ __forceinline__ float over(float x) const { return fmaf(x, hi, x * lo); }
};

// ------------------------------------------------------------------------------- matrices
// Where the scale of block j of row r lies (w8a8_fp4).
__host__ __device__ __forceinline__ size_t fp4_scale_at(int64_t r, int j, int groups) {
  return ((size_t)(r >> 7) * groups + (j >> 2)) * 512 + (size_t)(r & 31) * 16 + (size_t)((r >> 5) & 3) * 4 + (j & 3);
}
__host__ __device__ __forceinline__ int fp4_groups(int k, int block) { return (k / block + 3) / 4; }
constexpr int kMaxFp4Rows = 0x7fffff80;  // whole 128-row blocks of scales stay within an int
w8a8_status check_fp4(const char* who, const w8a8_fp4* q);
// (no argument checks).  pad: rows beyond q.rows, up to a multiple of 128, get scales of 0 as well.
w8a8_status launch_fp4_quantize(int dtype, const void* x, int64_t x_row, const w8a8_fp4& q, bool pad, cudaStream_t st);
inline int type_bytes(int dtype) { return dtype == W8A8_TYPE_F32 ? 4 : 2; }

// ------------------------------------------------------------------------------- cache
// A 4-bit cache as kernels see it: p holds the pages' shape and the codes' strides in bytes (its pointers are unused).
struct Fp4Pages {
  PagedCache p;
  int64_t s_page, s_slot, s_head;
  uint8_t *k, *v, *ks, *vs;
  int k_exp, v_exp;
  float k_unit = 1.0f, score = 0.0f;  // of attention: in K's operand (chunks), on sums of products
};
w8a8_status check_fp4_paged(const char* who, const w8a8_paged_cache_fp4* c, const w8a8_paged_batch* b, Fp4Pages* pc,
                            PagedBatch* pb);
// Byte offsets of the codes and of the scales of (sequence s, position p, head h); -1 where the page holds nothing.
__device__ __forceinline__ int64_t fp4_key_offset(const PagedBatch& b, const Fp4Pages& c, int s, int p, int h, int64_t& scales) {
  const int col = p >> c.p.page_shift;
  if (p < 0 || col >= b.max_pages) return -1;
  const int page = b.pages[(int64_t)s * b.max_pages + col];
  if (page < 0 || page >= c.p.n_pages) return -1;
  const int slot = p & ((1 << c.p.page_shift) - 1);
  scales = (int64_t)page * c.s_page + (int64_t)slot * c.s_slot + (int64_t)h * c.s_head;
  return (int64_t)page * c.p.page_stride + (int64_t)slot * c.p.slot_stride + (int64_t)h * c.p.head_stride;
}

}  // namespace w8a8
