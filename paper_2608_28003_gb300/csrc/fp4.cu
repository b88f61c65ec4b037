// Quantisation of matrix rows to floating point of 4 bits, and back (w8a8_fp4).
//
// Both kernels only move data, so HBM bounds them, or for few rows the launch.  A thread holds units of 16 columns: 32 or 64
// bytes in, 8 bytes of codes out; the scales of four neighbouring blocks meet in one lane, whose word is contiguous in the
// tiled order.  With blocks of 16 a row's largest magnitude comes first: the row stays in registers over that reduction (up to
// kHeld units a thread; what is beyond is read again, from L2).  At 8191 rows of 6912 bf16 numbers: quantised in 23.0 us with
// blocks of 32 (6.2 TB/s), in 27.8 with blocks of 16 (5.2; a row's reduction stands between its loads and stores), back in 24.0
// and 32.8 (6.0 and 4.4 TB/s; with a division a place blocks of 32 took 27.7); before the maxima and quotients were packed two to a
// register and four units flew together, 75 there and back with blocks of 32.
#include <algorithm>

#include "fp4.cuh"
#include "ops.cuh"

namespace w8a8 {

namespace {

template <int kType>
struct Unit16;  // 16 columns as loaded
template <>
struct Unit16<W8A8_TYPE_F32> {
  uint4 w[4];
};
template <>
struct Unit16<W8A8_TYPE_BF16> {
  uint4 w[2];
};
template <>
struct Unit16<W8A8_TYPE_F16> {
  uint4 w[2];
};

template <int kType>
__device__ __forceinline__ Unit16<kType> load_unit(const char* row, int unit) {
  Unit16<kType> u;
  const uint4* p = reinterpret_cast<const uint4*>(row + (size_t)unit * sizeof(u));
#pragma unroll
  for (int i = 0; i < (int)(sizeof(u) / 16); ++i) u.w[i] = p[i];
  return u;
}
template <int kType>
__device__ __forceinline__ void unit_floats(const Unit16<kType>& u, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof(u) / 16); ++i) {
    const uint32_t w[4] = {u.w[i].x, u.w[i].y, u.w[i].z, u.w[i].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (kType == W8A8_TYPE_F32) {
        x[4 * i + e] = __uint_as_float(w[e]);
      } else {
        const float2 f = unpack2<kType == W8A8_TYPE_BF16>(w[e]);
        x[8 * i + 2 * e] = f.x;
        x[8 * i + 2 * e + 1] = f.y;
      }
    }
  }
}
// The bits of the largest magnitude, as an fp32 number's: compared as integers, so that NaN and infinities are above everything.
template <int kType>
__device__ __forceinline__ uint32_t top_of(const Unit16<kType>& u) {
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(u) / 16); ++i) {
    if constexpr (kType == W8A8_TYPE_F32)
      t = max(max(max(t, u.w[i].x & 0x7fffffffu), max(u.w[i].y & 0x7fffffffu, u.w[i].z & 0x7fffffffu)), u.w[i].w & 0x7fffffffu);
    else
      t = __vmaxu2(__vmaxu2(__vmaxu2(t, u.w[i].x & 0x7fff7fffu), __vmaxu2(u.w[i].y & 0x7fff7fffu, u.w[i].z & 0x7fff7fffu)),
                   u.w[i].w & 0x7fff7fffu);
  }
  if constexpr (kType == W8A8_TYPE_F32) return t;
  t = max(t & 0xffffu, t >> 16);
  return kType == W8A8_TYPE_BF16 ? t << 16 : __float_as_uint(__half2float(__ushort_as_half((unsigned short)t)));
}

// One unit: its codes, and its block's scale byte (both lanes of a block of 32 have it).  `top` of this unit; s2 the reciprocal of
// the row's scale (blocks of 16).  All lanes of a warp.
template <int kType, int kBlock>
__device__ __forceinline__ uint32_t quantise_unit(const Unit16<kType>& u, uint32_t top, float s2, uint2& codes) {
  float x[16];
  unit_floats<kType>(u, x);
  f32x2 q[8], hi, lo = 0ull;
  uint32_t byte;
  bool nan;
  if constexpr (kBlock == 16) {
    Block16 b;
    b.unit(top, s2);
    byte = b.byte;
    nan = byte == kE4m3NaN;
    if (s2 > 0x1p60f || s2 < 0x1p-60f) {
      // a row of numbers near the type's ends: brought towards 1 first (exactly, but for numbers whose codes are 0), so that the
      // products below are normal numbers
      const float near = s2 > 1.0f ? 0x1p60f : 0x1p-60f;
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] *= near;
      s2 *= s2 > 1.0f ? 0x1p-60f : 0x1p60f;
    }
    hi = f2_pack(b.hi * s2, b.hi * s2);  // (s2 is a power of two)
    lo = f2_pack(b.lo * s2, b.lo * s2);
  } else {
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    nan = top >= 0x7f800000u;
    byte = nan ? kE8m0NaN : (uint32_t)max((int)(top >> 23) - 2, 0);  // 2^(byte - 127)
    // 2^(127 - byte), a normal number but for 254, which no finite block has (252 at most); x times it is exact, or so
    // small that its code is 0
    const float inv = __uint_as_float((254u - min(byte, 253u)) << 23);
    hi = f2_pack(inv, inv);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const f32x2 v = f2_pack(x[2 * e], x[2 * e + 1]);
    q[e] = f2_fma(v, hi, kBlock == 16 ? f2_fma(v, lo, 0ull) : 0ull);
  }
  codes = make_uint2(e2m1x8_of(q[0], q[1], q[2], q[3]), e2m1x8_of(q[4], q[5], q[6], q[7]));
  if (nan) codes = make_uint2(0u, 0u);
  return byte;
}

// kWarp: tpr (a power of two, kBlock / 4 to 32) neighbouring lanes take a row (all 32 where kHeld > 1), else a block takes one.
template <int kType, int kBlock, bool kWarp, int kHeld>
__global__ void __launch_bounds__(512) fp4_quantise_kernel(const char* __restrict__ x, int64_t x_row_bytes, int rows, int padded,
                                                           int k, int tpr, uint8_t* __restrict__ codes,
                                                           uint8_t* __restrict__ scales, float* __restrict__ row_scale) {
  __shared__ uint32_t s_top[16];
  pdl_wait();
  pdl_trigger();  // (behind the wait: a product may read its weights ahead of its own)
  const int units = k / 16, groups = fp4_groups(k, kBlock), lane = threadIdx.x & 31;
  const int step = kWarp ? tpr : (int)blockDim.x;
  const int64_t row = kWarp ? ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / tpr : (int64_t)blockIdx.x;
  const int u0 = kWarp ? (int)(threadIdx.x & (tpr - 1)) : (int)threadIdx.x;
  const bool live = row < rows;
  const char* src = x + row * x_row_bytes;
  Unit16<kType> held[kHeld];
  uint32_t tops[kHeld];
  float s2 = 1.0f;
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (live && u0 + i * step < units) held[i] = load_unit<kType>(src, u0 + i * step);
#pragma unroll
  for (int i = 0; i < kHeld; ++i) tops[i] = live && u0 + i * step < units ? top_of<kType>(held[i]) : 0u;
  if constexpr (kBlock == 16) {
    uint32_t top = 0;  // of the blocks that are finite
#pragma unroll
    for (int i = 0; i < kHeld; ++i) top = max(top, tops[i] < 0x7f800000u ? tops[i] : 0u);
    for (int u = u0 + kHeld * step; live && u < units; u += step) {
      const uint32_t t = top_of<kType>(load_unit<kType>(src, u));
      top = max(top, t < 0x7f800000u ? t : 0u);
    }
    if constexpr (kWarp) {
      for (int o = tpr / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    } else {
      top = __reduce_max_sync(0xffffffffu, top);
      if (lane == 0) s_top[threadIdx.x >> 5] = top;
      __syncthreads();
      top = __reduce_max_sync(0xffffffffu, lane < (int)(blockDim.x >> 5) ? s_top[lane] : 0u);
    }
    const int p = top == 0 ? 0 : row_exponent(top);
    s2 = two_to(-p);
    if (live && u0 == 0) row_scale[row] = two_to(p);
  }
  auto put = [&](int u, const Unit16<kType>& x, uint32_t top) {
    const bool here = live && u < units;
    uint2 c;
    uint32_t byte = quantise_unit<kType, kBlock>(x, top, s2, c);
    if (here) *reinterpret_cast<uint2*>(codes + row * (int64_t)(k / 2) + 8 * u) = c;
    // the bytes of four blocks in their first lane
    constexpr int kStep = kBlock / 16;  // lanes a block
    const int j = u / kStep;
    byte = here ? byte << (8 * (j & 3)) : 0u;
    byte |= __shfl_xor_sync(0xffffffffu, byte, kStep);
    byte |= __shfl_xor_sync(0xffffffffu, byte, 2 * kStep);
    if ((u & (4 * kStep - 1)) == 0 && u < units && row < padded)
      *reinterpret_cast<uint32_t*>(scales + fp4_scale_at(row, j, groups)) = byte;
  };
  // every lane makes the same trips: the scales' exchange is a whole warp's
  const int first = kWarp ? 0 : (int)(threadIdx.x & ~31u);
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (first + i * step < units) {
      if (!(live && u0 + i * step < units)) held[i] = Unit16<kType>{};
      put(u0 + i * step, held[i], tops[i]);
    }
  for (int i = kHeld; first + i * step < units; ++i) {
    Unit16<kType> x{};
    if (live && u0 + i * step < units) x = load_unit<kType>(src, u0 + i * step);
    put(u0 + i * step, x, top_of<kType>(x));
  }
}

// f b rounded to odd: cut off, and its last bit set where that lost something.  fp32 has more than two bits beyond the 16-bit types', so what
// is rounded from it to one of them is as if from f b itself.  The remainder is rounded away from zero: its last bits can lie below
// fp32's smallest number.
__device__ __forceinline__ float product_to_odd(float f, float b) {
  const float x = fabsf(f), y = fabsf(b), p = __fmul_rz(x, y);
  const uint32_t sign = (__float_as_uint(f) ^ __float_as_uint(b)) & 0x80000000u;
  return __uint_as_float(__float_as_uint(p) | (__fmaf_ru(x, y, -p) > 0.0f ? 1u : 0u) | sign);
}

// A thread has eight columns, so that a warp's loads and stores are contiguous, of kAhead places 256 threads apart.  per_row =
// ceil(2^64 / eighths): i per_row / 2^64 is less than i / 2^64 above i / eighths, and i < 2^44 and eighths <= 2^13.
constexpr int kAhead = 4;
template <int kType, int kBlock>
__global__ void __launch_bounds__(256) fp4_dequantise_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                             const float* __restrict__ row_scale, int64_t total, int eighths,
                                                             uint64_t per_row, int groups, char* __restrict__ y,
                                                             int64_t y_row_bytes) {
  pdl_wait();
  pdl_trigger();
  const int64_t i0 = (int64_t)blockIdx.x * (256 * kAhead) + threadIdx.x;
  uint32_t c[kAhead], byte[kAhead];
  float b[kAhead];
  int64_t row[kAhead];
  int e8[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) {
    const int64_t i = i0 + 256 * j;
    if (i >= total) continue;
    row[j] = (int64_t)__umul64hi((uint64_t)i, per_row);  // i / eighths
    e8[j] = (int)(i - row[j] * eighths);
    c[j] = *reinterpret_cast<const uint32_t*>(codes + i * 4);
    byte[j] = scales[fp4_scale_at(row[j], kBlock == 16 ? e8[j] >> 1 : e8[j] >> 2, groups)];
    if (kBlock == 16) b[j] = row_scale[row[j]];
  }
#pragma unroll
  for (int j = 0; j < kAhead; ++j) {
    if (i0 + 256 * j >= total) break;
    uint32_t h[4];
    float v[8];
    e2m1x8_to_f16(c[j], h);
    if constexpr (kBlock == 16) {
      const uint32_t a = e4m3x2_to_f16x2(byte[j] * 0x101u);
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = hmul2_bits(h[e], a);  // exact: six significant bits between 2^-10 and 2688
    } else {
      b[j] = byte[j] == kE8m0NaN ? NAN : byte[j] == 0 ? 0x1p-127f : __uint_as_float(byte[j] << 23);
    }
    // A row's scale that is a (normal) power of two, as the quantiser's are, costs the product no rounding; another would cost a 16-bit
    // value two (to odd: 38.8 us at 8191 x 6912, 32.8 with powers of two).
    if (kBlock == 16 && kType != W8A8_TYPE_F32 && (__float_as_uint(b[j]) << 9) != 0) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = unpack2<false>(h[e]);
        v[2 * e] = product_to_odd(f.x, b[j]);
        v[2 * e + 1] = product_to_odd(f.y, b[j]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = unpack2<false>(h[e]);
        v[2 * e] = f.x * b[j];
        v[2 * e + 1] = f.y * b[j];
      }
    }
    constexpr int kBytes = kType == W8A8_TYPE_F32 ? 32 : 16;
    uint4* to = reinterpret_cast<uint4*>(y + row[j] * y_row_bytes + (int64_t)e8[j] * kBytes);
    if constexpr (kType == W8A8_TYPE_F32) {
      to[0] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      to[1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
    } else {
      constexpr bool kBf = kType == W8A8_TYPE_BF16;
      to[0] = make_uint4(pack2<kBf>(v[0], v[1]), pack2<kBf>(v[2], v[3]), pack2<kBf>(v[4], v[5]), pack2<kBf>(v[6], v[7]));
    }
  }
}

w8a8_status check_matrix(const char* who, int dtype, int64_t row_stride, int k) {
  W8A8_CHECK_ARG(dtype >= W8A8_TYPE_BF16 && dtype <= W8A8_TYPE_F32, W8A8_ERR_INVALID_ARG, "%s: type %d", who, dtype);
  W8A8_CHECK_ARG(row_stride >= 0 && row_stride <= (1ll << 40) && row_stride * type_bytes(dtype) % 16 == 0, W8A8_ERR_SHAPE,
                 "%s: a row stride of %lld elements is not a multiple of 16 bytes", who, (long long)row_stride);
  return W8A8_OK;
}

}  // namespace

w8a8_status check_fp4(const char* who, const w8a8_fp4* q) {
  W8A8_CHECK_ARG(q != nullptr, W8A8_ERR_INVALID_ARG, "%s: null descriptor", who);
  W8A8_CHECK_ARG(q->block == 16 || q->block == 32, W8A8_ERR_INVALID_ARG, "%s: block %d must be 16 or 32", who, q->block);
  W8A8_CHECK_ARG(q->rows >= 0 && q->rows <= kMaxFp4Rows && q->k > 0 && q->k % 32 == 0 && q->k <= W8A8_MAX_K, W8A8_ERR_SHAPE,
                 "%s: rows %d, k %d: k must be a multiple of 32, at most %d", who, q->rows, q->k, W8A8_MAX_K);
  if (q->rows == 0) return W8A8_OK;
  W8A8_CHECK_ARG(q->codes && q->scales && (q->block == 32 || q->row_scale), W8A8_ERR_INVALID_ARG, "%s: null pointer", who);
  W8A8_CHECK_ARG(aligned16(q->codes) && aligned16(q->scales) && aligned16(q->row_scale), W8A8_ERR_ALIGN,
                 "%s: codes, scales and row_scale must be 16-byte aligned", who);
  return W8A8_OK;
}

// Lanes of a warp share its rows while a row's units fit; then a block a row.  What fills the SMs with a thread a unit more than once has
// lanes of up to four units, whose loads fly together (8191 rows of 6912: 23.0 us with blocks of 32, 27.8 with blocks of 16; with one 30.2
// and 39.1), and rows of up to 128 units a warp each, four a block (262144 rows of 1152: 149 and 207 us; 264 and 265 with one).  The
// others have one, for the shortest chain (2048 rows of 1152: 2.6 and 3.0 us; with up to four 2.8 and 3.5; 16 rows 1.4 and 1.7; 1.9 and
// 2.5).  Blocks of 16 are bound by instructions.
w8a8_status launch_fp4_quantize(int dtype, const void* x, int64_t x_row, const w8a8_fp4& q, bool pad, cudaStream_t st) {
  const int units = q.k / 16, padded = pad ? (int)round_up((size_t)q.rows, 128) : q.rows;
  int tpr = q.block / 4;  // four blocks' scales meet within a row's lanes
  while (tpr < units && tpr < 32) tpr *= 2;
  const int held = dtype == W8A8_TYPE_F32 ? 2 : 4;
  DevInfo d;
  W8A8_TRY(dev_info(&d));
  const bool many = (int64_t)q.rows * units >= (int64_t)d.sms * 2048, warp = units <= 32 || (many && units <= 32 * held);
  const int each = many ? held : 1;
  const int threads = warp ? 128 : std::min((int)round_up((size_t)(units + each - 1) / each, 32), 512);
  const int64_t blocks = warp ? ((int64_t)padded * tpr + 127) / 128 : padded;
  auto go = [&](auto kernel) {
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3((unsigned)threads), 0, st, static_cast<const char*>(x),
                      x_row * type_bytes(dtype), q.rows, padded, q.k, tpr, q.codes, q.scales, q.row_scale);
  };
  auto of = [&](auto type) {
    constexpr int kT = decltype(type)::value;
    constexpr int kH = kT == W8A8_TYPE_F32 ? 2 : 4;
    if (q.block == 16)
      return warp && units > 32 ? go(fp4_quantise_kernel<kT, 16, true, kH>)
             : warp ? go(fp4_quantise_kernel<kT, 16, true, 1>)
             : many ? go(fp4_quantise_kernel<kT, 16, false, kH>)
                    : go(fp4_quantise_kernel<kT, 16, false, 2>);
    return warp && units > 32 ? go(fp4_quantise_kernel<kT, 32, true, kH>)
           : warp ? go(fp4_quantise_kernel<kT, 32, true, 1>)
           : many ? go(fp4_quantise_kernel<kT, 32, false, kH>)
                  : go(fp4_quantise_kernel<kT, 32, false, 2>);
  };
  W8A8_CUDA(dtype == W8A8_TYPE_BF16  ? of(std::integral_constant<int, W8A8_TYPE_BF16>())
            : dtype == W8A8_TYPE_F16 ? of(std::integral_constant<int, W8A8_TYPE_F16>())
                                     : of(std::integral_constant<int, W8A8_TYPE_F32>()));
  return W8A8_OK;
}

}  // namespace w8a8

using namespace w8a8;

extern "C" w8a8_status w8a8_fp4_scale_bytes(int rows, int k, int block, size_t* bytes) {
  const char* who = "w8a8_fp4_scale_bytes";
  W8A8_CHECK_ARG(bytes != nullptr && (block == 16 || block == 32), W8A8_ERR_INVALID_ARG, "%s: null pointer, or block %d", who,
                 block);
  W8A8_CHECK_ARG(rows >= 0 && rows <= kMaxFp4Rows && k > 0 && k % 32 == 0 && k <= W8A8_MAX_K, W8A8_ERR_SHAPE,
                 "%s: rows %d, k %d: k must be a multiple of 32, at most %d", who, rows, k, W8A8_MAX_K);
  *bytes = round_up((size_t)rows, 128) / 128 * (size_t)fp4_groups(k, block) * 512;
  return W8A8_OK;
}

extern "C" w8a8_status w8a8_fp4_quantize(int dtype, const void* x, int64_t x_row, const w8a8_fp4* q, void* stream) {
  const char* who = "w8a8_fp4_quantize";
  W8A8_TRY(check_fp4(who, q));
  W8A8_TRY(check_matrix(who, dtype, x_row, q->k));
  if (q->rows == 0) return W8A8_OK;
  W8A8_CHECK_ARG(x != nullptr, W8A8_ERR_INVALID_ARG, "%s: null x", who);
  W8A8_CHECK_ARG(aligned16(x), W8A8_ERR_ALIGN, "%s: x must be 16-byte aligned", who);
  W8A8_TRY(check_device());
  return launch_fp4_quantize(dtype, x, x_row, *q, true, as_stream(stream));
}

extern "C" w8a8_status w8a8_fp4_dequantize(const w8a8_fp4* q, int dtype, void* y, int64_t y_row, void* stream) {
  const char* who = "w8a8_fp4_dequantize";
  W8A8_TRY(check_fp4(who, q));
  W8A8_TRY(check_matrix(who, dtype, y_row, q->k));
  if (q->rows == 0) return W8A8_OK;
  W8A8_CHECK_ARG(y != nullptr, W8A8_ERR_INVALID_ARG, "%s: null y", who);
  W8A8_CHECK_ARG(aligned16(y), W8A8_ERR_ALIGN, "%s: y must be 16-byte aligned", who);
  W8A8_CHECK_ARG(q->rows == 1 || y_row >= q->k, W8A8_ERR_SHAPE, "%s: y's rows overlap", who);
  W8A8_TRY(check_device());
  const int eighths = q->k / 8;
  const int64_t total = (int64_t)q->rows * eighths, blocks = (total + 256 * kAhead - 1) / (256 * kAhead);
  W8A8_CHECK_ARG(blocks <= 0x7fffffffll, W8A8_ERR_SHAPE, "%s: [%d, %d] is too large", who, q->rows, q->k);
  auto go = [&](auto kernel) {
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3(256), 0, as_stream(stream), (const uint8_t*)q->codes,
                      (const uint8_t*)q->scales, (const float*)q->row_scale, total, eighths, ~0ull / (uint64_t)eighths + 1,
                      fp4_groups(q->k, q->block), static_cast<char*>(y), y_row * type_bytes(dtype));
  };
  auto of = [&](auto type) {
    constexpr int kT = decltype(type)::value;
    return q->block == 16 ? go(fp4_dequantise_kernel<kT, 16>) : go(fp4_dequantise_kernel<kT, 32>);
  };
  W8A8_CUDA(dtype == W8A8_TYPE_BF16  ? of(std::integral_constant<int, W8A8_TYPE_BF16>())
            : dtype == W8A8_TYPE_F16 ? of(std::integral_constant<int, W8A8_TYPE_F16>())
                                     : of(std::integral_constant<int, W8A8_TYPE_F32>()));
  return W8A8_OK;
}
