// Quantisation of matrix rows to floating point of 4 bits, and back (w8a8_fp4).
//
// Both kernels only move data, so HBM bounds them, or for few rows the launch.  A thread holds a unit of 16 columns: 32 or 64
// bytes in, 8 bytes of codes out; the scales of four neighbouring blocks meet in one lane, whose word is contiguous in the
// tiled order.  With blocks of 16 a row's largest magnitude comes first: the row stays in registers over that reduction (up to
// kHeld units a thread; longer rows are read again, from L2).
#include "fp4.cuh"
#include "ops.cuh"

namespace w8a8 {

namespace {

constexpr int kHeld = 2;  // units of a row that a thread keeps

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
// The bits of the largest magnitude: as integers, so that NaN and infinities are above everything.
__device__ __forceinline__ uint32_t top_of(const float (&x)[16]) {
  uint32_t t = 0;
#pragma unroll
  for (int e = 0; e < 16; ++e) t = max(t, __float_as_uint(x[e]) & 0x7fffffffu);
  return t;
}
// Codes of 16 values in units already divided out.
__device__ __forceinline__ uint2 codes16(const float (&q)[16]) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    w[h] = e2m1x2_of(q[8 * h], q[8 * h + 1]) | e2m1x2_of(q[8 * h + 2], q[8 * h + 3]) << 8 |
           e2m1x2_of(q[8 * h + 4], q[8 * h + 5]) << 16 | e2m1x2_of(q[8 * h + 6], q[8 * h + 7]) << 24;
  return make_uint2(w[0], w[1]);
}

// One unit: its codes, and its block's scale byte (both lanes of a block of 32 have it).  `top` of this unit; s2 the reciprocal of
// the row's scale (blocks of 16).  All lanes of a warp.
template <int kBlock>
__device__ __forceinline__ uint32_t quantise_unit(const float (&x)[16], uint32_t top, float s2, uint2& codes) {
  float q[16];
  if constexpr (kBlock == 16) {
    Block16 b;
    b.unit(top, s2);
#pragma unroll
    for (int e = 0; e < 16; ++e) q[e] = b.byte == kE4m3NaN ? 0.0f : b.over(x[e] * s2);
    codes = codes16(q);
    return b.byte;
  } else {
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const int e8 = top >= 0x7f800000u ? (int)kE8m0NaN : max((int)(top >> 23) - 2, 0);  // 2^(e8 - 127)
    // 2^(127 - e8), a normal number but for e8 = 254, which no finite block has (253 - 2 at most); x times it is exact, or so
    // small that its code is 0
    const float inv = __uint_as_float((uint32_t)(254 - e8) << 23);
#pragma unroll
    for (int e = 0; e < 16; ++e) q[e] = top >= 0x7f800000u ? 0.0f : x[e] * inv;
    codes = codes16(q);
    return (uint32_t)e8;
  }
}

// kWarp: tpr (a power of two, kBlock / 4 to 32) neighbouring lanes take a row, else a block takes one.
template <int kType, int kBlock, bool kWarp>
__global__ void __launch_bounds__(512) fp4_quantise_kernel(const char* __restrict__ x, int64_t x_row_bytes, int rows, int padded,
                                                           int k, int tpr, uint8_t* __restrict__ codes,
                                                           uint8_t* __restrict__ scales, float* __restrict__ row_scale,
                                                           int settled) {
  __shared__ uint32_t s_top[16];
  if (settled) pdl_trigger();
  pdl_wait();
  if (!settled) pdl_trigger();
  const int units = k / 16, groups = fp4_groups(k, kBlock), lane = threadIdx.x & 31;
  const int step = kWarp ? tpr : (int)blockDim.x;
  const int64_t row = kWarp ? ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / tpr : (int64_t)blockIdx.x;
  const int u0 = kWarp ? (int)(threadIdx.x & (tpr - 1)) : (int)threadIdx.x;
  const bool live = row < rows;
  const char* src = x + row * x_row_bytes;
  Unit16<kType> held[kHeld];
  uint32_t tops[kHeld];
  float v[16], s2 = 1.0f;
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (live && u0 + i * step < units) held[i] = load_unit<kType>(src, u0 + i * step);
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    tops[i] = 0;
    if (live && u0 + i * step < units) {
      unit_floats<kType>(held[i], v);
      tops[i] = top_of(v);
    }
  }
  if constexpr (kBlock == 16) {
    uint32_t top = 0;  // of the blocks that are finite
#pragma unroll
    for (int i = 0; i < kHeld; ++i) top = max(top, tops[i] < 0x7f800000u ? tops[i] : 0u);
    for (int u = u0 + kHeld * step; live && u < units; u += step) {
      unit_floats<kType>(load_unit<kType>(src, u), v);
      const uint32_t t = top_of(v);
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
  // every lane makes the same trips: the scales' exchange is a whole warp's
  for (int i = 0, first = kWarp ? 0 : (int)(threadIdx.x & ~31u); first < units; ++i, first += step) {
    const int u = u0 + i * step;
    const bool here = live && u < units;
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = 0.0f;
    if (here) {
      if (i < kHeld) {  // (unrolled, so that what is held stays in registers)
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
          if (i == j) {
            unit_floats<kType>(held[j], v);
            top = tops[j];
          }
      } else {
        unit_floats<kType>(load_unit<kType>(src, u), v);
        top = top_of(v);
      }
    }
    uint2 c;
    uint32_t byte = quantise_unit<kBlock>(v, top, s2, c);
    if (here) *reinterpret_cast<uint2*>(codes + row * (int64_t)(k / 2) + 8 * u) = c;
    // the bytes of four blocks in their first lane
    constexpr int kStep = kBlock / 16;  // lanes a block
    const int j = u / kStep;
    byte = here ? byte : 0u;
    byte <<= 8 * (j & 3);
    byte |= __shfl_xor_sync(0xffffffffu, byte, kStep);
    byte |= __shfl_xor_sync(0xffffffffu, byte, 2 * kStep);
    if ((u & (4 * kStep - 1)) == 0 && u < units && row < padded)
      *reinterpret_cast<uint32_t*>(scales + fp4_scale_at(row, j, groups)) = byte;
  }
}

template <int kType>
__global__ void __launch_bounds__(256) fp4_dequantise_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                             const float* __restrict__ row_scale, int64_t total, int units,
                                                             int block, int groups, char* __restrict__ y, int64_t y_row_bytes) {
  pdl_wait();
  pdl_trigger();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const int64_t row = i / units;
  const int u = (int)(i - row * units);
  const uint2 c = *reinterpret_cast<const uint2*>(codes + i * 8);
  const uint32_t byte = scales[fp4_scale_at(row, block == 16 ? u : u >> 1, groups)];
  float a, b = 1.0f;
  if (block == 16) {
    a = e4m3_value(byte);
    b = row_scale[row];
  } else {
    a = byte == kE8m0NaN ? NAN : byte == 0 ? 0x1p-127f : __uint_as_float(byte << 23);
  }
  float v[16];
  uint32_t h[8];
  uint32_t(&h0)[4] = *reinterpret_cast<uint32_t(*)[4]>(h), (&h1)[4] = *reinterpret_cast<uint32_t(*)[4]>(h + 4);
  e2m1x8_to_f16(c.x, h0);
  e2m1x8_to_f16(c.y, h1);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float2 f = unpack2<false>(h[e]);
    v[2 * e] = f.x * a * b;
    v[2 * e + 1] = f.y * a * b;
  }
  constexpr int kBytes = kType == W8A8_TYPE_F32 ? 64 : 32;
  uint4* to = reinterpret_cast<uint4*>(y + row * y_row_bytes + (int64_t)u * kBytes);
  if constexpr (kType == W8A8_TYPE_F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      to[e] = make_uint4(__float_as_uint(v[4 * e]), __float_as_uint(v[4 * e + 1]), __float_as_uint(v[4 * e + 2]),
                         __float_as_uint(v[4 * e + 3]));
  } else {
    constexpr bool kBf = kType == W8A8_TYPE_BF16;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      to[e] = make_uint4(pack2<kBf>(v[8 * e], v[8 * e + 1]), pack2<kBf>(v[8 * e + 2], v[8 * e + 3]),
                         pack2<kBf>(v[8 * e + 4], v[8 * e + 5]), pack2<kBf>(v[8 * e + 6], v[8 * e + 7]));
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
  W8A8_CHECK_ARG(q->rows >= 0 && q->k > 0 && q->k % 32 == 0 && q->k <= W8A8_MAX_K, W8A8_ERR_SHAPE,
                 "%s: rows %d, k %d: k must be a multiple of 32, at most %d", who, q->rows, q->k, W8A8_MAX_K);
  if (q->rows == 0) return W8A8_OK;
  W8A8_CHECK_ARG(q->codes && q->scales && (q->block == 32 || q->row_scale), W8A8_ERR_INVALID_ARG, "%s: null pointer", who);
  W8A8_CHECK_ARG(aligned16(q->codes) && aligned16(q->scales) && aligned16(q->row_scale), W8A8_ERR_ALIGN,
                 "%s: codes, scales and row_scale must be 16-byte aligned", who);
  return W8A8_OK;
}

// Lanes of a warp share its rows while a row's units fit; then a block a row, of as few threads as leave kHeld units to each.
w8a8_status launch_fp4_quantize(int dtype, const void* x, int64_t x_row, const w8a8_fp4& q, bool pad, bool settled,
                                cudaStream_t st) {
  const int units = q.k / 16, padded = pad ? (int)round_up((size_t)q.rows, 128) : q.rows;
  int tpr = q.block / 4;  // four blocks' scales meet within a row's lanes
  while (tpr < units && tpr < 32) tpr *= 2;
  const bool warp = units <= 32;
  const int threads = warp ? 128 : units <= 512 ? (int)round_up((size_t)units, 32) : 512;
  const int64_t blocks = warp ? ((int64_t)padded * tpr + 127) / 128 : padded;
  auto go = [&](auto kernel) {
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3((unsigned)threads), 0, st, static_cast<const char*>(x),
                      x_row * type_bytes(dtype), q.rows, padded, q.k, tpr, q.codes, q.scales, q.row_scale, (int)settled);
  };
  auto of = [&](auto type) {
    constexpr int kT = decltype(type)::value;
    if (q.block == 16) return warp ? go(fp4_quantise_kernel<kT, 16, true>) : go(fp4_quantise_kernel<kT, 16, false>);
    return warp ? go(fp4_quantise_kernel<kT, 32, true>) : go(fp4_quantise_kernel<kT, 32, false>);
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
  W8A8_CHECK_ARG(rows >= 0 && k > 0 && k % 32 == 0 && k <= W8A8_MAX_K, W8A8_ERR_SHAPE,
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
  W8A8_CHECK_ARG(q->rows <= 0x7fffff80, W8A8_ERR_SHAPE, "%s: %d rows", who, q->rows);
  W8A8_TRY(check_device());
  return launch_fp4_quantize(dtype, x, x_row, *q, true, false, as_stream(stream));
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
  const int units = q->k / 16;
  const int64_t total = (int64_t)q->rows * units, blocks = (total + 255) / 256;
  W8A8_CHECK_ARG(blocks <= 0x7fffffffll, W8A8_ERR_SHAPE, "%s: [%d, %d] is too large", who, q->rows, q->k);
  auto go = [&](auto kernel) {
    return launch_pdl(kernel, dim3((unsigned)blocks), dim3(256), 0, as_stream(stream), (const uint8_t*)q->codes,
                      (const uint8_t*)q->scales, (const float*)q->row_scale, total, units, q->block,
                      fp4_groups(q->k, q->block), static_cast<char*>(y), y_row * type_bytes(dtype));
  };
  W8A8_CUDA(dtype == W8A8_TYPE_BF16  ? go(fp4_dequantise_kernel<W8A8_TYPE_BF16>)
            : dtype == W8A8_TYPE_F16 ? go(fp4_dequantise_kernel<W8A8_TYPE_F16>)
                                     : go(fp4_dequantise_kernel<W8A8_TYPE_F32>));
  return W8A8_OK;
}
