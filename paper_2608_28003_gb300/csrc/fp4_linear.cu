// The linear in floating point of 4 bits, in its simplest form: a block takes 16 x 64 outputs and walks k 32 columns at a time.
#include "fp4.cuh"
#include "ops.cuh"

namespace w8a8 {

namespace {

struct Side {
  const uint8_t *codes, *scales;
  const float* row_scale;
};

__device__ __forceinline__ float unit_of(const Side& s, int64_t row, int col, int block, int groups) {
  const uint32_t byte = s.scales[fp4_scale_at(row, col / block, groups)];
  if (block == 16) return e4m3_value(byte);
  return byte == kE8m0NaN ? NAN : byte == 0 ? 0x1p-127f : __uint_as_float(byte << 23);
}

__global__ void __launch_bounds__(256) fp4_linear_kernel(Side w, Side x, int M, int N, int k, int block, const float* bias,
                                                         int out, void* y, int64_t y_row) {
  __shared__ float sx[16][33], sw[64][33];
  pdl_wait();
  pdl_trigger();
  const int n0 = blockIdx.x * 64, groups = fp4_groups(k, block);
  for (int m0 = blockIdx.y * 16; m0 < M; m0 += gridDim.y * 16) {
    float acc[4] = {};
    const int tm = threadIdx.x >> 4, tn = threadIdx.x & 15;
    for (int k0 = 0; k0 < k; k0 += 32) {
      __syncthreads();
      for (int i = threadIdx.x; i < 80 * 4; i += 256) {  // eight columns of a row
        const int r = i >> 2, c = k0 + 8 * (i & 3);
        const bool is_x = r < 16;
        const int64_t row = is_x ? m0 + r : n0 + r - 16;
        const Side& s = is_x ? x : w;
        uint32_t codes = 0;
        float u = 0.0f;
        if (row < (is_x ? M : N)) {
          codes = *reinterpret_cast<const uint32_t*>(s.codes + (row * k + c) / 2);
          u = unit_of(s, row, c, block, groups);
        }
        uint32_t h[4];
        e2m1x8_to_f16(codes, h);
        float* to = is_x ? &sx[r][8 * (i & 3)] : &sw[r - 16][8 * (i & 3)];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = unpack2<false>(h[e]);
          to[2 * e] = f.x * u;
          to[2 * e + 1] = f.y * u;
        }
      }
      __syncthreads();
#pragma unroll
      for (int c = 0; c < 32; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = fmaf(sx[tm][c], sw[tn + 16 * j][c], acc[j]);
    }
    const int m = m0 + tm;
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + tn + 16 * j;
      if (m >= M || n >= N) continue;
      float v = acc[j];
      if (block == 16) v = v * w.row_scale[n] * x.row_scale[m];
      if (bias) v += bias[n];
      if (out == W8A8_TYPE_F32)
        static_cast<float*>(y)[m * y_row + n] = v;
      else
        static_cast<uint16_t*>(y)[m * y_row + n] =
            (uint16_t)(out == W8A8_TYPE_BF16 ? pack2<true>(v, 0.0f) : pack2<false>(v, 0.0f));
    }
  }
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
  W8A8_CHECK_ARG(M >= 0 && N >= 0 && K > 0 && K % 32 == 0 && K <= W8A8_MAX_K, W8A8_ERR_SHAPE, "%s: M=%d N=%d K=%d", who, M, N,
                 K);
  *bytes = linear_fp4_ws(M, K, block).total;
  return W8A8_OK;
}

extern "C" w8a8_status w8a8_fp4_linear(const w8a8_fp4* w, int dtype, const void* X, int64_t x_row, int M, const float* bias,
                                       int out_dtype, void* Y, int64_t y_row, void* workspace, size_t ws_bytes, void* stream) {
  const char* who = "w8a8_fp4_linear";
  W8A8_TRY(check_fp4(who, w));
  W8A8_CHECK_ARG(M >= 0, W8A8_ERR_INVALID_ARG, "%s: M=%d is negative", who, M);
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
  W8A8_TRY(launch_fp4_quantize(dtype, X, x_row, x, false, false, st));
  const Side ws{w->codes, w->scales, w->row_scale}, xs{x.codes, x.scales, x.row_scale};
  const unsigned gy = (unsigned)((M + 15) / 16 < 65535 ? (M + 15) / 16 : 65535);
  W8A8_CUDA(launch_pdl(fp4_linear_kernel, dim3((unsigned)((N + 63) / 64), gy), dim3(256), 0, st, ws, xs, M, N, K, (int)w->block,
                       bias, out_dtype, Y, y_row));
  return W8A8_OK;
}
