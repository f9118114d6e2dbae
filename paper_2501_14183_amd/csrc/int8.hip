// Products in 8-bit integers with a scale for each token and each output channel, for a model that answers.
//
//   s_t = max |x_t| / 127,  q_t = round(x_t (127 / max |x_t|));  the same for the columns of W;  y = act(s_t s_c (q_t . q_c) + b_c)
//
// Integer products and sums are exact; what is rounded is the codes, and the result.  Codes lie along k in rows of whole 128-byte
// stages, zeros behind the last, which is what the matrix instruction's tiles (tile_gemm.h) read.
#include "pack8.h"
#include "tile_gemm.h"

namespace {

constexpr int kMaxI8K = 65536;                        // 127^2 K < 2^31
constexpr float kLeastRow = 7.8886090522101181e-31f;  // 2^-100: rows below count as zeros (127 / max would not be finite for the smallest)

__host__ __device__ inline int i8_pitch(int K) { return (K + 127) / 128 * 128; }

// scale and its reciprocal of a row whose largest magnitude has these bits; a row that holds an infinity or NaN gets NaN
__device__ inline void i8_scales(uint32_t most, float& scale, float& up) {
  const float m = __uint_as_float(most);
  const bool some = m >= kLeastRow;
  scale = most >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : (some ? m / 127.f : 0.f);
  up = some && most < 0x7f800000u ? 127.f / m : 0.f;
}
// (the product is rounded before it is rounded to a whole number: a fused one would break ties of its own)
__device__ inline uint32_t i8_code(float v, float up) {
#pragma clang fp contract(off)
  const float p = v * up;
  return __float_as_uint(p + 12582912.f) & 0xffu;
}

__device__ inline uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m, 64));
  return v;
}

// A wavefront a row, any width and alignment.
template <typename T>
__global__ __launch_bounds__(256) void i8_rows_kernel(const T* x, long long rows, int K, uint8_t* q, float* scale) {
  const int lane = threadIdx.x & 63, pitch = i8_pitch(K);
  for (long long r = blockIdx.x * 4ll + (threadIdx.x >> 6); r < rows; r += gridDim.x * 4ll) {
    const T* row = x + r * K;
    uint32_t most = 0;
    for (int k = lane; k < K; k += 64) most = max(most, magnitude(to_float(row[k])));
    most = wave_max(most);
    float s, up;
    i8_scales(most, s, up);
    for (int k = lane; k < pitch; k += 64) q[r * pitch + k] = k < K ? (uint8_t)i8_code(up == 0.f ? 0.f : to_float(row[k]), up) : 0;
    if (lane == 0) scale[r] = s;
  }
}
// The same for rows of whole groups of eight that 64 lanes hold in U groups each: read once.
template <typename T, int U>
__global__ __launch_bounds__(256) void i8_rows_whole_kernel(const T* x, long long rows, int K, uint8_t* q, float* scale) {
  const int lane = threadIdx.x & 63, pitch = i8_pitch(K);
  for (long long r = blockIdx.x * 4ll + (threadIdx.x >> 6); r < rows; r += gridDim.x * 4ll) {
    float v[U][8];
    uint32_t most = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = (u * 64 + lane) * 8;
      if (k < K) load_eight(x + r * K + k, v[u]);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] = 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, magnitude(v[u][e]));
    most = wave_max(most);
    float s, up;
    i8_scales(most, s, up);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = (u * 64 + lane) * 8;
      uint32_t c[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = i8_code(up == 0.f ? 0.f : v[u][e], up);
      if (k < pitch)
        *reinterpret_cast<u32x2*>(q + r * pitch + k) = u32x2{pack_four(c[0], c[1], c[2], c[3]), pack_four(c[4], c[5], c[6], c[7])};
    }
    if (lane == 0) scale[r] = s;
  }
}

// Columns of W [K][N] as rows of codes: 32 columns a workgroup, their largest magnitudes first, then 32 x 32 blocks turned in LDS.
template <typename T>
__global__ __launch_bounds__(256) void i8_weight_kernel(const T* W, int K, int N, uint8_t* q, float* scale) {
  __shared__ uint32_t red[8][32];
  __shared__ uint8_t tile[32][33];
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5, n = blockIdx.x * 32 + c, pitch = i8_pitch(K);
  uint32_t most = 0;
  if (n < N)
    for (int k = g; k < K; k += 8) most = max(most, magnitude(to_float(W[(long long)k * N + n])));
  red[g][c] = most;
  __syncthreads();
  for (int i = 0; i < 8; ++i) most = max(most, red[i][c]);
  float s, up;
  i8_scales(most, s, up);
  if (g == 0 && n < N) scale[n] = s;
  for (int k0 = 0; k0 < pitch; k0 += 32) {
    __syncthreads();
    for (int i = g; i < 32; i += 8) {
      const int k = k0 + i;
      tile[i][c] = n < N && k < K && up != 0.f ? (uint8_t)i8_code(to_float(W[(long long)k * N + n]), up) : 0;
    }
    __syncthreads();
    for (int i = g; i < 32; i += 8) {
      const int row = blockIdx.x * 32 + i;
      if (row < N) q[(long long)row * pitch + k0 + c] = tile[c][i];
    }
  }
}

template <typename T, int ACT>
struct EpiI8 {
  struct Args {
    T* y;
    const float *sx, *sw;
    const T* bias;
    int N, whole;              // whole: rows of y can be stored in groups of eight
  } a;
  float w[8], b[8];
  __device__ void columns(int n, int N) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = n + e < N ? a.sw[n + e] : 0.f;
      b[e] = a.bias && n + e < N ? to_float(a.bias[n + e]) : 0.f;
    }
  }
  __device__ void done(int, int, bool) {}
  __device__ void row(int, int m, int n, bool live, float (&v)[8]) {
    if (!live) return;
    const float s = a.sx[m];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act_value<ACT, sizeof(T) == 4>(v[e] * s * w[e] + b[e]);
    T* p = a.y + (long long)m * a.N + n;
    if (a.whole) {
      store_eight(p, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (n + e < a.N) from_float(p + e, v[e]);
    }
  }
};

template <typename T, int ACT>
int i8_product(vardrop_ctx* ctx, const void* q, const float* sx, int rows, int K, int N, const void* wq, const float* sw, const void* bias, void* y,
               hipStream_t s) {
  TileArgs g = {};
  g.A = q; g.B = wq;
  g.K = i8_pitch(K);
  g.lda = g.ldb = g.K;
  g.M = rows; g.N = N; g.slices = 1;
  const typename EpiI8<T, ACT>::Args epi = {(T*)y, sx, sw, (const T*)bias, N, N % 8 == 0 && vd_aligned(y, 16)};
  const long long t128 = (long long)vd_ceil_div(N, 128) * vd_ceil_div(rows, 128);
  if (t128 >= 512) return launch_tile_gemm<true, true, true, Tile128, EpiI8<T, ACT>>(ctx, VARDROP_K_LINEAR_I8, g, epi, s);
  return launch_tile_gemm<true, true, true, Tile64, EpiI8<T, ACT>>(ctx, VARDROP_K_LINEAR_I8, g, epi, s);
}

template <typename T>
int quantize(vardrop_ctx* ctx, const T* x, long long rows, int K, uint8_t* q, float* scale, hipStream_t s) {
  const dim3 grid((unsigned)((rows + 3) / 4 > 8192 ? 8192 : (rows + 3) / 4));
  const bool whole = K % 8 == 0 && vd_aligned(x, 16) && i8_pitch(K) <= 2048;
  VdTimer timer(ctx, VARDROP_K_QUANTIZE, s);
  if (!whole) VD_KERNEL(ctx, i8_rows_kernel<T>, grid, dim3(256), 0, s, x, rows, K, q, scale);
  else if (i8_pitch(K) <= 512) VD_KERNEL(ctx, (i8_rows_whole_kernel<T, 1>), grid, dim3(256), 0, s, x, rows, K, q, scale);
  else if (i8_pitch(K) <= 1024) VD_KERNEL(ctx, (i8_rows_whole_kernel<T, 2>), grid, dim3(256), 0, s, x, rows, K, q, scale);
  else VD_KERNEL(ctx, (i8_rows_whole_kernel<T, 4>), grid, dim3(256), 0, s, x, rows, K, q, scale);
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

bool is_type(int dtype) { return dtype == VARDROP_F32 || dtype == VARDROP_BF16; }
size_t element(int dtype) { return dtype == VARDROP_BF16 ? 2 : 4; }

}  // namespace

extern "C" int vardrop_i8_pitch(int K) { return K < 1 || K > kMaxI8K ? 0 : i8_pitch(K); }

extern "C" int vardrop_quantize_rows(vardrop_ctx* ctx, const void* x, int rows, int K, int dtype, void* codes, float* scale, void* stream) {
  if (!ctx || rows < 0 || K < 1 || !is_type(dtype)) return VARDROP_EINVAL;
  if (K > kMaxI8K) return VARDROP_EUNSUPPORTED;
  if (rows == 0) return VARDROP_OK;
  if (!x || !codes || !scale || !vd_aligned(x, element(dtype)) || !vd_aligned(codes, 16) || !vd_aligned(scale, 4)) return VARDROP_EINVAL;
  if (dtype == VARDROP_BF16) return quantize<bf16_t>(ctx, (const bf16_t*)x, rows, K, (uint8_t*)codes, scale, (hipStream_t)stream);
  return quantize<float>(ctx, (const float*)x, rows, K, (uint8_t*)codes, scale, (hipStream_t)stream);
}

extern "C" int vardrop_quantize_weight(vardrop_ctx* ctx, const void* W, int K, int N, int dtype, void* codes, float* scale, void* stream) {
  if (!ctx || K < 1 || N < 1 || !is_type(dtype)) return VARDROP_EINVAL;
  if (K > kMaxI8K) return VARDROP_EUNSUPPORTED;
  if (!W || !codes || !scale || !vd_aligned(W, element(dtype)) || !vd_aligned(codes, 16) || !vd_aligned(scale, 4)) return VARDROP_EINVAL;
  VdTimer timer(ctx, VARDROP_K_QUANTIZE, (hipStream_t)stream);
  const dim3 grid((unsigned)vd_ceil_div(N, 32));
  if (dtype == VARDROP_BF16) VD_KERNEL(ctx, i8_weight_kernel<bf16_t>, grid, dim3(256), 0, (hipStream_t)stream, (const bf16_t*)W, K, N, (uint8_t*)codes, scale);
  else VD_KERNEL(ctx, i8_weight_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, (const float*)W, K, N, (uint8_t*)codes, scale);
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

extern "C" size_t vardrop_linear_i8_workspace_bytes(int rows, int K, int N) {
  if (rows < 0 || K < 1 || N < 1 || K > kMaxI8K) return 0;
  return vd_align_up((size_t)rows * i8_pitch(K), 256) + vd_align_up((size_t)rows * 4, 256);
}

extern "C" int vardrop_linear_i8(vardrop_ctx* ctx, const void* x, const float* sx, int rows, int K, int N, int x_dtype, const void* codes,
                                 const float* scale, const void* bias, int act, void* y, int dtype, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx || rows < 0 || K < 1 || N < 1 || !is_type(dtype) || (!is_type(x_dtype) && x_dtype != VARDROP_I8)) return VARDROP_EINVAL;
  if (act != VARDROP_ACT_NONE && act != VARDROP_ACT_RELU && act != VARDROP_ACT_GELU) return VARDROP_EINVAL;
  if (K > kMaxI8K || (long long)vd_ceil_div(rows, 64) * vd_ceil_div(N, 128) >= (1ll << 31)) return VARDROP_EUNSUPPORTED;
  if ((x_dtype == VARDROP_I8) != (sx != nullptr) && rows > 0) return VARDROP_EINVAL;
  if (rows == 0) return VARDROP_OK;
  if (!x || !codes || !scale || !y || x == y) return VARDROP_EINVAL;
  if (!vd_aligned(x, x_dtype == VARDROP_I8 ? 16 : element(x_dtype)) || !vd_aligned(codes, 16) || !vd_aligned(scale, 4) || !vd_aligned(sx, 4) ||
      !vd_aligned(y, element(dtype)) || !vd_aligned(bias, element(dtype)))
    return VARDROP_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  const void* q = x;
  if (x_dtype != VARDROP_I8) {
    if (!ws || !vd_aligned(ws, 256) || ws_bytes < vardrop_linear_i8_workspace_bytes(rows, K, N)) return VARDROP_EWORKSPACE;
    float* made = (float*)((char*)ws + vd_align_up((size_t)rows * i8_pitch(K), 256));
    const int rc = vardrop_quantize_rows(ctx, x, rows, K, x_dtype, ws, made, stream);
    if (rc) return rc;
    q = ws;
    sx = made;
  }
#define VD_I8(T)                                                                                                       \
  (act == VARDROP_ACT_NONE ? i8_product<T, kActNone>(ctx, q, sx, rows, K, N, codes, scale, bias, y, s)                 \
   : act == VARDROP_ACT_RELU ? i8_product<T, kActRelu>(ctx, q, sx, rows, K, N, codes, scale, bias, y, s)               \
                             : i8_product<T, kActGelu>(ctx, q, sx, rows, K, N, codes, scale, bias, y, s))
  return dtype == VARDROP_BF16 ? VD_I8(bf16_t) : VD_I8(float);
#undef VD_I8
}
