// Products in 8-bit integers with a scale for each token and each output channel, for a model that answers.
//
//   s_t = max |x_t| / 127,  q_t = round(x_t (127 (1 / max |x_t|)));  the same for the columns of W;  y = act(s_t s_c (q_t . q_c) + b_c)
//
// Integer products and sums are exact; what is rounded is the codes, and the result.  Codes lie along k in rows of whole 128-byte
// stages, zeros behind the last, which is what the matrix instruction's tiles (tile_gemm.h) read.
#include "pack8.h"
#include "tile_gemm.h"

namespace {

constexpr int kMaxI8K = 65536;                        // 127^2 K < 2^31
constexpr int kMaxI8Rows = 1 << 30;
constexpr float kLeastRow = 7.8886090522101181e-31f;  // 2^-100: rows below count as zeros (1 / max would not be finite for the smallest)

__host__ __device__ inline int i8_pitch(int K) { return (K + 127) / 128 * 128; }

// scale and 127 / max of a row whose largest magnitude has these bits; a row that holds an infinity or NaN gets NaN.
// (127 (1 / max), two roundings, is how array libraries divide a number by a tensor: who quantises weights with one gets the same codes.)
__device__ inline void i8_scales(uint32_t most, float& scale, float& up) {
  const float m = __uint_as_float(most);
  const bool some = m >= kLeastRow;
  scale = most >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : (some ? m / 127.f : 0.f);
  up = some && most < 0x7f800000u ? 127.f * (1.f / m) : 0.f;
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

// A wavefront a row, any width and alignment: rows are read twice, the second time from the caches.
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
// The same for rows of whole groups of eight that 64 lanes hold in U groups each: read once, 16 bytes at a time.  us, by elements -> by groups:
// 27 584 x 512 in bf16 21.7 -> 9.3 (4.6 TB/s), 65 536 x 768 in bf16 64.6 -> 25.9, in fp32 76.8 -> 36.3, 2000 x 2048 in bf16 12.0 -> 3.8.
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

// Columns of W [K][N] as rows of codes: 32 columns a workgroup, their largest magnitudes first, then 32 x 32 blocks turned in LDS.  Bound by each workgroup's
// own chain over K, twice, with a two-byte load a lane: 512 x 2048 in bf16 25 us (64 workgroups), 2048 x 2048 94.  It runs once for a weight.
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

// act(v) chosen at run time: what it costs beside the product is a branch
template <typename T>
__device__ inline float i8_act(float v, int act) {
  return act == kActNone ? v : act == kActRelu ? act_value<kActRelu, true>(v) : act_value<kActGelu, sizeof(T) == 4>(v);
}

template <typename T>
struct EpiI8 {
  static constexpr bool kFetch = false, kSums = false;
  static constexpr int kPartsA = 1, kPartsB = 1, kRowSums = 0;
  struct Args {
    T* y;
    const float *sx, *sw;      // sx[0] is row m0's
    const T* bias;
    int m0, N, act, whole;     // whole: rows of y can be stored in groups of eight
    int past;
  } a;
  float w[8], b[8];
  __device__ void columns(int n, int N) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = n + e < N ? a.sw[n + e] : 0.f;
      b[e] = a.bias && n + e < N ? to_float(a.bias[n + e]) : 0.f;
    }
  }
  __device__ void row(int, int, int m, int n, bool live, float (&v)[8]) {
    if (!live) return;
    const float s = a.sx[m - a.m0];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] * s * w[e] + b[e];
    if (a.act == kActRelu) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = act_value<kActRelu, true>(v[e]);
    } else if (a.act == kActGelu) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = act_value<kActGelu, sizeof(T) == 4>(v[e]);
    }
    T* p = a.y + (long long)m * a.N + n;
    if (a.whole) {
      store_eight(p, v, a.past);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (n + e < a.N) from_float(p + e, v[e]);
    }
  }
};

// What a call has in hand.
struct I8Call {
  vardrop_ctx* ctx;
  const void* x;
  const float* sx;
  int rows, K, N;
  const uint8_t* codes;
  const float* scale;
  const void* bias;
  int act;
  void* y;
  hipStream_t s;
};

template <typename T>
int i8_product(const I8Call& c) {
  TileArgs g = {};
  g.A = c.x; g.B = c.codes;
  g.K = i8_pitch(c.K);
  g.lda = g.ldb = g.K;
  g.M = c.rows; g.N = c.N; g.slices = 1;
  const typename EpiI8<T>::Args epi = {(T*)c.y, c.sx, c.scale, (const T*)c.bias, 0, c.N, c.act, c.N % 8 == 0 && vd_aligned(c.y, 16),
                                      (long long)c.rows * c.N * (long long)sizeof(T) >= kPastCaches};
#define VD_CALL(S) launch_tile_gemm<true, true, true, S, EpiI8<T>>(c.ctx, VARDROP_K_LINEAR_I8, g, epi, c.s)
  return VD_BY_SHAPE(product_shape(kRowShapes, c.rows, c.N, g.K / 2), VD_CALL, TileWide);
#undef VD_CALL
}

// ---- quantisation and product in one launch, while a tile's rows of codes fit LDS beside the stages of the weight: every workgroup makes
// the codes of its own 32 rows (16 lanes a row), which the workgroups of the other columns make again.  32 and not 64 rows: twice the
// workgroups, half the rows for each to wait for.  A chain too: launch, rows, their codes, four stages, the end; 862 x 512 x 720 7.4 us (86 TOPS).
template <typename X>
__device__ inline void load_some(const X* row, int k, int K, bool whole, float (&v)[8]) {
  if (whole && k + 8 <= K) {
    load_eight(row + k, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = k + e < K ? to_float(row[k + e]) : 0.f;
  }
}
typedef TileShape<32, 128, 1, 4, 128, 3> I8Shape;
constexpr int kFusedPitch = 512, kI8Ring = I8Shape::NS * I8Shape::B_BYTES;
inline int i8_fused_lds(int K) { return kI8Ring + 256 + I8Shape::BM * i8_pitch(K); }
template <typename X, typename T>
__global__ __launch_bounds__(256, 2) void i8_fused_kernel(const X* x, int rows, int K, int N, const uint8_t* codes, typename EpiI8<T>::Args args, int whole_x) {
  typedef I8Shape S;
  constexpr int NS = S::NS, LPS = S::B_BYTES / 4096, J = kFusedPitch / 128;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float* sx = reinterpret_cast<float*>(smem + kI8Ring);
  unsigned char* tile = smem + kI8Ring + 256;             // [stage][32 rows][128 bytes], swizzled
  const int pitch = i8_pitch(K), nk = pitch >> 7, gx = (N + 127) >> 7, total = gx * ((rows + 31) >> 5);
  const int t = xcd_contiguous(blockIdx.x, total), n0 = t % gx * 128, m0 = t / gx * 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 31, half = lane >> 5;
  const copy_src src = tile_source(codes + (long long)n0 * pitch, (long long)(N - n0) * pitch);
  uint32_t off[LPS];
#pragma unroll
  for (int u = 0; u < LPS; ++u) {
    const int row = (u * 4 + wave) * 8 + (lane >> 3);
    off[u] = (uint32_t)row * (uint32_t)pitch + (((lane & 7) ^ swz_kc<64>(row)) * 16);
  }
  auto issue = [&](int k, int buf) {
#pragma unroll
    for (int u = 0; u < LPS; ++u) dma16_buf(src, off[u], k * 128u, smem + buf * S::B_BYTES + (u * 4 + wave) * 1024);
  };
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (s < nk) issue(s, s);
  // ---- codes of the tile's rows
  const int l = threadIdx.x & 15;
  float v[2][J][8];
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int m = m0 + p * 16 + (threadIdx.x >> 4);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (m < rows && j < nk) {
        load_some(x + (long long)m * K, (l + 16 * j) * 8, K, whole_x != 0, v[p][j]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[p][j][e] = 0.f;
      }
    }
  }
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int r = p * 16 + (threadIdx.x >> 4);
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, magnitude(v[p][j][e]));
#pragma unroll
    for (int i = 1; i < 16; i <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, i, 64));
    float scale, up;
    i8_scales(most, scale, up);
    if (l == 0) sx[r] = scale;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (j < nk) {
        uint32_t c[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = i8_code(up == 0.f ? 0.f : v[p][j][e], up);
        *reinterpret_cast<u32x2*>(tile + j * S::A_BYTES + r * 128 + (((l >> 1) ^ swz_kc<64>(r)) * 16) + (l & 1) * 8) =
            u32x2{pack_four(c[0], c[1], c[2], c[3]), pack_four(c[4], c[5], c[6], c[7])};
      }
    }
  }
  __syncthreads();
  // ---- product
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;
  const int rb = wave * 32 + col;
  uint32_t addrA[4], addrB[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    addrA[ks] = lds0 + kI8Ring + 256 + col * 128 + (((2 * ks + half) ^ swz_kc<64>(col)) * 16);
    addrB[ks] = lds0 + rb * 128 + (((2 * ks + half) ^ swz_kc<64>(rb)) * 16);
  }
  intx16 acc[1][1];
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[0][0][e] = 0;
  for (int t0 = 0; t0 < nk; t0 += NS) {
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int k = t0 + s;
      if (k < nk) {
        wait_stages<NS - 2, LPS>(nk - 1 - k);
        __builtin_amdgcn_s_barrier();
        if (k + NS - 1 < nk) issue(k + NS - 1, (s + NS - 1) % NS);
        Frag fa[4], fb[4];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          lds_read16(fa[ks].q, addrA[ks] + k * S::A_BYTES);
          lds_read16(fb[ks].q, addrB[ks] + s * S::B_BYTES);
        }
        wait_lds<6>(fa[0], fb[0]);
        acc[0][0] = tile_mfma(fb[0], fa[0], acc[0][0]);
        wait_lds<4>(fa[1], fb[1]);
        acc[0][0] = tile_mfma(fb[1], fa[1], acc[0][0]);
        wait_lds<2>(fa[2], fb[2]);
        acc[0][0] = tile_mfma(fb[2], fa[2], acc[0][0]);
        wait_lds<0>(fa[3], fb[3]);
        acc[0][0] = tile_mfma(fb[3], fa[3], acc[0][0]);
      }
    }
  }
  __syncthreads();
  args.sx = sx;
  args.m0 = m0;
  EpiI8<T> epi{args};
  tile_finish<S, EpiI8<T>>(acc, smem, epi, 0, rows, N, m0, n0);
}

// ---- up to four rows: a workgroup makes their codes and takes 16 columns, 16 lanes each, with the byte dot product.  Its time is a chain: launch,
// rows twice, weights, sums; 1 x 512 x 512 4.3 us.
constexpr int kFewRows = 4, kFewPitch = 1024;
template <typename X, typename T, int R>
__global__ __launch_bounds__(256) void i8_few_kernel(const X* x, int rows, int K, int N, const uint8_t* codes, typename EpiI8<T>::Args a) {
  __shared__ __attribute__((aligned(16))) uint8_t q[R][kFewPitch];
  __shared__ float sx[R];
  constexpr int J = kFewPitch / 256;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, pitch = i8_pitch(K);
  const int n = blockIdx.x * 16 + wave * 4 + (lane >> 4);
  u32x4 w[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int at = (l + 16 * j) * 16;
    w[j] = n < N && at < pitch ? *reinterpret_cast<const u32x4*>(codes + (long long)n * pitch + at) : u32x4{0, 0, 0, 0};
  }
  for (int r = wave; r < R; r += 4) {
    if (r >= rows) break;
    uint32_t most = 0;
    for (int k = lane; k < K; k += 64) most = max(most, magnitude(to_float(x[(long long)r * K + k])));
    most = wave_max(most);
    float scale, up;
    i8_scales(most, scale, up);
    for (int k = lane; k < pitch; k += 64) q[r][k] = k < K && up != 0.f ? (uint8_t)i8_code(to_float(x[(long long)r * K + k]), up) : 0;
    if (lane == 0) sx[r] = scale;
  }
  __syncthreads();
  int sum[R];
#pragma unroll
  for (int r = 0; r < R; ++r) sum[r] = 0;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int at = (l + 16 * j) * 16;
    if (at < pitch) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(&q[r][at]);       // (rows behind the last: whatever is there, not stored)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[r] = __builtin_amdgcn_sdot4((int)v[e], (int)w[j][e], sum[r], false);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 1; i < 16; i <<= 1) sum[r] += __shfl_xor(sum[r], i, 64);
  if (n >= N) return;
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (l == r && r < rows)
      from_float(a.y + (long long)r * N + n, i8_act<T>((float)sum[r] * sx[r] * a.sw[n] + (a.bias ? to_float(a.bias[n]) : 0.f), a.act));
}

template <typename X, typename T>
int i8_one_launch(const I8Call& c) {
  const typename EpiI8<T>::Args a = {(T*)c.y, nullptr, c.scale, (const T*)c.bias, 0, c.N, c.act, c.N % 8 == 0 && vd_aligned(c.y, 16), 0};
  const X* x = (const X*)c.x;
  if (c.rows <= kFewRows && i8_pitch(c.K) <= kFewPitch) {
    const dim3 grid((unsigned)vd_ceil_div(c.N, 16));
    VdTimer timer(c.ctx, VARDROP_K_LINEAR_I8, c.s);
    if (c.rows == 1) VD_KERNEL(c.ctx, (i8_few_kernel<X, T, 1>), grid, dim3(256), 0, c.s, x, c.rows, c.K, c.N, c.codes, a);
    else VD_KERNEL(c.ctx, (i8_few_kernel<X, T, kFewRows>), grid, dim3(256), 0, c.s, x, c.rows, c.K, c.N, c.codes, a);
    VD_LAUNCH_CHECK(c.ctx);
    return VARDROP_OK;
  }
  const int lds = i8_fused_lds(c.K), whole = c.K % 8 == 0 && vd_aligned(x, 16);
  const dim3 grid((unsigned)(vd_ceil_div(c.N, 128) * vd_ceil_div(c.rows, 32)));
  static int configured = -1;
  const int rc = tile_allow_lds(c.ctx, (const void*)i8_fused_kernel<X, T>, i8_fused_lds(kFusedPitch), configured);
  if (rc) return rc;
  VdTimer timer(c.ctx, VARDROP_K_LINEAR_I8, c.s);
  VD_KERNEL(c.ctx, (i8_fused_kernel<X, T>), grid, dim3(256), lds, c.s, x, c.rows, c.K, c.N, c.codes, a, whole);
  VD_LAUNCH_CHECK(c.ctx);
  return VARDROP_OK;
}
// One launch: few rows, or rows whose codes fit beside the stages twice a compute unit while all tiles are resident together.  us, two launches -> one
// (replayed from a graph; issued one by one, two cost the host 2 us more): few rows, 1 x 128 x 512 5.4 -> 3.1, 4 x 512 x 4096 6.2 -> 5.3, 4 x 1024 x
// 4096 7.5 -> 7.2, but 8 x 512 x 512 6.1 -> 8.4, 1 x 2048 x 2048 9.3 -> 9.6; tiles, 2247 x 97 x 321 8.5 -> 7.9, 4000 x 128 x 512 7.6 -> 5.8, 862 x 512 x 720 7.0
// -> 7.4 (bf16) and 7.4 -> 7.0 (fp32), but 64 x 1024 x 1024 7.8 -> 10.6.
bool i8_is_one_launch(const I8Call& c) {
  const int pitch = i8_pitch(c.K);
  if (c.rows <= kFewRows && pitch <= kFewPitch) return true;
  return pitch <= kFusedPitch && (long long)vd_ceil_div(c.rows, 32) * vd_ceil_div(c.N, 128) <= 2 * c.ctx->num_cus;
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
  if (K > kMaxI8K || rows > kMaxI8Rows) return VARDROP_EUNSUPPORTED;
  if (rows == 0) return VARDROP_OK;
  if (!x || !codes || !scale || !vd_aligned(x, element(dtype)) || !vd_aligned(codes, 16) || !vd_aligned(scale, 4)) return VARDROP_EINVAL;
  if (dtype == VARDROP_BF16) return quantize<bf16_t>(ctx, (const bf16_t*)x, rows, K, (uint8_t*)codes, scale, (hipStream_t)stream);
  return quantize<float>(ctx, (const float*)x, rows, K, (uint8_t*)codes, scale, (hipStream_t)stream);
}

extern "C" int vardrop_quantize_weight(vardrop_ctx* ctx, const void* W, int K, int N, int dtype, void* codes, float* scale, void* stream) {
  if (!ctx || K < 1 || N < 1 || !is_type(dtype)) return VARDROP_EINVAL;
  if (K > kMaxI8K || N > kMaxI8Rows) return VARDROP_EUNSUPPORTED;
  if (!W || !codes || !scale || !vd_aligned(W, element(dtype)) || !vd_aligned(codes, 16) || !vd_aligned(scale, 4)) return VARDROP_EINVAL;
  VdTimer timer(ctx, VARDROP_K_QUANTIZE, (hipStream_t)stream);
  const dim3 grid((unsigned)vd_ceil_div(N, 32));
  if (dtype == VARDROP_BF16) VD_KERNEL(ctx, i8_weight_kernel<bf16_t>, grid, dim3(256), 0, (hipStream_t)stream, (const bf16_t*)W, K, N, (uint8_t*)codes, scale);
  else VD_KERNEL(ctx, i8_weight_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, (const float*)W, K, N, (uint8_t*)codes, scale);
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

extern "C" size_t vardrop_linear_i8_workspace_bytes(int rows, int K, int N) {
  if (rows < 0 || K < 1 || N < 1 || K > kMaxI8K || rows > kMaxI8Rows || N > kMaxI8Rows) return 0;
  return vd_align_up((size_t)rows * i8_pitch(K), 256) + vd_align_up((size_t)rows * 4, 256);
}

extern "C" int vardrop_linear_i8(vardrop_ctx* ctx, const void* x, const float* sx, int rows, int K, int N, int x_dtype, const void* codes,
                                 const float* scale, const void* bias, int act, void* y, int dtype, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx || rows < 0 || K < 1 || N < 1 || !is_type(dtype) || (!is_type(x_dtype) && x_dtype != VARDROP_I8)) return VARDROP_EINVAL;
  if (act != VARDROP_ACT_NONE && act != VARDROP_ACT_RELU && act != VARDROP_ACT_GELU) return VARDROP_EINVAL;
  if (K > kMaxI8K || rows > kMaxI8Rows || N > kMaxI8Rows || (long long)vd_ceil_div(rows, 32) * vd_ceil_div(N, 64) >= (1ll << 31)) return VARDROP_EUNSUPPORTED;
  if ((x_dtype == VARDROP_I8) != (sx != nullptr) && rows > 0) return VARDROP_EINVAL;
  if (rows == 0) return VARDROP_OK;
  if (!x || !codes || !scale || !y || x == y) return VARDROP_EINVAL;
  if (!vd_aligned(x, x_dtype == VARDROP_I8 ? 16 : element(x_dtype)) || !vd_aligned(codes, 16) || !vd_aligned(scale, 4) || !vd_aligned(sx, 4) ||
      !vd_aligned(y, element(dtype)) || !vd_aligned(bias, element(dtype)))
    return VARDROP_EINVAL;
  I8Call c = {ctx, x, sx, rows, K, N, (const uint8_t*)codes, scale, bias, act, y, (hipStream_t)stream};
  if (x_dtype != VARDROP_I8) {
    if (!ws || !vd_aligned(ws, 256) || ws_bytes < vardrop_linear_i8_workspace_bytes(rows, K, N)) return VARDROP_EWORKSPACE;
    if (i8_is_one_launch(c)) {
      if (x_dtype == VARDROP_BF16) return dtype == VARDROP_BF16 ? i8_one_launch<bf16_t, bf16_t>(c) : i8_one_launch<bf16_t, float>(c);
      return dtype == VARDROP_BF16 ? i8_one_launch<float, bf16_t>(c) : i8_one_launch<float, float>(c);
    }
    float* made = (float*)((char*)ws + vd_align_up((size_t)rows * i8_pitch(K), 256));
    const int rc = vardrop_quantize_rows(ctx, x, rows, K, x_dtype, ws, made, stream);
    if (rc) return rc;
    c.x = ws;
    c.sx = made;
  }
  return dtype == VARDROP_BF16 ? i8_product<bf16_t>(c) : i8_product<float>(c);
}
