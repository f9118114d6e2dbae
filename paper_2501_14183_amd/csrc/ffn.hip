// The feed-forward block, the other half of an encoder layer beside the attention (Sec. 4.1), whose activations wait for the
// backward pass in 8 bits.
//
//   h = x W1 + b1,  a = act(h),  y = a W2 + b2            kept: x and h, packed (pack8.h)
//   dh = (dy W2^T) act'(h'),  dx = dh W1^T,  dW1 = x'^T dh,  db1 = sum dh,  dW2 = act(h')^T dy,  db2 = sum dy
//
// with x', h' what the checkpoints stand for.  bf16: the element-wise work is done on the products' sums before they are
// stored (tile_gemm.h): h never exists outside a tile, dy W2^T neither.
#include "gemm_f32.h"
#include "pack8.h"
#include "tile_gemm.h"

namespace {

// ---- what is done to the rows of a product
// eight columns' biases
__device__ inline void bias_eight(const bf16_t* b, int n, int N, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  if (b && n < N) load_eight(b + n, v);
}

struct EpiOut {              // C = sums + bias, bf16
  struct Args {
    bf16_t* C;
    const bf16_t* bias;
    int N;
  } a;
  float b[8];
  __device__ void columns(int n, int N) { bias_eight(a.bias, n, N, b); }
  __device__ void row(int, int m, int n, bool live, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += b[e];
    if (live) store_eight(a.C + (long long)m * a.N + n, v);
  }
};

template <int ACT, bool KEEP>
struct EpiAct {              // h = sums + bias, packed with KEEP; a = act(h)
  struct Args {
    bf16_t* C;
    const bf16_t* bias;
    uint8_t *codes, *exps;
    int N;
  } a;
  float b[8];
  __device__ void columns(int n, int N) { bias_eight(a.bias, n, N, b); }
  __device__ void row(int, int m, int n, bool live, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += b[e];
    const long long at = (long long)m * a.N + n;
    if constexpr (KEEP) {
      uint32_t e;
      const u32x2 c = pack_eight(v, e);
      if (live) {
        *reinterpret_cast<u32x2*>(a.codes + at) = c;
        if ((n & 31) == 0) a.exps[at >> 5] = (uint8_t)e;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act_value<ACT, false>(v[e]);
    if (live) store_eight(a.C + at, v);
  }
};

template <int ACT>
struct EpiActBwd {           // sums = da; dh = da act'(h'), a = act(h')
  struct Args {
    bf16_t *dh, *act;
    const uint8_t *codes, *exps;
    int N;
  } a;
  __device__ void columns(int, int) {}
  __device__ void row(int, int m, int n, bool live, float (&v)[8]) {
    if (!live) return;
    const long long at = (long long)m * a.N + n;
    float h[8];
    unpack_eight(*reinterpret_cast<const u32x2*>(a.codes + at), a.exps[at >> 5], h);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float slope;
      h[e] = act_both<ACT, false>(h[e], slope);
      v[e] *= slope;
    }
    store_eight(a.dh + at, v);
    store_eight(a.act + at, h);
  }
};

struct EpiGrad {             // weight gradients: the result in the type of the gradients, or a slice's fp32 partial product
  struct Args {
    void* C;
    float* part;
    int M, N, bf16;
  } a;
  __device__ void columns(int, int) {}
  __device__ void row(int slice, int m, int n, bool live, float (&v)[8]) {
    if (!live) return;
    const long long at = (long long)m * a.N + n;
    if (a.part) store_eight(a.part + (long long)slice * a.M * a.N + at, v);
    else if (a.bf16) store_eight((bf16_t*)a.C + at, v);
    else store_eight((float*)a.C + at, v);
  }
};

// ---- column sums of dh and dy: partial sums of a range of rows each (grid: columns / 64, ranges, matrices), rows in order
constexpr int kColRanges = 64;
struct ColArgs {
  const void* src[2];
  int cols[2];
  float* part;               // [kColRanges][cols[0] + cols[1]]
  int B, n, ranges;
  const int32_t* n_dev;
};
template <typename T>
__global__ __launch_bounds__(256) void ffn_colsum_kernel(ColArgs c) {
  int n;
  if (!vd_count(c.n_dev, c.n, n)) return;
  const bool second = blockIdx.z != 0;
  const int cols = second ? c.cols[1] : c.cols[0], col = blockIdx.x * 64 + (threadIdx.x & 63), wave = threadIdx.x >> 6;
  const T* src = (const T*)(second ? c.src[1] : c.src[0]);
  if (!src || (int)blockIdx.x * 64 >= cols) return;
  __shared__ float red[4][64];
  const long long rows = (long long)c.B * n, per = (rows + c.ranges - 1) / c.ranges;
  const long long r0 = blockIdx.y * per, r1 = min(rows, r0 + per);
  float s = 0.f;
  if (col < cols) {
    long long r = r0 + wave;
    for (; r + 28 < r1; r += 32) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = to_float(src[(r + 4 * i) * cols + col]);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
    for (; r < r1; r += 4) s += to_float(src[r * cols + col]);
  }
  red[wave][threadIdx.x & 63] = s;
  __syncthreads();
  if (wave == 0 && col < cols)
    c.part[(long long)blockIdx.y * (c.cols[0] + c.cols[1]) + (second ? c.cols[0] : 0) + col] =
        ((red[0][threadIdx.x] + red[1][threadIdx.x]) + red[2][threadIdx.x]) + red[3][threadIdx.x];
}

// ---- sums over slices and ranges, in order: dW1, dW2, db1, db2
struct FinishArgs {
  const float* part[2];      // [slices][d f]; null: already there
  const float* colpart;
  void* dW[2];
  void* db[2];
  int cols[2];
  long long count;
  int slices, ranges, bf16;
  const int32_t* n_dev;
  int n;
};
__device__ inline void put(void* p, long long i, float v, int bf16) {
  if (bf16) ((bf16_t*)p)[i] = f2bf(v);
  else ((float*)p)[i] = v;
}
__global__ __launch_bounds__(256) void ffn_finish_kernel(FinishArgs f) {
  int n;
  if (!vd_count(f.n_dev, f.n, n)) return;
  const int z = blockIdx.y;
  const long long step = (long long)gridDim.x * 256;
  if (z < 2) {
    const float* p = z ? f.part[1] : f.part[0];
    if (!p) return;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < f.count; i += step) {
      float s = 0.f;
      for (int k = 0; k < f.slices; ++k) s += p[k * f.count + i];
      put(z ? f.dW[1] : f.dW[0], i, s, f.bf16);
    }
    return;
  }
  void* db = z == 2 ? f.db[0] : f.db[1];
  if (!db) return;
  const int cols = z == 2 ? f.cols[0] : f.cols[1], all = f.cols[0] + f.cols[1];
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < cols; i += step) {
    float s = 0.f;
    for (int k = 0; k < f.ranges; ++k) s += f.colpart[(long long)k * all + (z == 2 ? 0 : f.cols[0]) + i];
    put(db, i, s, f.bf16);
  }
}

// ---- sizes
bool is_act(int act) { return act == VARDROP_ACT_RELU || act == VARDROP_ACT_GELU; }
int check_sizes(int B, int n, int d, int f, int dtype) {
  if (B < 0 || n < 0 || d < 1 || f < 1 || (dtype != VARDROP_F32 && dtype != VARDROP_BF16)) return VARDROP_EINVAL;
  const long long T = (long long)B * n;
  if (T >= (1ll << 31) || T * d >= (1ll << 31) || T * f >= (1ll << 31) || (long long)d * f >= (1ll << 31)) return VARDROP_EUNSUPPORTED;
  if (dtype == VARDROP_BF16 && (d % 64 != 0 || f % 64 != 0)) return VARDROP_EUNSUPPORTED;
  return VARDROP_OK;
}
// K slices of the two weight gradients: tiles for two workgroups a compute unit, at least 256 tokens each.  Grows with T.
int grad_slices(long long T, int d, int f) {
  const long long tiles = 2ll * vd_ceil_div(d, 128) * vd_ceil_div(f, 128);
  long long s = (512 + tiles - 1) / tiles;
  if (s > 16) s = 16;
  if (s > T / 256) s = T / 256;
  return s < 1 ? 1 : (int)s;
}
struct FfnWorkspace {        // bytes from its start
  size_t wide, act, x, part, second, col, total;
};
FfnWorkspace ffn_workspace(long long T, int d, int f, int dtype) {
  const size_t es = dtype == VARDROP_BF16 ? 2 : 4;
  FfnWorkspace w;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += vd_align_up(bytes, 256);
    return here;
  };
  w.wide = take((size_t)T * f * es);       // a in the forward (fp32: h); dh in the backward
  w.act = take((size_t)T * f * es);        // act(h')
  w.x = take((size_t)T * d * es);          // x'
  const size_t slices = dtype == VARDROP_BF16 ? grad_slices(T, d, f) : vd_f32_splitk(d, f, 1, T);
  w.part = take(slices * d * f * 4);
  w.second = take(slices * d * f * 4);
  w.col = take((size_t)kColRanges * (d + f) * 4);
  w.total = at;
  return w;
}

struct FfnCall {
  vardrop_ctx* ctx;
  int B, n, d, f, dtype, act;
  long long T;
  VdDevCount dn;
  hipStream_t s;
};

template <bool BKC, typename Epi>
int product(const FfnCall& c, int kid, const void* A, const void* Bm, int K, int N, const typename Epi::Args& epi, bool status) {
  TileArgs g = {};
  g.A = A; g.B = Bm;
  g.lda = (long long)K * 2; g.ldb = (long long)(BKC ? K : N) * 2;
  g.M = (int)c.T; g.N = N; g.K = K; g.slices = 1;
  g.n_dev = c.dn.dev; g.status = status ? c.dn.status : nullptr; g.n_max = c.n; g.n_mul = c.B; g.n_role = 0;
  const long long t128 = (long long)vd_ceil_div(N, 128) * vd_ceil_div(g.M, 128);
  if (t128 >= 512) return launch_tile_gemm<false, true, BKC, 128, 2, Epi>(c.ctx, kid, g, epi, c.s);
  return launch_tile_gemm<false, true, BKC, 64, 3, Epi>(c.ctx, kid, g, epi, c.s);
}
// C [M][N] = A^T B over the tokens
int weight_gradient(const FfnCall& c, const void* A, const void* Bm, int M, int N, int slices, void* C, float* part, int grad_dtype) {
  TileArgs g = {};
  g.A = A; g.B = Bm;
  g.lda = (long long)M * 2; g.ldb = (long long)N * 2;
  g.M = M; g.N = N; g.K = (int)c.T; g.slices = slices;
  g.n_dev = c.dn.dev; g.n_max = c.n; g.n_mul = c.B; g.n_role = 1;
  const EpiGrad::Args epi = {C, slices > 1 ? part : nullptr, M, N, grad_dtype == VARDROP_BF16};
  return launch_tile_gemm<false, false, false, 128, 2, EpiGrad>(c.ctx, VARDROP_K_FFN_WEIGHTS, g, epi, c.s);
}

template <int ACT>
int fwd_bf16(const FfnCall& c, const void* x, const void* W1, const void* b1, const void* W2, const void* b2, void* y, uint8_t* hc, uint8_t* he,
             char* ws) {
  const FfnWorkspace w = ffn_workspace(c.T, c.d, c.f, c.dtype);
  const bf16_t* bias = (const bf16_t*)b1;
  bf16_t* a = (bf16_t*)(ws + w.wide);
  const int rc = hc ? product<false, EpiAct<ACT, true>>(c, VARDROP_K_FFN_UP, x, W1, c.d, c.f, {a, bias, hc, he, c.f}, true)
                    : product<false, EpiAct<ACT, false>>(c, VARDROP_K_FFN_UP, x, W1, c.d, c.f, {a, bias, nullptr, nullptr, c.f}, true);
  return rc ? rc : product<false, EpiOut>(c, VARDROP_K_FFN_DOWN, a, W2, c.f, c.d, {(bf16_t*)y, (const bf16_t*)b2, c.d}, false);
}

int fwd_f32(const FfnCall& c, const float* x, const float* W1, const float* b1, const float* W2, const float* b2, float* y, uint8_t* hc, uint8_t* he,
            char* ws) {
  const FfnWorkspace w = ffn_workspace(c.T, c.d, c.f, c.dtype);
  float* h = (float*)(ws + w.wide);
  GemmF32 g = {};
  g.set(0, x, W1, h, b1);
  g.lda = c.d; g.ldb = c.f; g.ldc = c.f;
  g.M = (int)c.T; g.N = c.f; g.K = c.d; g.nz = 1; g.nseg = 1;
  g.count(c.dn, true, c.n, c.B, 0);
  int rc = vd_gemm_f32(c.ctx, VARDROP_K_FFN_UP, g, false, c.s);
  if (rc) return rc;
  if ((rc = vd_pack8(c.ctx, VARDROP_K_FFN_ACT, h, c.B, c.n, c.f, VARDROP_F32, c.act, hc, he, h, c.s, {c.dn.dev, nullptr}))) return rc;
  g.set(0, h, W2, y, b2);
  g.lda = c.f; g.ldb = c.d; g.ldc = c.d;
  g.N = c.d; g.K = c.f;
  return vd_gemm_f32(c.ctx, VARDROP_K_FFN_DOWN, g, false, c.s);
}

int forward(vardrop_ctx* ctx, const void* x, int B, int n, int d, int f, int dtype, int act, const void* W1, const void* b1, const void* W2,
            const void* b2, void* y, void* saved, void* ws, size_t ws_bytes, hipStream_t s, VdDevCount dn) {
  if (!ctx || !is_act(act)) return VARDROP_EINVAL;
  int rc = check_sizes(B, n, d, f, dtype);
  if (rc) return rc;
  const long long T = (long long)B * n;
  if (T == 0) return VARDROP_OK;
  if (!x || !W1 || !W2 || !y || x == y) return VARDROP_EINVAL;
  const uintptr_t all = (uintptr_t)x | (uintptr_t)W1 | (uintptr_t)W2 | (uintptr_t)y | (uintptr_t)b1 | (uintptr_t)b2;
  if (all % (dtype == VARDROP_BF16 ? 16 : 4) != 0) return VARDROP_EINVAL;
  if (!vd_aligned(saved, 256)) return VARDROP_EWORKSPACE;
  if (!ws || !vd_aligned(ws, 256) || ws_bytes < ffn_workspace(T, d, f, dtype).total) return VARDROP_EWORKSPACE;
  const FfnCall c = {ctx, B, n, d, f, dtype, act, T, dn, s};
  uint8_t* hc = saved ? (uint8_t*)saved + pack_bytes(T, d) : nullptr;
  uint8_t* he = saved ? hc + pack_exponents_at(T, f) : nullptr;
  if (dtype == VARDROP_F32) {
    rc = fwd_f32(c, (const float*)x, (const float*)W1, (const float*)b1, (const float*)W2, (const float*)b2, (float*)y, hc, he, (char*)ws);
  } else {
    rc = act == VARDROP_ACT_RELU ? fwd_bf16<kActRelu>(c, x, W1, b1, W2, b2, y, hc, he, (char*)ws)
                                 : fwd_bf16<kActGelu>(c, x, W1, b1, W2, b2, y, hc, he, (char*)ws);
  }
  if (rc || !saved) return rc;
  return vd_pack8(ctx, VARDROP_K_PACK8, x, B, n, d, dtype, VARDROP_ACT_NONE, saved, (char*)saved + pack_exponents_at(T, d), nullptr, s, {dn.dev, nullptr});
}

int backward(vardrop_ctx* ctx, const void* dy, int B, int n, int d, int f, int dtype, int act, const void* W1, const void* W2, const void* saved,
             void* dx, void* dW1, void* dW2, void* db1, void* db2, int grad_dtype, void* ws, size_t ws_bytes, hipStream_t s, VdDevCount dn) {
  if (!ctx || !is_act(act) || (grad_dtype != VARDROP_F32 && grad_dtype != VARDROP_BF16)) return VARDROP_EINVAL;
  int rc = check_sizes(B, n, d, f, dtype);
  if (rc) return rc;
  if (dtype == VARDROP_F32 && grad_dtype != VARDROP_F32) return VARDROP_EUNSUPPORTED;
  const long long T = (long long)B * n;
  if (!dW1 || !dW2) return VARDROP_EINVAL;
  if (T > 0 && (!dy || !W1 || !W2 || !saved || dx == dy)) return VARDROP_EINVAL;
  const uintptr_t all = (uintptr_t)dy | (uintptr_t)W1 | (uintptr_t)W2 | (uintptr_t)dx | (uintptr_t)dW1 | (uintptr_t)dW2;
  if (all % (dtype == VARDROP_BF16 ? 16 : 4) != 0) return VARDROP_EINVAL;
  if (((uintptr_t)db1 | (uintptr_t)db2) % (grad_dtype == VARDROP_BF16 ? 2 : 4) != 0) return VARDROP_EINVAL;
  const FfnWorkspace w = ffn_workspace(T, d, f, dtype);
  if (!vd_aligned(saved, 256) || !ws || !vd_aligned(ws, 256) || ws_bytes < w.total) return VARDROP_EWORKSPACE;
  const FfnCall c = {ctx, B, n, d, f, dtype, act, T, dn, s};
  char* at = (char*)ws;
  const uint8_t* xc = (const uint8_t*)saved;
  const uint8_t* xe = xc + pack_exponents_at(T, d);
  const uint8_t* hc = xc + pack_bytes(T, d);
  const uint8_t* he = hc + pack_exponents_at(T, f);
  void *dh = at + w.wide, *a = at + w.act, *xv = at + w.x;
  float *part = (float*)(at + w.part), *second = (float*)(at + w.second), *col = (float*)(at + w.col);
  const VdDevCount quiet = {dn.dev, nullptr};
  FinishArgs fin = {};
  fin.slices = 1;
  if (T > 0 && (rc = vd_unpack8(ctx, VARDROP_K_UNPACK8, xc, xe, B, n, d, dtype, xv, s, dn))) return rc;
  if (dtype == VARDROP_BF16) {
    if (T > 0) {
      rc = act == VARDROP_ACT_RELU ? product<true, EpiActBwd<kActRelu>>(c, VARDROP_K_FFN_DH, dy, W2, d, f, {(bf16_t*)dh, (bf16_t*)a, hc, he, f}, false)
                                   : product<true, EpiActBwd<kActGelu>>(c, VARDROP_K_FFN_DH, dy, W2, d, f, {(bf16_t*)dh, (bf16_t*)a, hc, he, f}, false);
      if (rc) return rc;
      if (dx && (rc = product<true, EpiOut>(c, VARDROP_K_FFN_DX, dh, W1, f, d, {(bf16_t*)dx, nullptr, d}, false))) return rc;
    }
    const int slices = grad_slices(T, d, f);
    if ((rc = weight_gradient(c, xv, dh, d, f, slices, dW1, part, grad_dtype))) return rc;
    if ((rc = weight_gradient(c, a, dy, f, d, slices, dW2, second, grad_dtype))) return rc;
    fin.slices = slices;
    if (slices > 1) {
      fin.part[0] = part;
      fin.part[1] = second;
    }
  } else {
    GemmF32 g = {};
    g.nz = 1; g.nseg = 1;
    if (T > 0) {
      g.set(0, (const float*)dy, (const float*)W2, (float*)dh, nullptr);
      g.lda = d; g.ldb = d; g.ldc = f; g.M = (int)T; g.N = f; g.K = d;
      g.count(dn, false, n, B, 0);
      if ((rc = vd_gemm_f32(ctx, VARDROP_K_FFN_DH, g, true, s))) return rc;
      if ((rc = vd_act_bwd_f32(ctx, VARDROP_K_FFN_ACT, (const float*)dh, hc, he, B, n, f, act, (float*)dh, (float*)a, s, quiet))) return rc;
      if (dx) {
        g.set(0, (const float*)dh, (const float*)W1, (float*)dx, nullptr);
        g.lda = f; g.ldb = f; g.ldc = d; g.N = d; g.K = f;
        if ((rc = vd_gemm_f32(ctx, VARDROP_K_FFN_DX, g, true, s))) return rc;
      }
    }
    g.count(dn, false, n, B, 1);
    g.K = (int)T;
    g.set(0, (const float*)xv, (const float*)dh, (float*)dW1, nullptr);
    g.lda = d; g.ldb = f; g.ldc = f; g.M = d; g.N = f; g.part = part;
    if ((rc = vd_gemm_f32_wgrad(ctx, VARDROP_K_FFN_WEIGHTS, g, s))) return rc;
    g.set(0, (const float*)a, (const float*)dy, (float*)dW2, nullptr);
    g.lda = f; g.ldb = d; g.ldc = d; g.M = f; g.N = d; g.part = second;
    if ((rc = vd_gemm_f32_wgrad(ctx, VARDROP_K_FFN_WEIGHTS, g, s))) return rc;
  }
  fin.ranges = T < 64 ? 1 : (T / 64 > kColRanges ? kColRanges : (int)(T / 64));
  if (db1 || db2) {
    ColArgs ca = {};
    ca.src[0] = db1 ? dh : nullptr; ca.src[1] = db2 ? dy : nullptr;
    ca.cols[0] = f; ca.cols[1] = d;
    ca.part = col; ca.B = B; ca.n = n; ca.ranges = fin.ranges; ca.n_dev = dn.dev;
    const dim3 grid((unsigned)vd_ceil_div(d > f ? d : f, 64), (unsigned)fin.ranges, 2);
    if (T > 0) {
      VdTimer timer(ctx, VARDROP_K_FFN_BIAS, s);
      if (dtype == VARDROP_BF16) VD_KERNEL(ctx, ffn_colsum_kernel<bf16_t>, grid, dim3(256), 0, s, ca);
      else VD_KERNEL(ctx, ffn_colsum_kernel<float>, grid, dim3(256), 0, s, ca);
      VD_LAUNCH_CHECK(ctx);
    } else {
      fin.ranges = 0;          // (no tokens: zeros)
    }
  }
  if (!fin.part[0] && !db1 && !db2) return VARDROP_OK;
  fin.dW[0] = dW1; fin.dW[1] = dW2; fin.db[0] = db1; fin.db[1] = db2;
  fin.colpart = col; fin.cols[0] = f; fin.cols[1] = d; fin.count = (long long)d * f;
  fin.bf16 = grad_dtype == VARDROP_BF16; fin.n_dev = dn.dev; fin.n = n;
  const long long blocks = (fin.count + 255) / 256;
  VdTimer timer(ctx, VARDROP_K_REDUCE_DW, s);
  VD_KERNEL(ctx, ffn_finish_kernel, dim3((unsigned)(blocks > 2048 ? 2048 : blocks), 4), dim3(256), 0, s, fin);
  VD_LAUNCH_CHECK(ctx);
  return VARDROP_OK;
}

}  // namespace

extern "C" size_t vardrop_ffn_saved_bytes(int B, int n, int d, int f) {
  if (check_sizes(B, n, d, f, VARDROP_F32) != VARDROP_OK) return 0;
  return pack_bytes((long long)B * n, d) + pack_bytes((long long)B * n, f);
}
extern "C" size_t vardrop_ffn_workspace_bytes(int B, int n, int d, int f, int dtype) {
  if (check_sizes(B, n, d, f, dtype) != VARDROP_OK) return 0;
  return ffn_workspace((long long)B * n, d, f, dtype).total;
}
extern "C" int vardrop_ffn_fwd(vardrop_ctx* ctx, const void* x, int B, int n, int d, int f, int dtype, int act, const void* W1, const void* b1,
                               const void* W2, const void* b2, void* y, void* saved, void* ws, size_t ws_bytes, void* stream) {
  return forward(ctx, x, B, n, d, f, dtype, act, W1, b1, W2, b2, y, saved, ws, ws_bytes, (hipStream_t)stream, {nullptr, nullptr});
}
extern "C" int vardrop_ffn_fwd_dev(vardrop_ctx* ctx, const void* x, int B, const int32_t* n_dev, int n_max, int32_t* status, int d, int f, int dtype,
                                   int act, const void* W1, const void* b1, const void* W2, const void* b2, void* y, void* saved, void* ws,
                                   size_t ws_bytes, void* stream) {
  if (!n_dev || n_max < 1) return VARDROP_EINVAL;
  return forward(ctx, x, B, n_max, d, f, dtype, act, W1, b1, W2, b2, y, saved, ws, ws_bytes, (hipStream_t)stream, {n_dev, status});
}
extern "C" int vardrop_ffn_bwd(vardrop_ctx* ctx, const void* dy, int B, int n, int d, int f, int dtype, int act, const void* W1, const void* W2,
                               const void* saved, void* dx, void* dW1, void* dW2, void* db1, void* db2, int grad_dtype, void* ws, size_t ws_bytes,
                               void* stream) {
  return backward(ctx, dy, B, n, d, f, dtype, act, W1, W2, saved, dx, dW1, dW2, db1, db2, grad_dtype, ws, ws_bytes, (hipStream_t)stream,
                  {nullptr, nullptr});
}
extern "C" int vardrop_ffn_bwd_dev(vardrop_ctx* ctx, const void* dy, int B, const int32_t* n_dev, int n_max, int32_t* status, int d, int f, int dtype,
                                   int act, const void* W1, const void* W2, const void* saved, void* dx, void* dW1, void* dW2, void* db1, void* db2,
                                   int grad_dtype, void* ws, size_t ws_bytes, void* stream) {
  if (!n_dev || n_max < 1) return VARDROP_EINVAL;
  return backward(ctx, dy, B, n_max, d, f, dtype, act, W1, W2, saved, dx, dW1, dW2, db1, db2, grad_dtype, ws, ws_bytes, (hipStream_t)stream,
                  {n_dev, status});
}
