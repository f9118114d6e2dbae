// The feed-forward block, the other half of an encoder layer beside the attention (Sec. 4.1), whose activations wait for the
// backward pass in 8 bits.
//
//   h = x W1 + b1,  a = act(h),  y = a W2 + b2            kept: x and h, packed (pack8.h)
//   dh = (dy W2^T) act'(h'),  dx = dh W1^T,  dW1 = x'^T dh,  db1 = sum dh,  dW2 = act(h')^T dy,  db2 = sum dy
//
// with x', h' what the checkpoints stand for.  bf16: the element-wise work is done on the products' sums before they are
// stored (tile_gemm.h): h never exists outside a tile, dy W2^T neither.
// Two launches forward and three backward.  Large calls are bound by the products' loops, which wait for their operands' copies, and where the rows
// are worked on by vector work: 65 536 x 768 x 1536, us, h and a 240 (640 TFLOP/s), y 142 (1090), dh and a 278 (560), dx, dW1 and dW2 441 (1050).
// Short calls are chains of dependent launches, each of which takes 4 us and its tiles' stages one after the other: 2784 x 512 x 512 8.2, 6.3,
// 9.0, 12.4 and 3.9 for the sums.
#include "ffn.h"

namespace {

// ---- what is done to the rows of a product
// eight columns' biases
__device__ inline void bias_eight(const bf16_t* b, int n, int N, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  if (b && n < N) load_eight(b + n, v);
}

struct EpiOut {
  static constexpr bool kFetch = false, kSums = false;
  static constexpr int kPartsA = 1, kPartsB = 1, kRowSums = 0;  // C = sums + bias, bf16
  struct Args {
    bf16_t* C;
    const bf16_t* bias;
    int N, past;
  } a;
  float b[8];
  __device__ void columns(int n, int N) { bias_eight(a.bias, n, N, b); }
  __device__ void row(int, int, int m, int n, bool live, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += b[e];
    if (live) store_eight(a.C + (long long)m * a.N + n, v, a.past);
  }
};

template <int ACT, bool KEEP>
struct EpiAct {
  static constexpr bool kFetch = false, kSums = false;
  static constexpr int kPartsA = 1, kPartsB = 1, kRowSums = 0;  // h = sums + bias, packed with KEEP; a = act(h)
  struct Args {
    bf16_t* C;
    const bf16_t* bias;
    uint8_t *codes, *exps;
    int N, past;
  } a;
  float b[8];
  __device__ void columns(int n, int N) { bias_eight(a.bias, n, N, b); }
  __device__ void row(int, int, int m, int n, bool live, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += b[e];
    const long long at = (long long)m * a.N + n;
    if constexpr (KEEP) {
      uint32_t e;
      const u32x2 c = pack_eight(v, e);
      if (live) {
        store_past(reinterpret_cast<u32x2*>(a.codes + at), c, a.past);
        if ((n & 31) == 0) a.exps[at >> 5] = (uint8_t)e;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act_value<ACT, false>(v[e]);
    if (live) store_eight(a.C + at, v, a.past);
  }
};

struct ActBwdArgs {
  bf16_t *dh, *act;
  const uint8_t *codes, *exps;
  float* sums;                 // of dh over a tile's rows, before it is rounded; null: not wanted
  int N, past;
};
template <int ACT, int MI, int NJ>
struct EpiActBwd {
  static constexpr bool kFetch = true, kSums = false;
  static constexpr int kPartsA = 1, kPartsB = 1, kRowSums = 1;  // sums = da; dh = da act'(h'), a = act(h')
  typedef ActBwdArgs Args;
  Args a;
  float total[8];
  u32x2 codes[2 * MI * NJ];
  uint32_t exps[2 * MI * NJ];
  __device__ void fetch(int k, int m, int n, bool live) {
    const long long at = live ? (long long)m * a.N + n : 0;
    codes[k] = *reinterpret_cast<const u32x2*>(a.codes + at);
    exps[k] = a.exps[at >> 5];
  }
  __device__ void columns(int, int) {
#pragma unroll
    for (int e = 0; e < 8; ++e) total[e] = 0.f;
  }
  __device__ void row(int, int k, int m, int n, bool live, float (&v)[8]) {
    if (!live) return;
    const long long at = (long long)m * a.N + n;
    float h[8];
    unpack_eight(codes[k], exps[k], h);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float slope;
      h[e] = act_both<ACT, false>(h[e], slope);
      v[e] *= slope;
      total[e] += v[e];
    }
    store_eight(a.dh + at, v, a.past);
    store_eight(a.act + at, h, a.past);
  }
};

template <bool SUMS>
struct EpiGrad {
  static constexpr bool kFetch = false, kSums = SUMS;
  static constexpr int kPartsA = 1, kPartsB = 1, kRowSums = 0;  // weight gradients: the result in the type of the gradients, or a slice's fp32 partial product
  struct Args {
    void* C;
    float* part;
    float* sums;             // column sums of B, [pieces][N]; null: not wanted
    int M, N, bf16;
  } a;
  __device__ void sums(int piece, int n, bool live, float v) {
    if (live && a.sums) a.sums[(long long)piece * a.N + n] = v;
  }
  __device__ void columns(int, int) {}
  __device__ void row(int slice, int, int m, int n, bool live, float (&v)[8]) {
    if (!live) return;
    const long long at = (long long)m * a.N + n;
    if (a.part) store_eight(a.part + (long long)slice * a.M * a.N + at, v);
    else if (a.bf16) store_eight((bf16_t*)a.C + at, v);
    else store_eight((float*)a.C + at, v);
  }
};

// ---- what else a launch carries: element-wise work in workgroups behind those of the product, which has no need of it.  (Between them, eight
// pieces and so many tiles in turn, the activation of 65 536 x 768 x 1536 took 250 us instead of 215, of 2784 x 512 x 512 11.3 instead of 8.6.)
// x into 8 bits, or x' out of them: groups of eight elements, `pieces` workgroups (d is a multiple of 32)
struct PieceArgs {
  const bf16_t* x;
  bf16_t* values;
  uint8_t *codes, *exps;
  int B, n, d, pieces;
  const int32_t* n_dev;
};
template <int THREADS, bool PACK>
__device__ __forceinline__ void piece_8(const PieceArgs& p, int piece) {
  int n;
  if (!vd_count(p.n_dev, p.n, n)) return;
  const long long groups = (long long)p.B * n * (p.d >> 3), step = (long long)p.pieces * THREADS;
  for (long long i0 = (long long)piece * THREADS + threadIdx.x; i0 < groups; i0 += 4 * step) {
    float v[4][8];
    u32x2 c[4];
    uint32_t e[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = i0 + u * step;
      if (i < groups) {
        if constexpr (PACK) {
          load_eight(p.x + i * 8, v[u]);
        } else {
          c[u] = *reinterpret_cast<const u32x2*>(p.codes + i * 8);
          e[u] = p.exps[i >> 2];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = i0 + u * step;
      if (i < groups) {                        // (a block's four lanes agree)
        if constexpr (PACK) {
          const u32x2 code = pack_eight(v[u], e[u]);
          *reinterpret_cast<u32x2*>(p.codes + i * 8) = code;
          if ((i & 3) == 0) p.exps[i >> 2] = (uint8_t)e[u];
        } else {
          unpack_eight(c[u], e[u], v[u]);
          store_eight(p.values + i * 8, v[u]);
        }
      }
    }
  }
}
template <typename S, int ACT, bool KEEP>
__global__ __launch_bounds__(S::THREADS, S::simd) void ffn_up_kernel(TileArgs g, typename EpiAct<ACT, KEEP>::Args args, PieceArgs p) {
  const int tiles = gridDim.x - p.pieces;
  if ((int)blockIdx.x >= tiles) {
    if constexpr (KEEP) piece_8<S::THREADS, true>(p, blockIdx.x - tiles);
    return;
  }
  int M, K;
  if (!tile_dims(g, M, K)) return;
  const int total = (int)tile_count<S>(g, M);
  if ((int)blockIdx.x < total) tile_gemm<false, true, false, S, EpiAct<ACT, KEEP>>(g, args, M, K, xcd_contiguous(blockIdx.x, total));
}

template <typename S, int ACT>
__global__ __launch_bounds__(S::THREADS, S::simd) void ffn_dh_kernel(TileArgs g, ActBwdArgs args, PieceArgs p) {
  const int tiles = gridDim.x - p.pieces;
  if ((int)blockIdx.x >= tiles) {
    piece_8<S::THREADS, false>(p, blockIdx.x - tiles);
    return;
  }
  int M, K;
  if (!tile_dims(g, M, K)) return;
  const int total = (int)tile_count<S>(g, M);
  if ((int)blockIdx.x < total) tile_gemm<false, true, true, S, EpiActBwd<ACT, S::MI, S::NJ>>(g, args, M, K, xcd_contiguous(blockIdx.x, total));
}

// ---- sums over slices and pieces: dW1, dW2 (four elements a thread), then db1, db2 (16 columns a workgroup, 16 threads for each)
__device__ inline bool vd_aligned_16(const void* p) { return ((uintptr_t)p & 15) == 0; }
__device__ inline void put_four(float* p, const float4& v, int count) {
  p[0] = v.x;
  if (count > 1) p[1] = v.y;
  if (count > 2) p[2] = v.z;
  if (count > 3) p[3] = v.w;
}
__global__ __launch_bounds__(256) void ffn_finish_kernel(FfnFinish f, int blocks, const int32_t* n_dev, int n_max) {
  int n;
  if (!vd_count(n_dev, n_max, n)) return;
  const int weights = (f.part[0] ? 2 : 0) * blocks;
  if ((int)blockIdx.x < weights) {
    const int z = (int)blockIdx.x >= blocks;
    const int rows = z ? f.rows[1] : f.rows[0], cols = z ? f.cols[1] : f.cols[0], pitch4 = (z ? f.pitch[1] : f.pitch[0]) >> 2;
    const long long n4 = (long long)(z ? f.part_rows[1] : f.part_rows[0]) * pitch4;
    const float4* p = reinterpret_cast<const float4*>(z ? f.part[1] : f.part[0]);
    void* out = z ? f.dW[1] : f.dW[0];
    for (long long i = (long long)(blockIdx.x - z * blocks) * 256 + threadIdx.x; i < n4; i += (long long)blocks * 256) {
      float4 s = p[i];
      int k = 1;
      for (; k + 4 <= f.slices; k += 4) {
        float4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = p[(long long)(k + u) * n4 + i];
#pragma unroll
        for (int u = 0; u < 4; ++u) { s.x += v[u].x; s.y += v[u].y; s.z += v[u].z; s.w += v[u].w; }
      }
      for (; k < f.slices; ++k) {
        const float4 v = p[(long long)k * n4 + i];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
      if (cols == 4 * pitch4) {              // (rows behind the last are behind the end)
        if (i >= (long long)rows * pitch4) continue;
        if (f.bf16) reinterpret_cast<u32x2*>(out)[i] = u32x2{pack2(s.x, s.y), pack2(s.z, s.w)};
        else if (vd_aligned_16(out)) reinterpret_cast<float4*>(out)[i] = s;
        else put_four((float*)out + 4 * i, s, 4);
      } else {
        const int r = (int)(i / pitch4), c = (int)(i - (long long)r * pitch4) * 4;
        if (r < rows && c < cols) put_four((float*)out + (long long)r * cols + c, s, cols - c);
      }
    }
    return;
  }
  __shared__ float red[16][17];
  const int at = blockIdx.x - weights, b0 = f.col[0] ? (f.cols[0] + 15) / 16 : 0, z = at >= b0;
  const int c = threadIdx.x & 15, group = threadIdx.x >> 4, cols = z ? f.cols[1] : f.cols[0], pitch = z ? f.pitch[1] : f.pitch[0];
  const int column = (at - z * b0) * 16 + c, pieces = z ? f.pieces : (f.B * n + f.tile_rows - 1) / f.tile_rows;
  const float* p = (z ? f.col[1] : f.col[0]) + min(column, cols - 1);
  float s = 0.f;
  int k = group;
  for (; k + 48 < pieces; k += 64) {
    float v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = p[(long long)(k + 16 * u) * pitch];
#pragma unroll
    for (int u = 0; u < 4; ++u) s += v[u];
  }
  for (; k < pieces; k += 16) s += p[(long long)k * pitch];
  red[group][c] = s;
  __syncthreads();
  if (group == 0 && column < cols) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += red[i][c];
    void* db = z ? f.db[1] : f.db[0];
    if (f.bf16) ((bf16_t*)db)[column] = f2bf(s);
    else ((float*)db)[column] = s;
  }
}

// ---- sizes
constexpr int kMostChannels = 65536;
bool is_act(int act) { return act == VARDROP_ACT_RELU || act == VARDROP_ACT_GELU; }
int check_sizes(int B, int n, int d, int f, int dtype) {
  if (B < 0 || n < 0 || d < 1 || f < 1 || (dtype != VARDROP_F32 && dtype != VARDROP_BF16)) return VARDROP_EINVAL;
  // (fp32 rows are padded to multiples of 64 channels in the workspace)
  const long long T = (long long)B * n, D = dtype == VARDROP_F32 ? vd_align_up(d, 64) : d, F = dtype == VARDROP_F32 ? vd_align_up(f, 64) : f;
  if (T >= (1ll << 31) || T * D >= (1ll << 31) || T * F >= (1ll << 31) || D * F >= (1ll << 31)) return VARDROP_EUNSUPPORTED;
  if (d > kMostChannels || f > kMostChannels) return VARDROP_EUNSUPPORTED;      // (a tile's rows are within 32 bits of each other)
  if (dtype == VARDROP_BF16 && (d % 64 != 0 || f % 64 != 0)) return VARDROP_EUNSUPPORTED;
  return VARDROP_OK;
}
struct FfnWorkspace {        // bytes from its start
  size_t wide, act, x, part, second, col, col2, total;
};
FfnWorkspace ffn_workspace(long long T, int d, int f) {
  FfnWorkspace w;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += vd_align_up(bytes, 256);
    return here;
  };
  w.wide = take((size_t)T * f * 2);        // a in the forward, dh in the backward
  w.act = take((size_t)T * f * 2);         // act(h')
  w.x = take((size_t)T * d * 2);           // x'
  const size_t slices = most_slices(T);
  w.part = take(slices * d * f * 4);
  w.second = take(slices * d * f * 4);
  w.col = take((T + 63) / 64 * f * 4);                        // a piece for each row of tiles at most
  w.col2 = take(slices * vd_ceil_div(f, 64) * 2 * d * 4);     // two for each slice and row of tiles
  w.total = at;
  return w;
}
size_t workspace_bytes(long long T, int d, int f, int dtype) {
  return dtype == VARDROP_BF16 ? ffn_workspace(T, d, f).total : vd_ffn_workspace_f32(T, d, f);
}
// workgroups for `groups` of eight elements, about four each a thread
int pieces_8(long long groups, int threads) {
  const long long p = (groups + threads * 4 - 1) / (threads * 4);
  return p > 1024 ? 1024 : (int)p;
}

template <typename S, int ACT, bool KEEP>
int launch_up(const FfnCall& c, const TileArgs& g, const typename EpiAct<ACT, KEEP>::Args& e, PieceArgs p) {
  p.pieces = KEEP ? pieces_8(c.T * c.d / 8, S::THREADS) : 0;
  VD_FFN_LAUNCH(VARDROP_K_FFN_UP, (ffn_up_kernel<S, ACT, KEEP>), S, tile_count<S>(g, g.M) + p.pieces, g, e, p)
}
template <typename S, int ACT>
int launch_dh(const FfnCall& c, const TileArgs& g, const ActBwdArgs& e, PieceArgs p, int& tile_rows) {
  tile_rows = S::BM;
  p.pieces = pieces_8(c.T * c.d / 8, S::THREADS);
  VD_FFN_LAUNCH(VARDROP_K_FFN_DH, (ffn_dh_kernel<S, ACT>), S, tile_count<S>(g, g.M) + p.pieces, g, e, p)
}
template <int ACT>
int fwd_bf16(const FfnCall& c, const void* x, const void* W1, const void* b1, const void* W2, const void* b2, void* y, uint8_t* kept,
             char* ws) {
  uint8_t* hc = kept ? kept + pack_bytes(c.T, c.d) : nullptr;
  uint8_t* he = kept ? hc + pack_exponents_at(c.T, c.f) : nullptr;
  const FfnWorkspace w = ffn_workspace(c.T, c.d, c.f);
  bf16_t* a = (bf16_t*)(ws + w.wide);
  PieceArgs p = {};
  p.x = (const bf16_t*)x; p.codes = kept; p.exps = kept ? kept + pack_exponents_at(c.T, c.d) : nullptr;
  p.B = c.B; p.n = c.n; p.d = c.d; p.n_dev = c.dn.dev;
  const TileArgs up = rows_product(c, x, W1, c.d, c.f, c.f, true);
  const int shape = product_shape(kRowShapes, c.T, c.f, c.d);
  int rc;
  if (kept) {
    const typename EpiAct<ACT, true>::Args e = {a, (const bf16_t*)b1, hc, he, c.f, c.past(c.f, 2)};
#define VD_CALL(S) launch_up<S, ACT, true>(c, up, e, p)
    rc = VD_BY_SHAPE(shape, VD_CALL, TileWide);
#undef VD_CALL
  } else {
    const typename EpiAct<ACT, false>::Args e = {a, (const bf16_t*)b1, nullptr, nullptr, c.f, c.past(c.f, 2)};
#define VD_CALL(S) launch_up<S, ACT, false>(c, up, e, p)
    rc = VD_BY_SHAPE(shape, VD_CALL, TileWide);
#undef VD_CALL
  }
  if (rc) return rc;
  const TileArgs down = rows_product(c, a, W2, c.f, c.d, c.d, false);
  const EpiOut::Args e = {(bf16_t*)y, (const bf16_t*)b2, c.d, c.past(c.d, 2)};
#define VD_CALL(S) launch_tile_gemm<false, true, false, S, EpiOut>(c.ctx, VARDROP_K_FFN_DOWN, down, e, c.s)
  return VD_BY_SHAPE(product_shape(kShapes, c.T, c.d, c.f), VD_CALL, Tile256);
#undef VD_CALL
}

template <int ACT>
int bwd_bf16(const FfnCall& c, const void* dy, const void* W1, const void* W2, const uint8_t* saved, void* dx, void* dW1, void* dW2, void* db1, void* db2,
             int grad_dtype, char* ws, FfnFinish& fin) {
  const FfnWorkspace w = ffn_workspace(c.T, c.d, c.f);
  const uint8_t* hc = saved + pack_bytes(c.T, c.d);
  bf16_t *dh = (bf16_t*)(ws + w.wide), *a = (bf16_t*)(ws + w.act), *xv = (bf16_t*)(ws + w.x);
  float *part = (float*)(ws + w.part), *second = (float*)(ws + w.second), *col = (float*)(ws + w.col), *col2 = (float*)(ws + w.col2);
  if (c.T > 0) {
    PieceArgs p = {};
    p.values = xv; p.codes = const_cast<uint8_t*>(saved); p.exps = const_cast<uint8_t*>(saved) + pack_exponents_at(c.T, c.d);
    p.B = c.B; p.n = c.n; p.d = c.d; p.n_dev = c.dn.dev;
    const TileArgs g = rows_product(c, dy, W2, c.d, c.f, c.d, true);
    const ActBwdArgs e = {dh, a, hc, hc + pack_exponents_at(c.T, c.f), db1 ? col : nullptr, c.f, c.past(c.f, 2)};
#define VD_CALL(S) launch_dh<S, ACT>(c, g, e, p, fin.tile_rows)
    const int rc = VD_BY_SHAPE(product_shape(kRowShapes, c.T, c.f, c.d), VD_CALL, TileWide);
#undef VD_CALL
    if (rc) return rc;
  }
  const GradPlan plan = plan_grads(kShapes, c.T, c.d, c.f);
  const bool split = plan.slices > 1, low = grad_dtype == VARDROP_BF16;
  if (split) {
    fin.part[0] = part;
    fin.part[1] = second;
    fin.slices = plan.slices;
  }
  fin.col[0] = db1 ? col : nullptr;
  fin.col[1] = db2 ? col2 : nullptr;
  const TileArgs gx = dx && c.T > 0 ? rows_product(c, dh, W1, c.f, c.d, c.f, false) : TileArgs{};
  const TileArgs g1 = tokens_product(c, xv, dh, c.d, c.f, plan.slices), g2 = tokens_product(c, a, dy, c.f, c.d, plan.slices);
  const EpiOut::Args ax = {(bf16_t*)dx, nullptr, c.d, c.past(c.d, 2)};
  const EpiGrad<false>::Args a1 = {dW1, split ? part : nullptr, nullptr, c.d, c.f, low};
  const EpiGrad<true>::Args a2 = {dW2, split ? second : nullptr, fin.col[1], c.f, c.d, low};
#define VD_CALL(S) launch_grads<S, EpiOut, EpiGrad<false>, EpiGrad<true>>(c, gx, ax, g1, a1, g2, a2, fin.pieces)
  return VD_BY_SHAPE(plan.shape, VD_CALL, Tile256);
#undef VD_CALL
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
  if (!ws || !vd_aligned(ws, 256) || ws_bytes < workspace_bytes(T, d, f, dtype)) return VARDROP_EWORKSPACE;
  const FfnCall c = {ctx, B, n, d, f, act, T, dn, s};
  if (dtype == VARDROP_F32)
    return vd_ffn_fwd_f32(c, (const float*)x, (const float*)W1, (const float*)b1, (const float*)W2, (const float*)b2, (float*)y, (uint8_t*)saved, (char*)ws);
  return act == VARDROP_ACT_RELU ? fwd_bf16<kActRelu>(c, x, W1, b1, W2, b2, y, (uint8_t*)saved, (char*)ws)
                                 : fwd_bf16<kActGelu>(c, x, W1, b1, W2, b2, y, (uint8_t*)saved, (char*)ws);
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
  if (!vd_aligned(saved, 256) || !ws || !vd_aligned(ws, 256) || ws_bytes < workspace_bytes(T, d, f, dtype)) return VARDROP_EWORKSPACE;
  const FfnCall c = {ctx, B, n, d, f, act, T, dn, s};
  char* at = (char*)ws;
  const uint8_t* xc = (const uint8_t*)saved;
  FfnFinish fin = {};
  fin.slices = 1;
  fin.B = B;
  fin.tile_rows = 64;
  fin.rows[0] = fin.part_rows[0] = fin.cols[1] = fin.pitch[1] = d;
  fin.rows[1] = fin.part_rows[1] = fin.cols[0] = fin.pitch[0] = f;
  if (dtype == VARDROP_BF16) {
    rc = act == VARDROP_ACT_RELU ? bwd_bf16<kActRelu>(c, dy, W1, W2, xc, dx, dW1, dW2, db1, db2, grad_dtype, at, fin)
                                 : bwd_bf16<kActGelu>(c, dy, W1, W2, xc, dx, dW1, dW2, db1, db2, grad_dtype, at, fin);
  } else {
    rc = vd_ffn_bwd_f32(c, (const float*)dy, (const float*)W1, (const float*)W2, xc, (float*)dx, (float*)dW1, (float*)dW2, (float*)db1, (float*)db2, at, fin);
  }
  if (rc || (!fin.part[0] && !fin.col[0] && !fin.col[1])) return rc;
  fin.dW[0] = dW1; fin.dW[1] = dW2; fin.db[0] = db1; fin.db[1] = db2;
  fin.bf16 = grad_dtype == VARDROP_BF16;
  const long long most = (long long)fin.part_rows[0] * fin.pitch[0], other = (long long)fin.part_rows[1] * fin.pitch[1];
  const long long want = ((most > other ? most : other) / 4 + 255) / 256;
  const int blocks = want > 1024 ? 1024 : (int)want;
  const int grid = (fin.part[0] ? 2 * blocks : 0) + (fin.col[0] ? vd_ceil_div(f, 16) : 0) + (fin.col[1] ? vd_ceil_div(d, 16) : 0);
  VdTimer timer(ctx, VARDROP_K_REDUCE_DW, s);
  VD_KERNEL(ctx, ffn_finish_kernel, dim3((unsigned)grid), dim3(256), 0, s, fin, blocks, dn.dev, n);
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
  return workspace_bytes((long long)B * n, d, f, dtype);
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
