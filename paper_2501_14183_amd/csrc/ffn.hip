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

struct EpiOut {
  static constexpr bool kFetch = false, kSums = false;              // C = sums + bias, bf16
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
  static constexpr bool kFetch = false, kSums = false;              // h = sums + bias, packed with KEEP; a = act(h)
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
  int N, past;
};
template <int ACT, int MI, int NJ>
struct EpiActBwd {
  static constexpr bool kFetch = true, kSums = false;           // sums = da; dh = da act'(h'), a = act(h')
  typedef ActBwdArgs Args;
  Args a;
  u32x2 codes[2 * MI * NJ];
  uint32_t exps[2 * MI * NJ];
  __device__ void fetch(int k, int m, int n, bool live) {
    const long long at = live ? (long long)m * a.N + n : 0;
    codes[k] = *reinterpret_cast<const u32x2*>(a.codes + at);
    exps[k] = a.exps[at >> 5];
  }
  __device__ void columns(int, int) {}
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
    }
    store_eight(a.dh + at, v, a.past);
    store_eight(a.act + at, h, a.past);
  }
};

struct EpiGrad {
  static constexpr bool kFetch = false, kSums = true;             // weight gradients: the result in the type of the gradients, or a slice's fp32 partial product
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

// dx, dW1 and dW2 need the results of the launch before and nothing of each other.  The kind whose tiles are longer comes first; a die takes
// a contiguous range of either kind.
template <typename S>
__global__ __launch_bounds__(S::THREADS, S::simd) void ffn_grads_kernel(TileArgs gx, EpiOut::Args ax, TileArgs g1, EpiGrad::Args a1, TileArgs g2,
                                                                        EpiGrad::Args a2) {
  int Mx, Kx, M1, K1, M2, K2;
  if (!tile_dims(gx, Mx, Kx) || !tile_dims(g1, M1, K1) || !tile_dims(g2, M2, K2)) return;
  const int nx = gx.A ? (int)tile_count<S>(gx, Mx) : 0, n1 = (int)tile_count<S>(g1, M1), nw = n1 + (int)tile_count<S>(g2, M2);
  if ((int)blockIdx.x >= nx + nw) return;
  const bool w_first = K1 / g1.slices > Kx;
  const int first = w_first ? nw : nx, xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const int of_first = (first >> 3) + (xcd < (first & 7) ? 1 : 0), from = xcd_range_start(xcd, first);
  const bool in_first = slot < of_first;
  const int t = in_first ? from + slot : xcd_range_start(xcd, nx + nw) - from + (slot - of_first);
  if (in_first != w_first) tile_gemm<false, true, true, S, EpiOut>(gx, ax, Mx, Kx, t);
  else if (t < n1) tile_gemm<false, false, false, S, EpiGrad>(g1, a1, M1, K1, t);
  else tile_gemm<false, false, false, S, EpiGrad>(g2, a2, M2, K2, t - n1);
}

// ---- fp32: column sums of dh and dy (grid: columns / 64, pieces, matrices), rows in order
struct ColArgs {
  const float* src;
  float* part;                 // [pieces][d]
  int B, n, d, pieces;
  const int32_t* n_dev;
};
__global__ __launch_bounds__(256) void ffn_columns_f32_kernel(ColArgs c0, ColArgs c1) {
  const ColArgs c = blockIdx.z ? c1 : c0;
  int n;
  if (!c.src || !vd_count(c.n_dev, c.n, n)) return;
  const int col = blockIdx.x * 64 + (threadIdx.x & 63), wave = threadIdx.x >> 6;
  if ((int)blockIdx.x * 64 >= c.d) return;
  __shared__ float red[4][64];
  const long long rows = (long long)c.B * n, per = (rows + c.pieces - 1) / c.pieces;
  const long long r0 = blockIdx.y * per, r1 = min(rows, r0 + per);
  float s = 0.f;
  if (col < c.d) {
    long long r = r0 + wave;
    for (; r + 28 < r1; r += 32) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c.src[(r + 4 * i) * c.d + col];
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
    for (; r < r1; r += 4) s += c.src[r * c.d + col];
  }
  red[wave][threadIdx.x & 63] = s;
  __syncthreads();
  if (wave == 0 && col < c.d)
    c.part[(long long)blockIdx.y * c.d + col] = ((red[0][threadIdx.x] + red[1][threadIdx.x]) + red[2][threadIdx.x]) + red[3][threadIdx.x];
}

// ---- sums over slices and pieces, in an order of their own: dW1, dW2 (four elements a thread), then db1, db2 (16 columns a workgroup, 16
// threads for each)
struct FinishArgs {
  const float* part[2];        // [slices][count]; null: already there
  float* col[2];               // [pieces][cols]; null: not wanted
  void* dW[2];
  void* db[2];
  int cols[2], pieces[2];
  long long count;
  int slices, blocks, bf16;    // blocks: workgroups of a weight
  const int32_t* n_dev;
  int n;
};
__global__ __launch_bounds__(256) void ffn_finish_kernel(FinishArgs f) {
  int n;
  if (!vd_count(f.n_dev, f.n, n)) return;
  const int weights = (f.part[0] ? 2 : 0) * f.blocks;
  if ((int)blockIdx.x < weights) {
    const int z = (int)blockIdx.x >= f.blocks;
    const long long n4 = f.count >> 2;
    const float4* p = reinterpret_cast<const float4*>(z ? f.part[1] : f.part[0]);
    void* out = z ? f.dW[1] : f.dW[0];
    for (long long i = (long long)(blockIdx.x - z * f.blocks) * 256 + threadIdx.x; i < n4; i += (long long)f.blocks * 256) {
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
      if (f.bf16) reinterpret_cast<u32x2*>(out)[i] = u32x2{pack2(s.x, s.y), pack2(s.z, s.w)};
      else reinterpret_cast<float4*>(out)[i] = s;
    }
    return;
  }
  __shared__ float red[16][17];
  const int at = blockIdx.x - weights, b0 = f.col[0] ? (f.cols[0] + 15) / 16 : 0, z = at >= b0;
  const int c = threadIdx.x & 15, group = threadIdx.x >> 4, cols = z ? f.cols[1] : f.cols[0], column = (at - z * b0) * 16 + c;
  const int pieces = z ? f.pieces[1] : f.pieces[0];
  const float* p = (z ? f.col[1] : f.col[0]) + min(column, cols - 1);
  float s = 0.f;
  int k = group;
  for (; k + 48 < pieces; k += 64) {
    float v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = p[(long long)(k + 16 * u) * cols];
#pragma unroll
    for (int u = 0; u < 4; ++u) s += v[u];
  }
  for (; k < pieces; k += 16) s += p[(long long)k * cols];
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
bool is_act(int act) { return act == VARDROP_ACT_RELU || act == VARDROP_ACT_GELU; }
int check_sizes(int B, int n, int d, int f, int dtype) {
  if (B < 0 || n < 0 || d < 1 || f < 1 || (dtype != VARDROP_F32 && dtype != VARDROP_BF16)) return VARDROP_EINVAL;
  const long long T = (long long)B * n;
  if (T >= (1ll << 31) || T * d >= (1ll << 31) || T * f >= (1ll << 31) || (long long)d * f >= (1ll << 31)) return VARDROP_EUNSUPPORTED;
  if (dtype == VARDROP_BF16 && (d % 64 != 0 || f % 64 != 0)) return VARDROP_EUNSUPPORTED;
  return VARDROP_OK;
}
// ---- the plan of the gradients' launch
// The launch of dx (T x d over f) and of the weight gradients (2 d f over T in slices): time until the last place is done when the longer
// tiles come first, and the sum of the slices behind it.
constexpr int kMostSlices = 16, kLeastSlice = 256;
struct GradPlan {
  int shape, slices;
};
int most_slices(long long T) {
  const long long s = T / kLeastSlice;
  return s < 1 ? 1 : (s > kMostSlices ? kMostSlices : (int)s);
}
GradPlan plan_grads(long long T, int d, int f) {
  GradPlan best = {0, 1};
  double least = -1;
  for (int i = 0; i < 3; ++i) {
    const ShapeCost& c = kShapes[i];
    const long long nx = tiles_of(c, T, d);
    for (int s = 1; s <= most_slices(T); ++s) {
      const long long nw = (tiles_of(c, d, f) + tiles_of(c, f, d)) * s;
      const double tw = tile_time(c, (double)T / s), tx = tile_time(c, f);
      const double tl = tw > tx ? tw : tx, ts = tw > tx ? tx : tw;
      const long long nl = tw > tx ? nw : nx, ns = tw > tx ? nx : nw;
      const long long full = nl / c.places, rest = nl % c.places;              // `rest` places have a long tile more than the others
      double end = (full + (rest ? 1 : 0)) * tl;
      if (ns > 0) {
        // short tiles fill the places up: level at which all fit
        double level = (nl * tl + ns * ts) / c.places;
        long long fit = -1;
        while (true) {
          const double over = level - full * tl, under = level - (full + 1) * tl;
          fit = (c.places - rest) * (long long)(over > 0 ? over / ts + 1e-9 : 0) + rest * (long long)(under > 0 ? under / ts + 1e-9 : 0);
          if (fit >= ns) break;
          level += 0.25 * ts;
        }
        end = end > level ? end : level;
      }
      if (s > 1) end += 2.0 * d * f * s * 2e-4 + 400;                          // (written and read at memory's rate; a launch)
      if (least < 0 || end < least) {
        least = end;
        best = {i, s};
      }
    }
  }
  return best;
}

constexpr int kColPieces = 256;
int column_pieces(long long T) { return T < 64 ? 1 : (T / 32 > kColPieces ? kColPieces : (int)(T / 32)); }
struct FfnWorkspace {        // bytes from its start
  size_t wide, act, x, part, second, col, col2, total;
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
  const size_t slices = dtype == VARDROP_BF16 ? most_slices(T) : vd_f32_splitk(d, f, 1, T);
  w.part = take(slices * d * f * 4);
  w.second = take(slices * d * f * 4);
  // column sums: two pieces for each slice and row of tiles at most
  w.col = take((dtype == VARDROP_BF16 ? slices * vd_ceil_div(d, 64) * 2 : (size_t)kColPieces) * f * 4);
  w.col2 = take((dtype == VARDROP_BF16 ? slices * vd_ceil_div(f, 64) * 2 : (size_t)kColPieces) * d * 4);
  w.total = at;
  return w;
}

struct FfnCall {
  vardrop_ctx* ctx;
  int B, n, d, f, dtype, act;
  long long T;
  VdDevCount dn;
  hipStream_t s;
  int past(int N) const { return T * N * 2 >= kPastCaches; }
};

// C [T][N] = A B, over the tokens
TileArgs rows_product(const FfnCall& c, const void* A, const void* Bm, bool bkc, int K, int N, bool status) {
  TileArgs g = {};
  g.A = A; g.B = Bm;
  g.lda = (long long)K * 2; g.ldb = (long long)(bkc ? K : N) * 2;
  g.M = (int)c.T; g.N = N; g.K = K; g.slices = 1;
  g.n_dev = c.dn.dev; g.status = status ? c.dn.status : nullptr; g.n_max = c.n; g.n_mul = c.B; g.n_role = 0;
  return g;
}
// C [M][N] = A^T B, summed over the tokens
TileArgs tokens_product(const FfnCall& c, const void* A, const void* Bm, int M, int N, int slices) {
  TileArgs g = {};
  g.A = A; g.B = Bm;
  g.lda = (long long)M * 2; g.ldb = (long long)N * 2;
  g.M = M; g.N = N; g.K = (int)c.T; g.slices = slices;
  g.n_dev = c.dn.dev; g.n_max = c.n; g.n_mul = c.B; g.n_role = 1;
  return g;
}
// workgroups for `groups` of eight elements, about four each a thread
int pieces_8(long long groups, int threads) {
  const long long p = (groups + threads * 4 - 1) / (threads * 4);
  return p > 1024 ? 1024 : (int)p;
}

#define VD_FFN_LAUNCH(KID, KERNEL, S, GRID, ...)                                                     \
  {                                                                                                  \
    static int configured = -1;                                                                      \
    const int rc_ = tile_allow_lds(c.ctx, (const void*)KERNEL, S::lds, configured);                  \
    if (rc_) return rc_;                                                                             \
    if ((GRID) >= (1ll << 31)) return VARDROP_EUNSUPPORTED;                                          \
    VdTimer timer(c.ctx, KID, c.s);                                                                  \
    VD_KERNEL(c.ctx, (KERNEL), dim3((unsigned)(GRID)), dim3(S::THREADS), S::lds, c.s, __VA_ARGS__);  \
    VD_LAUNCH_CHECK(c.ctx);                                                                          \
    return VARDROP_OK;                                                                               \
  }
template <typename S, int ACT, bool KEEP>
int launch_up(const FfnCall& c, const TileArgs& g, const typename EpiAct<ACT, KEEP>::Args& e, PieceArgs p) {
  p.pieces = KEEP ? pieces_8(c.T * c.d / 8, S::THREADS) : 0;
  VD_FFN_LAUNCH(VARDROP_K_FFN_UP, (ffn_up_kernel<S, ACT, KEEP>), S, tile_count<S>(g, g.M) + p.pieces, g, e, p)
}
template <typename S, int ACT>
int launch_dh(const FfnCall& c, const TileArgs& g, const ActBwdArgs& e, PieceArgs p) {
  p.pieces = pieces_8(c.T * c.d / 8, S::THREADS);
  VD_FFN_LAUNCH(VARDROP_K_FFN_DH, (ffn_dh_kernel<S, ACT>), S, tile_count<S>(g, g.M) + p.pieces, g, e, p)
}
template <typename S>
int launch_grads(const FfnCall& c, const TileArgs& gx, const EpiOut::Args& ax, const TileArgs& g1, const EpiGrad::Args& a1, const TileArgs& g2,
                 const EpiGrad::Args& a2, int (&pieces)[2]) {
  pieces[0] = tile_pieces<S>(g1);
  pieces[1] = tile_pieces<S>(g2);
  VD_FFN_LAUNCH(VARDROP_K_FFN_GRADS, ffn_grads_kernel<S>, S, (gx.A ? tile_count<S>(gx, gx.M) : 0) + tile_count<S>(g1, g1.M) + tile_count<S>(g2, g2.M), gx, ax, g1,
                a1, g2, a2)
}
#undef VD_FFN_LAUNCH

template <int ACT>
int fwd_bf16(const FfnCall& c, const void* x, const void* W1, const void* b1, const void* W2, const void* b2, void* y, uint8_t* kept, uint8_t* hc,
             uint8_t* he, char* ws) {
  const FfnWorkspace w = ffn_workspace(c.T, c.d, c.f, c.dtype);
  bf16_t* a = (bf16_t*)(ws + w.wide);
  PieceArgs p = {};
  p.x = (const bf16_t*)x; p.codes = kept; p.exps = kept ? kept + pack_exponents_at(c.T, c.d) : nullptr;
  p.B = c.B; p.n = c.n; p.d = c.d; p.n_dev = c.dn.dev;
  const TileArgs up = rows_product(c, x, W1, false, c.d, c.f, true);
  const int shape = product_shape(kRowShapes, c.T, c.f, c.d);
  int rc;
  if (kept) {
    const typename EpiAct<ACT, true>::Args e = {a, (const bf16_t*)b1, hc, he, c.f, c.past(c.f)};
#define VD_CALL(S) launch_up<S, ACT, true>(c, up, e, p)
    rc = VD_BY_SHAPE(shape, VD_CALL, TileWide);
#undef VD_CALL
  } else {
    const typename EpiAct<ACT, false>::Args e = {a, (const bf16_t*)b1, nullptr, nullptr, c.f, c.past(c.f)};
#define VD_CALL(S) launch_up<S, ACT, false>(c, up, e, p)
    rc = VD_BY_SHAPE(shape, VD_CALL, TileWide);
#undef VD_CALL
  }
  if (rc) return rc;
  const TileArgs down = rows_product(c, a, W2, false, c.f, c.d, false);
  const EpiOut::Args e = {(bf16_t*)y, (const bf16_t*)b2, c.d, c.past(c.d)};
#define VD_CALL(S) launch_tile_gemm<false, true, false, S, EpiOut>(c.ctx, VARDROP_K_FFN_DOWN, down, e, c.s)
  return VD_BY_SHAPE(product_shape(kShapes, c.T, c.d, c.f), VD_CALL, Tile256);
#undef VD_CALL
}

template <int ACT>
int bwd_bf16(const FfnCall& c, const void* dy, const void* W1, const void* W2, const uint8_t* saved, void* dx, void* dW1, void* dW2, void* db1, void* db2,
             int grad_dtype, char* ws, FinishArgs& fin) {
  const FfnWorkspace w = ffn_workspace(c.T, c.d, c.f, c.dtype);
  const uint8_t* hc = saved + pack_bytes(c.T, c.d);
  bf16_t *dh = (bf16_t*)(ws + w.wide), *a = (bf16_t*)(ws + w.act), *xv = (bf16_t*)(ws + w.x);
  float *part = (float*)(ws + w.part), *second = (float*)(ws + w.second), *col = (float*)(ws + w.col), *col2 = (float*)(ws + w.col2);
  if (c.T > 0) {
    PieceArgs p = {};
    p.values = xv; p.codes = const_cast<uint8_t*>(saved); p.exps = const_cast<uint8_t*>(saved) + pack_exponents_at(c.T, c.d);
    p.B = c.B; p.n = c.n; p.d = c.d; p.n_dev = c.dn.dev;
    const TileArgs g = rows_product(c, dy, W2, true, c.d, c.f, true);
    const ActBwdArgs e = {dh, a, hc, hc + pack_exponents_at(c.T, c.f), c.f, c.past(c.f)};
#define VD_CALL(S) launch_dh<S, ACT>(c, g, e, p)
    const int rc = VD_BY_SHAPE(product_shape(kRowShapes, c.T, c.f, c.d), VD_CALL, TileWide);
#undef VD_CALL
    if (rc) return rc;
  }
  const GradPlan plan = plan_grads(c.T, c.d, c.f);
  const bool split = plan.slices > 1, low = grad_dtype == VARDROP_BF16;
  if (split) {
    fin.part[0] = part;
    fin.part[1] = second;
    fin.slices = plan.slices;
  }
  fin.col[0] = db1 ? col : nullptr;
  fin.col[1] = db2 ? col2 : nullptr;
  const TileArgs gx = dx && c.T > 0 ? rows_product(c, dh, W1, true, c.f, c.d, false) : TileArgs{};
  const TileArgs g1 = tokens_product(c, xv, dh, c.d, c.f, plan.slices), g2 = tokens_product(c, a, dy, c.f, c.d, plan.slices);
  const EpiOut::Args ax = {(bf16_t*)dx, nullptr, c.d, c.past(c.d)};
  const EpiGrad::Args a1 = {dW1, split ? part : nullptr, fin.col[0], c.d, c.f, low};
  const EpiGrad::Args a2 = {dW2, split ? second : nullptr, fin.col[1], c.f, c.d, low};
#define VD_CALL(S) launch_grads<S>(c, gx, ax, g1, a1, g2, a2, fin.pieces)
  return VD_BY_SHAPE(plan.shape, VD_CALL, Tile256);
#undef VD_CALL
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

int bwd_f32(const FfnCall& c, const float* dy, const float* W1, const float* W2, const uint8_t* saved, float* dx, float* dW1, float* dW2, bool db1, bool db2,
            char* ws, FinishArgs& fin) {
  const FfnWorkspace w = ffn_workspace(c.T, c.d, c.f, c.dtype);
  const uint8_t* hc = saved + pack_bytes(c.T, c.d);
  float *dh = (float*)(ws + w.wide), *a = (float*)(ws + w.act), *xv = (float*)(ws + w.x);
  const VdDevCount quiet = {c.dn.dev, nullptr};
  int rc;
  GemmF32 g = {};
  g.nz = 1; g.nseg = 1;
  if (c.T > 0) {
    if ((rc = vd_unpack8(c.ctx, VARDROP_K_UNPACK8, saved, saved + pack_exponents_at(c.T, c.d), c.B, c.n, c.d, VARDROP_F32, xv, c.s, c.dn))) return rc;
    g.set(0, dy, W2, dh, nullptr);
    g.lda = c.d; g.ldb = c.d; g.ldc = c.f; g.M = (int)c.T; g.N = c.f; g.K = c.d;
    g.count(c.dn, false, c.n, c.B, 0);
    if ((rc = vd_gemm_f32(c.ctx, VARDROP_K_FFN_DH, g, true, c.s))) return rc;
    if ((rc = vd_act_bwd_f32(c.ctx, VARDROP_K_FFN_ACT, dh, hc, hc + pack_exponents_at(c.T, c.f), c.B, c.n, c.f, c.act, dh, a, c.s, quiet))) return rc;
    if (dx) {
      g.set(0, dh, W1, dx, nullptr);
      g.lda = c.f; g.ldb = c.f; g.ldc = c.d; g.N = c.d; g.K = c.f;
      if ((rc = vd_gemm_f32(c.ctx, VARDROP_K_FFN_GRADS, g, true, c.s))) return rc;
    }
  }
  g.count(c.dn, false, c.n, c.B, 1);
  g.K = (int)c.T;
  g.set(0, xv, dh, dW1, nullptr);
  g.lda = c.d; g.ldb = c.f; g.ldc = c.f; g.M = c.d; g.N = c.f; g.part = (float*)(ws + w.part);
  if ((rc = vd_gemm_f32_wgrad(c.ctx, VARDROP_K_FFN_GRADS, g, c.s))) return rc;
  g.set(0, a, dy, dW2, nullptr);
  g.lda = c.f; g.ldb = c.d; g.ldc = c.d; g.M = c.f; g.N = c.d; g.part = (float*)(ws + w.second);
  if ((rc = vd_gemm_f32_wgrad(c.ctx, VARDROP_K_FFN_GRADS, g, c.s))) return rc;
  if (!db1 && !db2) return VARDROP_OK;
  const int pieces = column_pieces(c.T);
  fin.col[0] = db1 ? (float*)(ws + w.col) : nullptr;
  fin.col[1] = db2 ? (float*)(ws + w.col2) : nullptr;
  if (c.T == 0) return VARDROP_OK;       // (sums over no pieces)
  fin.pieces[0] = fin.pieces[1] = pieces;
  const ColArgs c0 = {db1 ? dh : nullptr, (float*)(ws + w.col), c.B, c.n, c.f, pieces, c.dn.dev};
  const ColArgs c1 = {db2 ? dy : nullptr, (float*)(ws + w.col2), c.B, c.n, c.d, pieces, c.dn.dev};
  VdTimer timer(c.ctx, VARDROP_K_FFN_BIAS, c.s);
  VD_KERNEL(c.ctx, ffn_columns_f32_kernel, dim3((unsigned)vd_ceil_div(c.d > c.f ? c.d : c.f, 64), (unsigned)pieces, 2), dim3(256), 0, c.s, c0, c1);
  VD_LAUNCH_CHECK(c.ctx);
  return VARDROP_OK;
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
    uint8_t* kept = (uint8_t*)saved;
    return act == VARDROP_ACT_RELU ? fwd_bf16<kActRelu>(c, x, W1, b1, W2, b2, y, kept, hc, he, (char*)ws)
                                   : fwd_bf16<kActGelu>(c, x, W1, b1, W2, b2, y, kept, hc, he, (char*)ws);
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
  if (!vd_aligned(saved, 256) || !ws || !vd_aligned(ws, 256) || ws_bytes < ffn_workspace(T, d, f, dtype).total) return VARDROP_EWORKSPACE;
  const FfnCall c = {ctx, B, n, d, f, dtype, act, T, dn, s};
  char* at = (char*)ws;
  const uint8_t* xc = (const uint8_t*)saved;
  FinishArgs fin = {};
  fin.slices = 1;
  fin.cols[0] = f; fin.cols[1] = d;
  if (dtype == VARDROP_BF16) {
    rc = act == VARDROP_ACT_RELU ? bwd_bf16<kActRelu>(c, dy, W1, W2, xc, dx, dW1, dW2, db1, db2, grad_dtype, at, fin)
                                 : bwd_bf16<kActGelu>(c, dy, W1, W2, xc, dx, dW1, dW2, db1, db2, grad_dtype, at, fin);
  } else {
    rc = bwd_f32(c, (const float*)dy, (const float*)W1, (const float*)W2, xc, (float*)dx, (float*)dW1, (float*)dW2, db1 != nullptr, db2 != nullptr, at, fin);
  }
  if (rc || (!fin.part[0] && !fin.col[0] && !fin.col[1])) return rc;
  fin.dW[0] = dW1; fin.dW[1] = dW2; fin.db[0] = db1; fin.db[1] = db2;
  fin.count = (long long)d * f;
  fin.bf16 = grad_dtype == VARDROP_BF16; fin.n_dev = dn.dev; fin.n = n;
  const long long blocks = (fin.count / 4 + 255) / 256;
  fin.blocks = blocks > 1024 ? 1024 : (int)blocks;
  const int grid = (fin.part[0] ? 2 * fin.blocks : 0) + (fin.col[0] ? vd_ceil_div(f, 16) : 0) + (fin.col[1] ? vd_ceil_div(d, 16) : 0);
  VdTimer timer(ctx, VARDROP_K_REDUCE_DW, s);
  VD_KERNEL(ctx, ffn_finish_kernel, dim3((unsigned)grid), dim3(256), 0, s, fin);
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
