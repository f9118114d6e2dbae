// What the bf16 and the fp32 feed-forward block share (ffn.hip, ffn_f32.hip).
#ifndef VARDROP_FFN_H
#define VARDROP_FFN_H
#include "pack8.h"
#include "tile_gemm.h"

struct FfnCall {
  vardrop_ctx* ctx;
  int B, n, d, f, act;
  long long T;
  VdDevCount dn;
  hipStream_t s;
  int past(int N, int bytes) const { return T * N * bytes >= kPastCaches; }
};

// What the last launch of a backward pass adds up, in an order of its own: slices of dW1 and dW2, pieces of db1 and db2.
struct FfnFinish {
  const float* part[2];        // [slices][rows][pitch]; null: already there
  float* col[2];               // [pieces][pitch of the columns]; null: not wanted
  void* dW[2];
  void* db[2];
  int rows[2], cols[2], pitch[2], part_rows[2];     // dW[z] is [rows][cols], a slice [part_rows][pitch]
  int slices, bf16;
  int B, tile_rows, pieces;    // db1 has a piece for every tile_rows of the B n tokens, db2 `pieces`
};

// the fp32 block (ffn_f32.hip); arguments are checked
size_t vd_ffn_workspace_f32(long long T, int d, int f);
int vd_ffn_fwd_f32(const FfnCall& c, const float* x, const float* W1, const float* b1, const float* W2, const float* b2, float* y, uint8_t* saved, char* ws);
int vd_ffn_bwd_f32(const FfnCall& c, const float* dy, const float* W1, const float* W2, const uint8_t* saved, float* dx, float* dW1, float* dW2, float* db1,
                   float* db2, char* ws, FfnFinish& fin);

namespace {

// ---- the plan of the gradients' launch
// The launch of dx (T x d over f) and of the weight gradients (2 d f over T in slices): time until the last place is done when the longer
// tiles come first, and the sum of the slices behind it.  Backward passes timed with every tile and number of slices, us, best -> by this plan:
// 31.0 -> 31.0 (1000 x 512 x 2048), 26.0 -> 26.0 (2784 x 512 x 512), 40.9 -> 40.9 (8000 x 512 x 512), 54.5 -> 55.7 (6000 x 768 x 768), 301 -> 316 (27 584 x 512 x
// 2048), 726 -> 731 (65 536 x 768 x 1536).
constexpr int kMostSlices = 16, kLeastSlice = 256;      // (tokens of a slice; in fp32, whose tokens count 3 and 6 times, a quarter)
struct GradPlan {
  int shape, slices;
};
inline int most_slices(long long T, int least = kLeastSlice) {
  const long long s = T / least;
  return s < 1 ? 1 : (s > kMostSlices ? kMostSlices : (int)s);
}
// parts: pairs of parts of dx and, in the mean, of the weight gradients (tile_pairs)
template <int SHAPES>
inline GradPlan plan_grads(const ShapeCost (&shapes)[SHAPES], long long T, int d, int f, int least_slice = kLeastSlice, double parts_x = 1, double parts_w = 1) {
  GradPlan best = {0, 1};
  double least = -1;
  for (int i = 0; i < SHAPES; ++i) {
    const ShapeCost& c = shapes[i];
    const long long nx = tiles_of(c, T, d);
    for (int s = 1; s <= most_slices(T, least_slice); ++s) {
      const long long nw = (tiles_of(c, d, f) + tiles_of(c, f, d)) * s;
      const double tw = tile_time(c, parts_w * T / s), tx = tile_time(c, parts_x * f);
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
      if (s > 1) end += 2.0 * d * f * s * 1e-3 + 1300;                         // (written and read; what the last launch takes longer)
      if (least < 0 || end < least) {
        least = end;
        best = {i, s};
      }
    }
  }
  return best;
}

// one product over the tokens' rows: A [T][K], B [K][N] or (bkc) [N][K], rows of `ldb` elements
inline TileArgs rows_product(const FfnCall& c, const void* A, const void* Bm, int K, int N, int ldb, bool status) {
  TileArgs g = {};
  g.A = A; g.B = Bm;
  g.lda = (long long)K * 2; g.ldb = (long long)ldb * 2;
  g.M = (int)c.T; g.N = N; g.K = K; g.slices = 1;
  g.n_dev = c.dn.dev; g.status = status ? c.dn.status : nullptr; g.n_max = c.n; g.n_mul = c.B; g.n_role = 0;
  return g;
}
// C [M][N] = A^T B, summed over the tokens
inline TileArgs tokens_product(const FfnCall& c, const void* A, const void* Bm, int M, int N, int slices) {
  TileArgs g = {};
  g.A = A; g.B = Bm;
  g.lda = (long long)M * 2; g.ldb = (long long)N * 2;
  g.M = M; g.N = N; g.K = (int)c.T; g.slices = slices;
  g.n_dev = c.dn.dev; g.n_max = c.n; g.n_mul = c.B; g.n_role = 1;
  return g;
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

// dx, dW1 and dW2 need the results of the launch before and nothing of each other.  The kind whose tiles are longer comes first; a die takes
// a contiguous range of either kind.
template <typename S, typename EpiX, typename Epi1, typename Epi2>
__global__ __launch_bounds__(S::THREADS, S::simd) void ffn_grads_kernel(TileArgs gx, typename EpiX::Args ax, TileArgs g1, typename Epi1::Args a1, TileArgs g2,
                                                                        typename Epi2::Args a2) {
  int Mx, Kx, M1, K1, M2, K2;
  if (!tile_dims(gx, Mx, Kx) || !tile_dims(g1, M1, K1) || !tile_dims(g2, M2, K2)) return;
  const int nx = gx.A ? (int)tile_count<S>(gx, Mx) : 0, n1 = (int)tile_count<S>(g1, M1), nw = n1 + (int)tile_count<S>(g2, M2);
  if ((int)blockIdx.x >= nx + nw) return;
  const bool w_first = (long long)(K1 / g1.slices) * tile_pairs<Epi1>() > (long long)Kx * tile_pairs<EpiX>();
  const int first = w_first ? nw : nx, xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const int of_first = (first >> 3) + (xcd < (first & 7) ? 1 : 0), from = xcd_range_start(xcd, first);
  const bool in_first = slot < of_first;
  const int t = in_first ? from + slot : xcd_range_start(xcd, nx + nw) - from + (slot - of_first);
  if (in_first != w_first) tile_gemm<false, true, true, S, EpiX>(gx, ax, Mx, Kx, t);
  else if (t < n1) tile_gemm<false, false, false, S, Epi1>(g1, a1, M1, K1, t);
  else tile_gemm<false, false, false, S, Epi2>(g2, a2, M2, K2, t - n1);
}

template <typename S, typename EpiX, typename Epi1, typename Epi2>
int launch_grads(const FfnCall& c, const TileArgs& gx, const typename EpiX::Args& ax, const TileArgs& g1, const typename Epi1::Args& a1, const TileArgs& g2,
                 const typename Epi2::Args& a2, int& pieces) {
  pieces = tile_pieces<S>(g2);
  VD_FFN_LAUNCH(VARDROP_K_FFN_GRADS, (ffn_grads_kernel<S, EpiX, Epi1, Epi2>), S, (gx.A ? tile_count<S>(gx, gx.M) : 0) + tile_count<S>(g1, g1.M) + tile_count<S>(g2, g2.M), gx, ax, g1,
                a1, g2, a2)
}
}  // namespace
#endif  // VARDROP_FFN_H
