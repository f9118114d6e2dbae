// The feed-forward block in fp32 (mathematics: ffn.hip), on the bf16 matrix instruction.
//
// An fp32 number is the sum of three bf16 numbers, hi + mid + lo, and a product of two such sums six exact products of parts
// (tile_gemm.h): with a sixth of the bf16 rate it is twice as fast as the fp32 instruction, and the products are the bf16 block's, with
// the element-wise work on their sums.  One launch lays the operands of a call out in parts, rows padded with zeros to multiples of 64
// channels, so that no width is odd to the products; what the products hand to each other (act(h), dh) they write in parts themselves.  A
// checkpoint's values are bf16 numbers, and x' has one part.  What three parts do not hold: bits below 2^-133; an infinity, or a magnitude
// that rounds to one in bf16 (from 0x1.ffp127 on), counts as NaN.
// Backward of 999 x 321 x 449, us: fp32 products with launches of their own for everything between 103 -> 42.
#include "ffn.h"

namespace {

__host__ __device__ inline int padded(int v) { return (v + 63) / 64 * 64; }

// parts of eight numbers, `plane` elements apart
__device__ inline void store_parts(bf16_t* p, long long plane, const float (&v)[8], bool past) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = v[e];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const u32x4 q = eight_bf16(r);
    store_past(reinterpret_cast<u32x4*>(p + k * plane), q, past);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      r[2 * w] -= __uint_as_float(q[w] << 16);
      r[2 * w + 1] -= __uint_as_float(q[w] & 0xffff0000u);
    }
  }
}
// eight neighbouring numbers of a row of `cols`, from column c on, zeros behind the last
__device__ inline void load_row(const float* row, int c, int cols, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? row[c + e] : 0.f;
}
__device__ inline void store_row(float* row, int c, int cols, const float (&v)[8], bool whole, bool past) {
  if (whole) {
    store_eight(row + c, v, past);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < cols) row[c + e] = v[e];
  }
}
// eight codes of a row, and back
__device__ inline void store_codes(uint8_t* row, int c, int cols, u32x2 codes) {
  if (cols % 8 == 0) {
    if (c < cols) *reinterpret_cast<u32x2*>(row + c) = codes;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < cols) row[c + e] = (uint8_t)((e < 4 ? codes.x : codes.y) >> (8 * (e & 3)));
  }
}
__device__ inline u32x2 load_codes(const uint8_t* row, int c, int cols) {
  if (cols % 8 == 0) return c < cols ? *reinterpret_cast<const u32x2*>(row + c) : u32x2{0, 0};
  uint32_t q[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (c + e < cols) q[e >> 2] |= (uint32_t)row[c + e] << (8 * (e & 3));
  return u32x2{q[0], q[1]};
}

// ---- the launch before the products.  A job's thread takes eight columns of a row; four threads are a block of 32.  Bound by memory: 27 584 x 512
// with weights of 512 x 2048 43 us (162 MB, 3.8 TB/s).
struct SplitJob {
  const float* src;            // null: values of a checkpoint, in one part
  bf16_t* dst;                 // [parts][rows][pitch]; null: only packed
  long long plane;             // elements from part to part
  uint8_t *codes, *exps;       // the checkpoint: written (src given) or read
  int rows, cols, all_rows;    // all_rows: those behind `rows` are zeros; tokens: rows is B n
  int tokens, blocks;
};
struct SplitArgs {
  SplitJob job[4];
  int B, n;
  const int32_t* n_dev;
  int32_t* status;
};
__global__ __launch_bounds__(256) void ffn_split_kernel(SplitArgs a) {
  int n;
  if (!vd_count(a.n_dev, a.n, n, a.status)) return;
  int block = blockIdx.x;
  SplitJob j = a.job[0];
#pragma unroll
  for (int k = 1; k < 4; ++k)
    if (block >= j.blocks) {
      block -= j.blocks;
      j = a.job[k];
    }
  if (j.tokens) j.rows = j.all_rows = a.B * n;
  const int pitch = padded(j.cols), per = pitch >> 3;
  const long long groups = (long long)j.all_rows * per;
  for (long long i = (long long)block * 256 + threadIdx.x; i < groups; i += (long long)j.blocks * 256) {
    const int r = groups <= 0x7fffffff ? (int)((uint32_t)i / (uint32_t)per) : (int)(i / per), c = (int)(i - (long long)r * per) * 8;
    float v[8];
    if (j.src) {
      load_row(j.src + (long long)r * j.cols, c, r < j.rows ? j.cols : 0, v);
      if (j.codes) {
        uint32_t e;
        const u32x2 q = pack_eight(v, e);
        store_codes(j.codes + (long long)r * j.cols, c, j.cols, q);
        if (c % 32 == 0 && c < j.cols) j.exps[(long long)r * pack_blocks(j.cols) + (c >> 5)] = (uint8_t)e;
      }
      if (j.dst) store_parts(j.dst + (long long)r * pitch + c, j.plane, v, false);
    } else {
      const u32x2 q = load_codes(j.codes + (long long)r * j.cols, c, j.cols);
      unpack_eight(q, c < j.cols ? j.exps[(long long)r * pack_blocks(j.cols) + (c >> 5)] : 1u, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = c + e < j.cols ? v[e] : 0.f;
      store_eight(j.dst + (long long)r * pitch + c, v);
    }
  }
}

// ---- what is done to the rows of a product (as in ffn.hip)
struct EpiOutF32 {           // C [rows][N] = sums + bias
  static constexpr bool kFetch = false, kSums = false;
  static constexpr int kPartsA = 3, kPartsB = 3, kRowSums = 0;
  struct Args {
    float* C;
    const float* bias;
    int N, whole, past;
  } a;
  float b[8];
  __device__ void columns(int n, int) {
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = a.bias && n + e < a.N ? a.bias[n + e] : 0.f;
  }
  __device__ void row(int, int, int m, int n, bool live, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += b[e];
    if (live && n < a.N) store_row(a.C + (long long)m * a.N, n, a.N, v, a.whole, a.past);
  }
};
template <int ACT, bool KEEP>
struct EpiActF32 {           // h = sums + bias, packed with KEEP; a = act(h) in parts, zeros behind the last channel
  static constexpr bool kFetch = false, kSums = false;
  static constexpr int kPartsA = 3, kPartsB = 3, kRowSums = 0;
  struct Args {
    bf16_t* act;
    long long plane;
    const float* bias;
    uint8_t *codes, *exps;
    int N, past;
  } a;
  float b[8];
  __device__ void columns(int n, int) {
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = a.bias && n + e < a.N ? a.bias[n + e] : 0.f;
  }
  __device__ void row(int, int, int m, int n, bool live, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = n + e < a.N ? v[e] + b[e] : 0.f;
    if constexpr (KEEP) {
      uint32_t e;
      const u32x2 c = pack_eight(v, e);
      if (live) {
        store_codes(a.codes + (long long)m * a.N, n, a.N, c);
        if (n % 32 == 0 && n < a.N) a.exps[(long long)m * pack_blocks(a.N) + (n >> 5)] = (uint8_t)e;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act_value<ACT, true>(v[e]);
    if (live) store_parts(a.act + (long long)m * padded(a.N) + n, a.plane, v, a.past);
  }
};
struct ActBwdF32Args {
  bf16_t *dh, *act;
  long long plane;
  const uint8_t *codes, *exps;
  float* sums;                 // of dh over a tile's rows; null: not wanted
  int N, past;
};
template <int ACT, int MI, int NJ>
struct EpiActBwdF32 {        // sums = da; dh = da act'(h'), a = act(h'), both in parts
  static constexpr bool kFetch = true, kSums = false;
  static constexpr int kPartsA = 3, kPartsB = 3, kRowSums = 1;
  typedef ActBwdF32Args Args;
  Args a;
  float total[8];
  u32x2 codes[2 * MI * NJ];
  uint32_t exps[2 * MI * NJ];
  __device__ void fetch(int k, int m, int n, bool live) {
    const int r = live ? m : 0;
    codes[k] = load_codes(a.codes + (long long)r * a.N, n, a.N);
    exps[k] = n < a.N ? a.exps[(long long)r * pack_blocks(a.N) + (n >> 5)] : 1u;
  }
  __device__ void columns(int, int) {
#pragma unroll
    for (int e = 0; e < 8; ++e) total[e] = 0.f;
  }
  __device__ void row(int, int k, int m, int n, bool live, float (&v)[8]) {
    if (!live) return;
    float h[8];
    unpack_eight(codes[k], exps[k], h);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float slope;
      h[e] = act_both<ACT, true>(h[e], slope);
      v[e] = n + e < a.N ? v[e] * slope : 0.f;
      total[e] += v[e];
      h[e] = n + e < a.N ? h[e] : 0.f;
    }
    const long long at = (long long)m * padded(a.N) + n;
    store_parts(a.dh + at, a.plane, v, a.past);
    store_parts(a.act + at, a.plane, h, a.past);
  }
};
template <int PARTS>
struct EpiGradF32 {          // a weight gradient [M][N], or a slice's partial product [slice][part_rows][pitch]
  static constexpr bool kFetch = false, kSums = PARTS == 3;       // (db2; db1 comes with dh)
  static constexpr int kPartsA = PARTS, kPartsB = 3, kRowSums = 0;
  struct Args {
    float *C, *part, *sums;
    int M, N, whole;         // M, N: the result's; the sums are [padded][padded]
  } a;
  __device__ void sums(int piece, int n, bool live, float v) {
    if (live && a.sums) a.sums[(long long)piece * padded(a.N) + n] = v;
  }
  __device__ void columns(int, int) {}
  __device__ void row(int slice, int, int m, int n, bool live, float (&v)[8]) {
    if (!live) return;
    if (a.part) store_eight(a.part + ((long long)slice * padded(a.M) + m) * padded(a.N) + n, v);
    else if (m < a.M && n < a.N) store_row(a.C + (long long)m * a.N, n, a.N, v, a.whole, false);
  }
};

// ---- a small block forward in one launch: a workgroup takes kSmallRows rows through both products, x and h in LDS (a channel's rows beside
// each other, so that a weight meets all of them), a thread a column of the result, or a part of its sum where columns are fewer
// than threads.  Its time is the chain of a row's steps, which more rows and columns do not lengthen.
constexpr int kSmallRows = 8, kSmallChannels = 512, kSmallWeights = 8192;
struct SmallArgs {
  const float *x, *W1, *b1, *W2, *b2;
  float* y;
  uint8_t *xc, *xe, *hc, *he;      // checkpoints; null: none
  int B, n, d, f;
  const int32_t* n_dev;
  int32_t* status;
};
typedef float SmallRow[kSmallRows];
// out[c][row] = bias[c] + sum_k in[k][row] W[k][c] for c < N; `part` has room for 256 columns' rows
__device__ __forceinline__ void small_product(const SmallRow* in, const float* W, const float* bias, int K, int N, SmallRow* out, SmallRow* part) {
  const int wide = min(256, (N + 63) / 64 * 64), groups = 256 / wide, g = threadIdx.x / wide, c0 = threadIdx.x % wide;
  const int per = (K + groups - 1) / groups, k0 = min(K, g * per), k1 = g < groups ? min(K, k0 + per) : k0;
  for (int c1 = 0; c1 < N; c1 += wide) {
    const int c = c1 + c0;
    float s[kSmallRows];
#pragma unroll
    for (int r = 0; r < kSmallRows; ++r) s[r] = 0.f;
    if (c < N) {
#pragma unroll 8
      for (int k = k0; k < k1; ++k) {
        const float w = W[(long long)k * N + c];
#pragma unroll
        for (int r = 0; r < kSmallRows; ++r) s[r] = fmaf(in[k][r], w, s[r]);
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallRows; ++r) part[threadIdx.x][r] = s[r];
    __syncthreads();
    if (g == 0 && c < N) {
      const float b = bias ? bias[c] : 0.f;
#pragma unroll
      for (int r = 0; r < kSmallRows; ++r) {
        for (int i = 1; i < groups; ++i) s[r] += part[threadIdx.x + i * wide][r];
        out[c][r] = s[r] + b;
      }
    }
  }
  __syncthreads();
}
// rows m0.. of `in`, packed: half a wavefront a block
__device__ __forceinline__ void small_pack(const SmallRow* in, int m0, int rows, int d, uint8_t* codes, uint8_t* exps) {
  const int nb = pack_blocks(d), l = threadIdx.x & 31;
  for (int b = threadIdx.x >> 5; b < rows * nb; b += 8) {
    const int r = b / nb, c = (b - r * nb) * kPackBlock + l;
    const float v = c < d ? in[c][r] : 0.f;
    uint32_t most = magnitude(v);
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, m, 64));
    const uint32_t e = pack_exponent(most);
    if (c < d) codes[(long long)(m0 + r) * d + c] = (uint8_t)pack_code(e >= 248u ? pack_limit(v) : v, pack_up(e));
    if (l == 0) exps[(long long)(m0 + r) * nb + (b - r * nb)] = (uint8_t)e;
  }
}
template <int ACT>
__global__ __launch_bounds__(256) void ffn_small_kernel(SmallArgs a) {
  __shared__ __attribute__((aligned(16))) SmallRow xs[kSmallChannels], hs[kSmallChannels], part[256];
  int n;
  if (!vd_count(a.n_dev, a.n, n, a.status)) return;
  const int T = a.B * n, m0 = blockIdx.x * kSmallRows, rows = min(kSmallRows, T - m0);
  if (rows <= 0) return;
  for (int i = threadIdx.x; i < kSmallRows * a.d; i += 256) {
    const int r = i / a.d, c = i - r * a.d;
    xs[c][r] = r < rows ? a.x[(long long)(m0 + r) * a.d + c] : 0.f;
  }
  __syncthreads();
  small_product(xs, a.W1, a.b1, a.d, a.f, hs, part);
  if (a.xc) {
    small_pack(xs, m0, rows, a.d, a.xc, a.xe);
    small_pack(hs, m0, rows, a.f, a.hc, a.he);
    __syncthreads();
  }
  for (int i = threadIdx.x; i < kSmallRows * a.f; i += 256) (&hs[0][0])[i] = act_value<ACT, true>((&hs[0][0])[i]);
  __syncthreads();
  small_product(hs, a.W2, a.b2, a.f, a.d, xs, part);
  for (int i = threadIdx.x; i < rows * a.d; i += 256) {
    const int r = i / a.d, c = i - r * a.d;
    a.y[(long long)(m0 + r) * a.d + c] = xs[c][r];
  }
}
// us, by the products -> in one launch: 40 x 64 x 128 11.6 -> 8.8, 2000 x 90 x 90 14.4 -> 10.9 (with checkpoints 12.0 -> 11.4, 15.3 -> 13.5), but 40 x 128 x 256
// 14.1 -> 17.1, 300 x 450 x 33 18.5 both (with checkpoints 14.6 -> 22.0, 19.6 -> 25.2).
bool is_small(const FfnCall& c) {
  return c.d <= kSmallChannels && c.f <= kSmallChannels && c.d * c.f <= kSmallWeights && c.T <= (long long)kSmallRows * c.ctx->num_cus;
}

template <typename S, int ACT, bool KEEP>
int launch_up(const FfnCall& c, const TileArgs& g, const typename EpiActF32<ACT, KEEP>::Args& e) {
  return launch_tile_gemm<false, true, false, S, EpiActF32<ACT, KEEP>>(c.ctx, VARDROP_K_FFN_UP, g, e, c.s);
}
template <typename S, int ACT>
int launch_dh(const FfnCall& c, const TileArgs& g, const ActBwdF32Args& e, int& tile_rows) {
  tile_rows = S::BM;
  return launch_tile_gemm<false, true, true, S, EpiActBwdF32<ACT, S::MI, S::NJ>>(c.ctx, VARDROP_K_FFN_DH, g, e, c.s);
}

struct WorkspaceF32 {        // bytes from its start; every operand in three parts
  size_t x, W1, W2, wide, act, kept, part, second, col, col2, total;
};
WorkspaceF32 workspace_f32(long long T, int d, int f) {
  const size_t D = padded(d), F = padded(f), t = T, slices = most_slices(T, kLeastSlice / 4);
  WorkspaceF32 w;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += vd_align_up(bytes, 256);
    return here;
  };
  w.x = take(6 * t * D);                   // x, or dy
  w.W1 = take(6 * D * F);
  w.W2 = take(6 * D * F);
  w.wide = take(6 * t * F);                // act(h) in the forward, dh in the backward
  w.act = take(6 * t * F);                 // act(h')
  w.kept = take(2 * t * D);                // x', one part
  w.part = take(slices * D * F * 4);
  w.second = take(slices * D * F * 4);
  w.col = take((t + 63) / 64 * F * 4);
  w.col2 = take(slices * (F / 64) * 2 * D * 4);
  w.total = at;
  return w;
}
int split_blocks(long long rows, int cols) {
  const long long b = (rows * (padded(cols) / 8) + 255) / 256;
  return b > 2048 ? 2048 : (int)b;
}
SplitJob weight_job(const float* W, void* dst, int rows, int cols) {
  SplitJob j = {};
  j.src = W; j.dst = (bf16_t*)dst;
  j.rows = rows; j.cols = cols; j.all_rows = padded(rows);
  j.plane = (long long)j.all_rows * padded(cols);
  j.blocks = split_blocks(j.all_rows, cols);
  return j;
}
int split(const FfnCall& c, const SplitJob& a, const SplitJob& b, const SplitJob& d, const SplitJob& e) {
  const SplitArgs s = {{a, b, d, e}, c.B, c.n, c.dn.dev, c.dn.status};
  VdTimer timer(c.ctx, VARDROP_K_FFN_SPLIT, c.s);
  VD_KERNEL(c.ctx, ffn_split_kernel, dim3((unsigned)(a.blocks + b.blocks + d.blocks + e.blocks)), dim3(256), 0, c.s, s);
  VD_LAUNCH_CHECK(c.ctx);
  return VARDROP_OK;
}
// operands in parts: A [T][K], B with rows of ldb
TileArgs parts_product(const FfnCall& c, const void* A, const void* Bm, int K, int N, int ldb, long long planeB) {
  TileArgs g = rows_product(c, A, Bm, K, N, ldb, false);
  g.planeA = c.T * K * 2;
  g.planeB = planeB * 2;
  return g;
}

template <int ACT>
int fwd(const FfnCall& c, const float* x, const float* W1, const float* b1, const float* W2, const float* b2, float* y, uint8_t* saved, char* ws) {
  if (is_small(c)) {
    uint8_t* hc = saved ? saved + pack_bytes(c.T, c.d) : nullptr;
    const SmallArgs a = {x, W1, b1, W2, b2, y, saved, saved ? saved + pack_exponents_at(c.T, c.d) : nullptr, hc, saved ? hc + pack_exponents_at(c.T, c.f) : nullptr,
                         c.B, c.n, c.d, c.f, c.dn.dev, c.dn.status};
    VdTimer timer(c.ctx, VARDROP_K_FFN_SMALL, c.s);
    VD_KERNEL(c.ctx, ffn_small_kernel<ACT>, dim3((unsigned)((c.T + kSmallRows - 1) / kSmallRows)), dim3(256), 0, c.s, a);
    VD_LAUNCH_CHECK(c.ctx);
    return VARDROP_OK;
  }
  const WorkspaceF32 w = workspace_f32(c.T, c.d, c.f);
  const int D = padded(c.d), F = padded(c.f);
  SplitJob jx = {};
  jx.src = x; jx.dst = (bf16_t*)(ws + w.x); jx.plane = c.T * D; jx.cols = c.d; jx.tokens = 1;
  jx.blocks = split_blocks(c.T, c.d);
  if (saved) {
    jx.codes = saved;
    jx.exps = saved + pack_exponents_at(c.T, c.d);
  }
  int rc = split(c, jx, weight_job(W1, ws + w.W1, c.d, c.f), weight_job(W2, ws + w.W2, c.f, c.d), SplitJob{});
  if (rc) return rc;
  const TileArgs up = parts_product(c, ws + w.x, ws + w.W1, D, F, F, (long long)D * F);
  bf16_t* a = (bf16_t*)(ws + w.wide);
  const int past = c.past(F, 6), shape = product_shape(kPartShapes, c.T, F, 6 * D);
  if (saved) {
    uint8_t* hc = saved + pack_bytes(c.T, c.d);
    const typename EpiActF32<ACT, true>::Args e = {a, c.T * F, b1, hc, hc + pack_exponents_at(c.T, c.f), c.f, past};
#define VD_CALL(S) launch_up<S, ACT, true>(c, up, e)
    rc = VD_BY_PARTS(shape, VD_CALL);
#undef VD_CALL
  } else {
    const typename EpiActF32<ACT, false>::Args e = {a, c.T * F, b1, nullptr, nullptr, c.f, past};
#define VD_CALL(S) launch_up<S, ACT, false>(c, up, e)
    rc = VD_BY_PARTS(shape, VD_CALL);
#undef VD_CALL
  }
  if (rc) return rc;
  const TileArgs down = parts_product(c, a, ws + w.W2, F, D, D, (long long)D * F);
  const EpiOutF32::Args e = {y, b2, c.d, c.d % 8 == 0 && vd_aligned(y, 16), c.past(c.d, 4)};
#define VD_CALL(S) launch_tile_gemm<false, true, false, S, EpiOutF32>(c.ctx, VARDROP_K_FFN_DOWN, down, e, c.s)
  return VD_BY_PARTS(product_shape(kPartShapes, c.T, D, 6 * F), VD_CALL);
#undef VD_CALL
}

template <int ACT>
int bwd(const FfnCall& c, const float* dy, const float* W1, const float* W2, const uint8_t* saved, float* dx, float* dW1, float* dW2, float* db1, float* db2,
        char* ws, FfnFinish& fin) {
  const WorkspaceF32 w = workspace_f32(c.T, c.d, c.f);
  const int D = padded(c.d), F = padded(c.f);
  const uint8_t* hc = saved + pack_bytes(c.T, c.d);
  bf16_t *dh = (bf16_t*)(ws + w.wide), *a = (bf16_t*)(ws + w.act), *xv = (bf16_t*)(ws + w.kept), *g0 = (bf16_t*)(ws + w.x);
  if (c.T > 0) {
    SplitJob jy = {}, jx = {};
    jy.src = dy; jy.dst = g0; jy.plane = c.T * D; jy.cols = c.d; jy.tokens = 1;
    jx.dst = xv; jx.codes = const_cast<uint8_t*>(saved); jx.exps = const_cast<uint8_t*>(saved) + pack_exponents_at(c.T, c.d); jx.cols = c.d; jx.tokens = 1;
    jy.blocks = jx.blocks = split_blocks(c.T, c.d);
    int rc = split(c, jy, weight_job(W2, ws + w.W2, c.f, c.d), jx, dx ? weight_job(W1, ws + w.W1, c.d, c.f) : SplitJob{});
    if (rc) return rc;
    const TileArgs g = parts_product(c, g0, ws + w.W2, D, F, D, (long long)D * F);
    const ActBwdF32Args e = {dh, a, c.T * F, hc, hc + pack_exponents_at(c.T, c.f), db1 ? (float*)(ws + w.col) : nullptr, c.f, c.past(F, 6)};
#define VD_CALL(S) launch_dh<S, ACT>(c, g, e, fin.tile_rows)
    rc = VD_BY_PARTS(product_shape(kPartShapes, c.T, F, 6 * D), VD_CALL);
#undef VD_CALL
    if (rc) return rc;
  }
  const GradPlan plan = plan_grads(kPartShapes, c.T, D, F, kLeastSlice / 4, 6, 4.5);
  float *part = (float*)(ws + w.part), *second = (float*)(ws + w.second);
  fin.part_rows[0] = fin.pitch[1] = D;
  fin.part_rows[1] = fin.pitch[0] = F;
  if (plan.slices > 1) {
    fin.part[0] = part;
    fin.part[1] = second;
    fin.slices = plan.slices;
  }
  fin.col[0] = db1 ? (float*)(ws + w.col) : nullptr;
  fin.col[1] = db2 ? (float*)(ws + w.col2) : nullptr;
  TileArgs gx = {}, g1 = tokens_product(c, xv, dh, D, F, plan.slices), g2 = tokens_product(c, a, g0, F, D, plan.slices);
  if (dx && c.T > 0) gx = parts_product(c, dh, ws + w.W1, F, D, F, (long long)D * F);
  g1.planeB = g2.planeA = c.T * F * 2;
  g2.planeB = c.T * D * 2;
  const EpiOutF32::Args ax = {dx, nullptr, c.d, c.d % 8 == 0 && vd_aligned(dx, 16), c.past(c.d, 4)};
  const EpiGradF32<1>::Args a1 = {dW1, (float*)fin.part[0], nullptr, c.d, c.f, c.f % 8 == 0 && vd_aligned(dW1, 16)};
  const EpiGradF32<3>::Args a2 = {dW2, (float*)fin.part[1], fin.col[1], c.f, c.d, c.d % 8 == 0 && vd_aligned(dW2, 16)};
#define VD_CALL(S) launch_grads<S, EpiOutF32, EpiGradF32<1>, EpiGradF32<3>>(c, gx, ax, g1, a1, g2, a2, fin.pieces)
  return VD_BY_PARTS(plan.shape, VD_CALL);
#undef VD_CALL
}

}  // namespace

size_t vd_ffn_workspace_f32(long long T, int d, int f) { return workspace_f32(T, d, f).total; }
int vd_ffn_fwd_f32(const FfnCall& c, const float* x, const float* W1, const float* b1, const float* W2, const float* b2, float* y, uint8_t* saved, char* ws) {
  return c.act == VARDROP_ACT_RELU ? fwd<kActRelu>(c, x, W1, b1, W2, b2, y, saved, ws) : fwd<kActGelu>(c, x, W1, b1, W2, b2, y, saved, ws);
}
int vd_ffn_bwd_f32(const FfnCall& c, const float* dy, const float* W1, const float* W2, const uint8_t* saved, float* dx, float* dW1, float* dW2, float* db1,
                   float* db2, char* ws, FfnFinish& fin) {
  return c.act == VARDROP_ACT_RELU ? bwd<kActRelu>(c, dy, W1, W2, saved, dx, dW1, dW2, db1, db2, ws, fin)
                                   : bwd<kActGelu>(c, dy, W1, W2, saved, dx, dW1, dW2, db1, db2, ws, fin);
}
